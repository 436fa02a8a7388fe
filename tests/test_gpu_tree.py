"""GPU tests of the draft-tree operators through the C ABI: tree attention, verification and commit against the numpy
oracle in double precision, alone and together as a decode loop uses them.

Tolerances of the attention, per element, with A = sum_k w_k |v_k| (w: softmax weights, from the oracle):
  the softmax weights reach the tensor core as bf16 (half a step: 2^-8 relative)      2^-8 A
  the output is rounded to bf16                                                       2^-8 |out|
  a logit is a sum of 128 exact products in fp32: off by at most 128 * 2^-23 * sum|q k| * scale, below 3e-4 for the
  inputs here (sum|q k| * scale < 20); a weight relative to the others is then off by twice that           6e-4 A
The log-sum-exp is off by a logit's error and by the sum of fp32 exponentials: 3e-4 + 1e-4.
Whole numbers (path, counts, tokens) and copies have to be equal."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as ot

pytestmark = pytest.mark.gpu

SCALE = 1.0 / math.sqrt(128.0)


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_08097_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def f64(t):
    return t.detach().double().cpu().numpy()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- attention -----------------------------------------------------------------------------------------------------
def random_tree(rng, B, T):
    return np.array([[-1] + [int(rng.integers(max(-1, t - 9), t)) for t in range(1, T)] for _ in range(B)], np.int32)


class AttnCase:
    """A working set whose rows hold `budget` random full blocks, the partial block in its local column, shuffled slots,
    and NaN, infinities and the largest values wherever no query may look."""

    def __init__(self, L, B, Hq, Hkv, T, lens, nodes, budget, parent=None, seed=0, dirty=True):
        rng, g = np.random.default_rng(seed), gen(seed)
        cols = budget + 2
        self.dims = L.Dims(B, Hq, Hkv, max(lens) // 16 + 1)
        self.T, self.lens, self.nodes = T, lens, nodes
        self.slot = rng.permutation(B * Hkv * cols).reshape(B, Hkv, cols).astype(np.int32)
        self.blk = np.full((B, Hkv, cols), -1, np.int32)
        pool = randn(g, B * Hkv * cols, 2, 16, 128)
        for b in range(B):
            full = lens[b] // 16
            for h in range(Hkv):
                k = min(budget, full)
                at = rng.permutation(budget)[:k]                     # holes among the columns
                self.blk[b, h, at] = rng.permutation(full)[:k]
                self.blk[b, h, budget + full % 2] = full             # the active local block, empty at a block's border
                if lens[b] % 16 == 0 and rng.random() < 0.5:
                    self.blk[b, h, budget + 1 - full % 2] = full + 1  # a block past the end
                if dirty:
                    for c in range(cols):
                        n = 0 if self.blk[b, h, c] < 0 else max(0, min(16, lens[b] - 16 * self.blk[b, h, c]))
                        pool[self.slot[b, h, c], :, n:] = float(rng.choice([np.nan, np.inf, -np.inf, 3e38]))
        self.parent = random_tree(rng, B, T) if parent is None else np.array(parent, np.int32)
        self.tree_kv, self.q = randn(g, B, T, Hkv, 2, 128), randn(g, B, T, Hq, 128) * 2
        if dirty:
            for b in range(B):
                n = max(0, min(nodes[b], T))
                self.tree_kv[b, n:] = float("nan")
                self.q[b, n:] = float("nan")
        self.pool = pool
        self.d_parent, self.d_nodes, self.d_lens = i32(self.parent.tolist()), i32(nodes), i32(lens)
        self.d_slot, self.d_blk = i32(self.slot.tolist()), i32(self.blk.tolist())
        self.need = L.tree_attn_workspace_bytes(self.dims, T, cols)
        self.ws = torch.full((max(self.need, 16),), 255, dtype=torch.uint8, device="cuda")       # NaN patterns
        self.fresh()

    def fresh(self):
        B, T, Hq = self.q.shape[:3]
        self.out = torch.full((B, T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((B, T, Hq), 7.0, device="cuda")

    def run(self, L, lse=True, stream=None, ws=True, out=None):
        L.tree_attn(self.dims, self.q, self.tree_kv, self.d_parent, self.d_nodes, self.pool, self.d_slot, self.d_blk, self.d_lens, SCALE,
                    self.out if out is None else out, lse=self.lse if lse else None, workspace=self.ws if ws else None, stream=stream)

    def check(self):
        out, lse = np.full(self.out.shape, 7.0), np.full(self.lse.shape, 7.0)
        a = ot.tree_attn(f64(self.q), f64(self.tree_kv), self.parent, self.nodes, f64(self.pool), self.slot, self.blk, self.lens, SCALE, out, lse)
        got, got_lse = f64(self.out), f64(self.lse)
        assert np.isfinite(got).all()
        assert np.all(np.abs(got - out) <= 2 ** -8 * (a + np.abs(out)) + 6e-4 * a), np.abs(got - out).max()
        assert np.all(np.abs(got_lse - lse) <= 4e-4), np.abs(got_lse - lse).max()
        for b, n in enumerate(self.nodes):                            # padding rows are left as they were
            n = max(0, min(n, self.T))
            assert (got[b, n:] == 7.0).all() and (got_lse[b, n:] == 7.0).all()


ATTN = [
    # B, Hq, Hkv, T, lens, nodes, budget
    (1, 8, 8, 1, [0], [1], 4),                        # the very first token
    (1, 1, 1, 1, [1], [1], 4),
    (2, 4, 2, 2, [15, 16], [2, 1], 6),
    (3, 12, 4, 5, [17, 0, 300], [5, 3, 0], 10),       # an empty request
    (2, 8, 2, 16, [129, 64], [16, 9], 12),            # 64 rows
    (2, 8, 2, 17, [200, 33], [17, 2], 3),             # 68 rows: two softmax sets; two blocks of the tree buffer
    (1, 32, 8, 33, [500], [33], 40),
    (2, 32, 8, 64, [333, 12], [64, 40], 24),          # 256 rows: two row groups, the second one empty of nodes 32..
    (1, 40, 8, 64, [90], [61], 8),                    # 320 rows in three groups, a node across a border
    (1, 128, 1, 3, [77], [3], 8),                     # one KV head, a node per row group
    (1, 64, 1, 64, [40], [64], 4),                    # 4,096 rows
    (5, 16, 2, 7, [1000, 999, 16, 31, 512], [7, 1, 7, 4, 9], 70),     # a count beyond n_tree is clamped
    (1, 8, 1, 4, [3000], [4], 190),                   # one row: split over many thread blocks
    (20, 16, 8, 4, [100 + 13 * i for i in range(20)], [4] * 20, 30),  # 160 rows: not split, more than the SMs
    (2, 8, 2, 20, [700, 650], [20, 13], 40),          # 80 rows
    (1, 8, 2, 8, [500], [8], 31),                     # 32 rows, splits that merge as a cluster of four
    (2, 24, 2, 5, [600, 20], [5, 4], 36),             # 60 rows
    (11, 16, 4, 16, [350, 20, 0, 16, 90, 333, 17, 15, 111, 400, 5], [16, 9, 16, 1, 0, 16, 16, 3, 16, 16, 7], 24),     # 64 rows, clusters of three
    (10, 16, 4, 20, [350, 20, 0, 16, 90, 333, 17, 15, 111, 400], [20, 9, 20, 1, 0, 20, 20, 3, 20, 19], 24),            # 80 rows, the same
    (10, 16, 4, 41, [350, 20, 0, 16, 90, 333, 17, 15, 111, 400], [41, 9, 33, 1, 0, 40, 41, 3, 41, 41], 24),            # 164 rows, the same
    (9, 16, 4, 64, [270, 20, 0, 16, 90, 260, 17, 15, 111], [64, 9, 33, 1, 0, 40, 64, 3, 64], 16),                      # 256 rows, clusters of two
    (1, 4, 1, 2, [4100], [2], 255),                   # 8 rows, splits that merge through the workspace
    (1, 16, 2, 16, [3300], [15], 200),                # 128 rows, the same
    (1, 8, 2, 64, [3400], [63], 210),                 # 256 rows, the same
]


@pytest.mark.parametrize("case", ATTN, ids=lambda c: "B%d_Hq%d_Hkv%d_T%d_k%d" % (c[0], c[1], c[2], c[3], c[6]))
def test_tree_attention(L, case):
    c = AttnCase(L, *case, seed=sum(case[:4]))
    c.run(L)
    torch.cuda.synchronize()
    c.check()
    first, first_lse = c.out.clone(), c.lse.clone()
    c.fresh()
    c.run(L)                                          # the same bits again, over a workspace that holds the first run's
    torch.cuda.synchronize()
    assert torch.equal(c.out, first) and torch.equal(c.lse, first_lse)
    c.fresh()
    c.run(L, lse=False)
    torch.cuda.synchronize()
    assert torch.equal(c.out, first) and (c.lse == 7.0).all()


@pytest.mark.parametrize("parent", [
    [-1, 0, 1, 2, 3, 4, 5, 6],                        # a chain
    [-1, -1, -1, -1, -1, -1, -1, -1],                 # eight roots
    [-1, 0, 0, 0, 0, 0, 0, 0],
    [-5, 99, 2, 7, 1, 4, 5, -1],                      # parents that are none: roots
])
def test_tree_shapes(L, parent):
    c = AttnCase(L, 2, 8, 2, 8, [70, 3], [8, 8], 6, parent=[parent, parent], seed=3)
    c.run(L)
    torch.cuda.synchronize()
    c.check()


def test_a_long_chain_sees_all_of_itself(L):
    chain = list(range(-1, 63))
    c = AttnCase(L, 1, 2, 1, 64, [0], [64], 4, parent=[chain], seed=4)
    c.run(L)
    torch.cuda.synchronize()
    c.check()


def test_a_long_cache(L):
    """Every block of 20,000 tokens, split over the SMs: the running maximum moves, sums are long."""
    c = AttnCase(L, 1, 4, 1, 3, [20011], [3], 1260, seed=5)
    c.q *= 3
    c.run(L)
    torch.cuda.synchronize()
    # (the logits are three times those that the module's bound of 20 is for)
    out, lse = np.zeros(c.out.shape), np.zeros(c.lse.shape)
    a = ot.tree_attn(f64(c.q), f64(c.tree_kv), c.parent, c.nodes, f64(c.pool), c.slot, c.blk, c.lens, SCALE, out, lse)
    assert np.all(np.abs(f64(c.out) - out) <= 2 ** -8 * (a + np.abs(out)) + 18e-4 * a)
    assert np.all(np.abs(f64(c.lse) - lse) <= 1e-3)


def test_a_chain_equals_the_chain_attention(L):
    """The same keys once in the tree buffer, once appended to the cache."""
    B, T, Hq, Hkv, budget, lens = 2, 5, 8, 2, 10, [100, 59]
    c = AttnCase(L, B, Hq, Hkv, T, lens, [T] * B, budget, parent=[[-1, 0, 1, 2, 3]] * B, seed=6, dirty=False)
    c.run(L)
    pool, blk = c.pool.clone(), c.d_blk.clone()
    table = torch.arange(B * c.dims.max_blocks, dtype=torch.int32, device="cuda").view(B, -1)
    L.append_kv(c.dims, c.tree_kv, 0, c.d_lens, table, c.d_slot, blk, budget, pool)
    out = torch.empty_like(c.out)
    ws = torch.empty(max(16, L.attn_workspace_bytes(c.dims, T, budget + 2)), dtype=torch.uint8, device="cuda")
    L.sparse_attn(c.dims, c.q, T, pool, c.d_slot, blk, budget + 2, c.d_lens, SCALE, out, workspace=ws)
    torch.cuda.synchronize()
    # two roundings of the weights and two of the outputs (values below 4): 2^-8 each way
    assert (c.out.float() - out.float()).abs().max() <= 4 * 2 ** -7


def test_graph_replay_and_two_streams(L):
    a = AttnCase(L, 2, 8, 2, 9, [120, 47], [9, 5], 12, seed=7)
    b = AttnCase(L, 1, 32, 8, 33, [400], [33], 30, seed=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    a.run(L)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a.run(L)
    for _ in range(3):
        a.out.fill_(7.0)
        a.lse.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        b.run(L, stream=s)
        torch.cuda.synchronize()
        a.check()
        b.check()
    a.q.neg_()                                        # replays read the inputs anew
    graph.replay()
    torch.cuda.synchronize()
    a.check()


# ---- verification --------------------------------------------------------------------------------------------------
def verify(L, logits, tokens, parent, nodes, u, temp, M, draft=None):
    B, T, V = logits.shape
    path = torch.full((B, M), 99, dtype=torch.int32, device="cuda")
    n, nxt = torch.full((B,), 99, dtype=torch.int32, device="cuda"), torch.full((B,), 99, dtype=torch.int32, device="cuda")
    L.verify_tree(logits, i32(tokens.tolist()), i32(parent.tolist()), i32(list(nodes)), torch.tensor(u, dtype=torch.float32, device="cuda"),
                  torch.tensor(temp, dtype=torch.float32, device="cuda"), path, n, nxt, draft_probs=draft)
    torch.cuda.synchronize()
    ref = ot.verify_tree(f64(logits), tokens, parent, nodes, np.array(u, np.float32), np.array(temp, np.float32), M,
                         None if draft is None else f64(draft))
    got = [t.cpu().numpy() for t in (path, n, nxt)]
    for name, g, r in zip(("path", "n_commit", "next_token"), got, ref):
        assert np.array_equal(g, r), (name, g, r)
    return got


def make_verify(rng, B, T, V, dtype, draft, spread=2.0):
    g = gen(int(rng.integers(1 << 30)))
    logits = (torch.randn((B, T, V), generator=g, device="cuda") * spread).to(dtype)
    q = torch.softmax(logits.float() + torch.randn((B, T, V), generator=g, device="cuda"), -1) if draft else None
    parent = np.array([[-1] + [int(rng.integers(max(0, t - 4), t)) for t in range(1, T)] for _ in range(B)], np.int32)
    top = logits.float().topk(min(3, V), -1).indices.cpu().numpy()
    tokens = np.array([[top[b, max(parent[b, t], 0), rng.integers(top.shape[2])] if rng.random() < 0.8 else rng.integers(V)
                        for t in range(T)] for b in range(B)], np.int32)
    return logits, q, parent, tokens, rng.random((B, T)).astype(np.float32)


@pytest.mark.parametrize("draft", [False, True], ids=["fixed", "drawn"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (2, 2, 2), (3, 5, 7), (2, 64, 33), (5, 9, 255), (4, 6, 4099), (3, 7, 20011), (40, 5, 1000), (160, 3, 515)])
def test_verification(L, B, T, V, dtype, draft):
    rng = np.random.default_rng(B * 1000 + T * 10 + V + draft)
    logits, q, parent, tokens, u = make_verify(rng, B, T, V, dtype, draft)
    temp = rng.choice([0.0, 0.4, 1.0, 1.7], B)
    nodes = rng.integers(0, T + 2, B) if B > 1 else [T]
    verify(L, logits, tokens, parent, nodes, u, temp, max(1, min(T, 6)), q)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_rows_at_any_alignment_and_stride(L, dtype):
    rng = np.random.default_rng(11)
    B, T, V = 3, 4, 5003
    logits, q, parent, tokens, u = make_verify(rng, B, T, V, dtype, True)
    for off in (1, 2, 3, 5):
        room = torch.full((B, T + 1, V + 13), float("nan"), dtype=dtype, device="cuda")        # what lies around the rows is not read
        room[:, :T, off:off + V] = logits
        dq = torch.full((B, T, V + 5), float("nan"), device="cuda")
        dq[:, :, off:off + V] = q if off + V <= V + 5 else 0
        verify(L, room[:, :T, off:off + V], tokens, parent, [T] * B, u, [0.0, 0.9, 1.3], T, dq[:, :, off:off + V])


def test_left_out_tokens_infinities_and_lowest_values(L):
    V, T = 1003, 3
    tokens, parent = np.array([[0, 4, 5]] * 8, np.int32), np.array([[-1, 0, 0]] * 8, np.int32)
    x = torch.randn((8, T, V), generator=gen(12), device="cuda")
    x[0, 0] = -math.inf                               # nothing is left
    x[1, 0] = -math.inf
    x[1, 0, 77] = 1.0                                 # one token is left
    x[2, 0] = math.nan
    x[2, 0, 5] = -3.0                                 # the second child's
    x[3, 0, [4, 600]] = math.inf                      # two tokens share everything
    x[4, 0] = torch.finfo(torch.float32).min          # the lowest value everywhere: all tokens alike
    x[5, 0, 6:] = torch.finfo(torch.float32).min
    x[6, 0] = math.nan
    x[7, 0, :] = 0.0
    for temp in (0.0, 0.3, 1.0):
        for u0 in (0.0, 0.5, 1.0 - 2.0 ** -24):
            verify(L, x, tokens, parent, [T] * 8, np.full((8, T), u0, np.float32), [temp] * 8, T)
            q = torch.full((8, T, V), 1.0 / V, device="cuda")
            verify(L, x, tokens, parent, [T] * 8, np.full((8, T), u0, np.float32), [temp] * 8, T, q)


def test_equal_logits_and_borders_between_tokens(L):
    """All tokens alike and a random number exactly on a border: the token behind the border; greedy: the first one."""
    V = 4096
    x = torch.zeros((6, 1, V), device="cuda")
    u = np.array([[0.0], [1 / V], [17 / V], [4095 / V], [1.0 - 2.0 ** -24], [0.5]], np.float32)
    got = verify(L, x, np.zeros((6, 1), np.int32), np.full((6, 1), -1, np.int32), [1] * 6, u, [1.0] * 6, 1)
    assert got[2].tolist() == [0, 1, 17, 4095, 4095, 2048]
    got = verify(L, x, np.zeros((6, 1), np.int32), np.full((6, 1), -1, np.int32), [1] * 6, u, [0.0] * 6, 1)
    assert got[2].tolist() == [0] * 6


def test_random_numbers_outside_their_range(L):
    x = torch.randn((5, 3, 300), generator=gen(13), device="cuda")
    tokens, parent = np.array([[0, 7, 9]] * 5, np.int32), np.array([[-1, 0, 1]] * 5, np.int32)
    u = np.array([[1.0] * 3, [2.0] * 3, [-1.0] * 3, [math.nan] * 3, [math.inf] * 3], np.float32)
    verify(L, x, tokens, parent, [3] * 5, u, [1.0] * 5, 3)


def test_siblings_with_the_same_token_and_tokens_outside_the_vocabulary(L):
    rng = np.random.default_rng(14)
    x = torch.randn((4, 6, 50), generator=gen(14), device="cuda")
    tokens = np.array([[0, 3, 3, 3, 8, 3], [0, -1, 50, 1 << 30, 2, -5], [0, 3, 4, 3, 4, 3], [9, 9, 9, 9, 9, 9]], np.int32)
    parent = np.array([[-1, 0, 0, 0, 0, 0]] * 3 + [[-1, 5, 2, 7, -9, 5]], np.int32)     # (the last: no valid child)
    for draft in (None, torch.softmax(x, -1)):
        for _ in range(6):
            verify(L, x, tokens, parent, [6] * 4, rng.random((4, 6)), [1.0, 0.8, 2.0, 1.0], 6, draft)
    verify(L, x, tokens, parent, [6] * 4, rng.random((4, 6)), [0.0] * 4, 6)


def test_a_draft_equal_to_the_target_and_one_that_takes_all(L):
    """q = p keeps every first child; q >= p everywhere leaves nothing when rejected: p stays as it was."""
    rng = np.random.default_rng(15)
    x = torch.randn((64, 4, 200), generator=gen(15), device="cuda")
    parent = np.array([[-1, 0, 0, 1]] * 64, np.int32)
    p = torch.softmax(x.double(), -1).float()
    tokens = rng.integers(0, 200, (64, 4)).astype(np.int32)
    verify(L, x, tokens, parent, [4] * 64, rng.random((64, 4)), [1.0] * 64, 4, p * 0.999)
    verify(L, x, tokens, parent, [4] * 64, rng.random((64, 4)), [1.0] * 64, 4, p + 0.5)


def test_random_numbers_next_to_the_decision(L):
    """Random numbers within a few fp32 steps of a child's share: decided by the fp64 value, as the oracle does."""
    x = torch.randn((32, 2, 3000), generator=gen(16), device="cuda")
    tokens, parent = np.full((32, 2), 11, np.int32), np.array([[-1, 0]] * 32, np.int32)
    p = torch.softmax(x.double(), -1)[:, 0, 11].cpu().numpy()
    u = np.zeros((32, 2), np.float32)
    for k in range(32):
        u[k, 1] = np.float32(p[k]) * np.float32(1 + (k - 16) * 2.0 ** -23)
        u[k, 0] = 0.25
    got = verify(L, x, tokens, parent, [2] * 32, u, [1.0] * 32, 2)
    assert 0 < (got[1] == 2).sum() < 32


def test_a_path_that_is_full_and_the_largest_vocabulary(L):
    rng = np.random.default_rng(17)
    V = 300007
    x = torch.randn((2, 8, V), generator=gen(17), device="cuda").to(torch.bfloat16)
    parent = np.array([list(range(-1, 7))] * 2, np.int32)
    tokens = np.zeros((2, 8), np.int32)
    best = x.float().argmax(-1).cpu().numpy()
    for t in range(1, 8):
        tokens[:, t] = best[:, t - 1]
    for M in (1, 3, 8):
        got = verify(L, x, tokens, parent, [8, 8], rng.random((2, 8)), [0.0, 0.02], M)
        assert got[1][0] == M
    big = torch.zeros((1, 1, 1 << 22), dtype=torch.float16, device="cuda")
    big[0, 0, (1 << 22) - 1] = 12.0
    verify(L, big, np.zeros((1, 1), np.int32), np.full((1, 1), -1, np.int32), [1], np.array([[0.9]]), [1.0], 1)
    verify(L, big, np.zeros((1, 1), np.int32), np.full((1, 1), -1, np.int32), [1], np.array([[0.9]]), [0.0], 1)


def test_verification_in_a_graph_and_on_a_stream(L):
    rng = np.random.default_rng(18)
    logits, q, parent, tokens, u = make_verify(rng, 6, 5, 9001, torch.bfloat16, True)
    args = [i32(tokens.tolist()), i32(parent.tolist()), i32([5] * 6), torch.tensor(u, device="cuda"), torch.full((6,), 0.9, device="cuda")]
    outs = [torch.zeros((6, 5), dtype=torch.int32, device="cuda")] + [torch.zeros(6, dtype=torch.int32, device="cuda") for _ in range(4)]
    L.verify_tree(logits, *args, outs[0], outs[1], outs[2], draft_probs=q)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs[:3]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.verify_tree(logits, *args, outs[0], outs[1], outs[2], draft_probs=q)
    outs[0].zero_(), outs[1].zero_(), outs[2].zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = torch.zeros((6, 5), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph.replay()
    L.verify_tree(logits, *args, other, outs[3], outs[4], draft_probs=q, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs[:3], want)) and torch.equal(other, want[0])
    ref = ot.verify_tree(f64(logits), tokens, parent, [5] * 6, u, np.full(6, np.float32(0.9)), 5, f64(q))
    assert all(np.array_equal(w.cpu().numpy(), r) for w, r in zip(want, ref))


@pytest.mark.parametrize("draft", [False, True], ids=["fixed", "drawn"])
def test_rows_larger_than_shared_memory(L, draft):
    """300 requests leave one thread block for each: its part of 70,001 tokens is read again for every pass."""
    rng = np.random.default_rng(19 + draft)
    logits, q, parent, tokens, u = make_verify(rng, 300, 3, 70001, torch.bfloat16, draft)
    verify(L, logits, tokens, parent, [3] * 300, u, rng.choice([0.0, 0.7, 1.0], 300), 3, q)


# ---- commit --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layers,B,Hkv,T,M,host", [(1, 1, 8, 1, 1, "device"), (1, 2, 1, 5, 5, "none"), (3, 5, 4, 64, 16, "pinned"),
                                                   (64, 2, 2, 7, 3, "device"), (2, 33, 3, 16, 11, "some")])
def test_commit(L, layers, B, Hkv, T, M, host):
    rng, g = np.random.default_rng(layers + B + T), gen(layers + B)
    cols, mb, col = 7, 6, 3
    lens = [int(rng.integers(0, 60)) for _ in range(B)]
    keep = [int(rng.integers(-1, M + 3)) for _ in range(B)]           # below none and beyond the path: clamped
    keep[0] = M
    path = rng.integers(0, T, (B, M)).astype(np.int32)               # the same node twice is allowed
    if B > 2:
        path[1, 0], path[2, M // 2] = -1, T                          # entries that name no node are skipped
    tree = [randn(g, B, T, Hkv, 2, 128) for _ in range(layers)]
    table = [torch.tensor(rng.permutation(B * mb).reshape(B, mb), dtype=torch.int32, device="cuda") for _ in range(layers)]
    slot = [torch.tensor(rng.permutation(B * Hkv * cols).reshape(B, Hkv, cols), dtype=torch.int32, device="cuda") for _ in range(layers)]
    blk = [torch.full((B, Hkv, cols), -9, dtype=torch.int32, device="cuda") for _ in range(layers)]
    pool = [torch.full((B * Hkv * cols, 2, 16, 128), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(layers)]
    kv = [torch.full((B * mb, Hkv, 2, 16, 128), 5.0, dtype=torch.bfloat16) for _ in range(layers)]
    kv = [None if host == "none" or (host == "some" and l == 0) else t.pin_memory() if host == "pinned" else t.cuda() for l, t in enumerate(kv)]
    want = []
    for l in range(layers):
        w = [f64(pool[l]), None if kv[l] is None else f64(kv[l]), blk[l].cpu().numpy(), np.zeros(B, np.int32)]
        ot.commit_kv(f64(tree[l]), path, keep, lens, table[l].cpu().numpy(), slot[l].cpu().numpy(), w[2], col, w[0], w[1], w[3])
        want.append(w)
    dims, nxt = L.Dims(B, Hkv, Hkv, mb), torch.zeros(B, dtype=torch.int32, device="cuda")
    d = [torch.tensor(path, device="cuda"), i32(keep), i32(lens)]
    if layers == 1:
        L.commit_kv(dims, tree[0], *d, table[0], slot[0], blk[0], col, pool[0], kv[0], next_len=nxt)
    else:
        plan = L.CommitPlan(dims, tree, table, slot, blk, col, pool, kv)
        L.commit_kv_layers(plan, *d)                                  # without the new lengths
        L.commit_kv_layers(plan, *d, next_len=nxt)
    torch.cuda.synchronize()
    for l in range(layers):
        assert np.array_equal(f64(pool[l]), want[l][0]) and np.array_equal(blk[l].cpu().numpy(), want[l][2])
        assert kv[l] is None or np.array_equal(f64(kv[l]), want[l][1])
    assert np.array_equal(nxt.cpu().numpy(), want[0][3])


def test_a_commit_past_the_last_block_is_skipped(L):
    B, Hkv, T, cols, mb = 1, 2, 8, 4, 2
    tree = randn(gen(20), B, T, Hkv, 2, 128)
    blk, pool = torch.full((B, Hkv, cols), -1, dtype=torch.int32, device="cuda"), torch.zeros((8, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros((mb, Hkv, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    slot, table = torch.arange(8, dtype=torch.int32, device="cuda").view(B, Hkv, cols), i32([[0, 1]])
    path = torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8)
    L.commit_kv(L.Dims(B, Hkv, Hkv, mb), tree, path, i32([8]), i32([28]), table, slot, blk, 2, pool, kv)
    torch.cuda.synchronize()
    assert torch.equal(kv[1, :, :, 12:], tree[0, :4].permute(1, 2, 0, 3)) and not kv[0].any() and not kv[1, :, :, :12].any()
    assert torch.equal(pool[[3, 7]][:, :, 12:], tree[0, :4].permute(1, 2, 0, 3))


def test_attention_verification_and_commit_in_one_graph(L):
    """Three steps of a loop whose lengths move on the device, replayed from one graph, against the same calls made one by one:
    the kernels overlap each other's ends in either case, and every one has to see what those before it wrote."""
    B, Hq, Hkv, T, V, M, layers, mb, cols = 4, 16, 2, 9, 700, 6, 2, 16, 10
    g, rng = gen(50), np.random.default_rng(50)
    dims, lens = L.Dims(B, Hq, Hkv, mb), [30, 16, 0, 47]
    slot = i32(np.arange(B * Hkv * cols).reshape(B, Hkv, cols).tolist())
    table = i32(rng.permutation(B * mb).reshape(B, mb).tolist())
    q, tree_kv = [randn(g, B, T, Hq, 128) for _ in range(3)], [[randn(g, B, T, Hkv, 2, 128) for _ in range(layers)] for _ in range(3)]
    logits, uniforms = torch.randn((3, B, T, V), generator=g, device="cuda"), torch.rand((3, B, T), generator=g, device="cuda") * 0.02
    temperature, parent, nodes = torch.tensor([0.0, 0.4, 0.7, 1.0], device="cuda"), i32(random_tree(rng, B, T).tolist()), i32([T, 1, T, 5])
    tokens = torch.gather(logits.argmax(-1), 2, parent.long().clamp(min=0).expand(3, B, T)).to(torch.int32)
    init = [(randn(gen(60 + l), B * Hkv * cols, 2, 16, 128), randn(gen(70 + l), B * mb * Hkv, 2, 16, 128)) for l in range(layers)]
    blk0 = torch.full((B, Hkv, cols), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(lens):
        for j in range((n + 15) // 16):
            blk0[b, :, 8 + (j & 1) if j >= n // 16 - 1 else j] = j

    class State:
        def __init__(self):
            self.blk = [blk0.clone() for _ in range(layers)]
            self.pools, self.kvs = [p.clone() for p, _ in init], [k.clone() for _, k in init]
            self.len, self.next = i32(lens), i32([0] * B)
            self.q, self.kv = q[0].clone(), [t.clone() for t in tree_kv[0]]
            self.x, self.u, self.tok = logits[0].clone(), uniforms[0].clone(), tokens[0].clone()
            self.out = [torch.zeros((B, T, Hq, 128), dtype=torch.bfloat16, device="cuda") for _ in range(layers)]
            self.path, self.n, self.token = i32([[0] * M] * B), i32([0] * B), i32([0] * B)
            self.ws = torch.empty(max(16, L.tree_attn_workspace_bytes(dims, T, cols)), dtype=torch.uint8, device="cuda")
            self.plan = L.CommitPlan(dims, self.kv, [table] * layers, [slot] * layers, self.blk, 8, self.pools, self.kvs)

        def load(self, k):
            for mine, new in zip((self.q, self.x, self.u, self.tok, *self.kv), (q[k], logits[k], uniforms[k], tokens[k], *tree_kv[k])):
                mine.copy_(new)

        def step(self):
            for l in range(layers):
                L.tree_attn(dims, self.q, self.kv[l], parent, nodes, self.pools[l], slot, self.blk[l], self.len, SCALE, self.out[l], workspace=self.ws)
            L.verify_tree(self.x, self.tok, parent, nodes, self.u, temperature, self.path, self.n, self.token)
            L.commit_kv_layers(self.plan, self.path, self.n, self.len, next_len=self.next)
            self.len.copy_(self.next)

        def all(self):
            return [*self.out, *self.pools, *self.kvs, *self.blk, self.len, self.path, self.n, self.token]

    eager, other = State(), State()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.step()
    moved = 0
    for k in range(3):
        eager.load(k)
        other.load(k)
        torch.cuda.synchronize()
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.all(), other.all())), k
        ref = ot.verify_tree(f64(logits[k]), tokens[k].cpu().numpy(), parent.cpu().numpy(), nodes.tolist(), uniforms[k].cpu().numpy(), temperature.cpu().numpy(), M)
        assert all(np.array_equal(a.cpu().numpy(), r) for a, r in zip((eager.path, eager.n, eager.token), ref))
        moved += int(eager.n.sum())
    assert eager.len.tolist() != lens and moved == sum(eager.len.tolist()) - sum(lens)


# ---- what the Python layer refuses ---------------------------------------------------------------------------------
def test_wrong_tensors_are_refused(L):
    c = AttnCase(L, 1, 4, 2, 3, [20], [3], 4, seed=30)
    good = dict(dims=c.dims, q=c.q, tree_kv=c.tree_kv, parent=c.d_parent, n_nodes=c.d_nodes, hbm_pool=c.pool, slot_tbl=c.d_slot, blk_tbl=c.d_blk,
                seq_len=c.d_lens, scale=SCALE, out=c.out, lse=c.lse, workspace=c.ws)
    for name, bad, err in (("q", c.q.float(), TypeError), ("q", c.q.cpu(), ValueError), ("tree_kv", c.tree_kv[:, :2], ValueError),
                           ("parent", c.d_parent.long(), TypeError), ("n_nodes", c.d_nodes.repeat(2), ValueError), ("out", c.out[:, :, :2], ValueError),
                           ("seq_len", c.d_lens.cpu(), ValueError), ("slot_tbl", c.d_slot[..., :3], ValueError), ("lse", c.lse.double(), TypeError),
                           ("hbm_pool", c.pool.cpu(), ValueError), ("q", c.q.transpose(1, 2).contiguous().transpose(1, 2), ValueError),
                           ("workspace", c.ws.cpu(), ValueError)):
        with pytest.raises(err):
            L.tree_attn(**{**good, name: bad})
    with pytest.raises(L.OasisError, match="scale"):
        L.tree_attn(**{**good, "scale": 0.0})
    x, u = torch.zeros((2, 3, 10), device="cuda"), torch.zeros((2, 3), device="cuda")
    z, n = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    good = dict(logits=x, tokens=z, parent=z, n_nodes=n, uniforms=u, temperature=u[:, 0].contiguous(), path=z, n_commit=n, next_token=n)
    for name, bad, err in (("logits", x.double(), TypeError), ("logits", x[0], ValueError), ("logits", x.cpu(), ValueError),
                           ("logits", x.transpose(1, 2).contiguous().transpose(1, 2), ValueError), ("uniforms", u.double(), TypeError),
                           ("temperature", u[:, 0], ValueError), ("tokens", z.long(), TypeError), ("logits", x[:, :1].expand(2, 3, 10), ValueError)):
        with pytest.raises(err):
            L.verify_tree(**{**good, name: bad})
    with pytest.raises(TypeError):
        L.verify_tree(**good, draft_probs=x.half())
    for name, bad, err in (("path", z[0], ValueError), ("path", z.long(), TypeError), ("n_commit", n[:1], ValueError), ("next_token", [1, 2], TypeError),
                           ("n_nodes", n.cpu(), ValueError), ("draft_probs", x[:, :, :5], ValueError), ("draft_probs", x.cpu(), ValueError)):
        with pytest.raises(err):
            L.verify_tree(**{**good, name: bad})
    dims, bf = L.Dims(2, 4, 2, 4), dict(dtype=torch.bfloat16, device="cuda")
    kv, pool, host = torch.zeros((2, 3, 2, 2, 128), **bf), torch.zeros((20, 2, 16, 128), **bf), torch.zeros((8, 2, 2, 16, 128), dtype=torch.bfloat16)
    table, cols = torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.zeros((2, 2, 4), dtype=torch.int32, device="cuda")
    plan = dict(dims=dims, tree_kvs=[kv], block_tables=[table], slot_tbls=[cols], blk_tbls=[cols.clone()], local_col=2, hbm_pools=[pool])
    for name, bad, err in (("tree_kvs", kv.float(), TypeError), ("tree_kvs", kv.cpu(), ValueError), ("block_tables", table[:, :2], ValueError),
                           ("slot_tbls", cols.long(), TypeError), ("hbm_pools", pool[:, :, :8], ValueError), ("host_kvs", host, ValueError)):
        with pytest.raises(err):
            L.CommitPlan(**{**plan, name: [bad]})
    layers = [kv]
    plan = L.CommitPlan(**{**plan, "tree_kvs": layers})
    layers.clear()                                                    # (the plan holds the tensors, not the list)
    assert plan._held[0][0] is kv
    good = dict(path=z, n_commit=n, seq_len=n.clone(), next_len=n.clone())
    for name, bad, err in (("path", z[0], ValueError), ("path", z.float(), TypeError), ("n_commit", n.cpu(), ValueError), ("seq_len", n.repeat(2), ValueError),
                           ("next_len", n.long(), TypeError)):
        with pytest.raises(err):
            L.commit_kv_layers(plan, **{**good, name: bad})
    with pytest.raises(L.OasisError, match="share memory"):
        L.commit_kv_layers(plan, z, n, good["seq_len"], next_len=good["seq_len"])


def test_empty_batches_do_nothing(L):
    e = lambda *shape, dt=torch.int32: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
    bf = torch.bfloat16
    L.tree_attn(L.Dims(0, 8, 2, 4), e(0, 3, 8, 128, dt=bf), e(0, 3, 2, 2, 128, dt=bf), e(0, 3), e(0), e(1, 2, 16, 128, dt=bf), e(0, 2, 4), e(0, 2, 4),
                e(0), SCALE, e(0, 3, 8, 128, dt=bf))
    L.verify_tree(e(0, 3, 9, dt=torch.float32), e(0, 3), e(0, 3), e(0), e(0, 3, dt=torch.float32), e(0, dt=torch.float32), e(0, 2), e(0), e(0))
    L.commit_kv(L.Dims(0, 8, 2, 4), e(0, 3, 2, 2, 128, dt=bf), e(0, 3), e(0), e(0), e(0, 4), e(0, 2, 4), e(0, 2, 4), 2, e(1, 2, 16, 128, dt=bf))


def test_bounds_check_build(L):
    """In a process of its own, because a process loads one build of the library."""
    import json
    import os
    import subprocess
    import sys
    from paper_2608_08097_b200 import build
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "tests", "tree_checked_worker.py")], capture_output=True, text=True, timeout=600,
                       env=dict(os.environ, OASIS_LIB=build.build(checked=True)))
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert json.loads(r.stdout.strip().splitlines()[-1])["ok"]


# ---- together ------------------------------------------------------------------------------------------------------
def test_a_decode_loop_with_draft_trees(L):
    """Steps of an engine with draft trees: attention of every layer, verification, commit; then the next step on the
    longer history.  The budget covers every block, so the attention has to be dense causal attention over the tokens
    that were kept, whichever path through summaries, top-k, plan, gather and local window their keys took."""
    from paper_2608_08097_b200 import pipeline
    B, Hq, Hkv, T, layers, V, mb, k = 3, 8, 2, 13, 2, 501, 16, 16
    g, rng = gen(40), np.random.default_rng(40)
    lens = [37, 16, 95]
    eng = pipeline.DecodeEngine(B, Hq, Hkv, mb, k, T, layers, mode="delta", cap=k, append=True, tree=True)
    hist = [[randn(g, lens[b], Hkv, 2, 128) for b in range(B)] for _ in range(layers)]          # the truth: [tokens][Hkv][2][128]
    for l in range(layers):
        kv = torch.zeros((B * mb, Hkv, 2, 16, 128), dtype=torch.bfloat16)
        table = torch.tensor(rng.permutation(B * mb).reshape(B, mb), dtype=torch.int32)
        for b in range(B):
            for pos in range(lens[b]):
                kv[table[b, pos // 16], :, :, pos % 16] = hist[l][b][pos].cpu()
        eng.attach(l, kv.pin_memory(), table.cuda())
    seq = i32(lens)
    q = [randn(g, B, T, Hq, 128) for _ in range(layers)]
    eng.prime(q, seq // 16, seq)
    nxt_len = torch.zeros_like(seq)
    path, n, token = torch.zeros((B, T), dtype=torch.int32, device="cuda"), torch.zeros_like(seq), torch.zeros_like(seq)
    before = seq // 16
    kept = []
    for step in range(5):
        q = [randn(g, B, T, Hq, 128) for _ in range(layers)]
        tree_kv = [randn(g, B, T, Hkv, 2, 128) for _ in range(layers)]
        parent = random_tree(rng, B, T)
        parent[:, 1:] = np.maximum(parent[:, 1:], 0)
        nodes = [T, 1, 7] if step % 2 else [9, T, T]
        d_parent, d_nodes = i32(parent.tolist()), i32(nodes)
        full = seq // 16
        torch.cuda.synchronize()
        eng.step(q, seq, before, full - before, full, seq, step_stamp=step + 1, new_kv=tree_kv, tree=(d_parent, d_nodes))
        before = full
        eng.join()
        torch.cuda.current_stream().wait_stream(eng.main)
        x = torch.randn((B, T, V), generator=g, device="cuda")
        at = d_parent.long().clamp(min=0)
        tokens = torch.gather(x.argmax(-1), 1, at).to(torch.int32)                               # likely drafts
        u = torch.rand((B, T), generator=g, device="cuda") * 0.05
        temp = torch.tensor([0.0, 0.3, 0.5], device="cuda")
        L.verify_tree(x, tokens, d_parent, d_nodes, u, temp, path, n, token)
        eng.commit(eng.commit_plan(tree_kv), path, n, seq, next_len=nxt_len)
        torch.cuda.synchronize()
        ref = ot.verify_tree(f64(x), tokens.cpu().numpy(), parent, nodes, u.cpu().numpy(), temp.cpu().numpy(), T)
        assert all(np.array_equal(a.cpu().numpy(), r) for a, r in zip((path, n, token), ref))
        for l in range(layers):
            out = f64(eng.layers[l].out)
            for b in range(B):
                H = f64(hist[l][b])
                for t in range(nodes[b]):
                    rows = np.concatenate([H, f64(tree_kv[l][b])[ot.ancestors(parent[b], t)]])
                    for a in range(Hq):
                        K, W = rows[:, a // (Hq // Hkv), 0], rows[:, a // (Hq // Hkv), 1]
                        z = K @ f64(q[l][b, t, a]) * SCALE
                        w = np.exp(z - z.max())
                        w /= w.sum()
                        want, amount = w @ W, w @ np.abs(W)
                        assert np.all(np.abs(out[b, t, a] - want) <= 2 ** -8 * (amount + np.abs(want)) + 6e-4 * amount), (step, l, b, t, a)
                keep = path[b, :int(n[b])].long()
                hist[l][b] = torch.cat([hist[l][b], tree_kv[l][b][keep]])
        kept += n.tolist()
        lens = [lens[b] + int(n[b]) for b in range(B)]
        assert nxt_len.tolist() == lens
        seq = nxt_len.clone()
    assert max(kept) > 2 and min(kept) >= 1
