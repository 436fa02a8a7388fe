"""GPU tests of the packed cache through the C ABI, against the numpy oracle in double precision.

Packing, unpacking and the gather are exact: bytes have to be equal.  Tolerances of the attention, per element, with
A = sum_k w_k |v_k| and Z = the row's largest sum |q k| * scale (both from the oracle):
  the softmax weights reach the tensor core as bf16 (half a step: 2^-8 relative)      2^-8 A
  the output is rounded to bf16                                                       2^-8 |out|
  a logit is a sum of 128 exact products in fp32 (off by at most 128 * 2^-23 Z) and is scaled, subtracted from and
  exponentiated in fp32 (a few 2^-23 of |logit| <= Z): E = 2^-15 Z; a weight relative to the others twice that  2 E A
The log-sum-exp is off by E and by the fp32 sum and logarithm: E + 1e-5 * (1 + |lse|)."""
import math

import numpy as np
import pytest
import torch

from oracle import packed as op

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


# ---- packing ---------------------------------------------------------------------------------------------------------
def odd_entries(g, n):
    """Random entries of different sizes, among them zeros, halfway cases, NaN, infinities and the far ends of the scales."""
    kv = randn(g, n, 2, 16, 128) * torch.exp2(torch.randint(-24, 14, (n, 1, 1, 1), generator=g, device="cuda").float()).to(torch.bfloat16)
    if n >= 6:
        kv[0] = 0
        whole = torch.randint(-15, 16, (2, 16, 128), generator=g, device="cuda").float() / 2    # multiples of 1/2 up to 7.5
        kv[1] = whole.to(torch.bfloat16)
        kv[1, 0, :, ::16], kv[1, 1, 0] = 7.0, 7.0                                               # .. against a scale of 1 (or 1.125)
        kv[2, :, 3, 5:40] = float("nan")
        kv[3, :, 2::5, 7::9] = float("inf")
        kv[4, :, 1::5, 3::7] = float("-inf")
        kv[4, 0, 7] = float("nan")
        kv[5] = 3e38
    return kv


@pytest.mark.parametrize("B, Hkv, counts, host", [(1, 1, [1], False), (3, 3, [4, 0, 2], False), (2, 8, [1, 3], True)])
def test_pack_blocks_writes_the_oracles_bytes_and_nothing_else(L, B, Hkv, counts, host):
    g, rng = gen(B), np.random.default_rng(B)
    mb, pages = 9, 17 * B
    pool = odd_entries(g, pages * Hkv).view(pages, Hkv, 2, 16, 128)
    src, dst = (rng.permutation(pages)[:B * 8].reshape(B, 8) for _ in range(2))
    src, dst = (np.concatenate([t, np.full((B, 1), 10 ** 6)], 1).astype(np.int32) for t in (src, dst))    # the last column is never asked for
    first = [2, 0, 5][:B]
    packed = torch.full((pages * Hkv, 2304), 171, dtype=torch.uint8, device="cpu" if host else "cuda")
    packed = packed.pin_memory() if host else packed
    summ = torch.full((B, Hkv, mb, 2, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    want_summ, dims = summ.clone(), L.Dims(B, 4 * Hkv, Hkv, mb)
    L.pack_blocks(dims, pool, i32(src.tolist()), i32(first), i32(counts), 4, packed, i32(dst.tolist()), summaries=summ)
    L.build_summaries(dims, pool, i32(src.tolist()), i32(first), i32(counts), 4, want_summ)
    torch.cuda.synchronize()
    want = np.full((pages * Hkv, 2304), 171, np.uint8)
    for b in range(B):
        for j in range(first[b], first[b] + counts[b]):
            for h in range(Hkv):
                want[dst[b, j] * Hkv + h] = op.pack(f64(pool[src[b, j], h]))
    assert np.array_equal(packed.cpu().numpy(), want)
    assert torch.equal(summ.view(torch.int16), want_summ.view(torch.int16))


def test_packing_is_bounded_by_the_block_array_and_by_max_new_blocks(L):
    pool = randn(gen(1), 8, 1, 2, 16, 128)
    table = i32([[0, 1, 2, 3]])
    dims = L.Dims(1, 1, 1, 4)
    for first, n, most, done in ((3, 5, 4, [3]), (-2, 4, 4, [0, 1]), (0, 4, 2, [0, 1]), (4, 1, 4, []), (0, -3, 4, [])):
        packed = torch.zeros((8, 2304), dtype=torch.uint8, device="cuda")
        L.pack_blocks(dims, pool, table, i32([first]), i32([n]), most, packed, table)
        got = packed.cpu().numpy()
        assert [j for j in range(8) if got[j].any()] == done
        for j in done:
            assert np.array_equal(got[j], op.pack(f64(pool[j, 0])))


def test_far_entries_and_pages_read_twice(L):
    """Entries whose offsets pass 32 bits, in both pools; one source page packed to two places, one packed entry read back twice."""
    n, m = (1 << 32) // 8192 + 7, (1 << 32) // 2304 + 9
    few = odd_entries(gen(2), 6)
    pool = torch.empty((n, 1, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    packed = torch.empty((m, 2304), dtype=torch.uint8, device="cuda")
    pool[n - 6:, 0] = few
    L.pack_blocks(L.Dims(1, 1, 1, 4), pool, i32([[n - 1, n - 3, n - 3, n - 5]]), i32([0]), i32([4]), 4, packed, i32([[m - 1, m - 4, 2, 0]]))
    out = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    L.unpack_blocks(packed, torch.tensor([m - 1, m - 4, m - 4, 2], device="cuda"), out)
    want = [op.pack(f64(few[k])) for k in (5, 3, 3, 1)]
    for at, w in zip((m - 1, m - 4, 2, 0), want):
        assert np.array_equal(packed[at].cpu().numpy(), w)
    got = out.view(torch.int16)
    assert torch.equal(got[1], got[2]) and torch.equal(got[1], got[3])
    again = torch.zeros((4, 2304), dtype=torch.uint8, device="cuda")
    L.pack_blocks(L.Dims(1, 1, 1, 4), out.view(4, 1, 2, 16, 128), i32([[0, 1, 2, 3]]), i32([0]), i32([4]), 4, again, i32([[0, 1, 2, 3]]))
    assert [np.array_equal(op.unpack(again[k].cpu().numpy()), f64(out[k])) for k in range(4)] == [True] * 4


@pytest.mark.parametrize("layers", [1, 3])
def test_pack_local_takes_the_column_of_the_blocks_parity(L, layers):
    B, Hkv, cols, col, mb, g, rng = 3, 2, 7, 4, 12, gen(9), np.random.default_rng(9)
    dims = L.Dims(B, 4, Hkv, mb)
    first, counts = [4, 7, 0], [1, 2, 0]
    pools = [odd_entries(g, B * Hkv * cols) for _ in range(layers)]
    slots = [rng.permutation(B * Hkv * cols).reshape(B, Hkv, cols).astype(np.int32) for _ in range(layers)]
    slots[0][1, 1, col + 1] = -1                                              # no entry there: skipped
    tables = [rng.permutation(B * mb).reshape(B, mb).astype(np.int32) for _ in range(layers)]
    packed = [torch.zeros((B * mb * Hkv, 2304), dtype=torch.uint8).pin_memory() if l % 2 else torch.zeros((B * mb * Hkv, 2304), dtype=torch.uint8, device="cuda")
              for l in range(layers)]
    summ = [torch.zeros((B, Hkv, mb, 2, 128), dtype=torch.bfloat16, device="cuda") if l != 1 else None for l in range(layers)]
    L.pack_local_layers(dims, pools, [i32(s.tolist()) for s in slots], col, i32(first), i32(counts), 2, packed, [i32(t.tolist()) for t in tables], summ)
    torch.cuda.synchronize()
    for l in range(layers):
        want, want_summ = np.zeros((B * mb * Hkv, 2304), np.uint8), torch.zeros((B, Hkv, mb, 2, 128), dtype=torch.bfloat16, device="cuda")
        for b in range(B):
            for j in range(first[b], first[b] + counts[b]):
                for h in range(Hkv):
                    s = int(slots[l][b, h, col + j % 2])
                    if s < 0:
                        continue
                    want[tables[l][b, j] * Hkv + h] = op.pack(f64(pools[l][s]))
                    fine = torch.nan_to_num(pools[l][s, 0].float(), nan=-math.inf, posinf=math.inf, neginf=-math.inf).amax(0)
                    want_summ[b, h, j, 1] = fine.to(torch.bfloat16)
                    want_summ[b, h, j, 0] = torch.nan_to_num(pools[l][s, 0].float(), nan=math.inf, posinf=math.inf, neginf=-math.inf).amin(0).to(torch.bfloat16)
        assert np.array_equal(packed[l].cpu().numpy(), want)
        if summ[l] is not None:
            assert torch.equal(summ[l].float(), want_summ.float())


def test_hand_over_from_a_dense_pool(L):
    B, Hkv, mb, P = 2, 3, 6, 20
    g, rng = gen(4), np.random.default_rng(4)
    kv = randn(g, P, Hkv, 2, 16, 128)
    k, v = kv[:, :, 0].contiguous(), kv[:, :, 1].contiguous()
    gpu, dst = (rng.permutation(P)[:B * mb].reshape(B, mb).astype(np.int32) for _ in range(2))
    dims, first, counts = L.Dims(B, 6, Hkv, mb), [0, 2], [6, 3]
    packed, summ = torch.zeros((P * Hkv, 2304), dtype=torch.uint8, device="cuda"), torch.zeros((B, Hkv, mb, 2, 128), dtype=torch.bfloat16, device="cuda")
    L.offload_blocks_packed(dims, k, v, i32(gpu.tolist()), i32(dst.tolist()), i32(first), i32(counts), mb, packed, summ)
    again, summ2 = torch.zeros_like(packed), torch.zeros_like(summ)
    L.pack_blocks(dims, kv, i32(gpu.tolist()), i32(first), i32(counts), mb, again, i32(dst.tolist()), summaries=summ2)
    assert torch.equal(packed, again) and torch.equal(summ, summ2)
    assert np.array_equal(packed[int(dst[1, 3]) * Hkv + 2].cpu().numpy(), op.pack(f64(kv[int(gpu[1, 3]), 2])))


@pytest.mark.parametrize("host", [False, True])
def test_unpack_and_gather(L, host):
    rng, n = np.random.default_rng(7), 37
    packed = torch.tensor(rng.integers(0, 256, (50, 2304), dtype=np.uint8))                 # any bytes are an entry
    packed = packed.pin_memory() if host else packed.cuda()
    idx = rng.integers(0, 50, n)
    idx[[3, 20]] = -1
    out = torch.full((n, 2, 16, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    L.unpack_blocks(packed, torch.tensor(idx, device="cuda"), out)
    want = op.unpack(packed.cpu().numpy()[idx])
    want[idx < 0] = 5.0
    assert np.array_equal(f64(out), want)
    for layers, m, ctas in ((1, n, 0), (3, 5, 0), (2, n, 1), (1, 1, 0)):
        pools = [torch.full((60, 2304), 9, dtype=torch.uint8, device="cuda") for _ in range(layers)]
        ids = [rng.integers(-1, 50, m) for _ in range(layers)]
        slots = [rng.permutation(60)[:m].astype(np.int32) for _ in range(layers)]
        L.stage_packed_layers([packed] * layers, [torch.tensor(i, device="cuda") for i in ids], [i32(s.tolist()) for s in slots], m, pools, max_ctas=ctas)
        torch.cuda.synchronize()
        for l in range(layers):
            ref = np.full((60, 2304), 9, np.uint8)
            ref[slots[l][ids[l] >= 0]] = packed.cpu().numpy()[ids[l][ids[l] >= 0]]
            assert np.array_equal(pools[l].cpu().numpy(), ref)


# ---- attention -------------------------------------------------------------------------------------------------------
class Case:
    """Rows with `budget` packed columns (random full blocks, holes among them), `near` bf16 columns, shuffled slots; NaN,
    infinities and huge values in the bf16 entries wherever no token of the request may look, random bytes in unused packed entries."""

    def __init__(self, L, B, Hq, Hkv, T, lens, budget, near=2, seed=0, size=1.0, ahead=False):
        rng, g = np.random.default_rng(seed), gen(seed)
        cols, self.budget, self.T, self.lens = budget + near, budget, T, np.array(lens)
        self.dims = L.Dims(B, Hq, Hkv, (max(lens) + T) // 16 + 3)
        self.slot = np.concatenate([rng.permutation(B * Hkv * budget + 3)[:B * Hkv * budget].reshape(B, Hkv, budget),
                                    rng.permutation(B * Hkv * near + 1)[:B * Hkv * near].reshape(B, Hkv, near)], 2).astype(np.int32)
        self.blk = np.full((B, Hkv, cols), -1, np.int32)
        self.local = randn(g, B * Hkv * near + 1, 2, 16, 128)
        self.packed = torch.randint(0, 256, (B * Hkv * budget + 3, 2304), generator=g, device="cuda", dtype=torch.int16).to(torch.uint8)
        kv = (randn(g, B * Hkv * budget, 2, 16, 128) * size).contiguous()
        if budget:
            at = i32(self.slot[:, :, :budget].reshape(1, -1).tolist())
            L.pack_blocks(L.Dims(1, 1, 1, at.numel()), kv, i32([list(range(at.numel()))]), i32([0]), i32([at.numel()]), at.numel(), self.packed, at)
        for b in range(B):
            last = lens[b] + T - 1
            full = lens[b] // 16 if not ahead else last // 16 + 1          # ahead: blocks that begin after the first token are packed too
            for h in range(Hkv):
                k = min(budget, full)
                self.blk[b, h, rng.permutation(budget)[:k]] = rng.permutation(full)[:k]
                if not ahead:
                    for j in range(full, last // 16 + 1):
                        if near and j - full < near:
                            self.blk[b, h, budget + (j % 2 if near == 2 else j - full)] = j
                if budget > k:
                    self.blk[b, h, np.nonzero(self.blk[b, h, :budget] < 0)[0][:1]] = last // 16 + 2    # a block past the end
                for c in range(budget, cols):
                    n = 0 if self.blk[b, h, c] < 0 else max(0, min(16, last + 1 - 16 * self.blk[b, h, c]))
                    self.local[self.slot[b, h, c], :, n:] = float(rng.choice([np.nan, np.inf, -np.inf, 3e38]))
        self.q = randn(g, B, T, Hq, 128) * 2
        self.d_slot, self.d_blk, self.d_lens = i32(self.slot.tolist()), i32(self.blk.tolist()), i32(list(lens))
        self.need = L.packed_attn_workspace_bytes(self.dims, T, cols, budget)
        self.ws = torch.full((max(self.need, 16),), 255, dtype=torch.uint8, device="cuda")                # NaN patterns
        self.fresh()

    def fresh(self):
        self.out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full(self.q.shape[:3], 7.0, device="cuda")

    def run(self, L, stream=None, lse=True, ws=None, out=None):
        L.packed_attn(self.dims, self.q, self.packed, self.local, self.d_slot, self.d_blk, self.budget, self.d_lens, SCALE,
                      self.out if out is None else out, lse=self.lse if lse else None, workspace=self.ws if ws is None else ws, stream=stream)

    def check(self):
        local = np.nan_to_num(f64(self.local), nan=0.0, posinf=0.0, neginf=0.0)
        out, lse, a, big = op.attn(f64(self.q), self.packed.cpu().numpy(), local, self.slot, self.blk, self.budget, self.lens, SCALE)
        got, got_lse = f64(self.out), f64(self.lse)
        e = 2.0 ** -15 * big
        assert np.isfinite(got).all()
        off = np.abs(got - out) - (2.0 ** -8 * (a + np.abs(out)) + 2 * e[..., None] * a)
        assert off.max() <= 0, (np.abs(got - out).max(), off.max())
        dead = np.isneginf(lse)
        assert np.array_equal(dead, np.isneginf(got_lse)) and not got[dead].any()
        assert np.all(np.abs(got_lse[~dead] - lse[~dead]) <= e[~dead] + 1e-5 * (1 + np.abs(lse[~dead])))


SHAPES = [  # B, Hq, Hkv, T, lengths, packed columns
    (1, 1, 1, 1, [0], 1), (1, 4, 1, 1, [1], 4), (1, 8, 2, 1, [15], 8), (1, 8, 2, 1, [16], 8), (2, 8, 2, 1, [17, 160], 8),
    (1, 32, 8, 1, [200], 16), (3, 32, 8, 5, [700, 0, 33], 43), (2, 16, 4, 16, [1000, 999], 64), (2, 24, 8, 2, [130, 2000], 125),
    (1, 16, 1, 1, [3000], 190), (1, 17, 1, 1, [500], 30), (2, 32, 1, 1, [64, 4000], 250), (1, 33, 1, 1, [800], 50),
    (1, 64, 1, 1, [900], 57), (1, 65, 1, 1, [900], 57), (2, 32, 4, 9, [2000, 77], 100), (1, 128, 1, 1, [1234], 70), (1, 16, 1, 8, [640], 41),
    (1, 40, 8, 3, [9000], 561), (40, 8, 4, 1, list(range(0, 400, 10)), 25), (70, 32, 8, 2, list(range(1, 701, 10)), 20),
    (1, 4, 4, 1, [20000], 1251), (160, 4, 4, 1, [48 + 5 * i for i in range(160)], 70),
]


@pytest.mark.parametrize("B, Hq, Hkv, T, lens, budget", SHAPES)
def test_attention_matches_the_oracle(L, B, Hq, Hkv, T, lens, budget):
    c = Case(L, B, Hq, Hkv, T, lens, budget, seed=B * 1000 + Hq + T)
    c.run(L)
    c.check()


@pytest.mark.parametrize("near, T, lens", [(0, 1, [160, 96]), (1, 1, [165, 7]), (5, 64, [100, 0]), (8, 128, [37, 12]), (2, 128, [16, 31])])
def test_no_or_many_local_columns(L, near, T, lens):
    c = Case(L, 2, 3 if T == 1 else 1, 1, T, lens, 10, near=near, seed=near)
    c.run(L)
    c.check()


def test_only_local_columns(L):
    c = Case(L, 3, 8, 2, 5, [0, 9, 13], 0)
    L.packed_attn(c.dims, c.q, None, c.local, c.d_slot, c.d_blk, 0, c.d_lens, SCALE, c.out, lse=c.lse, workspace=c.ws)
    c.check()


def test_packed_blocks_that_only_later_tokens_see(L):
    """Blocks at and past the first token's position among the packed columns: the causal border runs through them."""
    for T, lens in ((1, [0, 15, 16]), (16, [3, 40, 64]), (40, [0, 100, 5])):
        c = Case(L, 3, 2, 1, T, lens, 12, seed=T, ahead=True)
        c.run(L)
        c.check()


def test_rows_without_any_key(L):
    for budget in (1, 20, 600):                          # alone, in a cluster, through the workspace
        c = Case(L, 2, 8, 2, 3, [300, 300], budget, seed=budget)
        c.blk[1] = -1
        c.blk[0, 1, :budget] = -1
        c.d_blk = i32(c.blk.tolist())
        c.run(L)
        c.check()
        assert np.isneginf(f64(c.lse)[1]).all() and not f64(c.out)[1].any()


def test_requests_before_their_first_token(L):
    """A negative length hides everything that lies past it."""
    c = Case(L, 2, 4, 2, 2, [50, 50], 6, seed=3)
    c.lens = np.array([50, -40])
    c.d_lens = i32([50, -40])
    c.run(L)
    c.check()


@pytest.mark.parametrize("size", [1e-3, 30.0])
def test_small_and_large_keys(L, size):
    """Logits that hardly differ, and logits far apart, which raise the reference maximum again and again."""
    c = Case(L, 2, 8, 2, 2, [3000, 1500], 190, seed=11, size=size)
    c.run(L)
    c.check()


def test_rising_logits_rescale_in_every_tile(L):
    """Keys that grow from block to block: every tile has a new maximum, far above the last one's."""
    B, Hq, Hkv, T, n = 1, 4, 1, 1, 64
    c = Case(L, B, Hq, Hkv, T, [n * 16], n, seed=2)
    kv = randn(gen(5), n, 2, 16, 128)
    kv[:, 0] = (c.q[0, 0, 0] * 0.05).to(torch.bfloat16) * torch.arange(1, n + 1, device="cuda")[:, None, None].to(torch.bfloat16)
    c.blk[0, 0, :n] = np.arange(n)
    c.d_blk = i32(c.blk.tolist())
    at = i32(c.slot[:, :, :n].reshape(1, -1).tolist())
    L.pack_blocks(L.Dims(1, 1, 1, n), kv, i32([list(range(n))]), i32([0]), i32([n]), n, c.packed, at)
    c.run(L)
    c.check()


@pytest.mark.parametrize("T, Hq", [(1, 4), (9, 8)])
def test_values_near_the_end_of_the_range(L, T, Hq):
    """Local values of 10^38 beside packed ones: neither weights nor sums may carry them past it."""
    c = Case(L, 1, Hq, 1, T, [333], 20, seed=8)
    for col in (20, 21):
        j = int(c.blk[0, 0, col])
        if j >= 0:
            seen = min(16, 333 + T - 16 * j)
            c.local[int(c.slot[0, 0, col]), 1, :seen] = torch.sign(c.local[int(c.slot[0, 0, col]), 1, :seen]) * 1e38
    c.run(L)
    c.check()


def test_any_bytes_are_finite(L):
    """Entries of random bytes: code 0 (-8) and the largest scales among them."""
    c = Case(L, 1, 4, 1, 1, [320], 20, seed=4)
    c.packed[:, :2048] = torch.randint(0, 256, c.packed[:, :2048].shape, device="cuda", dtype=torch.int16, generator=gen(1)).to(torch.uint8)
    c.packed[:, 2048:] = torch.randint(130, 176, c.packed[:, 2048:].shape, device="cuda", dtype=torch.int16, generator=gen(2)).to(torch.uint8)
    c.run(L)
    c.check()
    c.packed[:, 2048:] = 255                             # logits of 10^6: weights of 0 and 1
    c.q *= 0.001
    c.run(L)
    c.check()


def test_shared_slots_and_far_slots(L):
    """Two columns of one slot, and slots whose offset passes 32 bits."""
    n = (1 << 32) // 2304 + 9
    c = Case(L, 1, 8, 2, 1, [160], 10, seed=6)
    c.slot[0, 0, 3] = c.slot[0, 0, 4]
    near, c.packed = c.packed, torch.zeros((n, 2304), dtype=torch.uint8, device="cuda")
    c.packed[n - 20:] = near[:20]                        # slots below 20 move to the end, the others stay
    c.packed[20:23] = near[20:23]
    few = c.slot.copy()
    c.slot[:, :, :10] += np.where(few[:, :, :10] < 20, n - 20, 0).astype(np.int32)
    c.d_slot = i32(c.slot.tolist())
    c.run(L)
    c.packed, c.slot = near, few
    c.check()


@pytest.mark.parametrize("B, T, budget", [(1, 1, 16), (4, 5, 128), (1, 1, 1200), (2, 16, 300)])
def test_results_do_not_depend_on_the_run_stream_or_graph(L, B, T, budget):
    c = Case(L, B, 16, 4, T, [budget * 16 + 3 * i for i in range(B)], budget, seed=budget)
    c.run(L)
    want, want_lse = c.out.clone(), c.lse.clone()
    for _ in range(3):
        c.fresh()
        c.ws.fill_(255)
        c.run(L, lse=False)
        assert torch.equal(c.out, want) and bool((c.lse == 7.0).all())
    c.fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(L, stream=side)
    side.synchronize()
    assert torch.equal(c.out, want) and torch.equal(c.lse, want_lse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run(L)
    for k in range(3):                                   # new queries and lengths in place
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
        c.q.copy_(torch.roll(c.q, 1, 2))
        c.lens = np.maximum(c.lens - 7 * k, 0)
        c.d_lens.copy_(i32(c.lens.tolist()))
        g.replay()
        c.check()


@pytest.mark.parametrize("T, Hq", [(1, 4), (2, 16), (3, 16), (4, 16), (9, 8), (10, 16), (16, 16)])
def test_a_key_that_decides_the_output(L, T, Hq):
    """All queries of a head look for one late key, so its value is the output: off by half a step of bf16, not by its weight's rounding.
    (The weight is no power of two: the reference comes from earlier keys.)"""
    c = Case(L, 2, Hq, 2, T, [1999, 1500], 124, seed=Hq + T)
    key = np.zeros((2, 2, 128))
    for b in range(2):
        for h in range(2):
            at = max(j for j in range(c.budget) if 0 <= c.blk[b, h, j] and 16 * c.blk[b, h, j] + 15 <= c.lens[b])
            entry = torch.zeros(1, 2, 16, 128, dtype=torch.bfloat16, device="cuda")
            L.unpack_blocks(c.packed, torch.tensor([int(c.slot[b, h, at])], device="cuda"), entry)
            key[b, h] = f64(entry[0, 0, 5 + b])
            rows = torch.linspace(1.5, 1.9, T * Hq // 2, device="cuda").view(T, Hq // 2, 1)
            c.q[b, :, h * Hq // 2:(h + 1) * Hq // 2] = (rows * entry[0, 0, 5 + b].float()).to(torch.bfloat16)
    c.run(L)
    out, lse, _, _ = op.attn(f64(c.q), c.packed.cpu().numpy(), np.nan_to_num(f64(c.local), nan=0.0, posinf=0.0, neginf=0.0), c.slot, c.blk, c.budget, c.lens, SCALE)
    others = 1 - np.exp(SCALE * np.einsum("bthd,bhd->bth", f64(c.q), np.repeat(key, Hq // 2, axis=1)) - lse)       # their share of the weights
    assert others.max() < 0.01
    # half a step is 2^-8 of the value; a weight that is 2^-8 off moves the output by that times the others' share of the difference of
    # two values (at most about 10); fp32 adds 2^-20 of a value
    assert np.all(np.abs(f64(c.out) - out) <= 2.0 ** -8 * np.abs(out) + (2.0 ** -8 * 10 * others + 2.0 ** -17)[..., None])
    assert np.all(np.abs(f64(c.lse) - lse) <= 1e-5 * (1 + np.abs(lse)))


@pytest.mark.parametrize("B, T, Hq, lens, budget", [(2, 1, 8, [40, 700], 12), (2, 3, 8, [900, 900], 130), (1, 9, 16, [900], 56), (1, 1, 8, [9600], 600), (1, 20, 8, [40000], 2500)])
def test_a_query_that_is_no_number_stays_alone(L, B, T, Hq, lens, budget):
    """NaN in one query row: its output and sum are NaN, every other row is what it was."""
    c = Case(L, B, Hq, 2, T, lens, budget, seed=T)
    c.run(L)
    want, want_lse = c.out.clone(), c.lse.clone()
    c.q[B - 1, T - 1, 3, 77] = float("nan")
    c.fresh()
    c.run(L)
    assert bool(c.out[B - 1, T - 1, 3].isnan().all()) and bool(c.lse[B - 1, T - 1, 3].isnan())
    c.out[B - 1, T - 1, 3], c.lse[B - 1, T - 1, 3] = want[B - 1, T - 1, 3], want_lse[B - 1, T - 1, 3]
    assert torch.equal(c.out, want) and torch.equal(c.lse, want_lse)


@pytest.mark.parametrize("shapes", [((1, 1, 1200), (16, 1, 130)), ((4, 9, 300), (2, 5, 600))])
def test_two_calls_at_once(L, shapes):
    """On two streams, and as two graphs that are replayed together, each with its own workspace."""
    cases = [Case(L, B, 16, 2, T, [budget * 16] * B, budget, seed=budget) for B, T, budget in shapes]
    streams, graphs, want = [torch.cuda.Stream() for _ in cases], [], []
    for c in cases:
        c.run(L)
        c.check()
        want.append((c.out.clone(), c.lse.clone()))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(4):
                c.run(L)
        graphs.append(g)
    for replay in (False, True):
        for c in cases:
            c.out.fill_(7.0)
            c.lse.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(20):
            for c, s, g in zip(cases, streams, graphs):
                with torch.cuda.stream(s):
                    g.replay() if replay else c.run(L)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert torch.equal(c.out, w[0]) and torch.equal(c.lse, w[1])


def test_back_to_back_calls_share_a_workspace_in_order(L):
    a, b = Case(L, 1, 8, 2, 1, [9600], 600, seed=1), Case(L, 1, 8, 2, 1, [9000], 600, seed=2)
    assert a.need == b.need > 0
    for _ in range(4):
        a.fresh()
        b.fresh()
        a.run(L)
        b.run(L, ws=a.ws)
        a.run(L)
        a.check()
        b.check()


def test_refusals(L):
    c = Case(L, 1, 8, 2, 2, [9600], 600, seed=1)
    good = [c.dims, c.q, c.packed, c.local, c.d_slot, c.d_blk, 600, c.d_lens, SCALE, c.out]
    kw = dict(lse=c.lse, workspace=c.ws)

    def call(i, v, **k):
        a = list(good)
        a[i] = v
        L.packed_attn(*a, **{**kw, **k})
    for i, v, e in ((1, c.q.float(), TypeError), (1, c.q[0], ValueError), (1, c.q.cpu(), ValueError), (1, c.q.transpose(0, 1), ValueError),
                    (2, c.packed.view(torch.int8), TypeError), (2, c.packed[:, :2048], ValueError), (2, c.packed.cpu(), ValueError),
                    (3, c.local.float(), TypeError), (4, c.d_slot.long(), TypeError), (4, c.d_slot[:, :, 1:].contiguous(), ValueError),
                    (5, c.d_blk[0], ValueError), (7, c.d_lens[:0], ValueError), (9, c.out[:, :1], ValueError), (8, 0.0, L.OasisError),
                    (6, 590, L.OasisError), (6, 603, L.OasisError), (6, -1, L.OasisError), (2, None, L.OasisError), (3, None, L.OasisError)):
        with pytest.raises(e):
            call(i, v)
    for k in (dict(workspace=None), dict(workspace=c.ws[:16]), dict(lse=c.lse[0]), dict(workspace=c.ws.cpu())):
        with pytest.raises((ValueError, L.OasisError)):
            call(8, SCALE, **k)
    big = torch.zeros((1, 2, 8 * 70, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(L.OasisError):
        L.packed_attn(L.Dims(1, 560, 2, 700), big, c.packed, c.local, c.d_slot, c.d_blk, 600, c.d_lens, SCALE, torch.zeros_like(big), workspace=c.ws)
    kv, t, n = randn(gen(1), 4, 1, 2, 16, 128), i32([[0, 1]]), i32([1])
    d, e = L.Dims(1, 1, 1, 2), torch.zeros((4, 2304), dtype=torch.uint8, device="cuda")
    for a in ((d, kv.float(), t, n, n, 1, e, t), (d, kv, t[0], n, n, 1, e, t), (d, kv, t, n, n, 1, e[:, :2300], t), (d, kv, t, n, n, 1, e.cpu(), t),
              (d, kv, t, n, n, 3, e, t), (d, kv, t, n, n, -1, e, t), (d, kv, t, n.long(), n, 1, e, t)):
        with pytest.raises((ValueError, TypeError, L.OasisError)):
            L.pack_blocks(*a)
    for a in ((e, n, kv.view(4, 2, 16, 128)), (e, n.long(), kv.view(4, 2, 16, 128)), (e[:, :5], n.long(), kv[:1, 0])):
        with pytest.raises((ValueError, TypeError)):
            L.unpack_blocks(*a)
    with pytest.raises(ValueError):
        L.stage_packed_layers([e], [n.long()], [n], 2, [e])
    with pytest.raises(ValueError):
        L.pack_local_layers(d, [kv], [], 0, n, n, 1, [e], [t])


def test_the_bounds_check_build_flags_and_skips(L):
    import json
    import os
    import subprocess
    import sys

    from paper_2608_08097_b200 import build
    env = dict(os.environ, OASIS_LIB=build.build(checked=True))
    worker = os.path.join(os.path.dirname(os.path.abspath(__file__)), "packed_checked_worker.py")
    r = subprocess.run([sys.executable, worker], env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    out = json.loads(r.stdout.strip().splitlines()[-1])
    assert out["ok"] and len(out["flagged"]) == 5
