"""GPU tests of a decode engine with draft trees: what padding nodes hold must not reach the next working set, and a request that
sits out a step, or whose step is thrown away, must come back to a working set that holds every block once."""
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


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


class Loop:
    """An engine over random histories; `hist` is the truth, one [tokens][Hkv][2][128] tensor per layer and request."""

    def __init__(self, lens, B, Hq, Hkv, T, layers, mb, k, cap, seed, **options):
        from paper_2608_08097_b200 import pipeline
        self.g, self.rng = torch.Generator(device="cuda"), np.random.default_rng(seed)
        self.g.manual_seed(seed)
        self.B, self.Hq, self.Hkv, self.T, self.layers, self.k = B, Hq, Hkv, T, layers, k
        self.lens = list(lens)
        self.eng = pipeline.DecodeEngine(B, Hq, Hkv, mb, k, T, layers, mode="delta", cap=cap, append=True, tree=True, **options)
        self.hist = [[self.randn(n, Hkv, 2, 128) for n in lens] for _ in range(layers)]
        for l in range(layers):
            kv = torch.zeros((B * mb, Hkv, 2, 16, 128), dtype=torch.bfloat16)
            table = torch.tensor(self.rng.permutation(B * mb).reshape(B, mb), dtype=torch.int32)
            for b in range(B):
                for pos in range(lens[b]):
                    kv[table[b, pos // 16], :, :, pos % 16] = self.hist[l][b][pos].cpu()
            self.eng.attach(l, kv.pin_memory(), table.cuda())
        self.seq = i32(self.lens)
        self.before = self.seq // 16
        self.stamp = 0
        self.sel = [torch.empty_like(x.sel) for x in self.eng.layers]
        self.eng.prime([self.randn(B, T, Hq, 128) for _ in range(layers)], self.seq // 16, self.seq)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda").to(torch.bfloat16)

    def step(self, nodes, fill=None, graph=False):
        """One step over chains of `nodes` nodes; padding rows of the queries and of the tree buffer hold `fill`."""
        self.q = [self.randn(self.B, self.T, self.Hq, 128) for _ in range(self.layers)]
        self.tree_kv = [self.randn(self.B, self.T, self.Hkv, 2, 128) for _ in range(self.layers)]
        if fill is not None:
            for b, n in enumerate(nodes):
                for t in (*self.q, *self.tree_kv):
                    t[b, n:] = fill
        self.parent, self.nodes = np.tile(np.arange(self.T) - 1, (self.B, 1)).astype(np.int32), list(nodes)
        self.stamp += 1
        full = self.seq // 16
        call = ((self.q, self.seq, self.before, full - self.before, full, self.seq),
                dict(step_stamp=self.stamp, new_kv=self.tree_kv, sel_log=self.sel, tree=(i32(self.parent.tolist()), i32(self.nodes))))
        torch.cuda.synchronize()
        if graph:
            g = self.eng.capture_step(*call[0], **call[1])
            self.eng.replay(g)
        else:
            self.eng.step(*call[0], **call[1])
            self.eng.join()
        torch.cuda.synchronize()
        self.before = full

    def commit(self, keep):
        """The first keep[b] nodes of every chain are kept."""
        path = np.full((self.B, self.T), -1, np.int32)
        for b, n in enumerate(keep):
            path[b, :n] = np.arange(n)
        nxt = torch.zeros_like(self.seq)
        self.eng.commit(self.eng.commit_plan(self.tree_kv), i32(path.tolist()), i32(list(keep)), self.seq, next_len=nxt)
        torch.cuda.synchronize()
        for l in range(self.layers):
            for b, n in enumerate(keep):
                self.hist[l][b] = torch.cat([self.hist[l][b], self.tree_kv[l][b][:n]])
        self.lens = [a + n for a, n in zip(self.lens, keep)]
        assert nxt.tolist() == self.lens
        self.seq = nxt

    def check_dense(self, requests):
        """The budget covers every block: the step's attention is dense causal attention (bounds as for the operator)."""
        for l in range(self.layers):
            out = f64(self.eng.layers[l].out)
            for b in requests:
                H = f64(self.hist[l][b])
                for t in range(self.nodes[b]):
                    rows = np.concatenate([H, f64(self.tree_kv[l][b])[ot.ancestors(self.parent[b], t)]])
                    for a in range(self.Hq):
                        K, W = rows[:, a // (self.Hq // self.Hkv), 0], rows[:, a // (self.Hq // self.Hkv), 1]
                        z = K @ f64(self.q[l][b, t, a]) * SCALE
                        w = np.exp(z - z.max())
                        w /= w.sum()
                        want, amount = w @ W, w @ np.abs(W)
                        assert np.all(np.abs(out[b, t, a] - want) <= 2 ** -8 * (amount + np.abs(want)) + 6e-4 * amount), (l, b, t, a)

    def check_no_block_twice(self):
        for l in range(self.layers):
            for row in self.eng.resident[l].view(-1, self.k + 2).tolist():
                held = [j for j in row if j >= 0]
                assert len(held) == len(set(held)), (l, row)


# ---- the scoring operator ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("reduce_mode", [0, 1], ids=["max", "sum"])
@pytest.mark.parametrize("Hq,Hkv,T,mb", [(4, 4, 1, 5), (8, 2, 9, 130), (6, 2, 64, 40), (32, 4, 13, 300), (32, 2, 20, 33), (128, 1, 3, 20), (3, 1, 50, 129)])
def test_scores_of_each_requests_own_drafts(L, Hq, Hkv, T, mb, reduce_mode):
    """Against the definition in 64 bits.  A score is a sum of 256 exact products (times the rows, where they are summed) in fp32."""
    nodes = [T, 0, 1, min(2, T), max(1, T - 1), T + 7, -3]
    B, G = len(nodes), Hq // Hkv
    rng, g = np.random.default_rng(T + mb), torch.Generator(device="cuda")
    g.manual_seed(T + mb)
    q = torch.randn((B, T, Hq, 128), generator=g, device="cuda").to(torch.bfloat16)
    s = torch.randn((B, Hkv, mb, 2, 128), generator=g, device="cuda").to(torch.bfloat16).sort(dim=3).values      # [min, max]
    for b, n in enumerate(nodes):
        q[b, max(n, 0):] = math.nan
    n_full = rng.integers(0, mb + 1, B)
    n_full[:3] = mb
    scores, cand = torch.full((B, Hkv, mb), math.nan, device="cuda"), i32([-9] * B)
    dims = L.Dims(B, Hq, Hkv, mb)
    L.score_tree(dims, q, i32(nodes), s, i32(n_full.tolist()), scores, reduce_mode=reduce_mode, n_candidates=cand)
    torch.cuda.synchronize()
    got, s64, q64 = scores.double().cpu().numpy(), f64(s), f64(q)
    assert cand.tolist() == [int(n_full[b]) if nodes[b] > 0 else 0 for b in range(B)]
    for b, n in enumerate(nodes):
        n, nf = max(0, min(n, T)), int(n_full[b])
        if n == 0:
            assert np.isneginf(got[b]).all()
            continue
        assert np.isneginf(got[b, :, nf:]).all()
        rows = q64[b, :1] if n == 1 else q64[b, 1:n][:128 // G]
        for h in range(Hkv):
            r = rows[:, h * G:(h + 1) * G].reshape(-1, 1, 128)
            u = np.maximum(r * s64[b, h, :nf, 0], r * s64[b, h, :nf, 1])
            want, size = u.sum(-1), np.abs(u).sum(-1) + np.minimum(np.abs(r * s64[b, h, :nf, 0]), np.abs(r * s64[b, h, :nf, 1])).sum(-1)
            want, size = (want.sum(0), size.sum(0)) if reduce_mode else (want.max(0), size.max(0))
            assert np.all(np.abs(got[b, h, :nf] - want) <= (256 + len(r)) * 2.0 ** -23 * size), (b, h)
    again = torch.full_like(scores, 1.0)
    L.score_tree(dims, q, i32(nodes), s, i32(n_full.tolist()), again, reduce_mode=reduce_mode)              # (without the count)
    assert torch.equal(again, scores)


def test_refusals_of_the_scoring(L):
    q, s = torch.zeros((2, 3, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 2, 5, 2, 128), dtype=torch.bfloat16, device="cuda")
    n, x = i32([1, 2]), torch.zeros((2, 2, 5), device="cuda")
    good = dict(dims=L.Dims(2, 4, 2, 5), q=q, n_nodes=n, summaries=s, n_full_blocks=n, scores=x, n_candidates=n.clone())
    L.score_tree(**good)
    for name, bad, err in (("q", q.float(), TypeError), ("q", q[:1], ValueError), ("q", q.cpu(), ValueError), ("n_nodes", n[:1], ValueError),
                           ("n_nodes", n.long(), TypeError), ("summaries", s[:, :, :4], ValueError), ("scores", x[..., :4], ValueError),
                           ("scores", x.double(), TypeError), ("n_candidates", n.cpu(), ValueError), ("n_full_blocks", i32([1, 2, 3]), ValueError)):
        with pytest.raises(err):
            L.score_tree(**{**good, name: bad})
    with pytest.raises(L.OasisError, match="reduce_mode"):
        L.score_tree(**good, reduce_mode=2)
    e = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    L.score_tree(L.Dims(0, 4, 2, 5), q[:0], e(0), s[:0], e(0), x[:0])


# ---- padding nodes -------------------------------------------------------------------------------------------------
def selections(fill, graph):
    """Three steps with a budget of 5 of up to 24 blocks; the last request has no node in any step."""
    loop = Loop([380, 200, 333, 90], 4, 8, 2, 9, 2, 32, 5, 5, seed=3)
    got = []
    for nodes, keep in (([9, 1, 4, 0], [3, 1, 2, 0]), ([2, 9, 1, 0], [1, 4, 1, 0]), ([1, 3, 9, 0], [1, 1, 1, 0])):
        loop.step(nodes, fill, graph)
        got += [t.clone() for t in loop.sel]
        got += [loop.eng.layers[l].out[b, :n].clone() for l in range(2) for b, n in enumerate(nodes)]
        loop.commit(keep)
        got += [t.clone() for t in loop.eng.resident]
    return got


@pytest.mark.parametrize("fill", [40.0, -3e38, math.inf, math.nan])
def test_padding_nodes_do_not_choose_the_working_set(L, fill):
    want, got = selections(0.0, False), selections(fill, False)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_padding_nodes_do_not_choose_the_working_set_in_a_graph(L):
    want, got = selections(0.0, False), selections(math.nan, True)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_priming_reads_no_padding_node(L):
    """The first working set, chosen by `prime` from queries whose padding rows hold NaN, equals that from clean ones."""
    nodes, got = [4, 1, 2], []
    for fill in (0.0, math.nan):
        loop = Loop([300, 200, 330], 3, 8, 2, 4, 2, 32, 5, 5, seed=8)
        q = [loop.randn(3, 4, 8, 128) for _ in range(2)]
        for t in q:
            for b, n in enumerate(nodes):
                t[b, n:] = fill
        loop.eng.prime(q, loop.seq // 16, loop.seq, n_nodes=i32(nodes))
        got.append([t.clone() for t in (*loop.eng.resident, *[x.sel for x in loop.eng.layers])])
    assert all(torch.equal(a, b) for a, b in zip(*got))


# ---- requests that keep nothing ------------------------------------------------------------------------------------
@pytest.mark.parametrize("nodes", [0, 5], ids=["sits out", "thrown away"])
@pytest.mark.parametrize("graph", [False, True], ids=["eager", "graph"])
def test_a_request_that_keeps_nothing_for_a_step(L, nodes, graph):
    """Request 0 commits across a block's border, keeps nothing for one or two steps, and goes on: block 2 is then in the working
    set once, as a selected block or in its local column."""
    loop = Loop([45, 60], 2, 8, 2, 6, 2, 16, 16, 16, seed=4)
    loop.step([6, 6], graph=graph)
    loop.commit([6, 6])                                   # 45 -> 51: blocks 2 and 3 are local now
    for _ in range(2):
        loop.step([nodes, 6], graph=graph)
        loop.check_dense([0, 1] if nodes else [1])
        loop.commit([0, 6])
        loop.check_no_block_twice()
    for _ in range(2):
        loop.step([6, 3], graph=graph)
        loop.check_dense([0, 1])
        loop.commit([4, 2])
        loop.check_no_block_twice()


def test_local_blocks_that_may_have_been_selected(L):
    """Rows of nine requests with the local blocks (even, odd) and candidates given: only a request that keeps nothing gives a
    column up, and only one whose block is below its number of candidates."""
    cols = [(4, 5), (4, 5), (4, 5), (4, 5), (-1, 5), (4, -1), (4, 5), (6, 5), (-9, -9)]
    cand, keep = [5, 4, 6, 0, 6, 6, 6, 6, 50], [0, 0, -2, 0, 0, 0, 2, 0, 0]
    want = [(-1, 5), (4, 5), (-1, -1), (4, 5), (-1, -1), (-1, -1), (6, 5), (6, -1), (-9, -9)]
    B, Hkv, n_cols, layers = 9, 3, 6, 2
    dims = L.Dims(B, Hkv, Hkv, 16)
    z = lambda *shape, dt=torch.bfloat16: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
    blk = [torch.tensor(cols, dtype=torch.int32, device="cuda")[:, None].expand(B, Hkv, 2).repeat(1, 1, 3).contiguous() for _ in range(layers)]
    before = [t.clone() for t in blk]
    plan = L.CommitPlan(dims, [z(B, 2, Hkv, 2, 128)] * layers, [z(B, 16, dt=torch.int32)] * layers, [z(B, Hkv, n_cols, dt=torch.int32) - 1] * layers,
                        blk, 4, [z(4, 2, 16, 128)] * layers)
    args, nxt = (plan, i32([[0, 1]] * B), i32(keep), i32([95] * B)), i32([0] * B)
    L.commit_kv_layers(*args, next_len=nxt, n_candidates=i32(cand))
    for a, was in zip(blk, before):
        assert a[:, :, :4].equal(was[:, :, :4]) and a[:, :, 4:].tolist() == [[list(w)] * Hkv for w in want]
        a.copy_(was)
    assert nxt.tolist() == [95 + max(n, 0) for n in keep]
    L.commit_kv_layers(*args)                             # no selection was made: those requests' columns stay
    for a, was in zip(blk, before):
        assert a[:6].equal(was[:6]) and a[7:].equal(was[7:])
    with pytest.raises(L.OasisError, match="share memory"):
        L.commit_kv_layers(*args, next_len=nxt, n_candidates=nxt)
    with pytest.raises(TypeError):
        L.commit_kv_layers(*args, n_candidates=nxt.long())


def test_more_layers_than_one_commit_takes(L):
    loop = Loop([30], 1, 2, 1, 3, 66, 8, 6, 6, seed=6)
    for keep in (3, 2, 1):
        loop.step([3])
        loop.check_dense([0])
        loop.commit([keep])
        loop.check_no_block_twice()
    with pytest.raises(ValueError, match="66 layers"):
        loop.eng.commit_plan(loop.tree_kv[:65])


@pytest.mark.parametrize("options", [{}, dict(transfer_group=2, wait_group=1, transfer_streams=2), dict(transfer_kind="bulk", wait_group=2, plan_stream="side")],
                         ids=["default", "grouped", "bulk"])
def test_a_loop_without_host_synchronisation(L, options):
    """Six steps whose order rests on streams and events alone give the bits of the same steps made one by one."""
    def run(sync):
        torch.cuda.synchronize()
        g = torch.Generator(device="cuda")
        g.manual_seed(9)
        B, T, layers, mb, k = 3, 7, 3, 32, 6
        loop = Loop([200, 310, 45], B, 8, 2, T, layers, mb, k, k, seed=9, **options)
        eng, now = loop.eng, torch.cuda.current_stream()
        parent, path = i32([[-1, 0, 1, 2, 3, 4, 5]] * B), i32([list(range(T))] * B)
        counts = [i32(n) for n in ([7, 3, 0], [1, 7, 5], [7, 7, 7], [0, 4, 7], [7, 1, 2], [7, 7, 7])]
        keeps = [i32(n) for n in ([6, 2, 0], [1, 7, 0], [3, 5, 7], [0, 4, 6], [7, 0, 2], [1, 2, 3])]
        seq, before, got = loop.seq, loop.seq // 16, []
        for s, (nodes, keep) in enumerate(zip(counts, keeps)):
            q = [torch.randn((B, T, 8, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(layers)]
            kv = [torch.randn((B, T, 2, 2, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(layers)]
            full, nxt = seq // 16, torch.empty_like(seq)
            if sync:
                torch.cuda.synchronize()
            for st in (eng.main, eng.pred):
                st.wait_stream(now)
            eng.step(q, seq, before, full - before, full, seq, step_stamp=s + 1, new_kv=kv, sel_log=loop.sel, tree=(parent, nodes))
            eng.join()
            now.wait_stream(eng.main)
            if sync:
                torch.cuda.synchronize()
            got += [x.clone() for x in loop.sel]
            got += [torch.where((torch.arange(T, device="cuda") < nodes[:, None])[..., None, None], x.out, 0) for x in eng.layers]
            eng.commit(eng.commit_plan(kv), path, keep, seq, next_len=nxt)
            got += [x.clone() for x in eng.resident]
            seq, before = nxt, full
        torch.cuda.synchronize()
        return got + [x.cpu() for x in eng.kv]

    want = run(True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(want, run(False)))
