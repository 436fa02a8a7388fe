"""CPU checks of the draft-tree operators: the oracle against brute force, an independent oracle and the law it has to
follow, and the refusals of the three entry points (made on the host, before anything is enqueued)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import tree as ot


def _chain(T):
    return np.arange(T, dtype=np.int32) - 1


def test_ancestors_of_a_small_tree_and_of_bad_parents():
    parent = [-1, 0, 0, 1, 3, 9, 6, -7]
    assert ot.ancestors(parent, 4) == [4, 3, 1, 0]
    assert ot.ancestors(parent, 2) == [2, 0]
    assert ot.ancestors(parent, 5) == [5]            # a parent that comes later: a root
    assert ot.ancestors(parent, 6) == [6]            # its own parent: a root
    assert ot.ancestors(parent, 7) == [7]


def test_tree_attention_of_a_chain_is_the_chain_attention(oracle):
    """A chain whose keys are in the tree buffer sees what the chain attention sees with the keys in the cache."""
    rng = np.random.default_rng(0)
    B, T, Hq, Hkv, cols, L = 2, 3, 4, 2, 4, 37                      # positions 37..39 are rows 5..7 of block 2

    def bits(*shape):
        return (rng.standard_normal(shape).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)

    pool, q = bits(B * Hkv * cols, 2, 16, 128), bits(B, T, Hq, 128)
    slot = np.arange(B * Hkv * cols, dtype=np.int32).reshape(B, Hkv, cols)
    blk = np.tile(np.array([1, 0, 2, -1], np.int32), (B, Hkv, 1))
    lens = np.full(B, L, np.int32)
    ref = oracle.sparse_attn(q, pool, slot, blk, lens, np.float32(0.1), Hkv)
    tree_kv = np.zeros((B, T, Hkv, 2, 128))
    for b in range(B):
        for h in range(Hkv):
            tree_kv[b, :, h] = ot.bf16(pool[slot[b, h, 2]])[:, 5:5 + T].transpose(1, 0, 2)
    out, lse = np.zeros((B, T, Hq, 128)), np.zeros((B, T, Hq))
    ot.tree_attn(ot.bf16(q), tree_kv, np.tile(_chain(T), (B, 1)), [T] * B, ot.bf16(pool), slot, blk, lens, np.float32(0.1), out, lse)
    # the other oracle sums 40 keys of 128 dims in fp32: a few hundred roundings of 2^-24 on sums of order 10
    np.testing.assert_allclose(out, ref["out32"], rtol=0, atol=2e-4)
    np.testing.assert_allclose(lse, ref["lse"], rtol=0, atol=2e-4)


@pytest.mark.parametrize("with_draft", [True, False])
def test_verified_tokens_follow_the_targets_distribution(with_draft):
    """The first token that comes out (the kept child, else the next token) is distributed as the target's own sample:
    with two children drawn independently from the draft's distribution, and with two fixed ones."""
    rng = np.random.default_rng(1)
    V, N = 4, 20000
    logits = np.tile(np.array([0.3, -0.4, 1.1, 0.0]), (1, 3, 1))
    p = ot.distribution(logits[0, 0], 0.7)
    q = np.array([0.5, 0.2, 0.1, 0.2])
    draft = np.tile(q, (1, 3, 1)) if with_draft else None
    seen = np.zeros(V)
    for _ in range(N):
        kids = rng.choice(V, 2, p=q) if with_draft else [2, 0]
        tok = np.array([[0, kids[0], kids[1]]])
        path, n, nxt = ot.verify_tree(logits, tok, np.array([[-1, 0, 0]]), [3], rng.random((1, 3)), [0.7], 3, draft)
        seen[tok[0, path[0, 1]] if n[0] > 1 else nxt[0]] += 1
    # five standard deviations of a share of N draws
    assert np.all(np.abs(seen / N - p) < 5 * np.sqrt(p * (1 - p) / N))


def test_greedy_walk_and_empty_requests():
    logits = np.zeros((3, 4, 6))
    logits[:, 0, 2] = logits[:, 0, 5] = 1.0                          # equal: the lower index
    logits[:, 2, 4] = 3.0
    logits[:, 3] = -np.inf
    tok = np.array([[9, 5, 2, 4]] * 3)
    parent = np.array([[-1, 0, 0, 2]] * 3)
    path, n, nxt = ot.verify_tree(logits, tok, parent, [4, 0, 3], np.zeros((3, 4)), [0, 0, 0], 4)
    assert path.tolist() == [[0, 2, 3, -1], [-1] * 4, [0, 2, -1, -1]] and n.tolist() == [3, 0, 2] and nxt.tolist() == [-1, -1, 4]
    path, n, nxt = ot.verify_tree(logits, tok, parent, [4, 0, 3], np.zeros((3, 4)), [0, 0, 0], 2)
    assert n.tolist() == [2, 0, 2] and nxt.tolist() == [4, -1, 4]     # the path is full: the walk ends there


def test_commit_of_a_chain_is_the_append(oracle):
    rng = np.random.default_rng(2)
    B, T, Hkv, cols, mb = 3, 7, 2, 5, 8
    new = rng.integers(0, 60000, (B, T, Hkv, 2, 128)).astype(np.uint16)
    lens = np.array([13, 16, 31], np.int32)
    table = rng.permutation(B * mb).reshape(B, mb).astype(np.int32)
    slot = np.arange(B * Hkv * cols, dtype=np.int32).reshape(B, Hkv, cols)

    def fresh():
        return (np.full((B, Hkv, cols), -1, np.int32), np.zeros((B * Hkv * cols, 2, 16, 128), np.uint16),
                np.zeros((B * mb, Hkv, 2, 16, 128), np.uint16))

    blk, pool, kv = fresh()
    oracle.append_kv(new, T, lens, table, slot, blk, 3, pool, kv)
    blk2, pool2, kv2 = fresh()
    nxt = np.zeros(B, np.int32)
    ot.commit_kv(new, np.tile(np.arange(T), (B, 1)), [T] * B, lens, table, slot, blk2, 3, pool2, kv2, nxt)
    assert np.array_equal(blk, blk2) and np.array_equal(pool, pool2) and np.array_equal(kv, kv2) and nxt.tolist() == [20, 23, 38]


# ---- refusals ------------------------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def L():
    from paper_2608_08097_b200 import binding, build
    build.build()
    return binding


ONE, ODD = 4096, 4104          # never dereferenced on the host; the second one is not 16-byte aligned


def test_refusals_of_tree_attention(L):
    lib = L.lib()

    def call(dims=L.Dims(2, 32, 8, 64), T=5, q=ONE, tree=ONE, parent=ONE, nodes=ONE, pool=ONE, slot=ONE, blk=ONE, cols=10, lens=ONE,
             scale=0.1, out=ONE, lse=None, ws=ONE, ws_bytes=1 << 30):
        d = dims.c()
        return lib.oasis_tree_attn(ctypes.byref(d), q, T, tree, parent, nodes, pool, slot, blk, cols, lens, scale, out, lse, ws, ws_bytes, None)

    for name in ("q", "tree", "parent", "nodes", "pool", "slot", "blk", "lens", "out"):
        assert call(**{name: None}) == 1, name
    for name in ("q", "tree", "pool", "out", "ws"):
        assert call(**{"cols": 4000, name: ODD}) == 1, name
    for bad in (dict(T=0), dict(T=65), dict(cols=0), dict(cols=-3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(dims=L.Dims(2, 30, 8, 64)), dict(dims=L.Dims(-1, 32, 8, 64))):
        assert call(**bad) == 1, bad
    for bad in (dict(dims=L.Dims(2, 32, 8, 64, head_dim=64)), dict(dims=L.Dims(2, 32, 8, 64, block_size=32)), dict(dims=L.Dims(2, 258, 2, 64))):
        assert call(**bad) == 2, bad
    need = L.tree_attn_workspace_bytes(L.Dims(2, 32, 8, 64), 5, 4000)      # split over more SMs than a cluster has
    assert need > 0 and call(cols=4000, ws=None) == 4 and call(cols=4000, ws_bytes=need - 1) == 4 and "workspace" in L.last_error()
    assert call(dims=L.Dims(0, 32, 8, 64), ws=None) == 0
    assert L.tree_attn_workspace_bytes(L.Dims(64, 32, 8, 64), 64, 130) == 0 == L.tree_attn_workspace_bytes(L.Dims(1, 32, 8, 64), 65, 130)


def test_refusals_of_verification(L):
    lib = L.lib()

    def call(B=2, T=5, V=100, logits=ONE, kind=0, lb=500, lr=100, tok=ONE, parent=ONE, nodes=ONE, u=ONE, temp=ONE, draft=None, db=0, dr=0,
             path=ONE, M=5, n=ONE, nxt=ONE):
        return lib.oasis_verify_tree(B, T, V, logits, kind, lb, lr, tok, parent, nodes, u, temp, draft, db, dr, path, M, n, nxt, None)

    for name in ("logits", "tok", "parent", "nodes", "u", "temp", "path", "n", "nxt"):
        assert call(**{name: None}) == 1, name
    for bad in (dict(T=0), dict(T=65), dict(V=0), dict(V=(1 << 22) + 1, lr=1 << 23), dict(M=0), dict(M=6), dict(kind=3), dict(kind=-1), dict(B=-1), dict(lr=99),
                dict(lb=-1), dict(logits=4097), dict(logits=4098), dict(draft=ONE, dr=99, db=500), dict(draft=4098, dr=100, db=500)):
        assert call(**bad) == 1, bad
    assert call(B=0) == 0


def test_refusals_of_the_commit(L):
    lib = L.lib()
    one = (ctypes.c_void_p * 2)(ONE, ONE)

    def call(dims=L.Dims(2, 32, 8, 64), layers=2, tree=one, T=5, path=ONE, M=5, n=ONE, lens=ONE, table=one, slot=one, blk=one, cols=10, col=8,
             pool=one, host=one, nxt=None):
        d = dims.c()
        return lib.oasis_commit_kv_layers(ctypes.byref(d), layers, tree, T, path, M, n, lens, table, slot, blk, cols, col, pool, host, nxt, None)

    for name in ("tree", "path", "n", "lens", "table", "slot", "blk", "pool"):
        assert call(**{name: None}) == 1, name
    for name in ("tree", "slot", "blk", "pool", "table"):
        assert call(**{name: (ctypes.c_void_p * 2)(ONE, None)}) == 1, name
    for name in ("tree", "pool", "host"):
        assert call(**{name: (ctypes.c_void_p * 2)(ONE, ODD)}) == 1, name
    for bad in (dict(T=0), dict(T=65), dict(M=0), dict(M=17), dict(col=-1), dict(col=9), dict(cols=1, col=0), dict(layers=65), dict(layers=-1),
                dict(nxt=ONE)):                                      # next_len is seq_len here
        assert call(**bad) == 1, bad
    far, off = 1 << 20, ONE + 4                                      # next_len overlaps one of its inputs by an element
    for inputs in (dict(path=far, n=far), dict(path=far, lens=far), dict(n=far, lens=far), dict(path=ONE - 36, n=far, lens=far)):
        assert call(nxt=off if "path" not in inputs or inputs["path"] == far else ONE, **inputs) == 1, inputs
        assert "share memory" in L.last_error()
    assert call(layers=0) == 0 and call(dims=L.Dims(0, 32, 8, 64)) == 0


def test_commit_plan_needs_one_tensor_per_layer(L):
    t = torch.zeros(1)
    with pytest.raises(ValueError, match="one tensor per layer"):
        L.CommitPlan(L.Dims(1, 8, 8, 8), [t, t], [t], [t, t], [t, t], 0, [t, t])
    with pytest.raises(ValueError, match="layers outside"):
        L.CommitPlan(L.Dims(1, 8, 8, 8), [], [], [], [], 0, [])


def test_dims_can_be_copied_after_a_call(L):
    import copy
    import pickle
    d = L.Dims(2, 32, 8, 64)
    L._cdims(d)
    assert pickle.loads(pickle.dumps(d)) == d == copy.deepcopy(d) and L._cdims(copy.copy(d)) != L._cdims(d)


def test_an_engine_refuses_trees_it_cannot_run():
    from paper_2608_08097_b200 import pipeline
    with pytest.raises(ValueError, match="KV append"):
        pipeline.DecodeEngine(1, 8, 8, 8, 4, 5, 1, mode="delta", cap=1, tree=True)
    with pytest.raises(ValueError, match="chains"):
        pipeline.DecodeEngine(1, 8, 8, 8, 4, 5, 1, mode="delta", cap=1, append=True, tree=True, fused=True)
