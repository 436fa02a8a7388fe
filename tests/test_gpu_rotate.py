"""GPU tests of the rotary positions through the C ABI, against the numpy oracle (angles in long double).

Tolerance of a rotated element u c - w s: the fraction of a turn is rounded to fp32 (at most half a turn: 2^-25 turns, 2 pi 2^-25
radians) after it was computed in 64 bits (below 1e-9 radians at the positions here), cos and sin are fp32 to 2 ulp, two products
and a sum in fp32: 2^-20 (|u| + |w|) factor covers them; and half a step of bf16 on the result, 2^-8 |y|.  Copies have to be equal."""
import numpy as np
import pytest
import torch

from oracle import packed as op

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


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


def make(shape, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * 3).to(TYPES[dtype])


def check(q, kv, qkv, pos, table, Hq, Hkv, live=None):
    x = qkv.double().cpu().numpy()
    want_q, want_kv = op.rotate(x, pos, table.freqs.cpu().numpy(), table.rot_dim, table.interleaved, table.factor, Hq, Hkv)
    big_q, big_kv = (np.abs(a) for a in op.rotate(x, np.zeros_like(pos), table.freqs.cpu().numpy(), table.rot_dim, table.interleaved, 1.0, Hq, Hkv))
    r, half = table.rot_dim, table.rot_dim // 2
    for got, want, big in ((q, want_q, big_q), (kv[:, :, :, 0], want_kv[:, :, :, 0], big_kv[:, :, :, 0])):
        got = got.double().cpu().numpy()
        mate = big.copy()
        if table.interleaved:
            mate[..., 0:r:2], mate[..., 1:r:2] = big[..., 1:r:2], big[..., 0:r:2]
        else:
            mate[..., :half], mate[..., half:r] = big[..., half:r], big[..., :half]
        tol = 2.0 ** -20 * table.factor * (big + mate) + 2.0 ** -8 * np.abs(want)
        tol[..., r:] = 0
        want = np.where(np.arange(128) < r, want, torch.tensor(want).to(torch.bfloat16).double().numpy())
        off = np.abs(got - want)
        rows = np.ones(off.shape[:2], bool) if live is None else live
        assert np.all(off[rows] <= tol[rows]), (off[rows] - tol[rows]).max()
        assert np.all(got[~rows] == 9.0)
    copied = torch.tensor(want_kv[:, :, :, 1]).to(torch.bfloat16).double().numpy()
    got = kv[:, :, :, 1].double().cpu().numpy()
    rows = np.ones(got.shape[:2], bool) if live is None else live
    assert np.array_equal(got[rows], copied[rows]) and np.all(got[~rows] == 9.0)


def outputs(B, T, Hq, Hkv):
    return (torch.full((B, T, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, T, Hkv, 2, 128), 9.0, dtype=torch.bfloat16, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rot, interleaved", [(128, False), (128, True), (64, False), (96, True), (52, False), (6, False), (2, False), (2, True), (122, True), (112, False), (126, False)])
def test_layouts_and_types(L, dtype, rot, interleaved):
    from paper_2608_08097_b200.rotary import RotaryTable
    B, T, Hq, Hkv = 2, 5, 6, 2
    table = RotaryTable(rot, interleaved=interleaved)
    qkv, (q, kv) = make((B, T, (Hq + 2 * Hkv) * 128), dtype, rot), outputs(B, T, Hq, Hkv)
    lens = [0, 70001]
    L.rotate_qkv(L.Dims(B, Hq, Hkv, 1), qkv, table, q, kv, seq_len=i32(lens))
    check(q, kv, qkv, np.array(lens)[:, None] + np.arange(T), table, Hq, Hkv)


@pytest.mark.parametrize("B, T, Hq, Hkv", [(1, 1, 1, 1), (1, 1, 32, 8), (3, 1, 40, 8), (1, 77, 1, 1), (2, 600, 2, 1), (1, 130, 64, 1), (700, 3, 3, 1)])
@pytest.mark.parametrize("scaling", [None, dict(kind="yarn", factor=8.0, trained=4096), dict(kind="bands", factor=8, trained=8192)])
def test_sizes_and_far_positions(L, B, T, Hq, Hkv, scaling):
    from paper_2608_08097_b200.rotary import RotaryTable
    table = RotaryTable(128, base=500000.0, scaling=scaling)
    rng = np.random.default_rng(T)
    pos = rng.integers(-5, 2 ** 24, (B, T))
    pos.flat[0] = 2 ** 31 - 1
    qkv, (q, kv) = make((B, T, (Hq + 2 * Hkv) * 128), "bf16", T), outputs(B, T, Hq, Hkv)
    L.rotate_qkv(L.Dims(B, Hq, Hkv, 1), qkv, table, q, kv, positions=i32(pos.tolist()))
    # (at 2^31 the turns carry 2^31 / 2 pi * 2^-53 of rounding: still below 1e-6 radians, inside 2^-20)
    check(q, kv, qkv, pos, table, Hq, Hkv)


@pytest.mark.parametrize("T", [1, 5, 33, 64])
def test_trees_and_padding(L, T):
    from paper_2608_08097_b200.rotary import RotaryTable
    B, Hq, Hkv, rng = 5, 4, 2, np.random.default_rng(T)
    parent = np.array([[-1] + [int(rng.integers(max(-1, t - 4), t)) for t in range(1, T)] for _ in range(B)])
    parent[1] = np.arange(T) - 1                                   # a chain
    parent[2] = np.arange(T) + 1                                   # no parent comes first: all are roots
    parent[3, T // 2] = -7
    nodes = np.array([T, T, T, max(1, T - 2), 0])
    depth = np.zeros((B, T), int)
    for b in range(B):
        for t in range(T):
            p = parent[b, t]
            depth[b, t] = depth[b, p] + 1 if 0 <= p < t else 0
    lens, table = [3, 0, 100000, 17, 5], RotaryTable(64, interleaved=True)
    qkv, (q, kv) = make((B, T, (Hq + 2 * Hkv) * 128), "bf16", T), outputs(B, T, Hq, Hkv)
    L.rotate_qkv(L.Dims(B, Hq, Hkv, 1), qkv, table, q, kv, seq_len=i32(lens), parent=i32(parent.tolist()), n_nodes=i32(nodes.tolist()))
    live = np.arange(T) < nodes[:, None]
    check(q, kv, qkv, np.array(lens)[:, None] + depth, table, Hq, Hkv, live)
    # a padded chain, counts outside the range
    q, kv = outputs(B, T, Hq, Hkv)
    counts = np.array([T + 5, -3, 0, 1, T])
    L.rotate_qkv(L.Dims(B, Hq, Hkv, 1), qkv, table, q, kv, seq_len=i32(lens), n_nodes=i32(counts.tolist()))
    check(q, kv, qkv, np.array(lens)[:, None] + np.arange(T), table, Hq, Hkv, np.arange(T) < counts[:, None])


def test_strided_rows_streams_and_graphs(L):
    from paper_2608_08097_b200.rotary import RotaryTable
    B, T, Hq, Hkv = 3, 4, 6, 2
    W = (Hq + 2 * Hkv) * 128
    whole = make((T, B + 1, W + 24), "bf16", 3)
    qkv = whole[:, 1:, 16:16 + W].transpose(0, 1)                  # [B][T][W], strides W + 24 and (B + 1)(W + 24)
    table, lens, (q, kv) = RotaryTable(128), i32([5, 6, 7000]), outputs(B, T, Hq, Hkv)
    d = L.Dims(B, Hq, Hkv, 1)
    pos = lens.cpu().numpy()[:, None] + np.arange(T)
    L.rotate_qkv(d, qkv, table, q, kv, seq_len=lens)
    check(q, kv, qkv, pos, table, Hq, Hkv)
    first = q.clone(), kv.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q.fill_(0)
    side.wait_stream(torch.cuda.current_stream())
    L.rotate_qkv(d, qkv, table, q, kv, seq_len=lens, stream=side)
    side.synchronize()
    assert torch.equal(q, first[0]) and torch.equal(kv, first[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.rotate_qkv(d, qkv, table, q, kv, seq_len=lens)
    lens.add_(1)
    g.replay()
    check(q, kv, qkv, pos + 1, table, Hq, Hkv)


def test_infinities_and_nan_stay_in_their_pair(L):
    from paper_2608_08097_b200.rotary import RotaryTable
    qkv, (q, kv) = make((1, 1, 3 * 128), "bf16"), outputs(1, 1, 1, 1)
    qkv[0, 0, 100], qkv[0, 0, 3], qkv[0, 0, 256 + 5] = float("inf"), float("nan"), float("nan")
    L.rotate_qkv(L.Dims(1, 1, 1, 1), qkv, RotaryTable(64), q, kv, seq_len=i32([9]))
    bad = ~torch.isfinite(q[0, 0, 0].float())
    assert torch.nonzero(bad).flatten().tolist() == [3, 35, 100] and torch.isinf(q[0, 0, 0, 100]) and torch.isfinite(kv[0, 0, 0, 0].float()).all()
    assert torch.nonzero(~torch.isfinite(kv[0, 0, 0, 1].float())).flatten().tolist() == [5]


def test_refusals(L):
    from paper_2608_08097_b200.rotary import RotaryTable
    B, T, Hq, Hkv = 2, 3, 4, 2
    d, table, lens = L.Dims(B, Hq, Hkv, 1), RotaryTable(128), i32([1, 2])
    qkv, (q, kv) = make((B, T, 8 * 128), "bf16"), outputs(B, T, Hq, Hkv)
    par, n = i32([[-1, 0, 1]] * B), i32([3, 3])
    for a, k, e in (((qkv.double(), table, q, kv), dict(seq_len=lens), TypeError), ((qkv[:, :, 1:], table, q, kv), dict(seq_len=lens), ValueError),
                    ((qkv.transpose(1, 2), table, q, kv), dict(seq_len=lens), ValueError), ((qkv.cpu(), table, q, kv), dict(seq_len=lens), ValueError),
                    ((qkv, table, q.float(), kv), dict(seq_len=lens), TypeError), ((qkv, table, q, kv[:, :1]), dict(seq_len=lens), ValueError),
                    ((qkv, table, q, kv), dict(), L.OasisError), ((qkv, table, q, kv), dict(seq_len=lens, parent=par), L.OasisError),
                    ((qkv, table, q, kv), dict(positions=par, parent=par, n_nodes=n), L.OasisError), ((qkv, table, q, kv), dict(seq_len=lens.long()), TypeError),
                    ((qkv, table, q, kv), dict(positions=par[:1]), ValueError), ((qkv, RotaryTable(128, device="cpu"), q, kv), dict(seq_len=lens), ValueError),
                    ((torch.zeros(B, T, 8 * 128 + 4, dtype=torch.bfloat16, device="cuda")[:, :, :1024], table, q, kv), dict(seq_len=lens), L.OasisError),
                    ((torch.zeros(B * T * 1024 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(B, T, 1024), table, q, kv), dict(seq_len=lens), L.OasisError)):
        with pytest.raises(e):
            L.rotate_qkv(d, *a, **k)
    assert bool((q == 9.0).all()) and bool((kv == 9.0).all())
    empty = torch.zeros((0, T, 1024), dtype=torch.bfloat16, device="cuda")
    L.rotate_qkv(L.Dims(0, Hq, Hkv, 1), empty, table, *outputs(0, T, Hq, Hkv), seq_len=i32([]))
