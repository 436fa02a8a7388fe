"""GPU tests of the packed attention where the reference that a row's weights are taken against has to be raised after its first
tile: sums and accumulators that exist already are scaled down, row by row.  All numbers of query rows (every variant of the two
kernels), rows that rise in different tiles, by little or by much or never, alone and in splits.  Bounds as in test_gpu_packed.py."""
import math

import numpy as np
import pytest
import torch

from oracle import packed as op
from tests.test_gpu_packed import SCALE, Case, L, f64, gen, i32  # noqa: F401

pytestmark = pytest.mark.gpu

AMP = 8.0                                                # of a query along its direction: logits of 1.02 times the key in log2 units


def heights(tile):
    """What the keys of a tile of eight columns have along the eight directions (dims 0, 16, .., 112)."""
    t = tile % 8
    return [7.0 * (0, 6, 12, 18, 24, 30, 36, 44)[t],     # far above the tile before, tile by tile (seven times a scale)
            1.5 * t,                                     # a little above: what was summed before still counts
            5.0, 30.0 - 3.0 * t,                         # never, and falling
            50.0 * (t >= 3), 34.0 * (t == 2), 20.0 * (t == 1) + 45.0 * (t == 6),
            0.0]


def direction(row):
    return (5 * row + 3) % 8


def rising(L, B, Hkv, G, T, n, near=2, seed=0):          # noqa: F811
    """n packed columns in order, all whole and visible, behind them the local window."""
    c = Case(L, B, G * Hkv, Hkv, T, [16 * n + (3 if near else 0)] * B, n, near=near, seed=seed)
    g = gen(seed + 1)
    c.blk[:, :, :n] = np.arange(n)
    c.d_blk = i32(c.blk.tolist())
    h = torch.tensor([heights(k // 8) for k in range(n)], device="cuda").repeat(B * Hkv, 1)              # [entries][8]
    kv = torch.randn((B * Hkv * n, 2, 16, 128), generator=g, device="cuda")
    kv[:, 0] *= 0.7
    kv[:, 0, :, ::16] += h[:, None]
    kv[:, 1] += (torch.arange(B * Hkv * n, device="cuda") % n // 8 % 5)[:, None, None] - 2.0              # values that tell the tiles apart
    kv = kv.to(torch.bfloat16)
    at = i32(c.slot[:, :, :n].reshape(1, -1).tolist())
    L.pack_blocks(L.Dims(1, 1, 1, at.numel()), kv, i32([list(range(at.numel()))]), i32([0]), i32([at.numel()]), at.numel(), c.packed, at)
    c.q.zero_()
    for t in range(T):
        for k in range(G):
            c.q[:, t, k::G, 16 * direction(t * G + k)] = AMP
    # the case is what it is meant to be: along direction 0 a tile is more than 2^32 above all of its group of eight so far, and
    # along direction 1 above it by less
    e = op.unpack(c.packed.cpu().numpy()[c.slot[0, 0, :n]])[:, 0]
    top = np.array([e[8 * k:8 * k + 8].max((0, 1)) for k in range(n // 8)]) * AMP * SCALE * math.log2(math.e)
    for k in range(1, n // 8):
        if k % 8:
            assert top[k, 0] - top[k - k % 8:k, 0].max() > 34
            assert -3 < top[k, 16] - top[k - k % 8:k, 16].max() < 20
    return c


@pytest.mark.parametrize("G, T", [(4, 1), (8, 1), (12, 1), (4, 4), (5, 4), (8, 3), (31, 1), (4, 8), (33, 1), (10, 4), (8, 8), (9, 8), (6, 16), (97, 1), (8, 16)])
@pytest.mark.parametrize("B, Hkv, n", [(1, 1, 64), (2, 2, 130), (1, 2, 2500)])
def test_references_rise_row_by_row(L, G, T, B, Hkv, n):  # noqa: F811
    """One request whose splits fit a cluster, and one that goes through the workspace."""
    c = rising(L, B, Hkv, G, T, n, seed=G + T)
    assert n < 2000 or c.need > 0
    c.run(L)
    c.check()


@pytest.mark.parametrize("G, T", [(4, 1), (4, 3), (4, 5), (8, 4), (8, 8), (8, 9), (8, 16)])
@pytest.mark.parametrize("near", [0, 2])
def test_references_rise_without_splits(L, G, T, near):  # noqa: F811
    """More rows than the GPU has places for: every thread block walks all tiles of its row."""
    c = rising(L, 150, 4, G, T, 40, near=near, seed=near + T)
    c.run(L)
    c.check()


@pytest.mark.parametrize("G, T", [(1, 32), (1, 8), (1, 20), (1, 40), (1, 90), (1, 128), (2, 64)])
def test_rows_that_see_nothing_at_first(L, G, T):        # noqa: F811
    """The blocks that only the last tokens see come first: the other rows have no reference until the others' sums are there."""
    c = rising(L, 76, 2, G, T, 96, near=0, seed=T)
    last = 319 + T - 1
    ahead = np.arange(last // 16, 19, -1)                                     # hidden from the first token, at position 319
    c.blk[:, :, :96] = np.concatenate([ahead, np.arange(20), np.arange(last // 16 + 1, 96)])
    c.lens = np.array([319 if b % 3 else 319 + T // 2 for b in range(76)])
    c.d_blk, c.d_lens = i32(c.blk.tolist()), i32(c.lens.tolist())
    c.run(L)
    c.check()


@pytest.mark.parametrize("Hq, Hkv, T", [(12, 1, 1), (20, 1, 1), (8, 1, 4), (40, 1, 1), (8, 1, 9), (16, 1, 8)])
def test_logits_far_apart(L, Hq, Hkv, T):                 # noqa: F811
    """Random keys 30 times as large: logits of a few hundred, whose maxima rise anywhere.

    Where the keys that decide have a value of zero, what is left of an output is as small as the other keys' weights, and small
    weights are zero: those below 2^-126 of their reference (the exponential flushes them), and a whole part of the keys, another
    split's or warp's, whose reference is that far below the others'.  A weight is at most 2^32 of its part's reference and the sum
    that divides them at least 1, so that n keys lose at most n 2^32 2^-126 max|v|.  Outputs as small as that are checked against it."""
    c = Case(L, 2, Hq, Hkv, T, [3000, 1500], 187, seed=Hq + T, size=30.0)
    c.run(L)
    local = np.nan_to_num(f64(c.local), nan=0.0, posinf=0.0, neginf=0.0)
    out, lse, a, big = op.attn(f64(c.q), c.packed.cpu().numpy(), local, c.slot, c.blk, c.budget, c.lens, SCALE)
    e = 2.0 ** -15 * big
    lost = c.blk.shape[2] * 16 * 2.0 ** -94 * 30 * 7                          # (values are 30 normally distributed ones)
    assert np.all(np.abs(f64(c.out) - out) <= 2.0 ** -8 * (a + np.abs(out)) + 2 * e[..., None] * a + lost)
    assert np.all(np.abs(f64(c.lse) - lse) <= e + 1e-5 * (1 + np.abs(lse)))


@pytest.mark.parametrize("G, T", [(4, 1), (4, 5), (8, 9)])
def test_a_raise_repeats_itself(L, G, T):                 # noqa: F811
    c = rising(L, 2, 2, G, T, 130, seed=T)
    c.run(L)
    want, want_lse = c.out.clone(), c.lse.clone()
    for _ in range(5):
        c.fresh()
        c.run(L)
        assert torch.equal(c.out, want) and torch.equal(c.lse, want_lse)
