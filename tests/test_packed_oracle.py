"""CPU tests of the packed cache and the rotary positions: the oracle against brute force, the frequency tables against their
closed forms, and what the C ABI and the binding refuse before anything is launched."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import packed as op

SCALES = np.array([(1 + m / 8) * 2.0 ** (e - 20) for e in range(32) for m in range(8)])


@pytest.fixture(scope="module")
def L():
    from paper_2608_08097_b200 import build, binding
    build.build()
    return binding


def bf16(x):
    return torch.as_tensor(x, dtype=torch.float64).to(torch.bfloat16).double().numpy()


def test_scales_are_in_order():
    assert np.array_equal(op.scale_of(np.arange(256)), SCALES) and np.all(np.diff(SCALES) > 0)


@pytest.mark.parametrize("size", [1e-6, 1e-5, 0.01, 1.0, 100.0, 3e4])
def test_a_group_takes_the_nearest_scale_and_the_nearest_multiples(size):
    rng = np.random.default_rng(int(size * 1e6))
    for _ in range(200):
        x = bf16(rng.standard_normal(16) * size)
        codes, byte = op.quantise(x)
        a = np.abs(x).max() / 7
        off = np.abs(SCALES - a)
        assert off[byte] == off.min()
        s = SCALES[byte]
        # every multiple, nearest first, ties to the smaller magnitude
        for v, c in zip(x, codes):
            best = min(range(-7, 8), key=lambda n: (abs(v - n * s), abs(n)))
            assert c - 8 == best or (best == 0 and c == 8)
        if 7 * SCALES[0] <= np.abs(x).max() <= 7 * SCALES[-1]:
            assert np.all(np.abs(x - (codes - 8) * s) <= s / 2)
        assert np.array_equal(bf16((codes - 8) * s), (codes - 8) * s)            # exact in bf16


def test_halfway_goes_to_the_smaller_magnitude_and_ties_of_scales_to_even():
    codes, byte = op.quantise(np.array([7.0, 0.5, -0.5, 1.5, -6.5, 6.515625] + [0.0] * 10))
    assert op.scale_of(byte) == 1.0 and list(codes[:6] - 8) == [7, 0, 0, 1, -6, 7]
    for odd in (17, 19, 29, 31):                        # a / 7 = odd / 16: halfway between two scales
        n = round(odd / 2)
        assert op.scale_of(op.group_byte(7 * odd / 16)) == n / 8 and n % 2 == 0


def test_zero_nan_and_infinity():
    assert list(op.quantise(np.zeros(16))[0]) == [8] * 16 and op.quantise(np.zeros(16))[1] == 0
    codes, byte = op.quantise(np.array([np.nan, 7.0, -3.0] + [0.0] * 13))
    assert op.scale_of(byte) == 1.0 and list(codes[:3]) == [8, 15, 5]
    codes, byte = op.quantise(np.array([np.inf, -np.inf, 1.0] + [0.0] * 13))
    assert byte == 255 and list(codes[:3]) == [15, 1, 8]
    codes, byte = op.quantise(np.array([3e38, -1e-30] + [0.0] * 14))
    assert byte == 255 and list(codes[:2]) == [15, 8]


def test_pack_and_unpack_agree_place_by_place():
    rng = np.random.default_rng(5)
    kv = bf16(rng.standard_normal((2, 16, 128)))
    e = op.pack(kv)
    got = op.unpack(e)
    for part in range(2):
        for i in range(16):
            for d in range(128):
                group = kv[0, i, d // 16 * 16:d // 16 * 16 + 16] if part == 0 else kv[1, :, d]
                codes, byte = op.quantise(group)
                assert got[part, i, d] == (codes[d % 16 if part == 0 else i] - 8) * op.scale_of(byte)
    # a single value shows up at its place alone
    for part, i, d, at, bit in ((0, 3, 37, 256 + 48 + 0, 24), (1, 9, 70, 1024 + 560 + 4, 16)):
        one = np.zeros((2, 16, 128))
        one[part, i, d] = 7.0
        w = op.pack(one)[at:at + 4]
        assert int.from_bytes(bytes(w), "little") == 0x88888888 ^ (8 << bit) ^ (15 << bit)


def test_rotation_is_a_rotation():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 3, 4 * 128))
    pos = rng.integers(0, 10 ** 6, (2, 3))
    f = 10000.0 ** (-np.arange(0, 52, 2) / 52)
    for inter in (0, 1):
        q, kv = op.rotate(x, pos, f, 52, inter, 1.0, 2, 1)
        back, _ = op.rotate(np.concatenate([q.reshape(2, 3, -1), kv.reshape(2, 3, -1)], -1), -pos, f, 52, inter, 1.0, 2, 1)
        assert np.allclose(back, x.reshape(2, 3, 4, 128)[:, :, :2], atol=1e-9)
        assert np.array_equal(q[..., 52:], x.reshape(2, 3, 4, 128)[:, :, :2, 52:]) and np.array_equal(kv[:, :, 0, 1], x.reshape(2, 3, 4, 128)[:, :, 3])
        assert np.allclose((q ** 2).sum(-1), (x.reshape(2, 3, 4, 128)[:, :, :2] ** 2).sum(-1))


def test_frequency_tables():
    from paper_2608_08097_b200.rotary import RotaryTable

    def table(r=128, **k):
        return RotaryTable(r, device="cpu", **k)
    plain = 10000.0 ** (-np.arange(64) / 64)
    t = table()
    assert t.freqs.dtype == torch.float64 and np.allclose(t.freqs, plain, rtol=1e-15) and t.factor == 1.0 and t.interleaved == 0
    assert np.allclose(table(scaling=dict(kind="linear", factor=4)).freqs, plain / 4)
    ntk = table(scaling=dict(kind="ntk", factor=4)).freqs
    assert ntk[0] == 1 and math.isclose(float(ntk[-1]), plain[-1] / 4, rel_tol=1e-12) and np.all(np.diff(ntk) < 0)
    y = table(scaling=dict(kind="yarn", factor=8, trained=4096))
    turns = 4096 * plain / (2 * math.pi)
    assert np.allclose(y.freqs[turns > 40], plain[turns > 40]) and np.allclose(y.freqs[turns < 0.8], plain[turns < 0.8] / 8)
    assert math.isclose(y.factor, 0.1 * math.log(8) + 1)
    b = table(base=500000.0, scaling=dict(kind="bands", factor=8, trained=8192))
    plain5 = 500000.0 ** (-np.arange(64) / 64)
    wave = 2 * math.pi / plain5
    assert np.allclose(b.freqs[wave < 8192 / 4], plain5[wave < 8192 / 4]) and np.allclose(b.freqs[wave > 8192], plain5[wave > 8192] / 8)
    mid = (wave >= 8192 / 4) & (wave <= 8192)
    smooth = (8192 / wave[mid] - 1) / 3
    assert np.allclose(b.freqs[mid], (1 - smooth) * plain5[mid] / 8 + smooth * plain5[mid])
    g = table(32, scaling=dict(kind="given", factors=np.arange(1, 17), attention_factor=1.5))
    assert np.allclose(g.freqs, 10000.0 ** (-np.arange(16) / 16) / np.arange(1, 17)) and g.factor == 1.5
    for bad in (dict(rot_dim=7), dict(rot_dim=130), dict(rot_dim=0), dict(base=0.5), dict(scaling=dict(kind="linear")), dict(scaling=dict(kind="yarn", factor=2)),
                dict(scaling=dict(kind="linear", factor=2, trained=3)), dict(scaling=dict(kind="spiral")), dict(scaling=dict(factor=2)),
                dict(scaling=dict(kind="yarn", factor=2, trained=100, sharp=1)), dict(scaling=dict(kind="given", factors=[1.0])),
                dict(scaling=dict(kind="linear", factor=0))):
        with pytest.raises(ValueError):
            RotaryTable(device="cpu", **bad)


def test_frequency_bands_must_be_in_order():
    from paper_2608_08097_b200.rotary import RotaryTable
    for kw in (dict(kind="bands", low_freq_factor=4.0, high_freq_factor=4.0), dict(kind="bands", low_freq_factor=0.0), dict(kind="bands", high_freq_factor=0.5),
               dict(kind="yarn", beta_fast=1.0), dict(kind="yarn", beta_slow=0.0), dict(kind="yarn", beta_fast=float("nan"))):
        with pytest.raises(ValueError):
            RotaryTable(64, scaling=dict(kw, factor=4.0, trained=8192), device="cpu")


def test_the_c_abi_refuses_without_a_gpu(L):
    lib, null, one, odd = L.lib(), ctypes.c_void_p(0), ctypes.c_void_p(4096), ctypes.c_void_p(4104)
    d = ctypes.byref(L.Dims(2, 32, 8, 64).c())
    assert L.PACKED_BYTES == op.BYTES

    def pack(kv=one, n=1, packed=one, summ=null, dims=d):
        return lib.oasis_pack_blocks(dims, kv, one, one, one, n, packed, one, summ, null)
    assert pack(kv=null) == 1 and pack(kv=odd) == 1 and pack(packed=null) == 1 and pack(packed=odd) == 1 and pack(summ=odd) == 1
    assert pack(n=-1) == 1 and pack(n=65) == 1 and pack(n=0) == 0 and pack(dims=ctypes.byref(L.Dims(0, 32, 8, 64).c())) == 0
    assert pack(dims=ctypes.byref(L.Dims(2, 32, 8, 64, head_dim=64).c())) == 2
    arr = (ctypes.c_void_p * 1)(4096)

    def local(n_layers=1, cols=10, col=8, n=1, packed=arr):
        return lib.oasis_pack_local_layers(d, n_layers, arr, arr, cols, col, one, one, n, packed, arr, null, null)
    assert local(n_layers=65) == 1 and local(col=9) == 1 and local(col=-1) == 1 and local(n=3) == 1 and local(packed=null) == 1 and local(n_layers=0) == 0
    assert local(n=0) == 0 and local(packed=(ctypes.c_void_p * 1)(4104)) == 1
    assert lib.oasis_offload_blocks_packed(d, one, null, one, one, one, one, 1, one, null, null) == 1
    assert lib.oasis_unpack_blocks(one, one, -1, one, null) == 1 and lib.oasis_unpack_blocks(one, one, 0, one, null) == 0
    assert lib.oasis_unpack_blocks(odd, one, 1, one, null) == 1 and lib.oasis_unpack_blocks(one, null, 1, one, null) == 1
    assert lib.oasis_stage_packed_layers(65, arr, arr, arr, 1, arr, 0, null) == 1 and lib.oasis_stage_packed_layers(1, arr, arr, arr, -1, arr, 0, null) == 1
    assert lib.oasis_stage_packed_layers(1, arr, arr, arr, 0, arr, 0, null) == 0 and lib.oasis_stage_packed_layers(1, null, arr, arr, 1, arr, 0, null) == 1

    def attn(T=5, cols=130, col=128, scale=0.1, packed=one, near=one, q=one, ws=null, n_ws=0, dims=d):
        return lib.oasis_packed_attn(dims, q, T, packed, near, one, one, cols, col, one, scale, one, null, ws, n_ws, null)
    assert attn(T=0) == 1 and attn(T=33) == 2 and attn(cols=0) == 1 and attn(col=131) == 1 and attn(col=121) == 1 and attn(col=-1) == 1
    assert attn(scale=0.0) == 1 and attn(scale=-1.0) == 1 and attn(scale=float("nan")) == 1 and attn(scale=float("inf")) == 1
    assert attn(packed=null) == 1 and attn(near=null) == 1 and attn(q=odd) == 1 and attn(q=null) == 1
    long = lib.oasis_packed_attn_workspace_bytes(d, 1, 4098, 4096)
    assert long > 0 and attn(T=1, cols=4098, col=4096) == 4 and attn(T=1, cols=4098, col=4096, ws=one, n_ws=long - 1) == 4
    assert attn(T=1, cols=4098, col=4096, ws=odd, n_ws=long) == 1
    assert lib.oasis_packed_attn_workspace_bytes(d, 0, 130, 128) == 0

    def rot(type=1, bs=48 * 128, ts=48 * 128, T=1, pos=null, lens=one, parent=null, nodes=null, rot_dim=128, qkv=one, q=one, dims=d):
        return lib.oasis_rotate_qkv(dims, qkv, type, bs, ts, T, pos, lens, parent, nodes, one, rot_dim, 0, 1.0, q, one, null)
    assert rot(type=3) == 1 and rot(bs=100) == 1 and rot(bs=48 * 128 + 4) == 1 and rot(T=2, ts=47 * 128) == 1 and rot(T=-1) == 1
    assert rot(rot_dim=0) == 1 and rot(rot_dim=3) == 1 and rot(rot_dim=130) == 1 and rot(lens=null) == 1 and rot(qkv=odd) == 1 and rot(q=null) == 1
    assert rot(parent=one) == 1 and rot(parent=one, nodes=one, pos=one) == 1 and rot(T=65, parent=one, nodes=one) == 1
    assert rot(T=0) == 0
