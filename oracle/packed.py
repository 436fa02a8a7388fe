"""The packed cache and the rotary positions in plain numpy, double precision: blocks of keys and values in 4 bits, attention over
them, rotation of a projection's rows.  Written from their definitions; no shared code with the product."""
import math

import numpy as np

BYTES = 2304


def scale_of(byte):
    """The scale that a byte stands for."""
    byte = np.asarray(byte, np.int64)
    return (1 + (byte & 7) / 8) * np.exp2((byte >> 3) - 20.0)


def group_byte(a):
    """The scale byte of a group with the largest magnitude a: a / 7 to four significant bits, ties to even."""
    if a == 0:
        return 0
    if math.isinf(a):
        return 255
    m, e = math.frexp(a / 7)                           # m in [1/2, 1)
    n = round(m * 16)                                  # 8 .. 16 (round() takes ties to even)
    if n == 16:
        n, e = 8, e + 1
    return min(max((e - 1 + 20) * 8 + n - 8, 0), 255)


def quantise(x):
    """x [16] -> (codes 1 .. 15, scale byte): the nearest whole multiple within +-7, halfway the one nearer to zero."""
    x = np.where(np.isnan(x), 0.0, x)
    byte = group_byte(float(np.abs(x).max()))
    s = float(scale_of(byte))
    q = [min(7, math.ceil(abs(v) / s - 0.5)) if not math.isinf(v) else 7 for v in x]
    return np.array([8 + int(math.copysign(max(n, 0), v)) for n, v in zip(q, x)]), byte


def _word(codes):
    w = 0
    for k, c in enumerate(codes):
        w |= int(c) << (4 * (k // 2) + 16 * (k % 2))
    return [(w >> (8 * i)) & 255 for i in range(4)]


def pack(kv):
    """kv [2][16][128] float64 -> [2304] uint8."""
    out = np.zeros(BYTES, np.uint8)
    for i in range(16):
        for g in range(8):
            c, out[2048 + 8 * i + g] = quantise(kv[0, i, 16 * g:16 * g + 16])
            for w in range(2):
                at = 256 * (g // 2) + 16 * i + 8 * (g % 2) + 4 * w
                out[at:at + 4] = _word(c[8 * w:8 * w + 8])
    for d in range(128):
        c, out[2176 + d] = quantise(kv[1, :, d])
        for w in range(2):
            out[1024 + 8 * d + 4 * w:1024 + 8 * d + 4 * w + 4] = _word(c[8 * w:8 * w + 8])
    return out


def unpack(entries):
    """[..., 2304] uint8 -> [..., 2][16][128] float64."""
    e = np.asarray(entries, np.uint8)
    lead = e.shape[:-1]

    def values(raw):                                   # [..., 4 n] bytes -> [..., 8 n] whole numbers
        w = raw.reshape(*raw.shape[:-1], raw.shape[-1] // 4, 4).astype(np.int64)
        w = w[..., 0] + (w[..., 1] << 8) + (w[..., 2] << 16) + (w[..., 3] << 24)
        c = np.stack([(w >> (4 * (k // 2) + 16 * (k % 2))) & 15 for k in range(8)], -1)
        return c.reshape(*c.shape[:-2], 2 * raw.shape[-1]) - 8.0

    k = values(np.moveaxis(e[..., :1024].reshape(*lead, 4, 16, 16), -2, -3).reshape(*lead, 16, 64))
    k = k * np.repeat(scale_of(e[..., 2048:2176].reshape(*lead, 16, 8)), 16, -1)
    v = values(e[..., 1024:2048].reshape(*lead, 128, 8)) * scale_of(e[..., 2176:])[..., None]
    return np.stack([k, np.swapaxes(v, -1, -2)], -3)


def attn(q, packed, local, slot_tbl, blk_tbl, local_col, seq_len, scale):
    """q [B][T][Hq][128], packed [slots][2304] uint8, local [slots][2][16][128] float64.  Returns out, lse, and for error
    bounds sum of weight * |value| and the rows' largest sum |q k| * scale."""
    B, T, Hq, _ = q.shape
    Hkv, cols = blk_tbl.shape[1:]
    G = Hq // Hkv
    out, out_abs = np.zeros(q.shape), np.zeros(q.shape)
    lse, big = np.full(q.shape[:3], -np.inf), np.zeros(q.shape[:3])
    for b in range(B):
        for h in range(Hkv):
            c = np.nonzero(blk_tbl[b, h] >= 0)[0]
            if not len(c):
                continue
            kv = np.concatenate([unpack(packed[slot_tbl[b, h, c[c < local_col]]]), local[slot_tbl[b, h, c[c >= local_col]]]])
            pos = (blk_tbl[b, h, c].astype(np.int64)[:, None] * 16 + np.arange(16)).ravel()
            k, v = kv[:, 0].reshape(-1, 128), kv[:, 1].reshape(-1, 128)
            for t in range(T):
                see = pos <= int(seq_len[b]) + t
                if not see.any():
                    continue
                ks, vs, rows = k[see], v[see], q[b, t, h * G:(h + 1) * G]
                z = rows @ ks.T * scale
                top = z.max(-1, keepdims=True)
                w = np.exp(z - top)
                den = w.sum(-1, keepdims=True)
                out[b, t, h * G:(h + 1) * G], out_abs[b, t, h * G:(h + 1) * G] = w / den @ vs, w / den @ np.abs(vs)
                lse[b, t, h * G:(h + 1) * G] = (top + np.log(den))[:, 0]
                big[b, t, h * G:(h + 1) * G] = (np.abs(rows) @ np.abs(ks).T).max(-1) * scale
    return out, lse, out_abs, big


def rotate(qkv, pos, freqs, rot, interleaved, factor, Hq, Hkv):
    """qkv [B][T][(Hq + 2 Hkv) * 128] float64, pos [B][T] -> q [B][T][Hq][128], kv [B][T][Hkv][2][128]."""
    B, T, _ = qkv.shape
    x = qkv.reshape(B, T, Hq + 2 * Hkv, 128).copy()
    for i in range(rot // 2):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        a = np.asarray(pos, np.longdouble) * np.longdouble(freqs[i])
        c, s = (factor * f(a).astype(np.float64)[:, :, None] for f in (np.cos, np.sin))
        u, w = x[:, :, :Hq + Hkv, lo].copy(), x[:, :, :Hq + Hkv, hi].copy()
        x[:, :, :Hq + Hkv, lo], x[:, :, :Hq + Hkv, hi] = u * c - w * s, w * c + u * s
    return x[:, :, :Hq], np.stack([x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]], 3)
