"""Cases and plain forms of the operators around a KV cache held in 4 bits: making and reading packed blocks (`pack_blocks`,
`unpack_blocks`), attention over the packed working set beside the bf16 local window (`packed_attn`), and the rotary positions
of a step's projections on their way into attention and cache (`rotate_qkv`).

`run` computes each operator in elementary torch operations where `own` is false and calls the library where it is true.

A packed entry is the 2,304 bytes of one (block, KV head), 16 tokens x 128 dims of keys and of values:
  [0, 1024)      key codes: dims 32c .. 32c + 31 of token i in 16 bytes at 256 c + 16 i
  [1024, 2048)   value codes: the 16 tokens of dim d in 8 bytes at 1024 + 8 d
  [2048, 2176)   key scales: one byte for dims 16g .. 16g + 15 of token i at 2048 + 8 i + g
  [2176, 2304)   value scales: one byte for the 16 tokens of dim d at 2176 + d
Eight codes are a little-endian 32-bit word: code 2p in bits 4p .. 4p + 3, code 2p + 1 in bits 16 + 4p .. 16 + 4p + 3.  A code c with
the scale byte b stands for (c - 8) * s, s = (1 + (b & 7) / 8) * 2^((b >> 3) - 20).
"""
import math

import numpy as np
import torch

own = False

D, BLK, PACKED = 128, 16, 2304
SCALE = 1.0 / math.sqrt(128.0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases --------------------------------------------------------------------------------------------------------
def listed():
    return [
        # packing (and reading back) --------------------------------------------------------------------------------
        # a decode step: the block that one request in sixteen has just filled, all its KV heads: latency
        dict(name="pack a step's full block", op="pack", batch=1, kv_heads=8, blocks=1, ragged=False),
        # requests that cross the threshold together, different lengths, a head count that is no power of two
        dict(name="pack ragged requests", op="pack", batch=5, kv_heads=3, blocks=301, ragged=True),
        # the hand-over of a request of 32 K tokens
        dict(name="pack 32 K tokens", op="pack", batch=1, kv_heads=8, blocks=2048, ragged=False),
        # attention -----------------------------------------------------------------------------------------------
        # one request that has just begun, one token: latency
        dict(name="attn one short request", op="attn", batch=1, q_heads=32, kv_heads=8, tokens=1, context=200, budget=16, ragged=False),
        # plain decoding, no drafts: one token a request over a 2,048-token budget
        dict(name="attn single tokens", op="attn", batch=16, q_heads=32, kv_heads=8, tokens=1, context=32768, budget=128, ragged=False),
        # the reasoning-style step: the same with four drafts behind the verified token
        dict(name="attn reasoning, 5 tokens", op="attn", batch=16, q_heads=32, kv_heads=8, tokens=5, context=32771, budget=128, ragged=False),
        # eight query heads per KV head, eight drafts: 72 query rows; requests of different lengths, one without any key
        dict(name="attn group of 8, ragged", op="attn", batch=7, q_heads=32, kv_heads=4, tokens=9, context=50003, budget=300, ragged=True),
        # every block of a long cache
        dict(name="attn whole long cache", op="attn", batch=2, q_heads=32, kv_heads=8, tokens=1, context=131072, budget=8192, ragged=False),
        # rotary positions --------------------------------------------------------------------------------------------
        # one token of one request: latency
        dict(name="rotate one token", op="rotate", batch=1, q_heads=32, kv_heads=8, tokens=1, dtype="bf16", rot=128, interleaved=False,
             scaling="none", place="chain", far=4096),
        # a draft tree per request, far positions stretched to eight times the trained length
        dict(name="rotate draft trees", op="rotate", batch=16, q_heads=32, kv_heads=8, tokens=16, dtype="bf16", rot=128, interleaved=False,
             scaling="yarn", place="tree", far=131072),
        # a prompt, pairs side by side, half of the head rotated
        dict(name="rotate prompt, half of the head", op="rotate", batch=1, q_heads=32, kv_heads=8, tokens=8192, dtype="bf16", rot=64,
             interleaved=True, scaling="none", place="given", far=8192),
        # fp32 projections of packed prompts, a part of the head that is no multiple of 16, very far positions
        dict(name="rotate odd part, fp32", op="rotate", batch=3, q_heads=20, kv_heads=4, tokens=1001, dtype="f32", rot=52, interleaved=False,
             scaling="linear", place="given", far=1000000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pack", "attn", "attn", "attn", "rotate", "rotate"])
    if op == "pack":
        c = dict(op="pack", batch=_log(rng, 1, 32), kv_heads=rng.choice([1, 2, 3, 4, 8]), blocks=_log(rng, 1, 2048), ragged=rng.random() < 0.7)
        while c["batch"] * c["kv_heads"] * c["blocks"] > 16384:
            c["batch" if c["batch"] > 1 else "blocks"] //= 2
        return c
    if op == "attn":
        group, kv = rng.choice([1, 2, 3, 4, 5, 8, 16]), rng.choice([1, 2, 3, 4, 8])
        c = dict(op="attn", batch=_log(rng, 1, 48), q_heads=group * kv, kv_heads=kv, tokens=rng.choice([1, 1, rng.randint(1, min(16, 128 // group))]),
                 context=_log(rng, 1, 131072), budget=_log(rng, 4, 8192), ragged=rng.random() < 0.7)
        while work(c)["flops"] > 1e10 or work(c)["bytes"] > 300e6 or c["batch"] * kv * c["budget"] > 131072:
            c["batch" if c["batch"] > 1 else "budget"] //= 2
        return c
    group, kv = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 2, 4, 8])
    place = rng.choice(["chain", "tree", "given"])
    c = dict(op="rotate", batch=_log(rng, 1, 32), q_heads=group * kv, kv_heads=kv, tokens=rng.randint(1, 64) if place == "tree" else _log(rng, 1, 8192),
             dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), rot=rng.choice([128, 128, 96, 64, 32, 2 * rng.randint(1, 64)]),
             interleaved=rng.random() < 0.4, scaling=rng.choice(["none", "linear", "yarn"]), place=place, far=_log(rng, 100, 1000000))
    while c["batch"] * c["tokens"] * (c["q_heads"] + 2 * kv) > 390000:
        c["batch" if c["batch"] > 1 else "tokens"] //= 2
    return c


# ---- sizes that go by the case alone ------------------------------------------------------------------------------
def _lengths(c):
    """History lengths; ragged: from the whole context down to half of it, one request at its very first token."""
    n, b = c["context"], c["batch"]
    if not c["ragged"]:
        return [n] * b
    got = [max(1, n - (n * i) // (2 * b) - 5 * i) for i in range(b)]
    if b > 2:
        got[1] = 0
    return got


def _block_counts(c):
    if not c["ragged"]:
        return [c["blocks"]] * c["batch"]
    return [max(0, c["blocks"] - (c["blocks"] * i) // c["batch"] - (i == 1)) for i in range(c["batch"])]


def _empty(c, i):
    """A padded place of the batch: no column holds a block."""
    return c["ragged"] and c["batch"] > 3 and i == c["batch"] - 1


def work(c):
    if c["op"] == "pack":
        n = sum(_block_counts(c)) * c["kv_heads"]
        return {"bytes": n * (8192 + PACKED + 512 + PACKED + 8192), "flops": 0}
    if c["op"] == "attn":
        h, g, t = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["tokens"]
        moved = flops = 0
        for i, n in enumerate(_lengths(c)):
            if _empty(c, i):
                continue
            full = min(c["budget"], n // BLK)
            local = (n + t - 1) // BLK - n // BLK + 1
            moved += h * (full * PACKED + local * 8192)
            flops += 4 * D * t * g * h * (full * BLK + n % BLK) + 2 * D * g * h * t * (t + 1)
        rows = c["batch"] * t * c["q_heads"]
        return {"bytes": moved + rows * (2 * D * 2 + 4), "flops": flops}
    n = c["batch"] * c["tokens"] * (c["q_heads"] + 2 * c["kv_heads"]) * D
    return {"bytes": n * (DTYPES[c["dtype"]].itemsize + 2), "flops": 3 * n}


# ---- inputs -------------------------------------------------------------------------------------------------------
def _randn(shape, g, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _kv_entries(n, g):
    """[n][2][16][128]: keys some of whose dims are large, as rotated keys have them, and values of one size."""
    kv = torch.randn((n, 2, BLK, D), generator=g, device="cuda", dtype=torch.float32)
    lift = torch.where(torch.arange(D, device="cuda") % 17 == 3, 8.0, 1.0)
    kv[:, 0] *= lift
    return kv.to(torch.bfloat16)


def _prepare_pack(c, g):
    b, h, m = c["batch"], c["kv_heads"], c["blocks"]
    counts = _block_counts(c)
    pages = b * m + 3
    pool = torch.empty((pages, h, 2, BLK, D), dtype=torch.bfloat16, device="cuda")
    for i in range(0, pages, 4096):
        n = min(4096, pages - i)
        pool[i:i + n] = _kv_entries(n * h, g).view(n, h, 2, BLK, D)
    pool[0, 0, :, :4] = 0.0                            # tokens of nothing but zeros
    mb = m + 2
    src = torch.rand(pages, generator=g, device="cuda").argsort()[:b * m].view(b, m)
    dst = torch.rand(pages, generator=g, device="cuda").argsort()[:b * m].view(b, m)
    pad = torch.zeros((b, 1), dtype=torch.int64, device="cuda")
    src, dst = (torch.cat([pad, t, pad], 1).to(torch.int32) for t in (src, dst))
    n_blocks = torch.tensor(counts, dtype=torch.int32, device="cuda")
    where = [(i, j) for i in range(b) for j in range(1, 1 + counts[i])]
    at = torch.tensor(where, device="cuda").view(-1, 2)
    idx = (dst[at[:, 0], at[:, 1]].long()[:, None] * h + torch.arange(h, device="cuda")).flatten()
    s = dict(case=c, pool=pool, src=src, dst=dst, at=at, idx=idx, n_blocks=n_blocks, first=torch.ones(b, dtype=torch.int32, device="cuda"),
             packed=torch.zeros((pages * h, PACKED), dtype=torch.uint8, device="cuda"),
             out=torch.zeros((idx.numel(), 2, BLK, D), dtype=torch.bfloat16, device="cuda"),
             summaries=torch.zeros((b, h, mb, 2, D), dtype=torch.bfloat16, device="cuda"))
    if own:
        from paper_2608_08097_b200 import binding
        s["dims"] = binding.Dims(b, h, h, mb)
    return s


def _pack_words(code):
    """[..., 8] codes -> [..., 4] bytes."""
    w = sum(code[..., 2 * p + hi] << (4 * p + 16 * hi) for p in range(4) for hi in range(2))
    return torch.stack([(w >> (8 * i)) & 255 for i in range(4)], -1).to(torch.uint8)


def _pack(kv):
    """[n][2][16][128] -> [n][2304], for the packed pools that the attention reads."""
    n = kv.shape[0]
    parts, scales = [], []
    for x in (kv[:, 0], kv[:, 1].transpose(1, 2)):     # keys [token][dim], values [dim][token]: groups of 16 along the last axis
        v, byte = _quantise(x.float().unflatten(-1, (-1, 16)))
        code = (v + 8).to(torch.int64).flatten(-2)
        parts.append(_pack_words(code.unflatten(-1, (-1, 8))).flatten(-2))
        scales.append(byte.to(torch.uint8).reshape(n, 128))
    keys = parts[0].view(n, BLK, 4, 16).transpose(1, 2).reshape(n, 1024)
    return torch.cat([keys, parts[1].reshape(n, 1024), scales[0], scales[1]], 1)


def _prepare_attn(c, g):
    b, hq, h, t, k = c["batch"], c["q_heads"], c["kv_heads"], c["tokens"], c["budget"]
    lens = torch.tensor(_lengths(c), device="cuda")
    n_full, last = lens // BLK, (lens + t - 1) // BLK
    most = max(1, int(max(_lengths(c)) // BLK))
    # the resident blocks of a row: distinct full blocks in no particular order, then the two local columns
    rank = torch.rand((b, h, most), generator=g, device="cuda")
    rank = rank.masked_fill(torch.arange(most, device="cuda") >= n_full[:, None, None], 2.0)
    order = rank.argsort(dim=-1)[..., :k]
    cols = k + 2
    tbl = torch.full((b, h, cols), -1, dtype=torch.int64, device="cuda")
    tbl[..., :order.shape[-1]] = torch.where(torch.arange(order.shape[-1], device="cuda") < n_full[:, None, None], order, -1)
    lo, hi = n_full[:, None], torch.where(last > n_full, last, -1)[:, None]
    even = lo % 2 == 0
    tbl[..., k] = torch.where(even, lo, hi)
    tbl[..., k + 1] = torch.where(even, hi, lo)
    for i in range(b):
        if _empty(c, i):
            tbl[i] = -1
    slot = torch.cat([torch.arange(b * h * k, device="cuda").view(b, h, k), torch.arange(b * h * 2, device="cuda").view(b, h, 2)], 2)
    packed = torch.empty((b * h * k, PACKED), dtype=torch.uint8, device="cuda")
    for i in range(0, b * h * k, 1 << 14):
        n = min(1 << 14, b * h * k - i)
        packed[i:i + n] = _pack(_kv_entries(n, g))
    s = dict(case=c, packed=packed, local=_kv_entries(b * h * 2, g), slot_tbl=slot.to(torch.int32), blk_tbl=tbl.to(torch.int32),
             seq_len=lens.to(torch.int32), q=_randn((b, t, hq, D), g),
             out=torch.zeros((b, t, hq, D), dtype=torch.bfloat16, device="cuda"), lse=torch.zeros((b, t, hq), dtype=torch.float32, device="cuda"))
    if own:
        from paper_2608_08097_b200 import binding
        s["dims"] = binding.Dims(b, hq, h, max(1, (max(_lengths(c)) + t + BLK) // BLK))
        s["workspace"] = torch.empty(max(16, binding.packed_attn_workspace_bytes(s["dims"], t, cols, k)), dtype=torch.uint8, device="cuda")
    return s


def _frequencies(c):
    """inverse frequencies (64 bits) and the factor on cos and sin: none, positions divided by 8, or the division blended in
    between the dims that turn 32 times and once over 4,096 trained positions."""
    r = c["rot"]
    f = 10000.0 ** (-np.arange(0, r, 2) / r)
    if c["scaling"] == "linear":
        return f / 8.0, 1.0
    if c["scaling"] == "yarn":
        edge = [r * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0)) for turns in (32, 1)]
        low, high = max(math.floor(edge[0]), 0), min(math.ceil(edge[1]), r - 1)
        ramp = np.clip((np.arange(r // 2) - low) / max(high - low, 0.001), 0, 1)
        return f / 8.0 * ramp + f * (1 - ramp), 0.1 * math.log(8.0) + 1.0
    return f, 1.0


def _prepare_rotate(c, g):
    b, hq, h, t = c["batch"], c["q_heads"], c["kv_heads"], c["tokens"]
    lens = (torch.rand(b, generator=g, device="cuda") * c["far"]).to(torch.int32)
    s = dict(case=c, qkv=_randn((b, t, (hq + 2 * h) * D), g, DTYPES[c["dtype"]], 2.0), seq_len=lens, positions=None, parent=None, n_nodes=None,
             q=torch.zeros((b, t, hq, D), dtype=torch.bfloat16, device="cuda"), kv=torch.zeros((b, t, h, 2, D), dtype=torch.bfloat16, device="cuda"))
    f, s["factor"] = _frequencies(c)
    s["freqs"] = torch.tensor(f, dtype=torch.float64, device="cuda")
    if c["place"] == "given":
        s["positions"] = (torch.rand((b, t), generator=g, device="cuda") * c["far"]).to(torch.int32)
    elif c["place"] == "tree":
        i = torch.arange(t, device="cuda")
        lag = (torch.rand((b, t), generator=g, device="cuda") * 2).long()
        s["parent"] = torch.where(i == 0, -1, (((i - 1).clamp(min=0) // 3).expand(b, t) - lag).clamp(min=0)).to(torch.int32).contiguous()
        s["n_nodes"] = torch.full((b,), t, dtype=torch.int32, device="cuda")
    if own:
        from paper_2608_08097_b200 import binding, rotary
        s["dims"] = binding.Dims(b, hq, h, 1)
        scaling = {"none": None, "linear": dict(kind="linear", factor=8.0), "yarn": dict(kind="yarn", factor=8.0, trained=4096)}[c["scaling"]]
        s["table"] = rotary.RotaryTable(c["rot"], interleaved=c["interleaved"], scaling=scaling)
    return s


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"pack": _prepare_pack, "attn": _prepare_attn, "rotate": _prepare_rotate}[c["op"]](c, g)


# ---- plain forms --------------------------------------------------------------------------------------------------
def _scale_of(byte):
    """The scale that a byte stands for (fp32, exact)."""
    return torch.ldexp(1 + (byte & 7).float() / 8, (byte >> 3).to(torch.int32) - 20)


def _quantise(x):
    """x [..., 16] fp32: the whole numbers q that q * s stands for (fp32), and the scale's byte [...]."""
    x = torch.where(x.isnan(), 0.0, x)
    mant, expo = torch.frexp(x.abs().amax(-1).double() / 7)            # a / 7 = mant * 2^expo, mant in [1/2, 1)
    step = torch.round(mant * 16).to(torch.int64)                      # 8 .. 16: four significant bits, ties to even
    byte = ((expo.to(torch.int64) - 1 + 20) * 8 + step - 8).clamp(0, 255)
    byte = torch.where(x.isinf().any(-1), 255, torch.where((x == 0).all(-1), 0, byte))
    s = _scale_of(byte)[..., None]
    q = sum((x.abs() > (k + 0.5) * s).float() for k in range(7))
    return torch.copysign(q, x), byte


def _plain_pack(s):
    h, at, out = s["case"]["kv_heads"], s["at"], []
    s["summaries"].zero_()
    for i in range(0, at.shape[0], 512):
        a = at[i:i + 512]
        kv = s["pool"][s["src"][a[:, 0], a[:, 1]].long()].float()      # [n][Hkv][2][16][128]
        k, v = kv[:, :, 0], kv[:, :, 1].transpose(2, 3)
        got = []
        for x in (k, v):
            q, byte = _quantise(x.unflatten(-1, (-1, 16)))
            got.append((q * _scale_of(byte)[..., None]).flatten(-2))
        out.append(torch.stack([got[0], got[1].transpose(2, 3)], 2).flatten(0, 1).to(torch.bfloat16))
        s["summaries"][a[:, 0], :, a[:, 1]] = torch.stack([k.amin(2), k.amax(2)], 2).to(torch.bfloat16)
    return torch.cat(out) if out else s["out"], s["summaries"]


def _codes(words):
    """[..., 4 n] bytes -> [..., 8 n] whole numbers in fp32."""
    w = words.unflatten(-1, (-1, 4)).to(torch.int64)
    w = w[..., 0] | w[..., 1] << 8 | w[..., 2] << 16 | w[..., 3] << 24
    return torch.stack([(w >> (4 * p + 16 * hi)) & 15 for p in range(4) for hi in range(2)], -1).flatten(-2).float() - 8


def _plain_values(e):
    """[..., 2304] bytes -> keys and values [..., 16][128] fp32."""
    k = _codes(e[..., :1024].unflatten(-1, (4, BLK, 16))).transpose(-3, -2)                  # [..., 16][4][32]
    k = k.unflatten(-1, (2, 16)) * _scale_of(e[..., 2048:2176].long().unflatten(-1, (BLK, 4, 2)))[..., None]
    v = _codes(e[..., 1024:2048].unflatten(-1, (D, 8))) * _scale_of(e[..., 2176:].long())[..., None]
    return k.flatten(-3), v.transpose(-1, -2)


def _plain_attn(s):
    c, q, tbl = s["case"], s["q"].float(), s["blk_tbl"].long()
    b, t, hq, _ = q.shape
    h, k_cols = c["kv_heads"], c["budget"]
    g = hq // h
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    now = torch.arange(t, device=q.device)
    for i in range(b):
        keys, vals = _plain_values(s["packed"][s["slot_tbl"][i, :, :k_cols].long()])          # [h][cols][16][128]
        loc = s["local"][s["slot_tbl"][i, :, k_cols:].long()].float()
        keys = torch.cat([keys, loc[:, :, 0]], 1).flatten(1, 2)
        vals = torch.cat([vals, loc[:, :, 1]], 1).flatten(1, 2)
        pos = tbl[i, :, :, None] * BLK + torch.arange(BLK, device=q.device)
        sees = ((tbl[i] >= 0)[..., None] & torch.ones_like(pos, dtype=torch.bool)).flatten(1)[:, None] & (
            pos.flatten(1)[:, None] <= (s["seq_len"][i].long() + now)[:, None])               # [h][t][keys]
        rows = q[i].view(t, h, g, D).permute(1, 0, 2, 3).reshape(h, t * g, D)
        logit = (rows @ keys.transpose(1, 2)).view(h, t, g, -1) * SCALE
        logit = torch.where(sees[:, :, None], logit, -math.inf)
        top = logit.amax(-1, keepdim=True)
        e = torch.where(sees[:, :, None], torch.exp(logit - top), 0.0)
        den = e.sum(-1, keepdim=True)
        o = (e.view(h, t * g, -1) @ vals).view(h, t, g, D) / torch.where(den > 0, den, 1.0)
        out[i] = o.permute(1, 0, 2, 3).reshape(t, hq, D).to(torch.bfloat16)
        lse[i] = torch.where(den > 0, top + torch.log(den), -math.inf)[..., 0].permute(1, 0, 2).reshape(t, hq)
    return out, lse


def _depth(parent):
    """[B][T]: how many ancestors a node has."""
    depth, at = torch.zeros_like(parent, dtype=torch.int64), parent.long()
    for _ in range(parent.shape[1]):
        depth = depth + (at >= 0)
        at = torch.where(at >= 0, torch.gather(parent.long(), 1, at.clamp(min=0)), -1)
    return depth


def _plain_rotate(s):
    c = s["case"]
    b, hq, h, t, r = c["batch"], c["q_heads"], c["kv_heads"], c["tokens"], c["rot"]
    x = s["qkv"].float().view(b, t, hq + 2 * h, D)
    if s["positions"] is not None:
        pos = s["positions"].double()
    elif s["parent"] is not None:
        pos = (s["seq_len"].long()[:, None] + _depth(s["parent"])).double()
    else:
        pos = (s["seq_len"].long()[:, None] + torch.arange(t, device=x.device)).double()
    angle = pos[:, :, None, None] * s["freqs"]                          # [b][t][1][r / 2], 64 bits: far positions
    cos, sin = torch.cos(angle).float() * s["factor"], torch.sin(angle).float() * s["factor"]
    y = x.clone()
    if c["interleaved"]:
        lo, hi = x[:, :, :hq + h, 0:r:2], x[:, :, :hq + h, 1:r:2]
        y[:, :, :hq + h, 0:r:2], y[:, :, :hq + h, 1:r:2] = lo * cos - hi * sin, hi * cos + lo * sin
    else:
        lo, hi = x[:, :, :hq + h, :r // 2], x[:, :, :hq + h, r // 2:r]
        y[:, :, :hq + h, :r // 2], y[:, :, :hq + h, r // 2:r] = lo * cos - hi * sin, hi * cos + lo * sin
    y = y.to(torch.bfloat16)
    return y[:, :, :hq].contiguous(), torch.stack([y[:, :, hq:hq + h], y[:, :, hq + h:]], 3)


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2608_08097_b200 import binding
        if op == "pack":
            binding.pack_blocks(s["dims"], s["pool"], s["src"], s["first"], s["n_blocks"], s["case"]["blocks"], s["packed"], s["dst"],
                                summaries=s["summaries"])
            binding.unpack_blocks(s["packed"], s["idx"], s["out"])
            return s["out"], s["summaries"]
        if op == "attn":
            binding.packed_attn(s["dims"], s["q"], s["packed"], s["local"], s["slot_tbl"], s["blk_tbl"], s["case"]["budget"], s["seq_len"],
                                SCALE, s["out"], lse=s["lse"], workspace=s["workspace"])
            return s["out"], s["lse"]
        binding.rotate_qkv(s["dims"], s["qkv"], s["table"], s["q"], s["kv"], seq_len=s["seq_len"], positions=s["positions"],
                           parent=s["parent"], n_nodes=s["n_nodes"])
        return s["q"], s["kv"]
    return {"pack": _plain_pack, "attn": _plain_attn, "rotate": _plain_rotate}[op](s)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def _nearest(x):
    """x [..., 16] in 64 bits: every value by the nearest whole multiple of its group's scale (halfway: the smaller one)."""
    a = x.abs().amax(-1, keepdim=True) / 7
    unit = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -20))) - 3)
    unit = torch.where(a >= 16 * unit, 2 * unit, torch.where(a < 8 * unit, unit / 2, unit))    # (where log2 was off by its last bit)
    s = (torch.round(a / unit) * unit).clamp(2.0 ** -20, 3840.0)
    return torch.sign(x) * torch.ceil(x.abs() / s - 0.5).clamp(0, 7) * s


def _exact_pack(s):
    out, summ = [], torch.zeros_like(s["summaries"], dtype=torch.float64)
    for a in s["at"].split(256):
        kv = s["pool"][s["src"][a[:, 0], a[:, 1]].long()].double()
        k = _nearest(kv[:, :, 0].reshape(*kv.shape[:2], BLK, 8, 16)).reshape(*kv.shape[:2], BLK, D)
        v = _nearest(kv[:, :, 1].movedim(-2, -1)).movedim(-1, -2)
        out.append(torch.stack((k, v), 2).reshape(-1, 2, BLK, D))
        summ[a[:, 0], :, a[:, 1]] = torch.stack((kv[:, :, 0].min(2).values, kv[:, :, 0].max(2).values), 2)
    return torch.cat(out) if out else s["out"].double(), summ


def _exact_entries(e):
    """[n][2304] -> keys, values [n][16][128] in 64 bits, code by code through an index of places."""
    dim, tok = torch.arange(D, device=e.device), torch.arange(BLK, device=e.device)[:, None]

    def values(byte0, order, scale_at):
        byte = e[:, byte0 + order // 8 * 4 + order % 2 * 2 + order % 8 // 4].long()            # two codes a byte, pairs 16 bits apart
        code = (byte >> (4 * (order % 4 // 2))) & 15
        b = e[:, scale_at].double()
        return (code.double() - 8) * (8 + b % 8) * 2.0 ** (torch.floor(b / 8) - 23)

    k = values(tok * 16 + dim // 32 * 256, dim % 32 + 0 * tok, 2048 + 8 * tok + dim // 16)
    v = values(1024 + 8 * dim + 0 * tok, tok + 0 * dim, 2176 + dim + 0 * tok)
    return k, v


def _exact_attn(s):
    c, q = s["case"], s["q"].double()
    b, t, hq, _ = q.shape
    h, g = c["kv_heads"], hq // c["kv_heads"]
    out, lse = torch.zeros((b, t, hq, D), dtype=torch.float64, device=q.device), torch.full((b, t, hq), -math.inf, dtype=torch.float64, device=q.device)
    for i in range(b):
        n = int(s["seq_len"][i])
        for j in range(h):
            ids, slots = s["blk_tbl"][i, j].long(), s["slot_tbl"][i, j].long()
            far, near = (ids >= 0) & (torch.arange(ids.numel(), device=q.device) < c["budget"]), ids >= 0
            near[:c["budget"]] = False
            if not bool(far.any() | near.any()):
                continue
            k, v = _exact_entries(s["packed"][slots[far]])
            loc = s["local"][slots[near]].double()
            k, v = torch.cat([k, loc[:, 0]]).reshape(-1, D), torch.cat([v, loc[:, 1]]).reshape(-1, D)
            pos = (torch.cat([ids[far], ids[near]])[:, None] * BLK + torch.arange(BLK, device=q.device)).reshape(-1)
            z = torch.einsum("tgd,kd->tgk", q[i, :, j * g:(j + 1) * g], k) * SCALE
            z = z.masked_fill((pos > n + torch.arange(t, device=q.device)[:, None])[:, None], -math.inf)
            lse[i, :, j * g:(j + 1) * g] = torch.logsumexp(z, -1)
            out[i, :, j * g:(j + 1) * g] = torch.einsum("tgk,kd->tgd", torch.softmax(z, -1), v)
    return out, lse


def _exact_rotate(s):
    c = s["case"]
    b, hq, h, t, r = c["batch"], c["q_heads"], c["kv_heads"], c["tokens"], c["rot"]
    lens = s["seq_len"].cpu().numpy().astype(np.float64)
    if c["place"] == "given":
        pos = s["positions"].cpu().numpy().astype(np.float64)
    else:
        pos = np.repeat(lens[:, None], t, 1)
        for j in range(1, t):
            pos[:, j] = pos[:, j - 1] + 1 if c["place"] == "chain" else pos[np.arange(b), s["parent"][:, j].cpu().numpy()] + 1
    f, factor = _frequencies(c)
    turn = torch.tensor(factor * np.exp(1j * pos[:, :, None] * f), device="cuda")[:, :, None]  # [b][t][1][r / 2] complex
    x = s["qkv"].double().view(b, t, hq + 2 * h, D).clone()
    part = x[:, :, :hq + h, :r]
    pair = part.unflatten(-1, (r // 2, 2)) if c["interleaved"] else part.unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * turn)
    x[:, :, :hq + h, :r] = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return x[:, :, :hq], torch.stack([x[:, :, hq:hq + h], x[:, :, hq + h:]], 3)


def exact(c, seed):
    s = prepare(c, seed)
    return {"pack": _exact_pack, "attn": _exact_attn, "rotate": _exact_rotate}[c["op"]](s)
