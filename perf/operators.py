"""Cases and plain forms of the operators that verify a tree of drafted tokens: attention of the tree over the
resident working set (`tree_attn`), the choice of the accepted path (`verify_tree`) and the write of the accepted
path's keys and values into the cache (`commit_kv_layers`).

`run` computes each operator in elementary torch operations where `own` is false and calls the library where it is true.
"""
import math

import numpy as np
import torch

own = False

D, BLK = 128, 16
SCALE = 1.0 / math.sqrt(128.0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CHILDREN = 3                # a draft tree's nodes have about this many children


# ---- cases --------------------------------------------------------------------------------------------------------
def listed():
    return [
        # attention -----------------------------------------------------------------------------------------------
        # a request that has just begun: a short history, all of it attended, one verified token and four drafts
        dict(name="attn first tokens", op="attn", batch=1, q_heads=32, kv_heads=8, nodes=5, context=200, budget=16, ragged=False),
        # the reasoning-style step: 32 K context, 2,048-token budget, a small draft tree
        dict(name="attn reasoning, 16 nodes", op="attn", batch=16, q_heads=32, kv_heads=8, nodes=16, context=32768, budget=128, ragged=False),
        # the same budget under a wide tree, more query rows than one tensor-core tile has
        dict(name="attn reasoning, 64 nodes", op="attn", batch=16, q_heads=32, kv_heads=8, nodes=64, context=32768, budget=128, ragged=False),
        # eight query heads per KV head, odd node count, requests of different lengths and tree sizes, one empty
        dict(name="attn group of 8, ragged", op="attn", batch=7, q_heads=32, kv_heads=4, nodes=13, context=50003, budget=300, ragged=True),
        # every block of a long cache: a budget that covers the whole history
        dict(name="attn whole long cache", op="attn", batch=2, q_heads=32, kv_heads=8, nodes=8, context=65536, budget=4096, ragged=False),
        # verification --------------------------------------------------------------------------------------------
        # one request, a chain, greedy decoding, a 32 K vocabulary: latency
        dict(name="verify greedy chain, one", op="verify", batch=1, nodes=5, vocab=32000, dtype="bf16", shape="chain", drafts="none", temperature=0.0),
        # sampling with the draft model's probabilities at hand
        dict(name="verify sampled chain", op="verify", batch=16, nodes=5, vocab=128256, dtype="f32", shape="chain", drafts="probs", temperature=1.0),
        # a wide tree of top-ranked drafts
        dict(name="verify tree of 64", op="verify", batch=16, nodes=64, vocab=151936, dtype="bf16", shape="tree", drafts="none", temperature=0.7),
        # many requests, a vocabulary whose rows are not aligned
        dict(name="verify many, odd vocabulary", op="verify", batch=128, nodes=6, vocab=50257, dtype="f16", shape="tree", drafts="none", temperature=1.0),
        # commit --------------------------------------------------------------------------------------------------
        # one layer, one request: latency
        dict(name="commit one layer", op="commit", layers=1, batch=1, kv_heads=8, nodes=5, path=5),
        # all layers of the reasoning-style step at once
        dict(name="commit 32 layers", op="commit", layers=32, batch=16, kv_heads=8, nodes=16, path=8),
        # a large batch with a wide tree, odd sizes
        dict(name="commit wide tree", op="commit", layers=9, batch=61, kv_heads=4, nodes=64, path=13),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "verify", "verify", "commit"])
    if op == "attn":
        group, kv = rng.choice([1, 2, 3, 4, 5, 8, 16]), rng.choice([1, 2, 3, 4, 8])
        c = dict(op="attn", batch=_log(rng, 1, 48), q_heads=group * kv, kv_heads=kv, nodes=rng.randint(1, 64),
                 context=_log(rng, 1, 65536), budget=_log(rng, 4, 1024), ragged=rng.random() < 0.7)
        while work(c)["flops"] > 3e10 or work(c)["bytes"] > 500e6:
            c["batch" if c["batch"] > 1 else "budget"] //= 2
        return c
    if op == "verify":
        c = dict(op="verify", batch=_log(rng, 1, 128), nodes=rng.randint(1, 64), vocab=_log(rng, 100, 152000),
                 dtype=rng.choice(["f32", "bf16", "f16"]), shape=rng.choice(["chain", "tree"]),
                 drafts=rng.choice(["none", "none", "probs"]), temperature=rng.choice([0.0, 0.5, 0.8, 1.0, 1.3]))
        while c["batch"] > 1 and c["batch"] * c["nodes"] * c["vocab"] > 150e6:
            c["batch"] //= 2
        return c
    c = dict(op="commit", layers=rng.randint(1, 40), batch=_log(rng, 1, 64), kv_heads=rng.choice([1, 2, 3, 4, 8]),
             nodes=rng.randint(1, 64), path=rng.randint(1, 16))
    while c["layers"] > 1 and c["layers"] * c["batch"] * c["kv_heads"] > 4096:
        c["layers"] //= 2
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


def _node_counts(c):
    """Nodes of each request's tree; ragged: fewer, and none for the last request (a padded place of the batch)."""
    t, b = c["nodes"], c["batch"]
    if not c["ragged"]:
        return [t] * b
    got = [max(1, t - (3 * i) % t) for i in range(b)]
    if b > 3:
        got[-1] = 0
    return got


def _path_lengths(c):
    """Tokens that each request keeps: from none to the whole path."""
    return [(c["path"] - i) % (c["path"] + 1) for i in range(c["batch"])]


def _commit_start(i, c):
    return 16 * (i % 3 + 1) + (7 * i + 3) % 16


def work(c):
    if c["op"] == "attn":
        h, g, t = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["nodes"]
        rows = moved = flops = 0
        for n, m in zip(_lengths(c), _node_counts(c)):
            if m == 0:
                continue
            blocks = min(c["budget"], n // BLK) + (n % BLK > 0)
            keys = min(c["budget"], n // BLK) * BLK + n % BLK + m
            moved += h * (blocks * 8192 + m * 512)
            rows += m * h * g
            flops += 4 * D * m * g * h * keys
        return {"bytes": moved + rows * (2 * D * 2 + 4), "flops": flops}
    if c["op"] == "verify":
        # the rows of the visited nodes: the walk stops where every child is rejected.  About 7 of 10 drafts of a
        # greedy tree are kept, half of the sampled ones, 9 of 10 of those drawn from a close draft distribution.
        keep = 0.7 if c["temperature"] == 0 else 0.9 if c["drafts"] == "probs" else 0.5
        depth = c["nodes"] if c["shape"] == "chain" else 4
        visited = sum(keep ** k for k in range(min(depth, c["nodes"], 16)))
        size = DTYPES[c["dtype"]].itemsize
        per = visited * c["vocab"] * size
        if c["drafts"] == "probs" and c["temperature"] > 0 and c["nodes"] > 1:
            per += c["vocab"] * 4              # the draft distribution of the node whose children were rejected
        return {"bytes": c["batch"] * per, "flops": c["batch"] * visited * c["vocab"] * 4}
    kept = sum(_path_lengths(c))
    return {"bytes": c["layers"] * c["kv_heads"] * kept * 512 * 3, "flops": 0}


# ---- inputs -------------------------------------------------------------------------------------------------------
def _randn(shape, g, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _tree(c, g, shape):
    """parent [B][T]: a chain, or a tree whose nodes come level by level with up to three children each."""
    b, t = c["batch"], c["nodes"]
    i = torch.arange(t, device="cuda")
    if shape == "chain":
        p = (i - 1).expand(b, t)
    else:
        lag = (torch.rand((b, t), generator=g, device="cuda") * 2).long()
        p = ((i - 1).clamp(min=0) // CHILDREN).expand(b, t) - lag
        p = torch.where(i == 0, -1, p.clamp(min=0))
    return p.to(torch.int32).contiguous()


def _prepare_attn(c, g):
    b, hq, h, t, k = c["batch"], c["q_heads"], c["kv_heads"], c["nodes"], c["budget"]
    lens = torch.tensor(_lengths(c), device="cuda")
    cols = k + 2
    n_full = lens // BLK
    most = max(1, int(max(_lengths(c)) // BLK))
    # the resident blocks of a row: distinct full blocks in no particular order, then the two local columns
    rank = torch.rand((b, h, most), generator=g, device="cuda")
    rank = rank.masked_fill(torch.arange(most, device="cuda") >= n_full[:, None, None], 2.0)
    order = rank.argsort(dim=-1)[..., :k]
    tbl = torch.full((b, h, cols), -1, dtype=torch.int64, device="cuda")
    tbl[..., :order.shape[-1]] = torch.where(torch.arange(order.shape[-1], device="cuda") < n_full[:, None, None], order, -1)
    part = torch.where(lens % BLK > 0, n_full, -1)[:, None]
    even = (n_full % 2 == 0)[:, None]
    tbl[..., k] = torch.where(even, part, -1)
    tbl[..., k + 1] = torch.where(even, -1, part)
    slots = torch.arange(b * h * cols, device="cuda").view(b, h, cols)
    pool = torch.empty((b * h * cols, 2, BLK, D), dtype=torch.bfloat16, device="cuda")
    for i in range(0, b * h * cols, 1 << 16):
        pool[i:i + (1 << 16)] = _randn((min(1 << 16, b * h * cols - i), 2, BLK, D), g)
    s = dict(case=c, pool=pool, slot_tbl=slots.to(torch.int32), blk_tbl=tbl.to(torch.int32), seq_len=lens.to(torch.int32),
             q=_randn((b, t, hq, D), g, scale=2.0), tree_kv=_randn((b, t, h, 2, D), g),
             parent=_tree(c, g, "tree"), n_nodes=torch.tensor(_node_counts(c), dtype=torch.int32, device="cuda"),
             out=torch.zeros((b, t, hq, D), dtype=torch.bfloat16, device="cuda"),
             lse=torch.zeros((b, t, hq), dtype=torch.float32, device="cuda"))
    if own:
        from paper_2608_08097_b200 import binding
        s["dims"] = binding.Dims(b, hq, h, max(1, (max(_lengths(c)) + BLK) // BLK))
        s["workspace"] = torch.empty(max(16, binding.tree_attn_workspace_bytes(s["dims"], t, cols)), dtype=torch.uint8, device="cuda")
    return s


def _prepare_verify(c, g):
    b, t, v = c["batch"], c["nodes"], c["vocab"]
    dt = DTYPES[c["dtype"]]
    # a row: a broad bulk and a few likely tokens, as a language model's logits have
    logits = torch.empty((b, t, v), dtype=dt, device="cuda")
    for i in range(b):
        logits[i] = _randn((t, v), g, torch.float32, 2.0).to(dt)
    likely = (torch.rand((b, t, 4), generator=g, device="cuda") * v).long()
    lift = 8 + 8 * torch.rand((b, t, 4), generator=g, device="cuda")
    logits.scatter_(2, likely, lift.to(dt))
    parent = _tree(c, g, c["shape"])
    at = parent.long().clamp(min=0)
    s = dict(case=c, logits=logits, parent=parent, n_nodes=torch.full((b,), t, dtype=torch.int32, device="cuda"),
             uniforms=torch.rand((b, t), generator=g, device="cuda"),
             temperature=torch.full((b,), c["temperature"], device="cuda"))
    if c["drafts"] == "probs":
        # the draft model: the target's logits with noise; the drafts are drawn from it
        q = torch.empty((b, t, v), dtype=torch.float32, device="cuda")
        tok = torch.empty((b, t), dtype=torch.int64, device="cuda")
        for i in range(b):
            q[i] = torch.softmax(logits[i].float() / max(c["temperature"], 0.5) + _randn((t, v), g, torch.float32, 0.5), dim=-1)
            tok[i] = torch.multinomial(q[i][at[i]], 1, generator=g)[:, 0]
        s["draft_probs"] = q
    else:
        # the r-th child of a node drafts one of the likely tokens, three times in ten another one
        nth = torch.arange(t, device="cuda") % CHILDREN if c["shape"] == "tree" else torch.zeros(t, dtype=torch.int64, device="cuda")
        lift_at = torch.gather(logits, 2, likely).float().argsort(dim=-1, descending=True)
        ranked = torch.gather(likely, 2, lift_at)
        tok = torch.gather(ranked, 1, at[..., None].expand(b, t, 4)).gather(2, nth.expand(b, t)[..., None])[..., 0]
        other = (torch.rand((b, t), generator=g, device="cuda") * v).long()
        tok = torch.where(torch.rand((b, t), generator=g, device="cuda") < 0.3, other, tok)
        s["draft_probs"] = None
    s["tokens"] = tok.to(torch.int32)
    m = min(t, 16)
    s.update(path=torch.zeros((b, m), dtype=torch.int32, device="cuda"), n_commit=torch.zeros(b, dtype=torch.int32, device="cuda"),
             next_token=torch.zeros(b, dtype=torch.int32, device="cuda"))
    return s


def _prepare_commit(c, g):
    n, b, h, t, m = c["layers"], c["batch"], c["kv_heads"], c["nodes"], c["path"]
    cols, mb = 6, 8
    start = torch.tensor([_commit_start(i, c) for i in range(b)], device="cuda")
    pick = torch.rand((b, m), generator=g, device="cuda")
    path = (pick * t).long().sort(dim=1).values
    keep = torch.tensor(_path_lengths(c), device="cuda")
    path = torch.where(torch.arange(m, device="cuda") < keep[:, None], path, -1)
    s = dict(case=c, tree_kv=_randn((n, b, t, h, 2, D), g), path=path.to(torch.int32), n_commit=keep.to(torch.int32),
             seq_len=start.to(torch.int32),
             block_table=torch.rand((n, b * mb), generator=g, device="cuda").argsort(dim=1).view(n, b, mb).to(torch.int32),
             slot_tbl=torch.arange(b * h * cols, device="cuda").view(b, h, cols).expand(n, b, h, cols).to(torch.int32).contiguous(),
             blk_tbl=torch.full((n, b, h, cols), -1, dtype=torch.int32, device="cuda"), local_col=cols - 2,
             pool=torch.zeros((n, b * h * cols, 2, BLK, D), dtype=torch.bfloat16, device="cuda"),
             kv=torch.zeros((n, b * mb, h, 2, BLK, D), dtype=torch.bfloat16, device="cuda"),
             next_len=torch.zeros(b, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2608_08097_b200 import binding
        s["plan"] = binding.CommitPlan(binding.Dims(b, h, h, mb), list(s["tree_kv"]), list(s["block_table"]), list(s["slot_tbl"]),
                                       list(s["blk_tbl"]), s["local_col"], list(s["pool"]), list(s["kv"]))
    return s


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"attn": _prepare_attn, "verify": _prepare_verify, "commit": _prepare_commit}[c["op"]](c, g)


# ---- plain forms --------------------------------------------------------------------------------------------------
def _ancestors(parent):
    """[B][T][T] bool: u is t or an ancestor of t (six squarings reach depth 64)."""
    t = parent.shape[1]
    i = torch.arange(t, device=parent.device)
    sees = ((parent[:, :, None] == i) | (i[:, None] == i)).float()
    for _ in range(6):
        sees = (sees @ sees > 0).float()
    return sees > 0


def _plain_attn(s):
    q, kv, tbl = s["q"].float(), s["tree_kv"].float(), s["blk_tbl"].long()
    b, t, hq, _ = q.shape
    h = kv.shape[2]
    entry = s["pool"][s["slot_tbl"].long()].float()                                   # [B][H][cols][2][16][128]
    pos = tbl[..., None] * BLK + torch.arange(BLK, device=q.device)
    old = ((tbl >= 0)[..., None] & (pos < s["seq_len"][:, None, None, None])).flatten(2)
    new = torch.arange(t, device=q.device) < s["n_nodes"][:, None]
    k = torch.cat([entry[:, :, :, 0].flatten(2, 3), kv[:, :, :, 0].transpose(1, 2)], 2)   # [B][H][keys][128]
    v = torch.cat([entry[:, :, :, 1].flatten(2, 3), kv[:, :, :, 1].transpose(1, 2)], 2)
    sees = torch.cat([old[:, :, None].expand(-1, -1, t, -1), (_ancestors(s["parent"]) & new[:, None])[:, None].expand(-1, h, -1, -1)], 3)
    sees = sees[:, :, :, None]                                                        # [B][H][T][1][keys]
    rows = q.view(b, t, h, hq // h, D).permute(0, 2, 1, 3, 4).reshape(b, h, -1, D)
    logit = (rows @ k.transpose(2, 3)).view(b, h, t, hq // h, -1) * SCALE
    logit = torch.where(sees, logit, -math.inf)
    top = logit.amax(-1, keepdim=True)
    e = torch.where(sees, torch.exp(logit - top), 0.0)
    den = e.sum(-1, keepdim=True)
    out = (e.view(b, h, -1, k.shape[2]) @ v).view(b, h, t, hq // h, D) / torch.where(den > 0, den, 1.0)
    lse = torch.where(den > 0, top + torch.log(den), -math.inf)[..., 0]
    live = new[:, :, None]
    out = torch.where(live[..., None], out.permute(0, 2, 1, 3, 4).reshape(b, t, hq, D).to(torch.bfloat16), s["out"])
    return out, torch.where(live, lse.permute(0, 2, 1, 3).reshape(b, t, hq), s["lse"])


def _plain_verify(s):
    """A node's children come after it, and siblings are tried in order, so one sweep over the nodes is the whole walk.
    The distribution of the current node is kept in 64 bits: a token goes by where a sum of all probabilities before it ends."""
    tok, parent, u = s["tokens"].long(), s["parent"].long(), s["uniforms"].double()
    b, t = tok.shape
    m = s["path"].shape[1]
    x = s["logits"].double()
    greedy = s["case"]["temperature"] == 0
    draft = s["draft_probs"]
    row = torch.arange(b, device=tok.device)
    cur = torch.zeros_like(row)
    n = torch.ones_like(row)
    path = torch.full_like(s["path"], -1)
    path[:, 0] = 0
    if greedy:
        best = x.argmax(-1)
    else:
        x = torch.exp((x - x.amax(-1, keepdim=True)) / s["temperature"].double()[:, None, None])
        x = x / x.sum(-1, keepdim=True)
        left = x[:, 0].clone()                                                        # what is left of the current node's distribution
    for c in range(1, t):
        child = (parent[:, c] == cur) & (n < m)
        if greedy:
            take = child & (tok[:, c] == best[row, cur])
        elif draft is None:
            share = left[row, tok[:, c]]
            whole = left.sum(-1) if c == 1 else whole
            take = child & (u[:, c] * whole < share)
            away = child & ~take
            left[row, tok[:, c]] = torch.where(away, 0.0, share)
            whole = torch.where(away, whole - share, whole)
        else:
            qc = draft[row, cur].double()
            take = child & (u[:, c] * qc[row, tok[:, c]] < left[row, tok[:, c]])
            rest = (left - qc).clamp(min=0)
            mass = rest.sum(-1, keepdim=True)
            left = torch.where(((child & ~take)[:, None]) & (mass > 0), rest / mass, left)
        cur = torch.where(take, c, cur)
        path[row, torch.where(take, n, 0)] = torch.where(take, c, 0).to(torch.int32)
        n = n + take
        if not greedy:
            left = torch.where(take[:, None], x[:, c], left)
            whole = torch.where(take, x[:, c].sum(-1), whole) if draft is None else None
    if greedy:
        return path, n.to(torch.int32), best[row, cur].to(torch.int32)
    run_sum = left.cumsum(-1)
    token = (run_sum > u[:, :1] * run_sum[:, -1:]).byte().argmax(-1)
    return path, n.to(torch.int32), token.to(torch.int32)


def _plain_commit(s):
    n, b, t, h = s["tree_kv"].shape[:4]
    m, dev = s["path"].shape[1], s["path"].device
    i = torch.arange(m, device=dev)
    live = i < s["n_commit"][:, None]                                                 # [B][M]
    pos = s["seq_len"].long()[:, None] + i
    blk, off = pos // BLK, pos % BLK
    layer = torch.arange(n, device=dev)[:, None, None, None]
    head = torch.arange(h, device=dev)[:, None]
    req = torch.arange(b, device=dev)[:, None, None]
    rows = s["tree_kv"][:, req[:, :, 0], s["path"].long().clamp(min=0)].transpose(2, 3)   # [n][B][H][M][2][128]
    slot = s["slot_tbl"].long()[layer, req, head, s["local_col"] + (blk & 1)[:, None]]    # [n][B][H][M]
    pick = live[None, :, None, :, None, None]
    o = off[:, None].expand(b, h, m)
    now = s["pool"][layer, slot, :, o]
    s["pool"][layer, slot, :, o] = torch.where(pick, rows, now)                       # a token that is not kept leaves its place as it was
    phys = s["block_table"].long()[layer, req, blk[:, None]]
    now = s["kv"][layer, phys, head, :, o]
    s["kv"][layer, phys, head, :, o] = torch.where(pick, rows, now)
    lo = s["seq_len"].long() // BLK
    last = s["seq_len"].long() + s["n_commit"] - 1
    hi = torch.where(last // BLK > lo, last // BLK, -1)
    even = lo % 2 == 0
    cols = torch.stack([torch.where(even, lo, hi), torch.where(even, hi, lo)], -1).to(torch.int32)[:, None]
    any_kept = (s["n_commit"] > 0)[:, None, None]
    at = s["blk_tbl"][..., s["local_col"]:]
    s["blk_tbl"][..., s["local_col"]:] = torch.where(any_kept, cols, at)
    s["next_len"].copy_(s["seq_len"] + s["n_commit"])
    return s["pool"], s["kv"], s["blk_tbl"], s["next_len"]


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2608_08097_b200 import binding
        if op == "attn":
            binding.tree_attn(s["dims"], s["q"], s["tree_kv"], s["parent"], s["n_nodes"], s["pool"], s["slot_tbl"], s["blk_tbl"],
                              s["seq_len"], SCALE, s["out"], lse=s["lse"], workspace=s["workspace"])
            return s["out"], s["lse"]
        if op == "verify":
            binding.verify_tree(s["logits"], s["tokens"], s["parent"], s["n_nodes"], s["uniforms"], s["temperature"], s["path"],
                                s["n_commit"], s["next_token"], draft_probs=s["draft_probs"])
            return s["path"], s["n_commit"], s["next_token"]
        binding.commit_kv_layers(s["plan"], s["path"], s["n_commit"], s["seq_len"], next_len=s["next_len"])
        return s["pool"], s["kv"], s["blk_tbl"], s["next_len"]
    return {"attn": _plain_attn, "verify": _plain_verify, "commit": _plain_commit}[op](s)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def _exact_attn(s):
    q, kv = s["q"].double(), s["tree_kv"].double()
    b, t, hq, _ = q.shape
    h = kv.shape[2]
    g = hq // h
    out, lse = s["out"].double(), s["lse"].double()
    parent, counts, lens = s["parent"].tolist(), s["n_nodes"].tolist(), s["seq_len"].tolist()
    for i in range(b):
        m = counts[i]
        if m == 0:
            continue
        chains = []
        for node in range(m):
            seen, at = [], node
            while at >= 0:
                seen.append(at)
                at = parent[i][at]
            chains.append(seen)
        sees = torch.zeros((m, m), dtype=torch.bool, device=q.device)
        sees[[n for n, c in enumerate(chains) for _ in c], [x for c in chains for x in c]] = True
        for j in range(h):
            ids = s["blk_tbl"][i, j].long()
            ent = s["pool"][s["slot_tbl"][i, j].long()[ids >= 0]].double()
            p = (ids[ids >= 0][:, None] * BLK + torch.arange(BLK, device=q.device)).reshape(-1)
            ent_k, ent_v = ent[:, 0].reshape(-1, D)[p < lens[i]], ent[:, 1].reshape(-1, D)[p < lens[i]]
            keys = torch.cat([ent_k, kv[i, :m, j, 0]])
            vals = torch.cat([ent_v, kv[i, :m, j, 1]])
            old = torch.ones((m, ent_k.shape[0]), dtype=torch.bool, device=q.device)
            ok = torch.cat([old, sees], 1)[:, None]
            z = torch.einsum("tgd,kd->tgk", q[i, :m, j * g:(j + 1) * g], keys) * SCALE
            z = z.masked_fill(~ok, -math.inf)
            lse[i, :m, j * g:(j + 1) * g] = torch.logsumexp(z, -1)
            out[i, :m, j * g:(j + 1) * g] = torch.einsum("tgk,kd->tgd", torch.softmax(z, -1), vals)
    return out, lse


def _exact_verify(s):
    tok, parent, u = s["tokens"].cpu().numpy(), s["parent"].cpu().numpy(), s["uniforms"].double().cpu().numpy()
    b, t = tok.shape
    m, temp = s["path"].shape[1], s["temperature"].double().cpu().numpy()
    path, n, nxt = np.full((b, m), -1, np.int64), np.zeros(b, np.int64), np.zeros(b, np.int64)
    for i in range(b):
        cur, walk = 0, [0]
        while True:
            row = s["logits"][i, cur].double().cpu().numpy()
            kids = [c for c in range(1, t) if parent[i, c] == cur] if len(walk) < m else []
            step = None
            if temp[i] == 0:
                token = int(np.argmax(row))
                step = next((c for c in kids if tok[i, c] == token), None)
            else:
                p = np.exp((row - row.max()) / temp[i])
                p /= p.sum()
                for c in kids:
                    q = np.zeros_like(p)
                    q[tok[i, c]] = 1.0
                    if s["draft_probs"] is not None:
                        q = s["draft_probs"][i, cur].double().cpu().numpy()
                    if u[i, c] * q[tok[i, c]] < p[tok[i, c]]:
                        step = c
                        break
                    rest = np.maximum(p - q, 0.0)
                    p = rest / rest.sum() if rest.sum() > 0 else p
                acc = np.cumsum(p)
                token = int(np.searchsorted(acc, u[i, 0] * acc[-1], side="right"))
            if step is None:
                break
            cur = step
            walk.append(step)
        path[i, :len(walk)], n[i], nxt[i] = walk, len(walk), token
    return path, n, nxt


def exact(c, seed):
    if c["op"] == "commit":
        return None                            # copies: nothing is computed
    s = prepare(c, seed)
    return (_exact_attn if c["op"] == "attn" else _exact_verify)(s)
