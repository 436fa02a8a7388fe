"""The draft-tree operators in plain numpy, double precision: attention of a tree over a working set, the choice of the
kept path, and the write of the kept rows.  Written from their definitions; loops, no shared code with the product."""
import math

import numpy as np


def bf16(bits):
    """uint16 bf16 patterns -> float64."""
    return (np.ascontiguousarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def ancestors(parent, t):
    """The nodes that node t sees inside the tree: itself and its ancestors (a parent outside [0, t) ends the line)."""
    line = [t]
    while 0 <= parent[line[-1]] < line[-1]:
        line.append(int(parent[line[-1]]))
    return line


def tree_attn(q, tree_kv, parent, n_nodes, pool, slot_tbl, blk_tbl, seq_len, scale, out, lse):
    """q [B][T][Hq][128], tree_kv [B][T][Hkv][2][128], pool [slots][2][16][128] float64; out and lse float64 are
    updated for the live nodes, out_abs (sum of weight * |value|, for error bounds) is returned."""
    B, T, Hq, _ = q.shape
    Hkv = tree_kv.shape[2]
    out_abs = np.zeros_like(out)
    for b in range(B):
        for t in range(max(0, min(int(n_nodes[b]), T))):
            line = ancestors(parent[b], t)
            for h in range(Hkv):
                keys, vals = [tree_kv[b, u, h, 0] for u in line], [tree_kv[b, u, h, 1] for u in line]
                for c in range(blk_tbl.shape[2]):
                    j = int(blk_tbl[b, h, c])
                    n = 0 if j < 0 else max(0, min(16, int(seq_len[b]) - 16 * j))
                    keys.extend(pool[slot_tbl[b, h, c], 0, :n])
                    vals.extend(pool[slot_tbl[b, h, c], 1, :n])
                keys, vals = np.array(keys), np.array(vals)
                for a in range(h * Hq // Hkv, (h + 1) * Hq // Hkv):
                    z = keys @ q[b, t, a] * scale
                    w = np.exp(z - z.max())
                    out[b, t, a] = w @ vals / w.sum()
                    out_abs[b, t, a] = w @ np.abs(vals) / w.sum()
                    lse[b, t, a] = z.max() + math.log(w.sum())
    return out_abs


def distribution(row, temperature):
    """softmax(row / temperature); NaN and -inf leave a token out, +inf shares everything; None: nothing is left."""
    x = np.where(np.isnan(row), -np.inf, row.astype(np.float64))
    m = x.max()
    if m == -np.inf:
        return None
    with np.errstate(invalid="ignore"):
        w = np.where(x == m, 1.0, np.exp((x - m) / float(temperature)))
    return w / w.sum()


def verify_tree(logits, tokens, parent, n_nodes, uniforms, temperature, max_path, draft=None):
    """logits [B][T][V] float64; -> path [B][max_path], n_commit [B], next_token [B]."""
    B, T, V = logits.shape
    path, count, token = np.full((B, max_path), -1, np.int32), np.zeros(B, np.int32), np.full(B, -1, np.int32)
    u = np.clip(np.nan_to_num(uniforms.astype(np.float64), nan=0.0), 0.0, 1.0 - 2.0 ** -24)
    for b in range(B):
        n = max(0, min(int(n_nodes[b]), T))
        if n == 0:
            continue
        walk, nxt = [0], -1
        while True:
            cur, step = walk[-1], None
            kids = [c for c in range(cur + 1, n) if parent[b, c] == cur] if len(walk) < max_path else []
            row = logits[b, cur]
            if not temperature[b] > 0:
                row = np.where(np.isnan(row), -np.inf, row)
                nxt = int(np.argmax(row)) if row.max() > -np.inf else -1
                step = next((c for c in kids if nxt >= 0 and tokens[b, c] == nxt), None)
            else:
                p = distribution(row, temperature[b])
                if p is None:
                    nxt = -1
                    break
                for c in kids:
                    v = int(tokens[b, c])
                    inside = 0 <= v < V
                    if draft is None:
                        q = np.zeros(V)
                        if inside:
                            q[v] = 1.0
                    else:
                        q = draft[b, cur].astype(np.float64)
                    if inside and u[b, c] * q[v] < p[v]:
                        step = c
                        break
                    rest = np.maximum(p - q, 0.0)
                    if rest.sum() > 0:
                        p = rest / rest.sum()
                if step is None:
                    run = np.cumsum(p)
                    at = np.nonzero((run > u[b, 0] * run[-1]) & (p > 0))[0]
                    nxt = int(at[0]) if len(at) else int(np.nonzero(p > 0)[0][-1])
            if step is None:
                break
            walk.append(step)
        path[b, :len(walk)], count[b], token[b] = walk, len(walk), nxt
    return path, count, token


def commit_kv(tree_kv, path, n_commit, seq_len, block_table, slot_tbl, blk_tbl, local_col, pool, host_kv, next_len):
    """All arrays are written in place (pool [slots][2][16][128], host_kv [P][Hkv][2][16][128] or None)."""
    B, T, Hkv = tree_kv.shape[:3]
    mb = block_table.shape[1]
    for b in range(B):
        n, L = max(0, min(int(n_commit[b]), path.shape[1])), int(seq_len[b])
        next_len[b] = L + n
        for h in range(Hkv):
            if n > 0:
                lo, hi = L // 16, (L + n - 1) // 16
                blk_tbl[b, h, local_col + lo % 2] = lo
                blk_tbl[b, h, local_col + 1 - lo % 2] = hi if hi > lo else -1
            for i in range(n):
                t, j, r = int(path[b, i]), (L + i) // 16, (L + i) % 16
                if not 0 <= t < T or j >= mb:
                    continue
                slot = int(slot_tbl[b, h, local_col + j % 2])
                for part in range(2):
                    if slot >= 0:
                        pool[slot, part, r] = tree_kv[b, t, h, part]
                    if host_kv is not None:
                        host_kv[block_table[b, j], h, part, r] = tree_kv[b, t, h, part]
