"""Secondary measurements of the sparse-decode path on one B200 (not part of the `bench.py` contract).

    python bench_sweep.py [--what c5,stage,shapes,packed]

Kernels alone (the whole step, every configuration and the fetch-ratio sweep are `bench.py --config / --sweep-ratios`).
Prints one JSON line per section:
  c5      the budget x draft-length sweep (configs[4]): solo kernel times and roofline fractions of
          scoring / top-k / attention and of the fused attention + scoring launch, and lookahead recall per cell.
  stage   the gather kernel alone on random entries of a pinned pool, against the DMA copy peak, and the
          dense -> sparse hand-over (device blocks -> pinned entries + summaries) alone.
  shapes  the kernels alone at the shapes of configs[0] to configs[3] (one layer, random
          summaries and pools): scoring, top-k, attention, and the fused attention + scoring launch where
          it takes the shape, each against the measured copy peak.
  packed  (not run by default) entries in 4 bits beside bf16 ones: the attention kernels on the same rows and columns, the hand-over
          into a pinned pool, and the whole step of the reasoning-style decode (bench.py's default workload) by DecodeEngine with
          kv_bits 16 and 4, with the pool in pinned memory and in HBM (--layers: fewer layers than that workload's).
Inputs are synthetic (the generators of `synth`); nothing here touches the CPU oracle.
"""
import argparse
import json
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, ROOT)

import bench as B                                        # noqa: E402
from paper_2608_08097_b200 import synth                  # noqa: E402


def graph_time(fn, n_rot, iters=32, warm=4):
    """Median of 5 graph replays of `iters` launches rotating over `n_rot` working sets (us per launch)."""
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        for i in range(warm):
            fn(i % n_rot)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        for i in range(iters):
            fn(i % n_rot)
    ts = []
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        g.replay()
        b.record()
        torch.cuda.synchronize()
        ts.append(a.elapsed_time(b) * 1e3 / iters)
    ts.sort()
    return ts[2]


def section_c5(args, dev, hbm_peak):
    """Budget x draft-length sweep: kernels alone (graph replay over rotating working sets) and recall."""
    from paper_2608_08097_b200 import binding, pipeline
    base = synth.scaled(synth.C5, n_draft=8, layers=1, steps=1)
    lay = synth.make_layer(base, seed=args.seed, layer=0, device=dev)
    kv = lay.host_kv.to(dev)
    table, n_full, seq = lay.block_table.to(dev), lay.n_full.to(dev), lay.seq_len.to(dev)
    Bq, Hq, Hkv, mb = base.batch, base.n_q_heads, base.n_kv_heads, base.max_blocks
    zeros = torch.zeros(Bq, dtype=torch.int32, device=dev)
    nf = int(lay.n_full[0])
    n_rot = 3                                                            # 3 x 268 MB of summaries > 2 x L2
    cells = []
    for K in (32, 64, 128, 256, 512):
        for Td in (1, 2, 4, 8):
            T = Td + 1
            Ls = [pipeline.DecodeLayer(Bq, Hq, Hkv, mb, K, T, dev) for _ in range(n_rot)]
            q = lay.q[:, :T].contiguous().to(dev)
            q_true = lay.q_true[:, :Td].contiguous().to(dev)
            for L in Ls:
                L.build_summaries(kv, table, zeros, n_full, mb)
                L.score(q, n_full)
                L.select(n_full, seq, table)
                L.stage(kv)
            torch.cuda.synchronize()
            t_score = graph_time(lambda i: Ls[i].score(q, n_full), n_rot)
            t_sel = graph_time(lambda i: Ls[i].select(n_full, seq, table), n_rot)
            t_attn = graph_time(lambda i: Ls[i].attend(q, seq), n_rot)
            t_layer = None
            if binding.attn_and_score_supported(Ls[0].dims, T, Ls[0].cols, Td):
                t_layer = graph_time(lambda i: Ls[i].attend_and_score(q, seq, n_full), n_rot)
            sel_draft = Ls[0].sel.clone()
            sel_true = torch.empty_like(sel_draft)
            Ls[0].score_queries(q_true, n_full)
            Ls[0].select(n_full, seq, table, sel=sel_true)
            torch.cuda.synchronize()
            a, b = sel_draft[..., :K], sel_true[..., :K]
            recall = (a[..., :, None] == b[..., None, :]).any(-1).float().mean().item()
            sb = Bq * Hkv * nf * 516
            ab = Bq * Hkv * (min(K, nf) + 1) * 8192 + 2 * Bq * T * Hq * 256
            cells.append({"K": K, "Td": Td, "score_us": round(t_score, 1), "score_frac": round(sb / t_score / 1e3 / hbm_peak, 3),
                          "select_us": round(t_sel, 1), "attn_us": round(t_attn, 1),
                          "attn_frac": round(ab / t_attn / 1e3 / hbm_peak, 3),
                          "layer_us": None if t_layer is None else round(t_layer, 1),
                          "layer_frac": None if t_layer is None else round((sb + ab) / t_layer / 1e3 / hbm_peak, 3),
                          "tokens_per_s_per_layer": round(Bq / ((t_score + t_sel + t_attn) * 1e-6), 1),
                          "tokens_per_s_per_layer_fused": None if t_layer is None else round(Bq / ((t_layer + t_sel) * 1e-6), 1),
                          "recall": round(recall, 4)})
            del Ls
            torch.cuda.empty_cache()
    print(json.dumps({"section": "c5", "workload": "configs[4]: batch 16, 32q/8kv heads, context 65536, one layer "
                      "(3 rotating copies of the summaries and pools), kernels alone; frac = algorithmic bytes / time / "
                      "measured copy peak; layer = the fused attention + scoring launch; tokens/s/layer from the serial sum score + "
                      "top-k + attention (and fused launch + top-k)",
                      "hbm_peak_GBps": hbm_peak, "cells": cells}))


def section_stage(args, dev, hbm_peak):
    """The gather kernels alone: random 8 KiB entries of a 2 GiB pinned pool into HBM slots."""
    from paper_2608_08097_b200 import binding as oasis
    h2d_peak = B.time_pinned_h2d(dev)
    P = 262144
    host = torch.empty((P, 2, 16, 128), dtype=torch.bfloat16, pin_memory=True)
    host.view(torch.int16).random_(0, 1000)
    pool = torch.zeros((4 * 16640, 2, 16, 128), dtype=torch.bfloat16, device=dev)
    g = torch.Generator()
    g.manual_seed(args.seed)
    rows = []
    for n, pad in ((896, 1024), (4096, 4096), (16640, 16640)):
        idxs, slots = [], []
        for _ in range(8):
            idx = torch.full((pad,), -1, dtype=torch.int64)
            idx[torch.randperm(pad, generator=g)[:n]] = torch.randint(0, P, (n,), generator=g)
            idxs.append(idx.to(dev))
            slots.append(torch.arange(pad, dtype=torch.int32, device=dev))
        us = graph_time(lambda i: oasis.stage_blocks(host, idxs[i], slots[i], pad, pool), 8, iters=8, warm=8)
        rows.append({"kernel": "warp per entry", "requests": n, "list_length": pad, "us": round(us, 1),
                     "GBps": round(n * 8192 / us / 1e3, 2), "frac_of_h2d_peak": round(n * 8192 / us / 1e3 / h2d_peak, 3)})
        slots4 = [torch.arange(j * pad, (j + 1) * pad, dtype=torch.int32, device=dev) for j in range(4)]
        # the same lists through the copy unit: one launch carries four layers' lists (here four of the eight lists)
        us = graph_time(lambda i: oasis.stage_blocks_bulk([host] * 4, [idxs[(i + j) % 8] for j in range(4)],
                                                          slots4, pad, [pool] * 4),
                        8, iters=8, warm=8)
        rows.append({"kernel": "bulk copies, 4 lists per launch", "requests": 4 * n, "list_length": pad, "us": round(us, 1),
                     "GBps": round(4 * n * 8192 / us / 1e3, 2), "frac_of_h2d_peak": round(4 * n * 8192 / us / 1e3 / h2d_peak, 3)})
    # the hand-over in the other direction: dense key / value blocks (HBM) -> entries of the pinned pool + summaries
    Bq, Hkv, mb = 8, 8, 2048                                            # 16,384 blocks x 8 heads x 8 KiB = 1 GiB
    dims = oasis.Dims(Bq, 32, Hkv, mb)
    dk = torch.randn((Bq * mb, Hkv, 16, 128), device=dev).to(torch.bfloat16)
    dv = torch.randn((Bq * mb, Hkv, 16, 128), device=dev).to(torch.bfloat16)
    tbl = torch.arange(Bq * mb, dtype=torch.int32, device=dev).view(Bq, mb)
    summ = torch.empty((Bq, Hkv, mb, 2, 128), dtype=torch.bfloat16, device=dev)
    first = torch.zeros(Bq, dtype=torch.int32, device=dev)
    n = torch.full((Bq,), mb, dtype=torch.int32, device=dev)
    host1 = host.view(-1)[:Bq * mb * Hkv * 2 * 16 * 128].view(Bq * mb, Hkv, 2, 16, 128)
    us = graph_time(lambda i: oasis.offload_blocks(dims, dk, dv, tbl, tbl, first, n, mb, host1, summ), 1, iters=2, warm=1)
    gb = Bq * mb * Hkv * 8192 / 1e9
    offload = {"blocks": Bq * mb, "GB": round(gb, 3), "ms": round(us / 1e3, 2), "GBps_to_host": round(gb / (us * 1e-6), 2)}
    print(json.dumps({"section": "stage", "pinned_h2d_peak_GBps": round(h2d_peak, 2), "rows": rows, "offload": offload}))


def section_shapes(args, dev, hbm_peak):
    """Kernels alone at the shapes of configs[0..3] (graph replay over 3 rotating working sets)."""
    from paper_2608_08097_b200 import binding, pipeline
    rows = []
    for name, base in (("configs[0]", synth.C1), ("configs[1]", synth.C2), ("configs[2]", synth.C3), ("configs[3]", synth.C4)):
        cfg = synth.scaled(base, layers=1, steps=1)
        Bq, Hq, Hkv, T, mb, K = cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.n_q_tokens, cfg.max_blocks, cfg.k_blocks
        n_rot = 3
        Ls = [pipeline.DecodeLayer(Bq, Hq, Hkv, mb, K, T, dev) for _ in range(n_rot)]
        g = torch.Generator(device=dev)
        g.manual_seed(args.seed)
        q = torch.randn((Bq, T, Hq, 128), device=dev, generator=g).to(torch.bfloat16)
        nf = cfg.context // 16
        n_full = torch.full((Bq,), nf, dtype=torch.int32, device=dev)
        seq = torch.full((Bq,), cfg.context, dtype=torch.int32, device=dev)
        table = torch.arange(Bq * mb, dtype=torch.int32, device=dev).view(Bq, mb)
        for L in Ls:
            L.summaries.copy_(torch.randn(L.summaries.shape, device=dev, generator=g).to(torch.bfloat16))
            L.pool.copy_(torch.randn(L.pool.shape, device=dev, generator=g).to(torch.bfloat16))
            L.score(q, n_full)
            L.select(n_full, seq, table)
        torch.cuda.synchronize()
        Td, stride = T - 1, T * Hq * 128
        sb = Bq * Hkv * nf * 516
        ab = Bq * Hkv * (K + 1) * 8192 + 2 * Bq * T * Hq * 256
        t_score = graph_time(lambda i: Ls[i].score(q, n_full), n_rot)
        t_sel = graph_time(lambda i: Ls[i].select(n_full, seq, table), n_rot)
        t_attn = graph_time(lambda i: Ls[i].attend(q, seq), n_rot)
        row = {"shape": name, "batch": Bq, "rows": Bq * Hkv, "context": cfg.context, "K": K, "Td": Td, "G": Hq // Hkv,
               "score_us": round(t_score, 1), "score_frac": round(sb / t_score / 1e3 / hbm_peak, 3),
               "select_us": round(t_sel, 1), "attn_us": round(t_attn, 1),
               "attn_frac": round(ab / t_attn / 1e3 / hbm_peak, 3), "layer_us": None, "layer_frac": None}
        if binding.attn_and_score_supported(Ls[0].dims, T, Ls[0].cols, Td):
            def fused(i):
                L = Ls[i]
                binding.attn_and_score(L.dims, q, T, L.pool, L.slot_tbl, L.sel, L.cols, seq, L.scale, L.out, q[:, 1:], Td,
                                       L.summaries, n_full, L.scores, q_batch_stride=stride, workspace=L.workspace)
            t_layer = graph_time(fused, n_rot)
            row["layer_us"] = round(t_layer, 1)
            row["layer_frac"] = round((sb + ab) / t_layer / 1e3 / hbm_peak, 3)
        if name == "configs[1]":
            # step 0 at full size: the summaries of every full block of the layer from a device-resident pool
            kvs = [torch.randn((Bq * mb, Hkv, 2, 16, 128), device=dev, generator=g, dtype=torch.float32).to(torch.bfloat16)
                   for _ in range(n_rot)]
            zeros = torch.zeros(Bq, dtype=torch.int32, device=dev)
            torch.cuda.synchronize()
            t_sum = graph_time(lambda i: Ls[i].build_summaries(kvs[i], table, zeros, n_full, mb), n_rot, iters=12)
            row["summaries_full_build_us"] = round(t_sum, 1)
            row["summaries_full_build_frac"] = round(Bq * Hkv * nf * (4096 + 512) / t_sum / 1e3 / hbm_peak, 3)
            del kvs
        rows.append(row)
        del Ls
        torch.cuda.empty_cache()
    print(json.dumps({"section": "shapes", "workload": "one layer of configs[0..3], 3 rotating copies of summaries and "
                      "pools (random contents), kernels alone by graph replay; frac = algorithmic bytes / time / measured "
                      "copy peak; layer = the fused attention + scoring launch (null where it does not take the shape)",
                      "hbm_peak_GBps": hbm_peak, "rows": rows}))


def attention_pair(dev, seed, batch, Hq, Hkv, T, K):
    """us of packed_attn, sparse_attn and tree_attn (None where it does not take the rows) for one list of K whole blocks and the
    local window, in a graph over more working sets than L2 holds."""
    from paper_2608_08097_b200 import binding, pipeline
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    randn = lambda *s: torch.randn(s, device=dev, generator=g).to(torch.bfloat16)
    q, seq = randn(batch, T, Hq, 128), torch.full((batch,), 16 * K, dtype=torch.int32, device=dev)
    sel = torch.arange(K + 2, dtype=torch.int32, device=dev).repeat(batch, Hkv, 1)
    sel[..., K + 1:] = K + 1 if T > 16 else -1
    n_ent, got = batch * Hkv * K, []
    one = torch.arange(n_ent, dtype=torch.int32, device=dev).view(1, -1)
    n, zero = torch.full((1,), n_ent, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    par = (torch.arange(T, dtype=torch.int32, device=dev) - 1).repeat(batch, 1).contiguous()
    nodes, tree_kv = torch.full((batch,), T, dtype=torch.int32, device=dev), randn(batch, T, Hkv, 2, 128)
    for kind in ("packed", "bf16", "tree"):
        if kind == "tree" and T > binding.MAX_TREE:
            got.append(None)
            continue
        size = n_ent * (2304 if kind == "packed" else 8192)
        n_rot = max(2, min(16, -(-300_000_000 // size)))
        Ls = []
        for _ in range(n_rot):
            L = pipeline.DecodeLayer(batch, Hq, Hkv, K + 16, K, T, dev, tree=kind == "tree", kv_bits=4 if kind == "packed" else 16)
            if kind == "packed":
                kv = randn(n_ent, 2, 16, 128)
                binding.pack_blocks(binding.Dims(1, 1, 1, n_ent), kv, one, zero, n, n_ent, L.pool, one)
                L.local.copy_(randn(*L.local.shape))
            else:
                L.pool.copy_(randn(*L.pool.shape))
            L.sel.copy_(sel)
            Ls.append(L)
        torch.cuda.synchronize()
        if kind == "tree":
            us = graph_time(lambda i: Ls[i].attend_tree(q, tree_kv, par, nodes, seq), n_rot)
        else:
            us = graph_time(lambda i: Ls[i].attend(q, seq), n_rot)
        got.append(round(us, 1))
        del Ls
        torch.cuda.empty_cache()
    return got


def section_packed(args, dev, hbm_peak):
    """Entries in 4 bits beside bf16 ones: attention kernels, hand-over, the engine's step."""
    from paper_2608_08097_b200 import binding, synth
    kernels = []
    for batch, Hq, Hkv, T, K in ((1, 32, 8, 1, 16), (16, 32, 8, 1, 128), (16, 32, 8, 5, 128), (16, 32, 8, 8, 128), (16, 32, 8, 16, 128),
                                 (16, 32, 4, 9, 128), (16, 32, 8, 32, 128), (2, 32, 8, 1, 4096), (2, 32, 8, 5, 4096), (2, 32, 8, 16, 4096),
                                 (2, 32, 8, 1, 8192)):
        p, b, t = attention_pair(dev, args.seed, batch, Hq, Hkv, T, K)
        kernels.append({"batch": batch, "q_heads": Hq, "kv_heads": Hkv, "tokens": T, "rows": T * Hq // Hkv, "columns": K + 2,
                        "packed_us": p, "bf16_us": b, "bf16_tree_us": t})
    # the hand-over of 16,384 dense blocks of 8 heads (1 GiB of bf16) into a packed pool
    Bq, Hkv, mb = 8, 8, 2048
    dims = binding.Dims(Bq, 32, Hkv, mb)
    dk, dv = (torch.randn((Bq * mb, Hkv, 16, 128), device=dev).to(torch.bfloat16) for _ in range(2))
    tbl = torch.arange(Bq * mb, dtype=torch.int32, device=dev).view(Bq, mb)
    summ = torch.empty((Bq, Hkv, mb, 2, 128), dtype=torch.bfloat16, device=dev)
    first, n = torch.zeros(Bq, dtype=torch.int32, device=dev), torch.full((Bq,), mb, dtype=torch.int32, device=dev)
    hand_over = {}
    for where in ("pinned", "hbm"):
        pool = torch.empty((Bq * mb, Hkv, 2304), dtype=torch.uint8, device="cpu" if where == "pinned" else dev, pin_memory=where == "pinned")
        us = graph_time(lambda i: binding.offload_blocks_packed(dims, dk, dv, tbl, tbl, first, n, mb, pool, summ), 1, iters=2, warm=1)
        hand_over[where] = {"us": round(us, 1), "GBps_written": round(Bq * mb * Hkv * 2304 / us / 1e3, 2), "GBps_read": round(Bq * mb * Hkv * 8192 / us / 1e3, 1)}
        del pool
    del dk, dv, summ
    torch.cuda.empty_cache()

    # the step of the reasoning-style decode
    opt = argparse.Namespace(config=1, layers=args.layers, batch=None, context=None, seed=args.seed, group=0, wait_group=0, transfer_group=0,
                             transfer_kind="", again=2, steps=20, warmup=5, fetch_ratio=0.05)
    cfg, _ = B.workload(opt)
    bench = B.Bench(opt, cfg, dev, 0)
    bench.h2d_peak, bench.hbm_peak = B.time_pinned_h2d(dev), hbm_peak
    bench.generate(want_mirror=False, want_host=True)
    w, cap = B.Work(bench, cfg.k_blocks, cfg.n_draft), B.cap_of(opt.fetch_ratio, cfg.k_blocks)
    steps = []

    def timed(eng, bits, where, group):
        ms, clocks, _, _ = bench.timed(eng, w, 1, opt.warmup, opt.steps)
        steps.append({"kv_bits": bits, "pool": where, "fused": eng.fused, "layers_per_gather": group, "ms_per_step": round(ms, 4),
                      "ms_per_step_again": list(bench.again_ms), "us_per_layer": round(ms * 1e3 / cfg.layers, 1),
                      "MB_gathered_per_layer": round(B.admitted_entries(eng) * (2304 if bits == 4 else 8192) / 1e6, 2),
                      "sm_mhz": clocks["sm_mhz"], "reasons": clocks["reasons"]})
    for where in ("pinned", "hbm"):
        pools = bench.host_kv if where == "pinned" else [kv.to(dev) for kv in bench.host_kv]
        eng = bench.engine(w, pools, cap)
        timed(eng, 16, where, eng.transfer_group)
        del eng, pools
        torch.cuda.empty_cache()
    n = cfg.layers
    P, Hkv = bench.host_kv[0].shape[:2]
    for where in ("pinned", "hbm"):
        pools = [torch.empty((P, Hkv, 2304), dtype=torch.uint8, pin_memory=True) if where == "pinned" else
                 torch.empty((P, Hkv, 2304), dtype=torch.uint8, device=dev) for _ in range(n)]
        ratio = bench.link_ratio(w, cap) * 2304 / 8192
        group = B.pick_transfer_group(ratio, n, bench.compute_us(w)) if where == "pinned" else 1
        eng = bench.pipeline.DecodeEngine(cfg.batch, cfg.n_q_heads, Hkv, cfg.max_blocks, w.k, w.T, n, dev, mode="delta", cap=cap, append=True,
                                          wait_group=bench.wait_group(), transfer_group=group, kv_bits=4)
        for l in range(n):
            eng.attach(l, pools[l], bench.tables[l])
            kv = bench.host_kv[l].to(dev)
            dense = kv[:, :, 0].contiguous(), kv[:, :, 1].contiguous()
            eng.handover(l, *dense, bench.tables[l], bench.seq_dev[0].contiguous())
            torch.cuda.synchronize()
            del kv, dense
        eng.prime([w.q_dev[l][0] for l in range(n)], bench.first_dev[0].contiguous(), bench.seq_dev[0].contiguous(), summaries_ready=True)
        timed(eng, 4, where, group)
        del eng, pools
        torch.cuda.empty_cache()
    print(json.dumps({"section": "packed", "workload": "kernels: one list of whole blocks and the local window, graph replay over working sets "
                      "that L2 does not hold; steps: reasoning-style decode (batch %d, context %d, %d layers, %d tokens a step, budget %d blocks, at most %d new "
                      "blocks per row), %d steps in one graph" % (cfg.batch, cfg.context, n, w.T, w.k, cap, opt.steps),
                      "hbm_peak_GBps": hbm_peak, "pinned_h2d_peak_GBps": round(bench.h2d_peak, 2), "attention": kernels, "hand_over": hand_over, "steps": steps}))


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--what", default="c5,stage,shapes")
    ap.add_argument("--layers", type=int, default=None, help="layers of the packed section's steps (default: the workload's)")
    args = ap.parse_args()
    if not torch.cuda.is_available():
        raise SystemExit("bench_sweep.py needs a CUDA device: the product path has no CPU fallback")
    torch.cuda.set_device(0)
    dev = torch.device("cuda", 0)
    from paper_2608_08097_b200 import build
    build.build()
    hbm_peak, _ = B.measured_peaks()
    for what in args.what.split(","):
        {"c5": section_c5, "stage": section_stage, "shapes": section_shapes, "packed": section_packed}[what](args, dev, hbm_peak)
        torch.cuda.empty_cache()


if __name__ == "__main__":
    main()
