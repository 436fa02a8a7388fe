"""GPU test of decoding over a cache in 4 bits as a user runs it: dense pools are handed over, every step's projections are
rotated, and the engine with kv_bits=4 appends, packs the blocks that fill up, scores, selects, gathers and attends -- step by
step against the oracle, whose cache holds the same bf16 keys and values, packed by the oracle's own packing."""
import math

import numpy as np
import pytest
import torch

from oracle import packed as op
from tests import parity_util as pu

pytestmark = pytest.mark.gpu

SCALE = 1.0 / math.sqrt(128.0)
B, HQ, HKV, T, K, MB, LAYERS, STEPS = 2, 8, 2, 3, 6, 16, 2, 20
SEQ0 = np.array([100, 77], np.int32)


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_08097_b200 import build
    build.build()
    from paper_2608_08097_b200 import binding, pipeline
    binding.lib()
    return binding, pipeline


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("graph, host, cap, group", [(False, True, 2, 1), (True, False, 2, 2), (False, False, K, 2)])
def test_decoding_over_packed_blocks(oracle, gpu, graph, host, cap, group):
    binding, pipeline = gpu
    from paper_2608_08097_b200.rotary import RotaryTable
    rng, g = np.random.default_rng(3), torch.Generator(device="cuda")
    g.manual_seed(3)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    eng = pipeline.DecodeEngine(B, HQ, HKV, MB, K, T, LAYERS, mode="delta", cap=cap, append=True, kv_bits=4, wait_group=group, transfer_group=group)
    assert not eng.fused
    table = RotaryTable(96, base=500000.0, scaling=dict(kind="bands", factor=8, trained=8192))
    P = B * MB
    dense = [randn(P, HKV, 2, 16, 128) for _ in range(LAYERS)]
    gpu_table, tables = rng.permutation(P).reshape(B, MB).astype(np.int32), [rng.permutation(P).reshape(B, MB).astype(np.int32) for _ in range(LAYERS)]
    pools = [torch.zeros((P, HKV, 2304), dtype=torch.uint8) for _ in range(LAYERS)]
    pools = [p.pin_memory() if host else p.cuda() for p in pools]
    kv_ref = [np.zeros((P, HKV, 2, 16, 128), np.uint16) for _ in range(LAYERS)]          # the oracle's cache, bf16
    for l in range(LAYERS):
        eng.attach(l, pools[l], i32(tables[l]))
        kv_ref[l][tables[l]] = pu.np_u16(dense[l])[gpu_table]
        eng.handover(l, dense[l][:, :, 0].contiguous(), dense[l][:, :, 1].contiguous(), i32(gpu_table), i32(SEQ0))
    qkv = randn(STEPS, LAYERS, B, T, (HQ + 2 * HKV) * 128)
    q = [randn(B, T, HQ, 128) for _ in range(LAYERS)]
    new_kv = [torch.zeros((B, T, HKV, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
    with pytest.raises(ValueError):
        eng.prime(q, i32(SEQ0 // 16), i32(SEQ0))
    torch.cuda.synchronize()
    eng.prime(q, i32(SEQ0 // 16), i32(SEQ0), summaries_ready=True)

    # ---- the oracle's side
    slot_tbl = eng.layers[0].slot_tbl.cpu().numpy()
    local = [np.zeros((2 * B * HKV, 2, 16, 128), np.uint16) for _ in range(LAYERS)]
    work = [np.zeros((B * HKV * K, 2304), np.uint8) for _ in range(LAYERS)]
    res = [np.full((B, HKV, K + 2), -1, np.int32) for _ in range(LAYERS)]
    stamp = [np.zeros((B, HKV, K + 2), np.int32) for _ in range(LAYERS)]
    made = [{} for _ in range(LAYERS)]                   # full blocks never change: each is packed once

    def predict(l, q_now, n_full, seq, gsel, cap_now, step):
        summ = oracle.build_summaries(kv_ref[l], tables[l], np.zeros(B, np.int32), n_full.astype(np.int32))
        s32, s64 = oracle.score_blocks(pu.np_u16(q_now)[:, 1:], summ, n_full.astype(np.int32))
        sel, _, _ = oracle.select_topk(s32, n_full.astype(np.int32), seq.astype(np.int32), T, K, tables[l])
        pu.assert_sel_parity(gsel, sel, s64, K)
        idx, slots, _ = oracle.plan_delta(gsel, tables[l], res[l], stamp[l], K, cap_now, step, K, n_res=K, n_local=0)
        flat = kv_ref[l].reshape(-1, 2, 16, 128)
        for i, s in zip(idx.ravel(), slots.ravel()):
            if i >= 0:
                if int(i) not in made[l]:
                    made[l][int(i)] = op.pack(pu.bf16_to_f32_np(torch.from_numpy(flat[i].view(np.int16)).view(torch.bfloat16)).astype(np.float64))
                work[l][s] = made[l][int(i)]

    for l in range(LAYERS):
        predict(l, q[l], SEQ0 // 16, SEQ0, eng.layers[l].sel.cpu().numpy(), K, 0)
        for b in range(B):                               # the block that still grows
            j = SEQ0[b] // 16
            local[l][slot_tbl[b, :, K + j % 2]] = kv_ref[l][tables[l][b, j]]
        oracle.local_window(SEQ0, T, tables[l], res[l], K, K + 2)
    sel_log = [torch.zeros_like(eng.layers[0].sel) for _ in range(LAYERS)]
    seq_d = {n: i32(np.zeros(B)) for n in ("seq", "first", "new", "full", "next")}
    args = (q, seq_d["seq"], seq_d["first"], seq_d["new"], seq_d["full"], seq_d["next"])
    captured = eng.capture_step(*args, step_stamp=1, new_kv=new_kv, sel_log=sel_log) if graph else None
    for s in range(STEPS):
        seq, stamp_now = SEQ0 + s, 1 if graph else s + 1
        for name, v in (("seq", seq), ("first", seq // 16), ("new", (seq + 1) // 16 - seq // 16), ("full", (seq + 1) // 16), ("next", seq + 1)):
            seq_d[name].copy_(i32(v))
        for l in range(LAYERS):
            eng.layers[l].rotate(qkv[s, l], table, q[l], new_kv[l], seq_d["seq"])
            want_q, want_kv = op.rotate(f64(qkv[s, l]), seq[:, None] + np.arange(T), table.freqs.cpu().numpy(), 96, 0, 1.0, HQ, HKV)
            # (half a step of bf16 below 8: 2^-8 * 8; tests/test_gpu_rotate.py is the closer check)
            assert np.abs(f64(q[l]) - want_q).max() < 0.04 and np.abs(f64(new_kv[l]) - want_kv).max() < 0.04
        torch.cuda.synchronize()
        if graph:
            eng.replay(captured)
        else:
            eng.step(*args, step_stamp=stamp_now, new_kv=new_kv, sel_log=sel_log)
            eng.join()
        torch.cuda.synchronize()
        for l in range(LAYERS):
            oracle.append_kv(pu.np_u16(new_kv[l]), 1, seq.astype(np.int32), tables[l], slot_tbl, res[l], K, local[l], kv_ref[l])
            near = f64(torch.from_numpy(local[l].view(np.int16)).view(torch.bfloat16))
            out, _, a, big = op.attn(f64(q[l]), work[l], near, slot_tbl, res[l], K, seq, SCALE)
            got = f64(eng.layers[l].out)
            # weights in bf16 and the output's rounding, logits within 2^-15 of the largest sum of |q k|
            assert np.all(np.abs(got - out) <= 2.0 ** -8 * (a + np.abs(out)) + 2.0 ** -14 * big[..., None] * a)
            predict(l, q[l], (seq + 1) // 16, seq + 1, sel_log[l].cpu().numpy(), cap, stamp_now)
            assert np.array_equal(eng.blk_tbl(l).cpu().numpy(), res[l]) and np.array_equal(eng.layers[l].pool.cpu().numpy(), work[l])
            assert np.array_equal(pu.np_u16(eng.layers[l].local), local[l])
    for l in range(LAYERS):                              # the pool holds every whole block, and the steps' blocks are summarised
        for i, e in made[l].items():
            assert np.array_equal(pools[l].view(-1, 2304)[i].cpu().numpy(), e)
        n_full = (SEQ0 + STEPS) // 16
        summ = oracle.build_summaries(kv_ref[l], tables[l], np.zeros(B, np.int32), n_full.astype(np.int32))
        pu.assert_summaries_equal(pu.np_u16(eng.layers[l].summaries), summ, n_full)


def test_what_a_packed_engine_refuses(gpu):
    _, pipeline = gpu
    for kw in (dict(mode="fetch_all"), dict(mode="delta", cap=2), dict(mode="delta", cap=2, append=True, tree=True), dict(mode="delta", cap=2, append=True, fused=True),
               dict(mode="delta", cap=2, append=True, transfer_kind="bulk")):
        with pytest.raises(ValueError):
            pipeline.DecodeEngine(1, 4, 1, 8, 2, 2, 1, kv_bits=4, **kw)
    with pytest.raises(ValueError):
        pipeline.DecodeEngine(1, 4, 1, 8, 2, 2, 1, mode="delta", cap=2, append=True, kv_bits=8)
