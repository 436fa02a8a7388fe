"""A decode loop over packed blocks (DecodeEngine(kv_bits=4)) against the oracle, step by step: the dense pools are handed over, and
every step's outputs, selections, tables, working sets, local windows and pools must be what the oracle's are, whose cache holds the
same bf16 keys and values and packs them by its own packing."""
import math

import numpy as np
import torch

from oracle import packed as op
from tests import parity_util as pu

SCALE = 1.0 / math.sqrt(128.0)


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def f64_of(bits):
    """bf16 patterns (uint16) as float64."""
    return f64(torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16))


class Loop:
    def __init__(self, oracle, pipeline, B, Hq, Hkv, T, K, max_blocks, layers, seq0, steps, cap, host=False, n_commit=1, seed=3, **engine):
        rng, g = np.random.default_rng(seed), torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.randn = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
        self.oracle, self.B, self.Hq, self.Hkv, self.T, self.K, self.layers = oracle, B, Hq, Hkv, T, K, layers
        self.seq0, self.steps, self.cap, self.n_commit = np.array(seq0, np.int32), steps, cap, n_commit
        self.eng = pipeline.DecodeEngine(B, Hq, Hkv, max_blocks, K, T, layers, mode="delta", cap=cap, append=True, kv_bits=4, n_commit=n_commit, **engine)
        P = B * max_blocks
        self.entries = P * Hkv                            # of a pool
        dense = [self.randn(P, Hkv, 2, 16, 128) for _ in range(layers)]
        gpu_table = rng.permutation(P).reshape(B, max_blocks).astype(np.int32)
        self.tables = [rng.permutation(P).reshape(B, max_blocks).astype(np.int32) for _ in range(layers)]
        pools = [torch.zeros((P, Hkv, 2304), dtype=torch.uint8) for _ in range(layers)]
        self.pools = [p.pin_memory() if host else p.cuda() for p in pools]
        self.kv_ref = [np.zeros((P, Hkv, 2, 16, 128), np.uint16) for _ in range(layers)]
        for l in range(layers):
            self.eng.attach(l, self.pools[l], i32(self.tables[l]))
            self.kv_ref[l][self.tables[l]] = pu.np_u16(dense[l])[gpu_table]
            self.eng.handover(l, dense[l][:, :, 0].contiguous(), dense[l][:, :, 1].contiguous(), i32(gpu_table), i32(self.seq0))
        self.q = self.randn(steps, layers, B, T, Hq, 128)
        self.new_kv = self.randn(steps, layers, B, T, Hkv, 2, 128)
        torch.cuda.synchronize()
        self.eng.prime(list(self.q[0]), i32(self.seq0 // 16), i32(self.seq0), summaries_ready=True)
        # the oracle's side
        self.slot_tbl = self.eng.layers[0].slot_tbl.cpu().numpy()
        self.local = [np.zeros((2 * B * Hkv, 2, 16, 128), np.uint16) for _ in range(layers)]
        self.work = [np.zeros((B * Hkv * K, 2304), np.uint8) for _ in range(layers)]
        self.res = [np.full((B, Hkv, K + 2), -1, np.int32) for _ in range(layers)]
        self.stamp = [np.zeros((B, Hkv, K + 2), np.int32) for _ in range(layers)]
        self.made = [{} for _ in range(layers)]          # whole blocks never change: each is packed once
        for l in range(layers):
            self._predict(l, self.q[0, l], self.seq0, self.eng.layers[l].sel.cpu().numpy(), K, 0)
            for b in range(B):                           # the block that still grows
                j = self.seq0[b] // 16
                self.local[l][self.slot_tbl[b, :, K + j % 2]] = self.kv_ref[l][self.tables[l][b, j]]
            oracle.local_window(self.seq0, T, self.tables[l], self.res[l], K, K + 2)

    def _predict(self, l, q, seq, gsel, cap, stamp):
        o, n_full = self.oracle, (seq // 16).astype(np.int32)
        summ = o.build_summaries(self.kv_ref[l], self.tables[l], np.zeros(self.B, np.int32), n_full)
        s32, s64 = o.score_blocks(pu.np_u16(q)[:, 1:], summ, n_full)
        sel, _, _ = o.select_topk(s32, n_full, seq.astype(np.int32), self.T, self.K, self.tables[l])
        pu.assert_sel_parity(gsel, sel, s64, self.K)
        idx, slots, _ = o.plan_delta(gsel, self.tables[l], self.res[l], self.stamp[l], self.K, cap, stamp, self.K, n_res=self.K, n_local=0)
        flat = self.kv_ref[l].reshape(-1, 2, 16, 128)
        for i, s in zip(idx.ravel(), slots.ravel()):
            if i >= 0:
                if int(i) not in self.made[l]:
                    self.made[l][int(i)] = op.pack(f64_of(flat[i]))
                self.work[l][s] = self.made[l][int(i)]

    def call(self, s, **more):
        """Arguments of step s.  The block that the step's first n_commit tokens fill is named in this step."""
        seq, after = self.seq0 + s * self.n_commit, self.seq0 + (s + 1) * self.n_commit
        self.sel_log.setdefault(s, [torch.zeros_like(L.sel) for L in self.eng.layers])
        args = (list(self.q[s]), i32(seq), i32(seq // 16), i32(after // 16 - seq // 16), i32(after // 16), i32(after))
        return args, dict(step_stamp=s + 1, new_kv=list(self.new_kv[s]), sel_log=self.sel_log[s], **more)

    def run(self, chunk=1, graph=False, e2e=None):
        """`chunk` steps between two synchronisations, as one graph or back to back; e2e: queries and outputs in pinned memory, one
        tensor per layer ("layers") or one for all ("stacked")."""
        eng, n, keep = self.eng, self.layers, []
        self.sel_log = {}
        q_pin = self.q.cpu().pin_memory()
        stage = torch.empty_like(self.q[0])
        outs = {}
        for s0 in range(0, self.steps, chunk):
            steps = range(s0, min(s0 + chunk, self.steps))
            calls = []
            for s in steps:
                args, kw = self.call(s)
                if e2e:
                    outs[s] = torch.zeros(self.q[0].shape, dtype=torch.bfloat16).pin_memory()
                    stacked = e2e == "stacked"
                    args = (stage if stacked else list(stage),) + args[1:]
                    kw.update(q_host=q_pin[s] if stacked else list(q_pin[s]), out_host=outs[s] if stacked else list(outs[s]))
                calls.append((args, kw))
            torch.cuda.synchronize()
            keep.append(calls)
            if graph:
                keep.append(eng.capture_steps(calls))
                eng.replay(keep[-1])
            else:
                for s, (args, kw) in zip(steps, calls):
                    eng.step(*args, **kw)
                    if not e2e:
                        with torch.cuda.stream(eng.main):
                            outs[s] = [L.out.clone() for L in eng.layers]
                eng.join()
            torch.cuda.synchronize()
            if graph and not e2e:
                assert chunk == 1
                outs[s0] = [L.out.clone() for L in eng.layers]
            for s in steps:
                for l in range(n):
                    self._check(s, l, outs[s][l], s == steps[-1])
        for l in range(n):                               # the pool holds every whole block that was asked for, and they are summarised
            for i, e in self.made[l].items():
                assert np.array_equal(self.pools[l].view(-1, 2304)[i].cpu().numpy(), e)
            n_full = (self.seq0 + self.steps * self.n_commit) // 16
            summ = self.oracle.build_summaries(self.kv_ref[l], self.tables[l], np.zeros(self.B, np.int32), n_full.astype(np.int32))
            pu.assert_summaries_equal(pu.np_u16(eng.layers[l].summaries), summ, n_full)

    def _check(self, s, l, got, last):
        eng, seq = self.eng, (self.seq0 + s * self.n_commit).astype(np.int32)
        self.oracle.append_kv(pu.np_u16(self.new_kv[s, l]), self.n_commit, seq, self.tables[l], self.slot_tbl, self.res[l], self.K, self.local[l], self.kv_ref[l])
        out, _, a, big = op.attn(f64(self.q[s, l]), self.work[l], f64_of(self.local[l]), self.slot_tbl, self.res[l], self.K, seq, SCALE)
        # weights in bf16 and the output's rounding, logits within 2^-15 of the largest sum of |q k|
        assert np.all(np.abs(f64(got) - out) <= 2.0 ** -8 * (a + np.abs(out)) + 2.0 ** -14 * big[..., None] * a)
        self._predict(l, self.q[s, l], seq + self.n_commit, self.sel_log[s][l].cpu().numpy(), self.cap, s + 1)
        if last:
            assert np.array_equal(eng.blk_tbl(l).cpu().numpy(), self.res[l]) and np.array_equal(eng.layers[l].pool.cpu().numpy(), self.work[l])
            assert np.array_equal(pu.np_u16(eng.layers[l].local), self.local[l])
