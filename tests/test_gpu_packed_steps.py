"""GPU tests of the engine over packed blocks beyond its smallest shape: many query rows, splits through the workspace, several steps
in one graph, queries and outputs in pinned memory, and the order of a step's launches."""
import pytest
import torch

from tests.packed_loop import Loop

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_08097_b200 import build
    build.build()
    from paper_2608_08097_b200 import binding, pipeline
    binding.lib()
    return binding, pipeline


SMALL = dict(B=2, Hq=8, Hkv=2, T=3, K=6, max_blocks=16, layers=3, seq0=[100, 77], steps=8, cap=2)


def test_the_attention_does_not_wait_for_the_packing(oracle, gpu, monkeypatch):
    """It reads the local window; what is packed goes to the pool, over the host link as a rule, and only scoring and gathers need it."""
    binding, pipeline = gpu
    loop, log = Loop(oracle, pipeline, **dict(SMALL, wait_group=2)), []
    eng, event, pack, wait = loop.eng, pipeline.DecodeEngine._event, binding.pack_local_layers, torch.cuda.Stream.wait_event

    def logged_event(stream):
        ev = event(stream)
        log.append(("event", stream, ev))
        return ev

    def logged_pack(*a, **k):
        log.append(("pack", torch.cuda.current_stream(), None))
        return pack(*a, **k)

    def logged_wait(stream, ev):
        log.append(("wait", stream, ev))
        return wait(stream, ev)
    monkeypatch.setattr(eng, "_event", logged_event)
    monkeypatch.setattr(binding, "pack_local_layers", logged_pack)
    monkeypatch.setattr(torch.cuda.Stream, "wait_event", logged_wait)
    loop.sel_log = {}
    args, kw = loop.call(0)
    eng.step(*args, **kw)
    eng.join()
    monkeypatch.undo()
    torch.cuda.synchronize()
    packs = [k for k, e in enumerate(log) if e[0] == "pack"]
    assert packs and all(log[k][1] == eng.pred for k in packs)
    from_pred = {id(e[2]): k for k, e in enumerate(log) if e[0] == "event" and e[1] == eng.pred}
    last = max(k for k, e in enumerate(log) if e[0] == "event" and e[1] == eng.main)                 # the last attention's
    waits = [from_pred[id(e[2])] for k, e in enumerate(log[:last]) if e[0] == "wait" and e[1] == eng.main and id(e[2]) in from_pred]
    assert len(waits) == 2 and max(waits) < min(packs)               # one per group of layers


def test_a_packed_layer_has_no_gather_list(gpu):
    """The slots of the top-k's list are those of a bf16 layer, k + 2 to a row."""
    _, pipeline = gpu
    lay = pipeline.DecodeLayer(1, 4, 1, 8, 2, 2, kv_bits=4)
    assert lay.stage_idx is None and lay.stage_slots is None
    lay.scores.copy_(torch.arange(8.0).view(1, 1, 8))
    n, length, table = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([6], [100], [list(range(8))]))
    lay.select(n, length, table)
    assert lay.sel.flatten().tolist() == [5, 4, 6, -1]
    with pytest.raises(ValueError, match="transfer plan"):
        lay.stage(torch.zeros((8, 1, 2304), dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("n_commit, T", [(3, 3), (2, 5), (16, 16)])
def test_steps_that_commit_several_tokens(oracle, gpu, n_commit, T):
    """A step adds n_commit tokens; the block that they fill is packed in that step."""
    _, pipeline = gpu
    Loop(oracle, pipeline, **dict(SMALL, T=T, layers=2, steps=6, n_commit=n_commit)).run(chunk=2)


@pytest.mark.parametrize("n_commit", [0, 4, -1])
def test_a_packed_engine_refuses_counts_that_no_step_has(gpu, n_commit):
    _, pipeline = gpu
    with pytest.raises(ValueError, match="n_commit"):
        pipeline.DecodeEngine(1, 4, 1, 8, 2, 3, 1, mode="delta", cap=2, append=True, kv_bits=4, n_commit=n_commit)


@pytest.mark.parametrize("shape", [
    dict(B=2, Hq=16, Hkv=2, T=9, K=12, max_blocks=40, layers=2, seq0=[500, 333], steps=5, cap=3),             # 72 query rows: tensor memory
    dict(B=1, Hq=4, Hkv=2, T=10, K=24, max_blocks=40, layers=1, seq0=[600], steps=4, cap=24),                 # 20 rows, splits in a cluster
    dict(B=1, Hq=2, Hkv=1, T=4, K=230, max_blocks=260, layers=1, seq0=[250 * 16 + 14], steps=4, cap=20),      # splits through the workspace
    dict(B=1, Hq=8, Hkv=1, T=8, K=230, max_blocks=260, layers=1, seq0=[250 * 16 + 14], steps=3, cap=20),      # the same with 64 rows
])
def test_rows_and_splits(oracle, gpu, shape):
    _, pipeline = gpu
    loop = Loop(oracle, pipeline, host=True, **shape)
    assert loop.eng.layers[0].splits == (shape["K"] == 230)
    loop.run(chunk=2)


@pytest.mark.parametrize("graph, e2e, chunk, group, streams", [
    (True, "stacked", 4, 2, 1), (True, "layers", 3, 1, 2), (False, "stacked", 4, 2, 2), (False, "layers", 8, 1, 1), (False, None, 8, 2, 2), (True, None, 1, 3, 1)])
def test_several_steps_and_pinned_queries_and_outputs(oracle, gpu, graph, e2e, chunk, group, streams):
    """No synchronisation between the steps of a chunk; blocks fill up and are gathered within it."""
    _, pipeline = gpu
    loop = Loop(oracle, pipeline, host=True, wait_group=group, transfer_group=group, transfer_streams=streams, **dict(SMALL, seq0=[109, 77], steps=9))
    loop.run(chunk=chunk, graph=graph, e2e=e2e)


def test_launches_are_counted(oracle, gpu):
    """Two launches for the appends and packs of a step, five per layer (attention, scoring, top-k, plan, gather)."""
    _, pipeline = gpu
    loop = Loop(oracle, pipeline, **dict(SMALL, steps=1, wait_group=3))
    before = loop.eng.launches
    loop.run()
    assert loop.eng.launches - before == 2 + 5 * 3


def test_the_gather_refuses_lists_in_host_memory(gpu):
    """Its kernel reads them on the device."""
    binding, _ = gpu
    packed, pool = (torch.zeros((4, 2304), dtype=torch.uint8, device="cuda") for _ in range(2))
    idx, slots = torch.tensor([1, 2], device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for i, s, e in ((idx.cpu(), slots, ValueError), (idx, slots.cpu(), ValueError), (idx.cpu().pin_memory(), slots, ValueError), (idx.int(), slots, TypeError),
                    (idx, slots.long(), TypeError), (idx.repeat(2)[::2], slots, ValueError), (idx[:1], slots, ValueError)):
        with pytest.raises(e):
            binding.stage_packed_layers([packed], [i], [s], 2, [pool])
    binding.stage_packed_layers([packed], [idx], [slots], 2, [pool])
    binding.stage_packed_layers([], [], [], 0, [])
