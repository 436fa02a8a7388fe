"""GPU tests of the tree attention with several row groups per request (more than 256 query rows per KV head), some of them without a
live node beside live ones, in each of the ways in which rows are split and merged."""
import pytest
import torch

from tests.test_gpu_tree import AttnCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_08097_b200 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("B,Hq,Hkv,T,lens,nodes,budget,workspace", [
    (40, 8, 1, 64, [30 + 7 * i for i in range(40)], [64, 20, 33, 32, 1, 0, 31, 50] * 5, 12, False),     # two groups of 32 nodes, not split
    (2, 8, 1, 64, [1100, 900], [20, 64], 62, True),                                       # the same, merged through the workspace
    (2, 8, 1, 64, [1100, 900], [33, 1], 62, True),
    (5, 8, 1, 64, [1200, 300, 1180, 16, 0], [20, 64, 32, 33, 7], 70, False),              # the same, merged in clusters
    (4, 16, 1, 40, [1210, 1000, 640, 1], [14, 15, 28, 40], 70, False),                    # three groups of 14 nodes, clusters
    (1, 16, 1, 40, [1210], [14], 70, True),                                               # the same, workspace
    (3, 64, 2, 30, [1150, 400, 77], [8, 9, 30], 64, False),                               # four groups of 8 nodes, two KV heads
])
def test_row_groups_without_a_live_node(L, B, Hq, Hkv, T, lens, nodes, budget, workspace):
    c = AttnCase(L, B, Hq, Hkv, T, lens, nodes, budget, seed=B + T)
    assert (c.need > 0) == workspace
    c.run(L)
    torch.cuda.synchronize()
    c.check()
    first, first_lse = c.out.clone(), c.lse.clone()
    c.fresh()
    c.run(L)
    torch.cuda.synchronize()
    assert torch.equal(c.out, first) and torch.equal(c.lse, first_lse)
