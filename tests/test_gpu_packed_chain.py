"""GPU test of the order of launches that may start before their predecessor has ended: packing, unpacking, attention (alone, merged in a
cluster, merged through the workspace) and rotation back to back, every one reading what the one before it wrote, against the same
calls with the GPU waited for after each."""
import pytest
import torch

from tests.test_gpu_packed import SCALE, L, gen, i32, randn  # noqa: F401

pytestmark = pytest.mark.gpu


class Chain:
    """entries -> packed -> unpacked -> packed again -> attention of 16 heads -> its output's rows as a projection, rotated to 12 heads
    -> attention of 12 heads over the same entries -> rotated to 8 heads and 2 key heads, whose rows become a block's -> packed from the
    local window -> attention of 8 heads over that block too."""

    def __init__(self, L, T, n):                          # noqa: F811
        from paper_2608_08097_b200.rotary import RotaryTable
        self.L, self.T, self.n = L, T, n
        self.table, self.g = RotaryTable(128), gen(n + T)
        dev, b16 = dict(device="cuda"), dict(device="cuda", dtype=torch.bfloat16)
        self.all = i32([list(range(2 * n))])
        self.first, self.count, self.length = i32([0]), i32([2 * n]), i32([16 * n - 1])
        self.idx = torch.randperm(2 * n, generator=torch.Generator().manual_seed(n)).cuda()
        self.pool = torch.empty((2 * n, 1, 2, 16, 128), **b16)
        self.far, self.near = (torch.empty((2 * n, 2304), dtype=torch.uint8, **dev) for _ in range(2))
        self.back = torch.empty((2 * n, 2, 16, 128), **b16)
        self.slots, self.blocks = i32(list(range(2 * n))).view(1, 2, n), i32(list(range(n)) * 2).view(1, 2, n)
        self.q = [torch.empty((1, T, h, 128), **b16) for h in (16, 12, 8)]
        self.out = [torch.empty((1, T, h, 128), **b16) for h in (16, 12, 8)]
        self.kv = [torch.empty((1, T, 2, 2, 128), **b16) for _ in range(2)]
        self.local = torch.zeros((4, 2, 16, 128), **b16)
        self.local_slots = i32([0, 1, 2, 3]).view(1, 2, 2)
        self.local_blocks = torch.empty((1, 2, 2), dtype=torch.int32, **dev)
        self.dims = [L.Dims(1, h, 2, n + 4) for h in (16, 12, 8)]
        self.ws = [torch.empty(max(16, L.packed_attn_workspace_bytes(d, T, n, n)), dtype=torch.uint8, **dev) for d in self.dims]
        self.page = i32([list(range(n + 4))])
        self.written = [self.far, self.near, self.back, *self.q[1:], *self.out, *self.kv]

    def fresh(self, k):
        """New inputs, and in the outputs what no call may leave behind."""
        self.g.manual_seed(k)
        self.pool.copy_(randn(self.g, *self.pool.shape))
        self.q[0].copy_(randn(self.g, *self.q[0].shape))
        for t in self.written:
            t.view(torch.uint8).fill_(255)
        self.local.zero_()
        self.local_blocks.fill_(-1)

    def attend(self, k):
        self.L.packed_attn(self.dims[k], self.q[k], self.near, None, self.slots, self.blocks, self.n, self.length, SCALE, self.out[k], workspace=self.ws[k])

    def calls(self):
        L, n, T = self.L, self.n, self.T                  # noqa: F841
        one = L.Dims(1, 1, 1, 2 * n)
        yield lambda: L.pack_blocks(one, self.pool, self.all, self.first, self.count, 2 * n, self.far, self.all)
        yield lambda: L.unpack_blocks(self.far, self.idx, self.back)
        yield lambda: L.pack_blocks(one, self.back.view(self.pool.shape), self.all, self.first, self.count, 2 * n, self.near, self.all)
        yield lambda: self.attend(0)
        yield lambda: L.rotate_qkv(L.Dims(1, 12, 2, 1), self.out[0].view(1, T, -1), self.table, self.q[1], self.kv[0], seq_len=self.length)
        yield lambda: self.attend(1)
        yield lambda: L.rotate_qkv(L.Dims(1, 8, 2, 1), self.out[1].view(1, T, -1), self.table, self.q[2], self.kv[1], seq_len=self.length)
        yield lambda: L.append_kv(self.dims[2], self.kv[1], 0, self.first, self.page, self.local_slots, self.local_blocks, 0, self.local, None)
        yield lambda: L.pack_local_layers(self.dims[2], [self.local], [self.local_slots], 0, self.first, self.one_block, 1, [self.near], [self.page])
        yield lambda: self.attend(2)

    def run(self, wait):
        for call in self.calls():
            call()
            if wait:
                torch.cuda.synchronize()
        return [t.clone() for t in self.written]


@pytest.mark.parametrize("T, n", [(1, 8), (2, 60), (8, 300), (16, 300), (1, 2000), (8, 2000)])
def test_launches_that_start_early_see_what_came_before(L, T, n):  # noqa: F811
    c = Chain(L, T, n)
    c.one_block = i32([1])
    want = []
    for k in range(12):
        c.fresh(k)
        torch.cuda.synchronize()
        want.append(c.run(wait=True))
    assert all(bool(torch.isfinite(t).all()) for w in want for t in w if t.dtype == torch.bfloat16)
    for k in range(12):
        c.fresh(k)
        for got, t in zip(c.run(wait=False), want[k]):
            assert torch.equal(got.view(torch.uint8), t.view(torch.uint8))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for call in c.calls():
            call()
    for k in range(12):
        c.fresh(k)
        g.replay()
        for got, t in zip(c.written, want[k]):
            assert torch.equal(got.view(torch.uint8), t.view(torch.uint8))
