"""Worker of test_gpu_tree.py: a process of its own with OASIS_LIB pointing at the bounds-check build.  Slots and entries of
the full-KV pool between a DECLARED extent and the (larger) size really allocated are flagged and skipped by the tree
attention and the commit, and nothing else is; nothing here can leave an allocation even if a check were wrong."""
import json
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2608_08097_b200 import binding  # noqa: E402
from oracle import tree as ot  # noqa: E402

HOST_ENTRY, SLOT, BLOCK_ID = 201, 202, 203
word = torch.zeros(1, dtype=torch.int32, device="cuda")


def take_code():
    torch.cuda.synchronize()
    c = int(word.item())
    word.zero_()
    return c


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def attention(declared):
    """Eight columns of one row; the entry of column 3 has slot 9."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    pool = torch.randn((12, 2, 16, 128), generator=g, device="cuda").to(torch.bfloat16)
    q = torch.randn((1, 3, 4, 128), generator=g, device="cuda").to(torch.bfloat16)
    kv = torch.randn((1, 3, 1, 2, 128), generator=g, device="cuda").to(torch.bfloat16)
    slot, blk, parent = [[[0, 1, 2, 9, 4, 5, 6, 7]]], [[list(range(8))]], [[-1, 0, 0]]
    binding.set_extents(0, declared)
    dims = binding.Dims(1, 4, 1, 8)
    out, lse = torch.zeros_like(q), torch.zeros((1, 3, 4), device="cuda")
    ws = torch.empty(max(16, binding.tree_attn_workspace_bytes(dims, 3, 8)), dtype=torch.uint8, device="cuda")
    binding.tree_attn(dims, q, kv, i32(parent), i32([3]), pool, i32(slot), i32(blk), i32([128]), 1 / math.sqrt(128), out, lse=lse, workspace=ws)
    code = take_code()
    seen = np.array(blk)
    if declared < 10:
        seen[0, 0, 3] = -1
    ref, ref_lse = np.zeros((1, 3, 4, 128)), np.zeros((1, 3, 4))
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    a = ot.tree_attn(f(q), f(kv), np.array(parent), [3], f(pool), np.array(slot), seen, [128], 1 / math.sqrt(128), ref, ref_lse)
    assert np.all(np.abs(f(out) - ref) <= 2 ** -8 * (a + np.abs(ref)) + 6e-4 * a), "attention with declared extent %d" % declared
    return code


def commit(slots, entries, mb=4):
    """Two tokens over a block border: blocks 0 and 1 in slots 4 and 5, entries 2 and 3."""
    binding.set_extents(entries, slots)
    kv = torch.ones((1, 2, 1, 2, 128), dtype=torch.bfloat16, device="cuda")
    pool, host = (torch.zeros((8, 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    blk = i32([[[-1, -1]]])
    binding.commit_kv(binding.Dims(1, 1, 1, mb), kv, i32([[0, 1]]), i32([2]), i32([15]), i32([[2, 3, 0, 1][:mb]]), i32([[[4, 5]]]), blk, 0, pool,
                      host.view(8, 1, 2, 16, 128))
    code = take_code()
    assert blk.tolist() == [[[0, 1]]]
    return code, [bool(pool[4, :, 15].all()), bool(pool[5, :, 0].all())], [bool(host[2, :, 15].all()), bool(host[3, :, 0].all())], \
        int(pool.sum()) + int(host.sum())


def main():
    assert binding.bounds_checked()
    binding.set_error_word(word)
    assert attention(12) == 0 and attention(9) == SLOT
    assert commit(8, 8) == (0, [True, True], [True, True], 4 * 256)
    assert commit(5, 8) == (SLOT, [True, False], [True, True], 3 * 256)
    assert commit(8, 3) == (HOST_ENTRY, [True, True], [True, False], 3 * 256)
    assert commit(8, 8, mb=1) == (BLOCK_ID, [True, False], [True, False], 2 * 256)
    binding.set_error_word(None)
    print(json.dumps({"ok": True}))


if __name__ == "__main__":
    main()
