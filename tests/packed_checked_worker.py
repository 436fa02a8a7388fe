"""Worker of test_gpu_packed.py: a process of its own with OASIS_LIB pointing at the bounds-check build.  Slots and entries
between a DECLARED extent and the (larger) size really allocated are flagged and skipped by the packed cache's calls, and nothing
else is; nothing here can leave an allocation even if a check were wrong."""
import json
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2608_08097_b200 import binding  # noqa: E402
from oracle import packed as op  # noqa: E402

HOST_ENTRY, SLOT, BLOCK_COUNT = 201, 202, 204
word = torch.zeros(1, dtype=torch.int32, device="cuda")


def take_code():
    torch.cuda.synchronize()
    c = int(word.item())
    word.zero_()
    return c


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def entries(n, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((n, 2, 16, 128), generator=g, device="cuda").to(torch.bfloat16)


def pack_all(kv):
    n = kv.shape[0]
    out, t = torch.zeros((n, 2304), dtype=torch.uint8, device="cuda"), i32([list(range(n))])
    binding.pack_blocks(binding.Dims(1, 1, 1, n), kv, t, i32([0]), i32([n]), n, out, t)
    return out


def attention(declared, heads):
    """Eight packed columns and a local one; column 3 has slot 9, the local column slot 10."""
    binding.set_extents(0, 0)
    packed, local = pack_all(entries(12, 1)), entries(12, 2)
    q = entries(1, 3).view(1, 1, -1, 128)[:, :, :heads].contiguous()
    slot, blk = [[[0, 1, 2, 9, 4, 5, 6, 7, 10]]], [[list(range(9))]]
    binding.set_extents(0, declared)
    out, lse = torch.zeros_like(q), torch.zeros((1, 1, heads), device="cuda")
    dims = binding.Dims(1, heads, 1, 10)
    ws = torch.empty(max(16, binding.packed_attn_workspace_bytes(dims, 1, 9, 8)), dtype=torch.uint8, device="cuda")
    binding.packed_attn(dims, q, packed, local, i32(slot), i32(blk), 8, i32([140]), 1 / math.sqrt(128), out, lse=lse, workspace=ws)
    code, seen = take_code(), np.array(blk)
    seen[np.array(slot) >= declared] = -1
    ref, _, a, big = op.attn(q.double().cpu().numpy(), packed.cpu().numpy(), local.double().cpu().numpy(), np.array(slot), seen, 8, [140], 1 / math.sqrt(128))
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= 2.0 ** -8 * (a + np.abs(ref)) + 2.0 ** -14 * big[..., None] * a)
    return code


def packing(declared_entries, declared_slots, first, local):
    """Two blocks of one head: sources 2 and 9 (slots) or 2 and 3 (pages), destinations 4 and 11."""
    kv, out = entries(12, 5), torch.zeros((12, 2304), dtype=torch.uint8, device="cuda")
    dims, table = binding.Dims(1, 1, 1, 4), i32([[4, 11, 0, 0]])
    binding.set_extents(declared_entries, declared_slots)
    if local:
        binding.pack_local_layers(dims, [kv], [i32([[[0, 2, 9]]])], 1, i32([first]), i32([2]), 2, [out], [table])
    else:
        binding.pack_blocks(dims, kv, i32([[2, 3, 0, 0]]), i32([first]), i32([2]), 2, out, table)
    code = take_code()
    return code, [j for j in range(12) if bool(out[j].any())]


def moving(declared_entries, declared_slots):
    """Entries 3, 8 and 2 into slots 1, 2 and 9 (gather) or unpacked."""
    binding.set_extents(0, 0)
    packed, idx, slots = pack_all(entries(10, 7)), torch.tensor([3, 8, 2], device="cuda"), i32([1, 2, 9])
    pool, out = torch.zeros((12, 2304), dtype=torch.uint8, device="cuda"), torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    binding.set_extents(declared_entries, declared_slots)
    binding.stage_packed_layers([packed], [idx], [slots], 3, [pool])
    a = take_code()
    binding.unpack_blocks(packed, idx, out)
    b = take_code()
    return a, [j for j in range(12) if bool(pool[j].any())], b, [j for j in range(3) if bool(out[j].any())]


assert binding.bounds_checked()
binding.set_error_word(word)
flagged = []
for heads in (4, 20, 32):                                # few rows and many
    assert attention(12, heads) == 0
    assert attention(9, heads) == SLOT                   # columns 3 and 8
    flagged.append("attention %d" % heads)
assert attention(10, 4) == SLOT                          # the local column alone
assert packing(12, 12, 0, False) == (0, [4, 11]) and packing(11, 12, 0, False) == (HOST_ENTRY, [4])
assert packing(12, 12, 0, True) == (0, [4, 11]) and packing(12, 9, 0, True) == (SLOT, [4]) and packing(11, 12, 0, True) == (HOST_ENTRY, [4])
assert packing(12, 12, 3, False)[0] == BLOCK_COUNT
flagged.append("packing")
assert moving(10, 12) == (0, [1, 2, 9], 0, [0, 1, 2])
assert moving(8, 12) == (HOST_ENTRY, [1, 9], HOST_ENTRY, [0, 2]) and moving(10, 9) == (SLOT, [1, 2], 0, [0, 1, 2])
flagged.append("moving")
print(json.dumps({"ok": True, "flagged": flagged}))
