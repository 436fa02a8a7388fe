"""Worker of test_gpu_packed_checked.py: a process of its own with OASIS_LIB pointing at the bounds-check build.  Indices between a
DECLARED extent and the (larger) size really allocated are flagged and skipped; nothing here can leave an allocation even if a check
were wrong."""
import json
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2608_08097_b200 import binding  # noqa: E402

HOST_ENTRY = 201
word = torch.zeros(1, dtype=torch.int32, device="cuda")


def take_code():
    torch.cuda.synchronize()
    c = int(word.item())
    word.zero_()
    return c


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def source_pages():
    """Three blocks of two heads from pages 2, 4 and 1 (entries 4, 5, 8, 9, 2, 3) to pages 0, 1 and 2; declared: all, or 8 entries."""
    kv = torch.randn((6, 2, 2, 16, 128), device="cuda").to(torch.bfloat16)
    dense = kv[:, :, 0].contiguous(), kv[:, :, 1].contiguous()
    dims, src, dst = binding.Dims(1, 2, 2, 4), i32([[2, 4, 1, 0]]), i32([[0, 1, 2, 3]])
    got = []
    for declared in (12, 8):
        for hand_over in (False, True):                  # (a dense pool has no declared extent)
            out = torch.zeros((12, 2304), dtype=torch.uint8, device="cuda")
            binding.set_extents(declared, 0)
            if hand_over:
                binding.offload_blocks_packed(dims, *dense, src, dst, i32([0]), i32([3]), 3, out)
            else:
                binding.pack_blocks(dims, kv, src, i32([0]), i32([3]), 3, out, dst)
            got.append((take_code(), [j for j in range(12) if bool(out[j].any())]))
    binding.set_extents(0, 0)
    return got


assert binding.bounds_checked()
binding.set_error_word(word)
every = [0, 1, 2, 3, 4, 5]
assert source_pages() == [(0, every), (0, every), (HOST_ENTRY, [0, 1, 4, 5]), (0, every)]
print(json.dumps({"ok": True}))
