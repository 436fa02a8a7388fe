"""Worker of test_gpu_packed_checked.py: a process of its own with OASIS_LIB pointing at the bounds-check build.  Indices between a
DECLARED extent and the (larger) size really allocated are flagged and skipped; nothing here can leave an allocation even if a check
were wrong."""
import json
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from oracle import oracle  # noqa: E402
from paper_2608_08097_b200 import binding, pipeline  # noqa: E402
from tests.packed_loop import Loop  # noqa: E402

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


def engine(K, **shape):
    """A loop over packed blocks against the oracle with the real extents declared: no check may fire."""
    B, Hkv, blocks = 2, 2, 16
    binding.set_extents(B * blocks * Hkv, B * Hkv * max(K, 2))
    loop = Loop(oracle, pipeline, B=B, Hq=8, Hkv=Hkv, K=K, max_blocks=blocks, layers=2, seq0=[100, 77], steps=7, cap=1, **shape)
    assert loop.eng.layers[0].pool.shape[0] == B * Hkv * K and loop.eng.layers[0].local.shape[0] == B * Hkv * 2
    assert take_code() == 0, "a check fired on valid indices"
    loop.run()
    code = take_code()
    binding.set_extents(0, 0)
    return code


assert binding.bounds_checked()
binding.set_error_word(word)
every = [0, 1, 2, 3, 4, 5]
assert source_pages() == [(0, every), (0, every), (HOST_ENTRY, [0, 1, 4, 5]), (0, every)]
oracle.lib()
assert [engine(6, T=3), engine(1, T=2), engine(4, T=9, host=True)] == [0, 0, 0]
print(json.dumps({"ok": True}))
