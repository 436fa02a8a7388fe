"""CPU test of the kernels' sources: kernels that may be brought onto the SMs while the launch before them still runs wait
(griddepcontrol.wait) before they read what it writes.  The read-only path is closed to them: its loads need data that nobody writes
while the kernel is resident, and a compiler that takes pointers for __restrict__ may move their loads above the wait."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def kernels():
    """(file, name, signature, body) of every kernel."""
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2608_08097_b200", "csrc", "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__ void __launch_bounds__\((?:[^()]|\([^()]*\))*\)\s*(\w+)\(", text):
            brace = text.index("{", m.end())
            depth, at = 1, brace + 1
            while depth:
                depth += {"{": 1, "}": -1}.get(text[at], 0)
                at += 1
            yield os.path.basename(path), m.group(1), text[m.end():brace], text[brace:at]


WAITING = [k for k in kernels() if "griddepcontrol.wait" in k[3]]


def test_the_kernels_are_found():
    names = {k[1] for k in kernels()}
    assert len(names) >= 25 and {"pack_blocks_kernel", "unpack_blocks_kernel", "rotate_qkv_kernel", "packed_attn_kernel", "packed_attn_few_kernel",
                                 "packed_combine_kernel"} <= {k[1] for k in WAITING}


@pytest.mark.parametrize("file, name, signature, body", WAITING, ids=[k[1] for k in WAITING])
def test_a_kernel_that_waits_reads_nothing_through_the_read_only_path(file, name, signature, body):
    assert "__restrict__" not in signature
    for closed in ("ld_stream_v4", "__ldg", "ld.global.nc", "__restrict__"):
        assert closed not in body, (file, name, closed)


@pytest.mark.parametrize("file", ["attn.cu", "attn_tc.cu", "layer_tc.cu", "tree_attn.cu", "packed_attn.cu"])
def test_attention_launches_let_a_successor_start_early(file):
    """As the header says of them and of their merge launches (oasis_attn_and_score)."""
    found = [k for k in kernels() if k[0] == file]
    assert found
    for _, name, _, body in found:
        assert "griddepcontrol.launch_dependents" in body, name


def test_a_merge_of_splits_waits_before_it_lets_the_next_launch_start():
    """What follows packed_combine_kernel may read before it waits: the splits' launch must be over by then."""
    body = next(k[3] for k in kernels() if k[1] == "packed_combine_kernel")
    assert body.index("griddepcontrol.wait") < body.index("griddepcontrol.launch_dependents")
