"""CPU checks of the draft-tree calls: refusals made on the host, lifetimes and the build."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2608_08097_b200 import binding, build
    build.build()
    return binding


ONE, ODD = 4096, 4104          # never dereferenced on the host; the second one is not 16-byte aligned


def test_refusals_of_the_tree_scoring(L):
    lib = L.lib()

    def call(dims=L.Dims(2, 32, 8, 64), q=ONE, T=5, nodes=ONE, summ=ONE, n_full=ONE, mode=0, scores=ONE, cand=None):
        d = dims.c()
        return lib.oasis_score_tree(ctypes.byref(d), q, T, nodes, summ, n_full, mode, scores, cand, None)

    for name in ("q", "nodes", "summ", "n_full", "scores"):
        assert call(**{name: None}) == 1, name
    for bad in (dict(q=ODD), dict(summ=ODD), dict(T=0), dict(T=65), dict(mode=2), dict(mode=-1), dict(dims=L.Dims(2, 30, 8, 64))):
        assert call(**bad) == 1, bad
    for bad in (dict(dims=L.Dims(2, 258, 2, 64)), dict(dims=L.Dims(1 << 12, 32, 8, 1 << 17)), dict(dims=L.Dims(2, 32, 8, 64, head_dim=64))):
        assert call(**bad) == 2, bad
    assert call(dims=L.Dims(0, 32, 8, 64), q=None) == 0


def test_a_dims_struct_is_made_once_whatever_the_threads_do(L, monkeypatch):
    """A second thread makes the struct while the first one is making it: both have to end with the same one, and the one whose
    address was handed out has to live on."""
    import threading
    d, inner, made = L.Dims(2, 32, 8, 64), [], []
    real = L.Dims.c

    def slow(self):
        made.append(real(self))
        if len(made) == 1:
            t = threading.Thread(target=lambda: inner.append(L._cdims(d)))
            t.start()
            t.join()
            return made[0]
        return made[-1]

    monkeypatch.setattr(L.Dims, "c", slow)
    outer = L._cdims(d)
    assert len(inner) == 1 and inner[0] == outer == L._cdims(d)
    assert ctypes.cast(outer, ctypes.POINTER(L._Dims)).contents.n_q_heads == 32


HARNESS = r"""
#include <cuda_runtime.h>
#include <chrono>
#include <cstdio>
#include <thread>
static cudaError_t slow_entry_point(const char *, void **ptr, unsigned long long, cudaDriverEntryPointQueryResult *q)
{
    std::this_thread::sleep_for(std::chrono::milliseconds(300));
    *ptr = (void *)0x1000;
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
#define cudaGetDriverEntryPoint slow_entry_point
#include "common.cuh"
#include "tc_common.cuh"
int main()
{
    bool got[4];
    std::thread t[4];
    for (int i = 0; i < 4; ++i) t[i] = std::thread([&, i] { got[i] = oasis::encode_tiled_fn() != nullptr; });
    for (auto &x : t) x.join();
    std::printf("%d %d %d %d\n", got[0], got[1], got[2], got[3]);
}
"""


def test_threads_that_ask_for_the_drivers_encoder_together(L, tmp_path):
    """The driver's answer takes a while: no thread may go on without it."""
    import os
    import subprocess
    from paper_2608_08097_b200 import build
    (tmp_path / "first.cu").write_text(HARNESS)
    exe = str(tmp_path / "first")
    subprocess.run([build.NVCC, *build.ARCH, "-std=c++17", "-I" + build.CSRC, "-o", exe, str(tmp_path / "first.cu"),
                    os.path.join(build.OBJ, "api.o")], check=True, capture_output=True)
    assert subprocess.run([exe], capture_output=True, text=True, timeout=60).stdout.split() == ["1"] * 4


def test_the_c_library_builds_without_torch(L, monkeypatch, tmp_path):
    import importlib.util
    from paper_2608_08097_b200 import build
    real = importlib.util.find_spec
    monkeypatch.setattr(build, "CALL", str(tmp_path / "_call.so"))      # (not built yet)
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else real(name, *a))
    assert build.build() == build.LIB and not (tmp_path / "_call.so").exists()


def test_the_python_calls_are_built_again_for_another_torch(L, monkeypatch):
    from paper_2608_08097_b200 import build
    ran = []

    class Failed:
        returncode, stdout, stderr = 1, "", "(not run)"

    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: ran.append(cmd) or Failed)
    assert build.build() == build.LIB and not ran                    # up to date: nothing is run
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "99.0")
    with pytest.raises(RuntimeError, match="g.. failed"):
        build.build()
    assert len(ran) == 1 and any("py_call.cpp" in x for x in ran[0])


def test_the_attention_lets_a_successor_start_only_after_its_own_wait(L):
    """oasis_attn_and_score reads its scoring inputs without a wait: a launch between it and their producer separates the two
    only if it lets a successor start after it has waited for the producer itself."""
    import os
    import re
    from paper_2608_08097_b200 import build
    text = open(os.path.join(build.CSRC, "tree_attn.cu")).read()
    kernel = text[text.index("tree_attn_tc_kernel(const"):text.index("tree_combine_kernel(const")]
    assert re.findall(r"griddepcontrol\.(\w+)", kernel) == ["wait", "launch_dependents"]
    for name in ("verify.cu", "commit.cu"):                          # these never let a successor start early
        assert re.findall(r"griddepcontrol\.(\w+)", open(os.path.join(build.CSRC, name)).read()) == ["wait"]


def test_steps_with_trees_are_captured_one_at_a_time():
    """No commit can lie between the steps of one graph."""
    from paper_2608_08097_b200 import pipeline
    eng = pipeline.DecodeEngine.__new__(pipeline.DecodeEngine)
    eng.tree = True
    with pytest.raises(ValueError, match="commit"):
        eng.capture_steps([((), {}), ((), {})])
