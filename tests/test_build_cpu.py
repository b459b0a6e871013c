"""What is built when, without a GPU: the CUDA library alone carries the bf16 path; the module that checks the 4-bit path's tensors
belongs to one torch and one Python."""
import ctypes
import subprocess
import types

import pytest
import torch

import paper_2609_34555_b200 as pkg
from paper_2609_34555_b200 import binding, build


@pytest.fixture
def no_compiler(monkeypatch):
    build.build()                                                # (whatever is out of date is built before there is none)
    build.build_front()
    monkeypatch.setenv("CXX", "/bin/false")
    monkeypatch.setenv("NVCC", "/bin/false")


def test_the_library_is_there_without_the_module(monkeypatch, no_compiler, tmp_path):
    """A program on bf16 blocks with a built library needs no C++ compiler and no headers of torch."""
    pkg.load_library()
    monkeypatch.setattr(build, "front_path", lambda: tmp_path / "none.so", raising=False)
    monkeypatch.setattr(build, "FRONT", tmp_path / "none.so", raising=False)
    assert build.build() == build.LIB
    with pytest.raises(subprocess.CalledProcessError):
        build.build_front()


def test_a_context_asks_for_the_module_with_the_first_call_that_needs_it(monkeypatch):
    def none():
        raise OSError("no module")

    lib = types.SimpleNamespace(pi_create=lambda cfg, out: 0, pi_kv4_block_bytes=lambda ctx: 20480, pi_destroy=lambda ctx: None, pi_clear_status=lambda ctx: 0)
    monkeypatch.setattr(binding, "load_library", lambda rebuild=False: lib)
    monkeypatch.setattr(binding, "load_front", none)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    pi = pkg.PulseInfer(n_layers=1, n_q_heads=32, n_kv_heads=8, block_tokens=16, budget_blocks=8, n_sink_blocks=1, n_local_blocks=1, pool_slots=8,
                        max_batch=1, max_blocks=8, solo_head=[0])
    pi.clear_status()
    with pytest.raises(OSError, match="no module"):
        pi.kv4_load(torch.zeros((1, 20480), dtype=torch.uint8), None, stream=0)
    with pytest.raises(AttributeError):
        pi.no_such_call
    pi._ctx = ctypes.c_void_p(1)
    pi.close()


def test_the_module_is_built_anew_for_another_torch_or_python(monkeypatch, no_compiler):
    monkeypatch.delenv("CXX")
    here = build.build_front()
    monkeypatch.setenv("CXX", "/bin/false")
    assert build.build_front() == here                           # up to date: nothing is compiled
    names = {here}
    for change in (lambda m: m.setattr(torch, "__version__", "9.9.9"), lambda m: m.setattr(torch._C, "_GLIBCXX_USE_CXX11_ABI", not torch._C._GLIBCXX_USE_CXX11_ABI),
                   lambda m: m.setattr(build.sysconfig, "get_config_var", lambda name: ".cpython-399-other.so")):
        with monkeypatch.context() as m:
            change(m)
            with pytest.raises(subprocess.CalledProcessError):
                build.build_front()
            names.add(build.front_path())
    assert len(names) == 4


def test_the_append_kernels_keep_their_state_in_registers(tmp_path):
    """What the compiler says of both forms, bf16 and 4-bit blocks: nothing is spilled, and the bf16 form stays at 32 registers."""
    import os
    import re
    said = subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xptxas=-v", f"-I{build.INCLUDE}",
                           f"-I{build.CSRC}", "-c", "-o", str(tmp_path / "a.o"), str(build.CSRC / "pi_append.cu")], check=True, capture_output=True, text=True).stderr
    assert re.findall(r"(\d+) bytes spill stores, (\d+) bytes spill loads", said) == [("0", "0")] * 2
    assert min(int(n) for n in re.findall(r"Used (\d+) registers", said)) <= 32
