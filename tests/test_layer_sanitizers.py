"""The C ABI layer of include/ress_layer.h under host sanitizers, as tests/test_sanitizers.py does it for ress.h (CPU
only: built with launchers that enqueue nothing, the checks run in a child process)."""
import glob
import os
import subprocess

import pytest

from test_sanitizers import HERE, HIPCC, ROOT, _run_child


def test_layer_abi_under_sanitizers(tmp_path):
    rt = sorted(glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so"))
    if not rt:
        pytest.skip("clang sanitizer runtime not found")
    inc = ["-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2609_35593_amd", "csrc")]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    base = [HIPCC, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Xclang", "-target-feature",
            "-Xclang", "-packed-fp32-ops", *inc, "-x", "hip", "-c"]
    api_o, stub_o, lib = tmp_path / "api.o", tmp_path / "stub.o", tmp_path / "libress_layer_san.so"
    subprocess.run([*base, *san, os.path.join(ROOT, "paper_2609_35593_amd", "csrc", "layer_api.cpp"), "-o", str(api_o)],
                   check=True, capture_output=True)
    subprocess.run([*base, os.path.join(HERE, "sanitize", "layer_stubs.cpp"), "-o", str(stub_o)], check=True,
                   capture_output=True)
    subprocess.run([HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", str(api_o), str(stub_o), "-o", str(lib)],
                   check=True, capture_output=True)
    out = _run_child([os.path.join(HERE, "sanitize", "layer_checks.py"), str(lib)], rt[-1])
    assert "layer checks ok" in out
