"""The C ABI layer and the plans of include/ress_pages.h under host sanitizers, as tests/test_sanitizers.py does it for ress.h
(CPU only: built with launchers that enqueue nothing, the checks run in a child process)."""
import glob
import os
import subprocess

import pytest

from test_sanitizers import HERE, HIPCC, ROOT, _run_child


def test_pages_under_sanitizers(tmp_path):
    rt = sorted(glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so"))
    if not rt:
        pytest.skip("clang sanitizer runtime not found")
    csrc = os.path.join(ROOT, "paper_2609_35593_amd", "csrc")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    base = [HIPCC, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Xclang", "-target-feature",
            "-Xclang", "-packed-fp32-ops", "-I" + os.path.join(ROOT, "include"), "-I" + csrc, "-x", "hip", "-c"]
    objs, lib = [], tmp_path / "libress_pages_san.so"
    for src, flags in ((os.path.join(csrc, "pages_api.cpp"), san), (os.path.join(csrc, "pages_plan.cpp"), san),
                       (os.path.join(HERE, "sanitize", "pages_stubs.cpp"), [])):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.run([*base, *flags, src, "-o", objs[-1]], check=True, capture_output=True)
    subprocess.run([HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", str(lib)], check=True, capture_output=True)
    out = _run_child([os.path.join(HERE, "sanitize", "pages_checks.py"), str(lib)], rt[-1])
    assert "pages checks ok" in out
