"""How the kernels of include/ress_layer.h spread over the chip (layer_plan.cpp), under host sanitizers: built with launchers
that enqueue nothing, the checks run in a child process (CPU only)."""
import glob
import os
import subprocess

import pytest

from test_sanitizers import HERE, HIPCC, ROOT, _run_child


def test_plans_under_sanitizers(tmp_path):
    rt = sorted(glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so"))
    if not rt:
        pytest.skip("clang sanitizer runtime not found")
    csrc = os.path.join(ROOT, "paper_2609_35593_amd", "csrc")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    base = [HIPCC, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Xclang", "-target-feature",
            "-Xclang", "-packed-fp32-ops", "-I" + os.path.join(ROOT, "include"), "-I" + csrc, "-x", "hip", "-c"]
    objs, lib = [], tmp_path / "libress_plans_san.so"
    for src, flags in ((os.path.join(csrc, "layer_api.cpp"), san), (os.path.join(csrc, "layer_plan.cpp"), san),
                       (os.path.join(HERE, "sanitize", "plan_stubs.cpp"), [])):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.run([*base, *flags, src, "-o", objs[-1]], check=True, capture_output=True)
    subprocess.run([HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", str(lib)], check=True, capture_output=True)
    out = _run_child([os.path.join(HERE, "sanitize", "plan_checks.py"), str(lib)], rt[-1])
    assert "plan checks ok" in out
