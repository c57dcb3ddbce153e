"""The ranges of a split context, checked on the host over lengths up to the largest (tests/native/attend_split_check.cpp
compiles the code that the attention's kernels share with it)."""
import os
import subprocess

import pytest

from paper_2606_03819_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_ranges_cover_a_context_of_any_length(tmp_path):
    hipcc = build.hipcc()
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    exe = tmp_path / "attend_split_check"
    rocm_inc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(hipcc))), "include")
    c = subprocess.run([hipcc, "-O1", "-std=c++17", "-x", "c++", "-D__HIP_PLATFORM_AMD__", "-I", rocm_inc, "-I", build.CSRC,
                        os.path.join(HERE, "native", "attend_split_check.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert c.returncode == 0, c.stderr[-3000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    print(r.stdout)
    assert r.returncode == 0 and r.stdout.strip().endswith(" 0 failures"), r.stdout
