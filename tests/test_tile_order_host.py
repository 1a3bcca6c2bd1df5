"""The order in which the step's plan lists tiles of many rows, on the host (no GPU)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.mark.skipif(not os.path.exists(os.path.join(ROCM, "include", "hip")), reason="no HIP headers")
def test_every_place_is_taken_once_whatever_the_lengths(tmp_path):
    exe = str(tmp_path / "order")
    r = subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error",
                        "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROCM, "include"), os.path.join(ROOT, "tests", "host", "tile_order_main.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "tile places agree" in r.stdout, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])
