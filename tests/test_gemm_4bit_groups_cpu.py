"""The tile kernel of mlt_gemm_w4 reads no scale and no zero point behind the last group (tests/host/gemm_4bit_groups_driver.cpp): what such a read would fetch lands where no product
looks, so that no comparison of results can show it."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def test_no_group_behind_the_last_one_is_read(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    exe = str(tmp_path / "gemm_4bit_groups_driver")
    r = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-Wno-inline-asm", "-x", "hip", os.path.join(ROOT, "tests", "host", "gemm_4bit_groups_driver.cpp"), "-o", exe],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout) > 0
