"""Launches of the 8-bit operators that would have more than 2^32 work-items are refused, with nothing enqueued (tests/host/fp8_limits_driver.cpp): the runtime would
take the number modulo 2^32 and leave workgroups out without an error."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LIB_DIR = os.path.join(ROOT, "paper_2503_14985_amd")


def test_launches_past_2_32_work_items_are_refused(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    exe = str(tmp_path / "fp8_limits_driver")
    r = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", os.path.join(ROOT, "tests", "host", "fp8_limits_driver.cpp"),
                        "-x", "none", "-o", exe, os.path.join(LIB_DIR, "libmlt.so"), "-Wl,-rpath," + LIB_DIR], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"))
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == ["-2"] * 12, r.stdout            # MLT_ERR_UNSUPPORTED
