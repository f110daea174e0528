"""Two threads that make calls on one stream: a call that leaves partial results to a second launch of its own enqueues both without another thread's in between, which would write the same scratch
(tests/host/threads_driver.cpp stands in for the HIP runtime; no kernel runs and no device is needed)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LIB_DIR = os.path.join(ROOT, "paper_2503_14985_amd")


def test_the_launches_of_a_call_stay_together(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    exe = str(tmp_path / "threads_driver")
    cmd = [HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", os.path.join(ROOT, "tests", "host", "threads_driver.cpp"),
           "-x", "none", "-o", exe, os.path.join(LIB_DIR, "libmlt.so"), "-Wl,-rpath," + LIB_DIR, "-pthread"]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    env = {k: v for k, v in os.environ.items() if not k.startswith("MLT_")}
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, r.stdout + r.stderr[-2000:]
    lines = [line.split() for line in r.stdout.splitlines()]
    assert [x[0] for x in lines] == ["packed", "prompt", "prefix", "w4", "mha", "paged", "paged_fp8"]
    assert all(x[1] == "2" for x in lines), r.stdout                 # each of them is one of two launches
    assert all(x[2] == "0" for x in lines), r.stdout
