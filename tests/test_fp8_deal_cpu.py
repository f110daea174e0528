"""Which batches decode attention over the 8-bit cache deals out by sequence length (tests/host/fp8_deal_driver.cpp), on both sides of each of the rule's bounds."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LIB_DIR = os.path.join(ROOT, "paper_2503_14985_amd")

CASES = [  # B, H, D, block, blocks, ranges, wide -> dealt
    ((64, 8, 128, 16, 256, 1, 1), 1), ((65, 8, 128, 16, 256, 1, 0), 1), ((250, 4, 128, 16, 256, 1, 0), 1),
    ((64, 4, 128, 16, 256, 1, 1), 0), ((64, 4, 128, 16, 256, 2, 1), 1),                    # 256 workgroups: none waits
    ((128, 8, 128, 16, 64, 1, 0), 1), ((128, 8, 128, 16, 63, 1, 0), 0),                    # 256 KiB a workgroup
    ((128, 8, 64, 32, 64, 1, 0), 1), ((128, 8, 64, 32, 62, 1, 0), 0),
    ((129, 8, 128, 16, 64, 1, 0), 0), ((192, 8, 128, 16, 96, 1, 0), 1), ((193, 8, 128, 16, 96, 1, 0), 0),      # 2 KiB a sequence
    ((256, 8, 128, 16, 512, 1, 0), 1), ((257, 8, 128, 16, 512, 1, 0), 0), ((512, 1, 128, 16, 512, 1, 1), 1), ((513, 1, 128, 16, 512, 1, 1), 0),   # a thread for each length
    ((1, 600, 128, 16, 512, 1, 0), 0)]


def test_batches_dealt_by_length(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    exe = str(tmp_path / "fp8_deal_driver")
    r = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", os.path.join(ROOT, "tests", "host", "fp8_deal_driver.cpp"),
                        "-x", "none", "-o", exe, os.path.join(LIB_DIR, "libmlt.so"), "-Wl,-rpath," + LIB_DIR], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c, _ in CASES) + "\n", capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    assert [int(x) for x in r.stdout.split()] == [want for _, want in CASES]
