"""Address and undefined-behaviour sanitizer run of the host side of the entry points for prompts, shared prefixes and 4-bit weights: calls that they must reject or accept as no-ops before anything
touches a GPU (tests/sanitize/abi_prompt_driver.cpp), built with the sanitizers and run as a child process."""
import os

import pytest

from test_sanitizers_cpu import CSRC, HIPCC, SAN, _run


def test_host_side_of_the_prompt_entry_points_under_sanitizers(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    others = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith(".o") and not f.endswith("_dbg.o") and f != "mlt_api.o"]
    if len(others) < 8:
        pytest.skip("library objects not built (run __graft_entry__.build_lib())")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
    api, drv, exe = (str(tmp_path / n) for n in ("mlt_api_san.o", "abi_prompt_driver.o", "san_abi_prompt"))
    _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"] + san +
         ["-c", os.path.join(CSRC, "mlt_api.hip"), "-o", api])
    _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17"] + san + ["-x", "hip", "-c", os.path.join(SAN, "abi_prompt_driver.cpp"), "-o", drv])
    _run([HIPCC, "--offload-arch=gfx950", "-fsanitize=address,undefined", "-fno-gpu-sanitize", "-o", exe, drv, api] + others)
    r = _run([exe])
    assert r.stdout.strip().endswith("ok"), r.stdout + r.stderr
