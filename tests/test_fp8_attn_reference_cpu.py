"""The cases and the bound of fp8_attn_util on the CPU: the kernel's arithmetic in numpy keeps the bound, and with a mistake in its rescaling it does not."""
import numpy as np
import pytest
import torch

import fp8_attn_util as a

BF16, FP16 = torch.bfloat16, torch.float16
WAVES, ROUNDS, D = 4, 6, 64


def _run(kind, step, dtype, wrong=""):
    c = a.units_case(kind, step, WAVES, ROUNDS, D, dtype, 3)
    n = int(c["lens"])
    o, more = a.exact(**c)
    tol = a.tolerance(o, more, n, D, dtype, ROUNDS, 2.0 ** -22)[0].numpy()
    at = c["table"][0].long()
    k, v, ks, vs = (c[x][at].double().numpy() for x in ("kc", "vc", "ks", "vs"))
    o = o[0].numpy()
    assert (tol < 0.1 * np.abs(o)).all()                                  # no result but the right one fits
    worst = 0.0
    for h in range(4):
        got = a.emulate(c["q"][0, h].double().numpy(), k[:, h // 2], ks[:, h // 2], v[:, h // 2], vs[:, h // 2], c["scale"], WAVES, n, wrong)
        got = torch.from_numpy(got).to(dtype).double().numpy()
        worst = max(worst, float((np.abs(got - o[h]) / tol[h]).max()))
    return worst


@pytest.mark.parametrize("kind,step", a.CASES)
def test_the_kernels_arithmetic_keeps_the_bound(kind, step):
    for dtype in (BF16, FP16):
        assert _run(kind, step, dtype) <= 1.0


@pytest.mark.parametrize("wrong", ["sum kept", "outputs kept"])
def test_a_reference_that_moves_without_its_sums_does_not(wrong):
    seen = [_run(kind, step, BF16, wrong) for kind, step in a.CASES]
    of_kind = {"sum kept": ("rise",), "outputs kept": ("rise", "scales_rise")}[wrong]
    assert all(w > 1.0 for w, (kind, _) in zip(seen, a.CASES) if kind in of_kind), seen


def test_weights_against_the_largest_scale_met_do_not():
    """... where that scale belongs to earlier keys of no weight: below 2^-24 of it the others' weights fall under fp16's smallest step."""
    for kind, step in a.CASES:
        if kind == "light_first" and step > 20:
            assert _run(kind, step, FP16, "scale reference") > 1.0, (kind, step)
