"""Appending to the paged cache where the other tests' sizes do not lead: scales at the ends of their range, and the row loop that a real model's prefill takes
(16 or more heads of 128 to a token, thousands of tokens). Against 64 bits."""
import numpy as np
import pytest
import torch

import fp8_util as u

pytestmark = pytest.mark.gpu
BF16, FP16, F8 = torch.bfloat16, torch.float16, u.F8


@pytest.fixture(autouse=True)
def _announce(request):
    print("\n[case] %s" % request.node.name, flush=True)
    yield


@pytest.fixture(scope="module")
def lib():
    from paper_2503_14985_amd import binding
    return binding


def dev():
    return torch.device("cuda:0")


def f64(t):
    return t.detach().cpu().to(torch.float32).double().numpy()


@pytest.mark.parametrize("exponent", [-100, -99.5, -60, 100, 119.5, 120, 120.5, 123, 125.25, 126])
def test_scales_at_the_ends_of_their_range(lib, exponent):
    """Earlier tokens with a scale of any size: a power of two is kept, another one raised to the next, and with it the tokens are rounded again, every e4m3 number among them."""
    H, D, block = 2, 64, 16
    codes = torch.arange(256, dtype=torch.uint8)
    codes[[127, 255]] = 0
    kc = codes.repeat(2 * H * block * D // 256).reshape(2, H, block, D).view(F8)
    vc = kc.clone().flip(0)
    scale = 2.0 ** exponent
    ks, vs = torch.full((2, H), scale), torch.full((2, H), scale * 0.5)
    if scale * 0.5 < 2.0 ** -100:
        vs = ks.clone()
    k = torch.randn((3, H, D), generator=torch.Generator().manual_seed(3)).mul(1e-30 if exponent > 0 else 1e-36).to(BF16)
    at = [t.to(dev()) for t in (k, k, torch.tensor([0, 1, 3], dtype=torch.int32), torch.tensor([9, 16], dtype=torch.int32), torch.tensor([[1], [0]], dtype=torch.int32))]
    Kc, Vc, Ks, Vs = (t.to(dev()) for t in (kc, vc, ks, vs))
    lib.mlt_paged_append_fp8(None, *at, None, None, Kc, Vc, Ks, Vs)
    spots = list(u.places([0, 1, 3], [9, 16], np.array([[1], [0]]), block, 2))
    for cache, scales, got, gots in ((kc, ks, Kc, Ks), (vc, vs, Vc, Vs)):
        want, wants = u.append_fp8(f64(k), f64(cache), f64(scales), spots)
        assert np.isfinite(want).all()
        assert np.array_equal(f64(gots), wants), (f64(gots), wants)
        assert np.array_equal(f64(got), want)
