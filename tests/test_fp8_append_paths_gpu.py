"""Appending to the paged cache where the other tests' sizes do not lead: scales at the ends of their range, and the row loop that a real model's prefill takes
(16 or more heads of 128 to a token, thousands of tokens). Against 64 bits."""
import numpy as np
import pytest
import torch

import fp8_util as u
from test_fp8_gpu import append_case

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


# ---- a prefill's rows: four accesses of a token at once, with 16 or more heads of 128 and 2048 or more tokens

@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("fp8,Hq,H", [(True, 16, 1), (True, 17, 2), (True, 19, 1), (True, 32, 8), (True, 33, 1), (False, 12, 2), (False, 9, 4), (False, 5, 7), (False, 0, 8), (False, 14, 3),
                                      (False, 40, 3)])
def test_prefill_rows(lib, fp8, Hq, H, interleaved):
    """Heads that fill the accesses and heads that do not, which of a token's rows are queries, keys and values falling anywhere in them; padding rows at the end."""
    new, before = [1300, 0, 1, 740, 9], [5, 40, 16, 0, 31]
    append_case(lib, new, before, Hq, H, 128, 16, 128, interleaved, BF16, fp8, 19, pad=6)
    assert sum(new) >= 2048


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 96])
def test_prefill_rows_partly_turned(lib, fp8, rot):
    append_case(lib, [2048, 3], [7, 0], 20, 2, 128, 32, rot, False, FP16, fp8, 23)


def test_prefill_rows_without_a_place(lib):
    """Positions past the table of angles and block numbers outside the cache, in the same loop."""
    def bad(t):
        t = t.clone()
        t[0, 3], t[1, 1] = -1, 1 << 30
        return t
    for fp8 in (False, True):
        append_case(lib, [1900, 200], [0, 4], 16, 2, 128, 16, 128, False, BF16, fp8, 29, tables=bad, positions=700)


def test_zero_scale_of_earlier_tokens(lib):
    """Earlier tokens with a scale of 0 are zeros, and stay so in the scale of the new ones."""
    H, D, block = 2, 64, 16
    kc = torch.full((1, H, block, D), 3.0).to(F8).to(dev())
    vc, ks, vs = kc.clone(), torch.zeros((1, H), device=dev()), torch.zeros((1, H), device=dev())
    k = torch.randn((2, H, D), generator=torch.Generator().manual_seed(5)).to(BF16).to(dev())
    k[:, 1] = 0.0                                                          # a head whose new tokens are zeros too
    at = [torch.tensor(v, dtype=torch.int32, device=dev()) for v in ([0, 2], [11], [[0]])]
    lib.mlt_paged_append_fp8(None, k, k, *at, None, None, kc, vc, ks, vs)
    for c, s in ((kc, ks), (vc, vs)):
        back = f64(c) * f64(s)[..., None, None]
        assert (back[0, :, :9] == 0).all()
        want, scales = u.append_fp8(f64(k), np.zeros((1, H, block, D)), np.full((1, H), 2.0 ** -100), [(0, 0, 9, 0, 9), (1, 0, 10, 0, 10)])
        assert np.array_equal(f64(s), scales) and np.array_equal(f64(c)[0, :, 9:11], want[0, :, 9:11])
        assert (f64(c)[0, :, 11:] == 3.0).all()
