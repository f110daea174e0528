"""Decode attention over the 8-bit cache where a wavefront's references move: scores and value scales that change from unit to unit. Against 64 bits."""
import pytest
import torch

import fp8_attn_util as a

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16
WEIGHT_HALF = 2.0 ** -22                                                  # the weights in the second product: 11 bits, and 11 of what they leave


@pytest.fixture(autouse=True)
def _announce(request):
    print("\n[case] %s" % request.node.name, flush=True)
    yield


@pytest.fixture(scope="module")
def lib():
    from paper_2503_14985_amd import binding
    return binding


@pytest.fixture
def key_split(lib):
    yield lib.mlt_diag_force_key_split
    lib.mlt_diag_force_key_split(0)


def dev():
    return torch.device("cuda:0")


def on_gpu(c):
    return {k: v.to(dev()) if torch.is_tensor(v) else v for k, v in c.items()}


def run(lib, c):
    return lib.mlt_paged_attn_decode_fp8(c["q"], c["kc"], c["vc"], c["ks"], c["vs"], c["table"], c["lens"], c["scale"])


def check(lib, c, rounds):
    O = run(lib, c)
    o, more = a.exact(**c)
    tol = a.tolerance(o, more, int(c["lens"].max()), o.shape[2], O.dtype, rounds, WEIGHT_HALF)
    assert bool((tol < 0.1 * o.abs()).all())                              # no result but the right one fits
    err = (O.double() - o).abs()
    print("   kernel=%s worst %.2f of the tolerance" % (lib.mlt_last_kernel(), float((err / tol).max())), flush=True)
    assert bool(torch.isfinite(O.float()).all()) and bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP16, 64)])
@pytest.mark.parametrize("kind,step", a.CASES)
def test_references_move(lib, key_split, kind, step, dtype, D):
    """Eight wavefronts, six units each; in three ranges, two units each."""
    c = on_gpu(a.units_case(kind, step, 8, 6, D, dtype, 5))
    for split in (1, 3):
        key_split(split)
        check(lib, c, 6)
        assert lib.mlt_last_kernel() == "paged_decode_fp8_d%d_w8%s" % (D, "_keysplit3" if split > 1 else "")


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (FP16, 128)])
@pytest.mark.parametrize("kind,step", a.CASES)
def test_references_move_with_four_wavefronts(lib, key_split, kind, step, dtype, D):
    """The same sequence many times over: more workgroups than two a CU, which have four wavefronts."""
    key_split(1)
    one = a.units_case(kind, step, 4, 6, D, dtype, 7)
    c = on_gpu(one)
    B = 300
    many = dict(c, q=c["q"].repeat(B, 1, 1), table=c["table"].repeat(B, 1).contiguous(), lens=c["lens"].repeat(B).contiguous())
    O = run(lib, many)
    assert lib.mlt_last_kernel() == "paged_decode_fp8_d%d_w4" % D
    o, more = a.exact(**c)
    tol = a.tolerance(o, more, int(one["lens"]), D, dtype, 6, WEIGHT_HALF)
    assert bool((tol < 0.1 * o.abs()).all()) and bool(((O[:1].double() - o).abs() <= tol).all())
    assert torch.equal(O, O[:1].expand_as(O))


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -12])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_keep_22_bits(lib, D, scale):
    """Few keys, (nearly) equal scores and value scales of any mantissa, positive values: nothing averages out, and a weight of 11 bits would show beside the
    output's rounding. The bound is that of `tolerance` with 2^-22 for the weights (11 bits, and 11 of what they leave) and half the output's own step instead of half
    of the largest relative one."""
    g = torch.Generator().manual_seed(17)
    H, G, block = 4, 2, 16
    lens = [1, 2, 5, 16, 17, 31, 32, 33, 64, 100]
    nb = len(lens) * 7
    kc, vc = (torch.randn((nb, H, block, D), generator=g).mul_(60).abs().add_(8).to(a.F8) for _ in range(2))
    ks, vs = (torch.exp2(torch.rand((nb, H), generator=g) * 3 - 8) for _ in range(2))
    c = on_gpu(dict(q=torch.randn((len(lens), H * G, D), generator=g).to(FP16), kc=kc, vc=vc, ks=ks, vs=vs, scale=scale,
                    table=torch.randperm(nb, generator=g).to(torch.int32).reshape(len(lens), 7).contiguous(), lens=torch.tensor(lens, dtype=torch.int32)))
    O = run(lib, c)
    o, more = a.exact(**c)
    n = c["lens"].double()[:, None, None]
    tol = a.tolerance(o, more, n, D, FP16, 1, WEIGHT_HALF) - (a.HALF[FP16] * o.abs() - a.half_step(o, FP16))
    err = (O.double() - o).abs()
    print("   worst %.2f of the tolerance, %.3f of the results beyond it" % (float((err / tol).max()), float((err > tol).double().mean())), flush=True)
    assert bool((tol < 1.5 * a.half_step(o, FP16)).all()) and bool((err <= tol).all())
