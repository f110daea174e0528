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


@pytest.mark.parametrize("split", [1, 3])
@pytest.mark.parametrize("size", [1e3, 1e5, 1e7, 3e8, 1e20, -1e5, -3e8, -1e20])
def test_scores_of_any_size(lib, key_split, size, split):
    """Equal scores, however large, weigh all keys alike: the mean of the values, whose scales differ. And with one key in front by any margin it is that key's value."""
    g = torch.Generator().manual_seed(23)
    H, D, block, n = 2, 64, 32, 1600
    nb = n // block
    q = torch.ones((1, 2 * H, D), dtype=BF16)
    kc = torch.ones((nb, H, block, D)).to(a.F8)
    vc = (torch.rand((nb, H, block, D), generator=g) * 200 + 100).to(a.F8)
    ks, vs = torch.ones((nb, H)), torch.exp2(torch.rand((nb, H), generator=g) * 12 - 12)
    c = on_gpu(dict(q=q, kc=kc, vc=vc, ks=ks, vs=vs, table=torch.randperm(nb, generator=g).to(torch.int32).reshape(1, -1).contiguous(),
                    lens=torch.tensor([n - 3], dtype=torch.int32), scale=size / D))
    key_split(split)
    O = run(lib, c).double()
    o, more = a.exact(**c)
    # fp32 sums over n keys, exp2 and the references' rescalings (sizes of at most 16 here, whatever the scores': the same number is taken off them first)
    rel = 2.0 ** -8 + 2.0 ** -22 + 2 * (n * 2.0 ** -24 + 8 * 16 * 3 * 2.0 ** -24)
    assert bool(((O - o).abs() <= rel * o.abs()).all()), float(((O - o).abs() / o.abs()).max())
    if size > 0:
        first = int(c["table"][0, 7])
        c["kc"].view(torch.uint8)[first, :, 5] = 0x40                      # 2.0: twice the others' score
        O = run(lib, c).double()
        want = (c["vc"][first, :, 5].double() * c["vs"][first].double()[:, None]).repeat_interleave(2, 0)
        assert bool(((O[0] - want).abs() <= rel * want).all())


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_zero_scales(lib, key_split, dtype):
    """Blocks whose values' scale is 0 (a quantiser's for a block of zeros) count as zeros and take no bits from the others, whose scales are small."""
    g = torch.Generator().manual_seed(29)
    H, D, block, n = 2, 128, 32, 2048
    nb = n // block
    vs = torch.exp2(torch.rand((nb, H), generator=g) - 12)
    q = torch.randn((1, 2 * H, D), generator=g).to(dtype)
    kc, vc = (torch.rand((nb, H, block, D), generator=g).mul(200).add(100).to(a.F8) for _ in range(2))
    table = torch.arange(nb, dtype=torch.int32).reshape(1, -1)
    key_split(1)
    c = on_gpu(dict(q=q, kc=kc, vc=vc, ks=torch.full((nb, H), 2.0 ** -12), vs=vs, table=table, lens=torch.tensor([n], dtype=torch.int32), scale=1 / D ** 0.5))
    for lo in (1.0, 2.0 ** -30, 2.0 ** -60):
        small = c["vs"] * lo
        none = small.clone()
        none[::3] = 0.0
        unit = 1.0 if lo == 1.0 else 1 / lo                                # (compared in units of the scales: the outputs themselves are small)
        O = run(lib, dict(c, vs=none)).double() * unit
        ref = dict(c, vs=c["vs"].clone())
        ref["vs"][::3] = 2.0 ** -100
        o, more = a.exact(**ref)
        tol = a.tolerance(o, more, n, D, dtype, 8, WEIGHT_HALF) + (2.0 ** -25 * unit if dtype == FP16 else 0.0)
        if dtype == BF16 or lo == 1.0:
            assert bool(((O - o).abs() <= tol).all()), (lo, float(((O - o).abs() / tol).max()))
