"""How mlt_gemm_fp8 adds up, as its header says: the products of an aligned group of 8 k in fixed point with 13 bits below the largest one's power of two, groups and
blocks in fp32. Sums that cancel show it. Every kernel."""
import numpy as np
import pytest
import torch

import fp8_util as u

pytestmark = pytest.mark.gpu
KERNELS = ["256pp16", "128pp16", "256x128kp", "224x128kp", "192x128kp", "128kp", "skinny"]


@pytest.fixture
def variant(request):
    from paper_2503_14985_amd import binding
    binding.mlt_diag_force_variant(gemm=request.param)
    binding.mlt_diag_force_k_parts(1)
    yield request.param
    binding.mlt_diag_force_variant(gemm="auto")
    binding.mlt_diag_force_k_parts(0)


def operands(small, apart, M, K, seed):
    """Rows of A, B all alike: in each row one group of 8 with +p and -p (p = 448 * 448, or 256 * 256 and another group of it) and `small` in up to six more places, of the
    same group or (apart) of other ones. small: (values of A, values of B) of those places."""
    g = np.random.default_rng(seed)
    a, b = np.zeros((M, K)), np.zeros(K)
    # B is shared, so places go by columns: position 8 i + e of every group has the same role in all of them
    b[0::8] = b[1::8] = 448.0
    b[2::8] = small[1]
    b[3:K:8], b[4:K:8], b[5:K:8], b[6:K:8], b[7:K:8] = (small[1],) * 5
    for m in range(M):
        i = g.integers(0, K // 8)
        a[m, 8 * i], a[m, 8 * i + 1] = 448.0, -448.0
        for e in range(2, 8):
            j = (i + 1 + g.integers(0, K // 8 - 1)) % (K // 8) if apart else i
            a[m, 8 * j + e] = small[0]
    return torch.from_numpy(a).to(u.F8), torch.from_numpy(b).to(u.F8)


def product(a, b, N, dtype):
    from paper_2503_14985_amd import binding
    dev, (M, K) = torch.device("cuda:0"), a.shape
    one = lambda *s: torch.ones(s, device=dev)  # noqa: E731
    C = binding.mlt_gemm_fp8(a.to(dev), one(K // 128, M), b[None].repeat(N, 1).to(dev), one(K // 128, -(-N // 128)), dtype=dtype)
    assert torch.equal(C, C[:, :1].expand_as(C))                          # every column alike
    return C[:, 0].double().cpu().numpy()


@pytest.mark.parametrize("variant", KERNELS, indirect=True)
@pytest.mark.parametrize("small", [(1.0, 1.0), (1.5, 3.0), (0.0625, 0.25), (5.0, 3.0)])
def test_cancelling_groups_keep_the_headers_bound(variant, small):
    M, N, K = 150, 200, 512
    for dtype in (torch.bfloat16, torch.float16):
        a, b = operands(small, False, M, K, 1)
        a64, b64 = a.double().numpy(), b.double().numpy()
        ref = a64 @ b64
        top = np.abs(a64 * b64).reshape(M, -1, 8).max(2).sum(1)           # of each group the largest product
        off = np.abs(product(a, b, N, dtype) - ref)
        assert (ref == 6 * small[0] * small[1]).all() and (off < 7 * 2.0 ** -13 * top).all(), float(off.max())
        # in groups of their own the same numbers are added exactly: 9 bits at most, and the cancelling group's sum is 0
        a, b = operands(small, True, M, K, 2)
        assert (product(a, b, N, dtype) == ref).all()


@pytest.mark.parametrize("variant", KERNELS, indirect=True)
def test_thirteen_bits_below_the_largest_product(variant):
    """Beside 2^16 in their group, products of 2^3 count; smaller ones may not, and are off by less than 2^3 each."""
    M, N, K = 70, 90, 256
    for value, exact in ((8.0, True), (24.0, True), (7.0, False), (0.5, False)):
        a, b = torch.zeros((M, K)), torch.ones(K)
        at = torch.arange(M) % 16
        row = torch.arange(M)
        for e in range(1, 8):
            a[row, 8 * at + e] = value
        a[row, 8 * at], a[row, 8 * (at + 16)] = 256.0, -256.0            # the sum's 2^16 goes away again in another group
        b[0::8] = 256.0
        got = product(a.to(u.F8), b.to(u.F8), N, torch.float16)
        off = np.abs(got - 7 * value)
        assert (off == 0).all() if exact else (off < 7 * 8.0).all(), (value, got[:4])


@pytest.mark.parametrize("variant", KERNELS, indirect=True)
def test_zero_scales(variant):
    """Blocks of A or B with a scale of 0 add nothing, whatever their numbers."""
    from paper_2503_14985_amd import binding
    dev, (M, N, K) = torch.device("cuda:0"), (150, 300, 512)
    g = torch.Generator().manual_seed(7)
    a, b = (torch.randint(-8, 9, (r, K), generator=g).float() for r in (M, N))
    sa, sb = torch.exp2(torch.randint(-2, 3, (4, M), generator=g).float()), torch.exp2(torch.randint(-2, 3, (4, 3), generator=g).float())
    sa[1, ::2], sb[2, 1] = 0.0, 0.0
    ref = ((a.double() * sa.t().double().repeat_interleave(128, 1)) @ (b.double() * sb.t().double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)).t())
    C = binding.mlt_gemm_fp8(a.to(u.F8).to(dev), sa.to(dev), b.to(u.F8).to(dev), sb.to(dev), dtype=torch.bfloat16)
    # whole numbers of at most 64 to a product: exact in a group's 13 bits and in fp32 but for the smallest scales' 2^-4; then the output's rounding
    assert torch.equal(C.double().cpu(), ref.float().to(torch.bfloat16).double())
