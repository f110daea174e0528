"""Few rows times 4-bit weights against the definition in 64 bits: rows from one to several tiles, any columns, groups and their last part, zero points, strides."""
import pytest
import torch

from prompt_util import check, w4_exact, w4_inputs, w4_tolerance

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding as b
    return b


SIZES = [(1, 1, 32), (1, 7, 96), (2, 64, 160), (3, 100, 256), (5, 257, 1024), (8, 33, 4096), (13, 512, 416), (16, 300, 2048), (17, 129, 544), (24, 1000, 640),
         (33, 48, 1280), (48, 515, 768), (57, 1040, 992), (64, 96, 8192), (65, 70, 512), (130, 200, 352), (1, 4096, 512), (4, 9000, 256)]


@pytest.mark.parametrize("zeros", [False, True], ids=["symmetric", "zeros"])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("size", SIZES, ids=["%dx%dx%d" % s for s in SIZES])
def test_sizes(binding, size, dtype, zeros):
    M, N, K = size
    for group in (32, 64, 128):
        A, Wq, S, Z, q = w4_inputs(M + N + K, M, N, K, group, zeros, dtype)
        C = binding.mlt_gemm_w4(A, Wq, S, Z, group=group)
        c, t = w4_exact(A, q, S, Z, group)
        check(C, c, w4_tolerance(c, t, K, group, dtype), "group %d %s" % (group, binding.mlt_last_kernel()))
        assert torch.equal(C, binding.mlt_gemm_w4(A, Wq, S, Z, group=group))


def test_every_weight(binding):
    """One-hot rows read single weights: each of the 16 numbers at each of 128 places, exactly."""
    K, N = 128, 16
    q = torch.stack([(torch.arange(K) + n) % 16 for n in range(N)]).to(torch.uint8).cuda()
    Wq = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()
    S = torch.full((1, N), 0.5, dtype=BF, device="cuda")
    Z = torch.arange(N, dtype=torch.uint8, device="cuda")[None].contiguous()
    eye = torch.eye(K, dtype=BF, device="cuda")
    for r in range(0, K, 32):
        assert torch.equal(binding.mlt_gemm_w4(eye[r:r + 32], Wq, S).float(), (q[:, r:r + 32].t().float() - 8) * 0.5)
        assert torch.equal(binding.mlt_gemm_w4(eye[r:r + 32], Wq, S, Z).float(), (q[:, r:r + 32].t().float() - Z.float()) * 0.5)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_strides_and_edges(binding, dtype):
    """Rows inside larger arrays; nothing beside C is written."""
    M, N, K, group = 19, 77, 352, 128
    A, Wq, S, Z, q = w4_inputs(1, M, N, K, group, True, dtype)

    def inside(x, left, right):
        big = torch.full((x.shape[0] + 2, x.shape[1] + left + right), 3, dtype=x.dtype, device="cuda")
        big[1:-1, left:left + x.shape[1]] = x
        return big, big[1:-1, left:left + x.shape[1]]

    _, a = inside(A, 8, 24)
    _, w = inside(Wq, 16, 32 - K // 2 % 16)
    _, s = inside(S, 3, 2)
    _, z = inside(Z, 5, 1)
    big, C = inside(torch.zeros((M, N), dtype=dtype, device="cuda"), 5, 6)
    binding.mlt_gemm_w4(a, w, s, z, group=group, C=C)
    c, t = w4_exact(A, q, S, Z, group)
    check(C, c, w4_tolerance(c, t, K, group, dtype))
    keep = torch.ones_like(big, dtype=torch.bool)
    keep[1:-1, 5:5 + N] = False
    assert bool((big[keep] == 3).all())


def test_large_values(binding):
    """Rows with a large mean: what a sum over weights with an offset would lose must not show."""
    M, N, K, group = 8, 256, 4096, 128
    A, Wq, S, Z, q = w4_inputs(4, M, N, K, group, False, FP)
    A += 100
    C = binding.mlt_gemm_w4(A, Wq, S, group=group)
    c, t = w4_exact(A, q, S, Z, group)
    check(C, c, w4_tolerance(c, t, K, group, FP))
    rel = (C.double() - c).norm() / c.norm()
    assert float(rel) <= 2.0 ** -11, float(rel)                      # a rounding is at most that


def test_empty(binding):
    for M, N, K in ((0, 5, 32), (5, 0, 32), (3, 4, 0)):
        C = binding.mlt_gemm_w4(torch.zeros((M, K), dtype=BF, device="cuda"), torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda"),
                                torch.zeros((-(-K // 128), N), dtype=BF, device="cuda"))
        assert C.shape == (M, N) and bool((C == 0).all())


@pytest.mark.parametrize("M", [1, 20, 40])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_values_that_are_not_finite(binding, M, group):
    """An infinite scale and rows with an infinity or NaN reach what they belong to and nothing else; the last part of K is shorter than what is read at a time."""
    N, K = 100, 544
    A, Wq, S, Z, q = w4_inputs(M, M, N, K, group, True, BF)
    clean = binding.mlt_gemm_w4(A, Wq, S, Z, group=group)
    S[-1, 7] = float("inf")
    C = binding.mlt_gemm_w4(A, Wq, S, Z, group=group)
    assert not bool(torch.isfinite(C[:, 7]).any())
    other = torch.arange(N, device="cuda") != 7
    assert torch.equal(C[:, other], clean[:, other])
    S[-1, 7] = 1
    A[M // 2, K - 1] = float("nan")
    A[0, 0] = float("inf")
    C = binding.mlt_gemm_w4(A, Wq, S, Z, group=group)
    rows = torch.arange(M, device="cuda")
    bad = (rows == M // 2) | (rows == 0)
    assert not bool(torch.isfinite(C[bad]).any()) and torch.equal(C[~bad][:, other], clean[~bad][:, other])
