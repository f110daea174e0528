"""mlt_gemm_w4 where every sum is exact in fp32, so that the result has to be the definition's, rounded once, bit for bit: K in one and in up to 8 parts with each width of a wavefront's pieces
(up to 16 rows: 512, groups of 32: 256; up to 32 rows: 256), tiles in parts and not, K that ends inside a piece, a chunk and a group.

A holds whole numbers up to 2 (1 beyond K = 32768), scales are 1/4, 1/2 or 1. The kernels add a (16 + q) and take (16 + z) sum a off, |a (16 + q)| <= 2 * 31: all sums, in any order, are multiples of
1/4 and below 2 * 31 * 32768 < 2^21 (31 * 65536 < 2^21), so they have 23 bits at most."""
import pytest
import torch

from prompt_util import w4_exact

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding as b
    return b


def whole_inputs(seed, M, N, K, group, zeros, dtype):
    g = torch.Generator().manual_seed(seed)
    groups, top = -(-K // group), 2 if K <= 32768 else 1
    q = torch.randint(0, 16, (N, K), generator=g, dtype=torch.uint8)
    A = torch.randint(-top, top + 1, (M, K), generator=g).to(dtype)
    S = (2.0 ** torch.randint(-2, 1, (groups, N), generator=g).float()).to(dtype)
    Z = torch.randint(0, 16, (groups, N), generator=g, dtype=torch.uint8) if zeros else None
    return [None if x is None else x.cuda() for x in (A, q[:, 0::2] | (q[:, 1::2] << 4), S, Z, q)]


# rows, columns, K, parts with groups of 32 and with others
SIZES = [(1, 300, 8192, 4, 2), (13, 515, 14336, 4, 2), (7, 900, 16416, 8, 4), (16, 100, 65536, 8, 8), (5, 33, 32288, 8, 8), (2, 2000, 8160, 4, 2), (9, 8200, 8192, 1, 1),
         (20, 300, 16384, 8, 8), (31, 1030, 4128, 2, 2), (32, 77, 8160, 4, 4), (33, 48, 1312, None, None), (48, 515, 8288, None, None), (64, 96, 32768, None, None), (57, 8200, 416, None, None),
         (130, 200, 4192, None, None)]


@pytest.mark.parametrize("zeros", [False, True], ids=["symmetric", "zeros"])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("size", SIZES, ids=["%dx%dx%d" % s[:3] for s in SIZES])
def test_exact_sums(binding, size, dtype, zeros):
    M, N, K, parts32, parts = size
    for group in (32, 64, 128):
        A, Wq, S, Z, q = whole_inputs(M + N + K, M, N, K, group, zeros, dtype)
        C = binding.mlt_gemm_w4(A, Wq, S, Z, group=group)
        name = binding.mlt_last_kernel()
        if parts is not None and torch.cuda.get_device_properties(0).multi_processor_count == 256:
            assert name.endswith("_parts%d" % (parts32 if group == 32 else parts)), name
        c, _ = w4_exact(A, q, S, Z, group)
        off = (C != c.to(dtype)).nonzero()
        assert off.numel() == 0, "group %d %s: %d values, first at %s" % (group, name, off.shape[0], off[0].tolist())


def test_weights_at_the_zero_point(binding):
    """Weights equal to their zero point count nothing, also beside large whole numbers in A: 300 * 31 * 64 < 2^24."""
    for M, K in ((3, 64), (40, 64), (16, 64)):
        A = torch.randint(-300, 301, (M, K), generator=torch.Generator().manual_seed(M)).to(FP).cuda()
        Z = torch.arange(16, dtype=torch.uint8, device="cuda")[None].repeat(2, 1).contiguous()
        q = Z[0][:, None].expand(16, K)
        S = torch.full((2, 16), 0.75, dtype=FP, device="cuda")
        assert bool((binding.mlt_gemm_w4(A, (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous(), S, Z, group=32) == 0).all())


def test_two_streams_and_repeats(binding):
    """K in parts: the counters and partial results of one stream's calls are not another's, and a counter is ready for the next call."""
    sizes = [(1, 300, 8192), (16, 100, 65536), (20, 300, 16384)]
    ins = [whole_inputs(i, *s, 128, True, BF) for i, s in enumerate(sizes)]
    want = [w4_exact(A, q, S, Z, 128)[0].to(BF) for A, _, S, Z, q in ins]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(12):
        for st, s in enumerate(streams):
            k = (i + st) % 3
            A, Wq, S, Z, _ = ins[k]
            C = torch.full(want[k].shape, 7.0, dtype=BF, device="cuda")
            s.wait_stream(torch.cuda.current_stream())
            outs.append((k, binding.mlt_gemm_w4(A, Wq, S, Z, group=128, C=C, stream=s)))
    torch.cuda.synchronize()
    for k, C in outs:
        assert torch.equal(C, want[k]), k
