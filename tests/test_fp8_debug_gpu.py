"""Race check of the 8-bit kernels that fetch into LDS rings and wait by count or barrier: the library and its debug build (libmlt_dbg.so, compiled with
-DMLT_DEBUG_BARRIERS: every pipeline barrier taken twice behind a wait for everything, waits for all loads where the product counts them) agree bit for bit."""
import ctypes
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DBG = os.path.join(ROOT, "paper_2503_14985_amd", "libmlt_dbg.so")
_i64, _i32, _p, _f = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


@pytest.fixture(scope="module")
def dbg():
    if not os.path.exists(DBG):
        pytest.skip("libmlt_dbg.so is not built (python -c 'import __graft_entry__ as g; g.build_debug_lib()')")
    lib = ctypes.CDLL(DBG)
    lib.mlt_gemm_fp8.argtypes = [_i64, _i64, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _i64, _i32, _p]
    lib.mlt_paged_attn_decode_fp8.argtypes = [_i64, _i64, _i64, _i64, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _f, _i32, _p]
    lib.mlt_diag_force_variant.argtypes = [ctypes.c_char_p, ctypes.c_char_p]
    lib.mlt_last_kernel.restype = ctypes.c_char_p
    yield lib


@pytest.fixture
def both(dbg):
    """Sets an override in both libraries, and takes it back."""
    from paper_2503_14985_amd import binding

    def force(variant="auto", parts=0, split=0):
        binding.mlt_diag_force_variant(gemm=variant)
        binding.mlt_diag_force_k_parts(parts)
        binding.mlt_diag_force_key_split(split)
        assert dbg.mlt_diag_force_variant(variant.encode(), None) == 0
        assert dbg.mlt_diag_force_k_parts(parts) == 0 and dbg.mlt_diag_force_key_split(split) == 0
    yield force
    force()


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


GEMM = [(M, N, K, variant, parts) for variant, parts in (("256pp16", 0), ("128pp16", 0), ("256x128kp", 1), ("224x128kp", 2), ("192x128kp", 1), ("128kp", 4))
        for M, N, K in ((1000, 1000, 4096), (300, 520, 2064))]
GEMM += [(16, 8192, 4096, "skinny", 1), (64, 1000, 4112, "skinny", 1), (33, 512, 8192, "skinny", 4), (333, 700, 4096, "skinny", 1), (777, 256, 6144, "skinny", 2)]


@pytest.mark.parametrize("M,N,K,variant,parts", GEMM)
def test_gemm_agrees_with_the_debug_build(dbg, both, M, N, K, variant, parts):
    from paper_2503_14985_amd import binding
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(M + N + K)
    for dtype, code in ((torch.bfloat16, 0), (torch.float16, 1)):
        a, sa = binding.mlt_quant_fp8(torch.randn((M, K), generator=gen, device=dev).to(dtype))
        b, sb = binding.mlt_quant_fp8(torch.randn((N, K), generator=gen, device=dev).to(dtype), 128)
        both(variant, parts)
        want = binding.mlt_gemm_fp8(a, sa, b, sb, dtype=dtype)
        name = binding.mlt_last_kernel()
        for _ in range(3):                                 # a race need not strike on the first launch
            got = torch.full_like(want, float("nan"))
            assert dbg.mlt_gemm_fp8(M, N, K, a.data_ptr(), a.stride(0), sa.data_ptr(), sa.stride(0), b.data_ptr(), b.stride(0), sb.data_ptr(), sb.stride(0),
                                    got.data_ptr(), got.stride(0), code, _stream()) == 0
            assert dbg.mlt_last_kernel().decode() == name
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)), name


@pytest.mark.parametrize("B,Hq,H,D,block,top,split", [(3, 8, 2, 128, 16, 3000, 1), (3, 8, 2, 64, 64, 3000, 3), (1, 16, 8, 128, 32, 9000, 24), (2, 34, 2, 128, 16, 2500, 8),
                                                      (40, 8, 8, 128, 16, 1400, 1), (70, 8, 8, 64, 16, 700, 1)])
def test_paged_attention_agrees_with_the_debug_build(dbg, both, B, Hq, H, D, block, top, split):
    from paper_2503_14985_amd import binding
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(B + top)
    per = -(-top // block)
    lens = torch.randint(0, top + 1, (B,), generator=gen, device=dev, dtype=torch.int32)
    lens[0] = top
    table = torch.randperm(B * per, generator=gen, device=dev).to(torch.int32).reshape(B, per).contiguous()
    kc, vc = (torch.randn((B * per, H, block, D), generator=gen, device=dev).mul_(60).to(binding.E4M3) for _ in range(2))
    ks, vs = (torch.rand((B * per, H), generator=gen, device=dev) * 0.05 + 0.001 for _ in range(2))
    both(split=split)
    for dtype, code in ((torch.bfloat16, 0), (torch.float16, 1)):
        q = torch.randn((B, Hq, D), generator=gen, device=dev).to(dtype)
        want = binding.mlt_paged_attn_decode_fp8(q, kc, vc, ks, vs, table, lens, 1.0 / math.sqrt(D))
        name = binding.mlt_last_kernel()
        for _ in range(3):
            got = torch.full_like(want, float("nan"))
            assert dbg.mlt_paged_attn_decode_fp8(B, Hq, H, D, block, per, B * per, q.data_ptr(), kc.data_ptr(), vc.data_ptr(), ks.data_ptr(), vs.data_ptr(),
                                                 table.data_ptr(), lens.data_ptr(), got.data_ptr(), 1.0 / math.sqrt(D), code, _stream()) == 0
            assert dbg.mlt_last_kernel().decode() == name
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)), name
