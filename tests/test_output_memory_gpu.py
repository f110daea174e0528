"""Outputs that a call allocates itself, on a stream that is given: never memory that the current stream has just let go of, whose pending work may still use it, nor memory
that the current stream's next tensor can take while the call is pending."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    from paper_2503_14985_amd import binding
    return binding


def dev():
    return torch.device("cuda:0")


def calls(lib):
    """name -> call(stream), which returns the allocated outputs"""
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g).to(dev())  # noqa: E731
    a, b = r(512, 1024).to(BF16), r(768, 1024).to(BF16)
    q = r(2, 4, 256, 128).to(BF16)
    aq, sa = lib.mlt_quant_fp8(a)
    bq, sb = lib.mlt_quant_fp8(b, 128)
    H, D, T = 8, 128, 256
    kv, new = torch.zeros((16, H, 16, D), dtype=BF16, device=dev()), r(T, H, D).to(BF16)
    kv8, one = torch.zeros((16, H, 16, D), device=dev()).to(lib.E4M3), torch.ones((16, H), device=dev())
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev())  # noqa: E731
    at = (i32([0, T]), i32([T]), torch.arange(16, dtype=torch.int32, device=dev())[None])
    many = r(256, 32, D).to(BF16)
    lens, table = torch.full((256,), 20, dtype=torch.int32, device=dev()), torch.arange(512, dtype=torch.int32, device=dev()).reshape(256, 2) % 16
    return {"mlt_gemm": lambda s: [lib.mlt_gemm(a, b, transB=True, stream=s)],
            "mlt_gemm_tiled": lambda s: [lib.mlt_gemm_tiled(a, b, 3, transB=True, stream=s)],
            "mlt_gemm_bias_act": lambda s: [lib.mlt_gemm_bias_act(a, b, None, 1, transB=True, stream=s)],
            "mlt_mha_fwd": lambda s: [lib.mlt_mha_fwd(q, q, q, 0.1, stream=s)],
            "mlt_quant_fp8": lambda s: list(lib.mlt_quant_fp8(a, stream=s)),
            "mlt_gemm_fp8": lambda s: [lib.mlt_gemm_fp8(aq, sa, bq, sb, stream=s)],
            "mlt_paged_append": lambda s: [lib.mlt_paged_append(new, new, new, *at, None, None, kv, kv.clone(), stream=s)],
            "mlt_paged_append_fp8": lambda s: [lib.mlt_paged_append_fp8(new, new, new, *at, None, None, kv8, kv8.clone(), one, one.clone(), stream=s)],
            "mlt_paged_attn_decode_fp8": lambda s: [lib.mlt_paged_attn_decode_fp8(many, kv8, kv8, one, one, table.contiguous(), lens, 0.1, stream=s)]}


NAMES = ["mlt_gemm", "mlt_gemm_tiled", "mlt_gemm_bias_act", "mlt_mha_fwd", "mlt_quant_fp8", "mlt_gemm_fp8", "mlt_paged_append", "mlt_paged_append_fp8", "mlt_paged_attn_decode_fp8"]


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_output_of_a_call_on_a_given_stream(lib, name, handle):
    call = calls(lib)[name]
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    want = [t.clone() for t in call(None)]                                # (the same block again and again, if each call lets its own go)
    torch.cuda.synchronize()
    held = call(None)
    sizes = [(t.untyped_storage().nbytes(), t.untyped_storage().data_ptr()) for t in held]
    busy = [torch.empty(n, dtype=torch.uint8, device=dev()) for n, _ in sizes]
    del held
    ranges = [(p, p + n) for n, p in sizes] + [(t.data_ptr(), t.data_ptr() + t.numel()) for t in busy]
    torch.cuda._sleep(20_000_000)
    for t in busy:
        t.fill_(7)                                                        # pending on the current stream when its memory is let go
    del busy, t
    got = call(stream)
    for o in got:
        p = o.untyped_storage().data_ptr()
        assert all(p + o.untyped_storage().nbytes() <= lo or p >= hi for lo, hi in ranges), name
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
    ends = [(o.untyped_storage().data_ptr(), o.untyped_storage().data_ptr() + o.untyped_storage().nbytes()) for o in got]
    sizes = [o.untyped_storage().nbytes() for o in got]
    del got, o, x, y
    again = [torch.empty(n, dtype=torch.uint8, device=dev()) for n in sizes for _ in range(4)]
    for t in again:
        assert all(t.data_ptr() + t.numel() <= lo or t.data_ptr() >= hi for lo, hi in ends), name
