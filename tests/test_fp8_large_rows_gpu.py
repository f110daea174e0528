"""The 8-bit operators at their largest: so many rows that the byte offset of a row's scale passes 2^32, and as many workgroups as a launch can have."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding
    return binding


@pytest.fixture(scope="module")
def operands():
    """A row's values are 1 to 5, its scale 1 to 64, neither with a period that 2^30 is a multiple of; all results are whole numbers that bf16 has."""
    dev = torch.device("cuda:0")
    M = (1 << 30) + 777
    row = torch.arange(M, dtype=torch.int32, device=dev)
    values = (row % 5 + 1).to(F8)
    sa = torch.exp2((row % 7).float())
    del row
    a = values.view(torch.uint8)[:, None].expand(M, 16).contiguous().view(F8)
    want = values.to(torch.bfloat16) * sa.to(torch.bfloat16) * 16
    yield a, sa[None], want
    del a, sa, want
    torch.cuda.empty_cache()


# (by 128 x 128 tiles these rows would take a launch of more than 2^32 work-items, which would leave most of them out: the last three choose another kernel)
@pytest.mark.parametrize("variant", ["256pp16", "256x128kp", "224x128kp", "192x128kp", "auto", "128pp16", "128kp"])
def test_scales_of_more_than_2_30_rows(binding, operands, variant):
    a, sa, want = operands
    b, sb = torch.ones((1, 16), device=a.device).to(F8), torch.ones((1, 1), device=a.device)
    print("\n[case] %s" % variant, flush=True)
    C = torch.full((a.shape[0], 1), float("nan"), dtype=torch.bfloat16, device=a.device)
    binding.mlt_diag_force_variant(gemm=variant)
    try:
        binding.mlt_gemm_fp8(a, sa, b, sb, C=C)
        torch.cuda.synchronize()
        print("   kernel=%s" % binding.mlt_last_kernel(), flush=True)
    finally:
        binding.mlt_diag_force_variant(gemm="auto")
    assert torch.equal(C[:, 0], want)


def test_the_largest_launches(binding):
    """2^24 - 1 workgroups of 256 work-items, the most that a launch can have, and one more: refused."""
    dev = torch.device("cuda:0")
    most = (1 << 24) - 1
    print("\n[case] quantisation", flush=True)
    M = 16 * most
    x = (torch.arange(M, dtype=torch.int32, device=dev) % 13 - 6).to(torch.bfloat16)[:, None].expand(M, 8).contiguous()
    q, s = torch.full((M, 16), 0x7F, dtype=torch.uint8, device=dev).view(F8)[:, :8], torch.full((1, M), -1.0, device=dev)
    binding.mlt_quant_fp8(x, Xq=q, S=s)
    assert torch.equal(q.to(torch.bfloat16) * s[0, :, None].to(torch.bfloat16), x)
    wide = torch.zeros((M + 1, 8), dtype=torch.bfloat16, device=dev)
    with pytest.raises(binding.MltError) as e:
        binding.mlt_quant_fp8(wide)
    assert e.value.status == binding.MLT_ERR_UNSUPPORTED
    del x, q, s, wide
    print("[case] append", flush=True)
    T, D = 4 * most, 64
    q = torch.arange(T * 8, dtype=torch.int32, device=dev).view(torch.int16).view(torch.bfloat16).reshape(T, 1, 16).repeat(1, 1, D // 16)
    none = torch.zeros((T, 0, D), dtype=torch.bfloat16, device=dev)
    cache = torch.zeros((1, 0, 16, D), dtype=torch.bfloat16, device=dev)
    out = torch.zeros_like(q)
    at = [torch.tensor(v, dtype=torch.int32, device=dev) for v in ([0, T], [T], [[0]])]
    binding.mlt_paged_append(q, none, none, *at, None, None, cache, cache, Qo=out)
    # (every bit pattern: NaN goes through fp32 and back, which sets a signalling one's quiet bit, 2^6 of a bfloat16, and leaves the others)
    bits = q.view(torch.int16)
    assert torch.equal(out.view(torch.int16), torch.where(torch.isnan(q), bits | 0x40, bits))
    del bits
    del q, out, none
    print("[case] attention", flush=True)
    B = most
    v = torch.randn((2, 1, 16, D), generator=torch.Generator().manual_seed(1)).to(F8).to(dev)
    one = torch.ones((2, 1), device=dev)
    q, O = torch.ones((B + 1, 1, D), dtype=torch.float16, device=dev), torch.zeros((B + 1, 1, D), dtype=torch.float16, device=dev)
    table, lens = (torch.arange(B + 1, dtype=torch.int32, device=dev) % 2)[:, None].contiguous(), torch.ones(B + 1, dtype=torch.int32, device=dev)
    binding.mlt_paged_attn_decode_fp8(q[:B], v, v, one, one, table[:B], lens[:B], 0.125, O=O[:B])
    assert torch.equal(O[:B:2, 0], v[0, 0, 0].to(torch.float16).expand(B // 2 + 1, D)) and torch.equal(O[1:B:2, 0], v[1, 0, 0].to(torch.float16).expand(B // 2, D))
    with pytest.raises(binding.MltError) as e:
        binding.mlt_paged_attn_decode_fp8(q, v, v, one, one, table, lens, 0.125, O=O)
    assert e.value.status == binding.MLT_ERR_UNSUPPORTED
    del q, O, table, lens
    torch.cuda.empty_cache()
