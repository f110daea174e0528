"""mlt_gemm_fp8 with so many rows that the byte offset of a row's scale passes 2^32."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


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


@pytest.mark.parametrize("variant", ["256pp16", "256x128kp", "224x128kp", "192x128kp"])
def test_scales_of_more_than_2_30_rows(operands, variant):
    from paper_2503_14985_amd import binding
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
