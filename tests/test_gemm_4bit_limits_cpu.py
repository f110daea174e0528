"""How many rows mlt_gemm_w4 takes: what the header says, asked of the C entry point with no device (the pointers are never followed)."""
import ctypes

import torch


def test_most_rows():
    from paper_2503_14985_amd import binding as b
    P = ctypes.c_void_p(0x10000)

    def call(M, K):
        return b.raw().mlt_gemm_w4(M, 8, K, P, 128, P, 64, 32, P, 8, None, 0, P, 8, 0, None)

    assert call(64 * 65535 + 1, 128) == b.MLT_ERR_UNSUPPORTED
    assert call((1 << 31) - 1, 128) == b.MLT_ERR_UNSUPPORTED
    if not torch.cuda.is_available():                                # (beyond the checks, where there is nothing to run it)
        assert call(64 * 65535, 128) == b.MLT_ERR_DEVICE
        assert call(64 * 65535 + 1, 0) == b.MLT_ERR_DEVICE
