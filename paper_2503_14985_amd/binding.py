"""ctypes binding of libmlt.so: the same names as the C ABI in include/mlt.h, argument marshalling
only. Every step of both operations runs in the HIP kernels; there is no fallback: if the
library has not been built, importing this module raises.

Tensors are torch tensors on the GPU (bf16 or fp16); torch is used for device memory and the
current stream, nothing else.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmlt.so")

MLT_BF16, MLT_FP16 = 0, 1
MLT_OK, MLT_ERR_INVALID_ARG, MLT_ERR_UNSUPPORTED, MLT_ERR_LAUNCH, MLT_ERR_DEVICE = 0, -1, -2, -3, -4
MLT_ERR_SCRATCH = -5

# include/mlt.h (the operations) and include/mlt_diag.h (probes, timing hooks, kernel-choice overrides)
EXPORTS = ("mlt_gemm", "mlt_gemm_noalloc", "mlt_gemm_acc", "mlt_gemm_tiled", "mlt_gemm_bias_act", "mlt_mha_fwd",
           "mlt_paged_attn_decode", "mlt_quant_fp8", "mlt_gemm_fp8", "mlt_paged_append", "mlt_paged_append_fp8",
           "mlt_paged_attn_decode_fp8", "mlt_mha_packed_fwd", "mlt_paged_attn_prompt", "mlt_paged_attn_decode_prefix",
           "mlt_paged_attn_decode_prefix_work", "mlt_gemm_w4", "mlt_status_string", "mlt_version")
DIAG_EXPORTS = ("mlt_probe_mfma", "mlt_probe_mfma16", "mlt_probe_hbm_read", "mlt_set_timing_events",
                "mlt_last_kernel", "mlt_query_tiling", "mlt_diag_force_variant",
                "mlt_diag_force_k_parts", "mlt_diag_force_key_split", "mlt_diag_set_persistent_grid")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libmlt.so is not built (%s). Run `python -c 'import __graft_entry__ as g; g.build_lib()'` "
        "from the repository root; there is no CPU fallback." % LIB_PATH)

_lib = ctypes.CDLL(LIB_PATH)
# What torch.cuda.current_stream(i).cuda_stream and torch.cuda.current_device() return, without the objects
# around it (a CPU-only build of torch has neither; no call gets that far there).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_i64, _p, _i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
_lib.mlt_gemm.restype = _i32
_lib.mlt_gemm.argtypes = [_i64, _i64, _i64, _p, _i64, _p, _i64, _i32, _p, _i64, _i32, _p]
_lib.mlt_gemm_noalloc.restype = _i32
_lib.mlt_gemm_noalloc.argtypes = [_i64, _i64, _i64, _p, _i64, _p, _i64, _i32, _p, _i64, _i32, _p]
_lib.mlt_gemm_acc.restype = _i32
_lib.mlt_gemm_acc.argtypes = [_i64, _i64, _i64, _p, _i64, _p, _i64, _i32, _p, _i64, _i32, _p]
_lib.mlt_gemm_tiled.restype = _i32
_lib.mlt_gemm_tiled.argtypes = [_i64, _i64, _i64, _p, _i64, _p, _i64, _i32, _p, _i64, _i32, _i32, _p]
_lib.mlt_gemm_bias_act.restype = _i32
_lib.mlt_gemm_bias_act.argtypes = [_i64, _i64, _i64, _p, _i64, _p, _i64, _i32, _p, _i32, _p, _i64, _i32, _p]
_lib.mlt_mha_fwd.restype = _i32
_lib.mlt_mha_fwd.argtypes = [_i64, _i64, _i64, _i64, _i64, _p, _p, _p, _p, ctypes.c_float, _i32,
                             _i32, _p]
_lib.mlt_paged_attn_decode.restype = _i32
_lib.mlt_paged_attn_decode.argtypes = [_i64, _i64, _i64, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p,
                                       ctypes.c_float, _i32, _p]
_lib.mlt_quant_fp8.restype = _i32
_lib.mlt_quant_fp8.argtypes = [_i64, _i64, _p, _i64, _i64, _p, _i64, _p, _i64, _i32, _p]
_lib.mlt_gemm_fp8.restype = _i32
_lib.mlt_gemm_fp8.argtypes = [_i64, _i64, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _i64, _i32, _p]
_lib.mlt_paged_append.restype = _i32
_lib.mlt_paged_append.argtypes = [_i64] * 8 + [_p, _i64] * 3 + [_p] * 5 + [_i64, _i64, _i32, _p, _p, _p, _i32, _p]
_lib.mlt_paged_append_fp8.restype = _i32
_lib.mlt_paged_append_fp8.argtypes = [_i64] * 8 + [_p, _i64] * 3 + [_p] * 5 + [_i64, _i64, _i32, _p, _p, _p, _p, _p, _i32, _p]
_lib.mlt_paged_attn_decode_fp8.restype = _i32
_lib.mlt_paged_attn_decode_fp8.argtypes = [_i64] * 7 + [_p] * 8 + [ctypes.c_float, _i32, _p]
_lib.mlt_mha_packed_fwd.restype = _i32
_lib.mlt_mha_packed_fwd.argtypes = [_i64] * 6 + [_p, _i64] * 3 + [_p, _p, _p, _i64, ctypes.c_float, _i32, _i32, _p]
_lib.mlt_paged_attn_prompt.restype = _i32
_lib.mlt_paged_attn_prompt.argtypes = [_i64] * 8 + [_p, _i64] + [_p] * 6 + [_i64, ctypes.c_float, _i32, _p]
_lib.mlt_paged_attn_decode_prefix.restype = _i32
_lib.mlt_paged_attn_decode_prefix.argtypes = [_i64] * 7 + [_p] * 4 + [_i64] + [_p] * 3 + [ctypes.c_float, _p, _i64, _i32, _p]
_lib.mlt_paged_attn_decode_prefix_work.restype = _i64
_lib.mlt_paged_attn_decode_prefix_work.argtypes = [_i64] * 7
_lib.mlt_gemm_w4.restype = _i32
_lib.mlt_gemm_w4.argtypes = [_i64, _i64, _i64, _p, _i64, _p, _i64, _i64, _p, _i64, _p, _i64, _p, _i64, _i32, _p]
_lib.mlt_probe_mfma.restype = _i32
_lib.mlt_probe_mfma.argtypes = [_i32, _p, _p, ctypes.POINTER(ctypes.c_double), _p]
_lib.mlt_probe_mfma16.restype = _i32
_lib.mlt_probe_mfma16.argtypes = [_i32, _p, _p, ctypes.POINTER(ctypes.c_double), _p]
_lib.mlt_probe_hbm_read.restype = _i32
_lib.mlt_probe_hbm_read.argtypes = [_p, _i64, _p, _p]
_lib.mlt_set_timing_events.restype = None
_lib.mlt_set_timing_events.argtypes = [_p, _p]
_lib.mlt_last_kernel.restype = ctypes.c_char_p
_lib.mlt_query_tiling.restype = _i32
_lib.mlt_query_tiling.argtypes = [_i32, ctypes.POINTER(_i64), _i32, ctypes.POINTER(ctypes.c_int32)]
_lib.mlt_diag_force_variant.restype = _i32
_lib.mlt_diag_force_variant.argtypes = [ctypes.c_char_p, ctypes.c_char_p]
_lib.mlt_diag_force_k_parts.restype = _i32
_lib.mlt_diag_force_k_parts.argtypes = [_i32]
_lib.mlt_diag_force_key_split.restype = _i32
_lib.mlt_diag_force_key_split.argtypes = [_i32]
_lib.mlt_diag_set_persistent_grid.restype = _i32
_lib.mlt_diag_set_persistent_grid.argtypes = [_i32]
_lib.mlt_status_string.restype = ctypes.c_char_p
_lib.mlt_status_string.argtypes = [_i32]
_lib.mlt_version.restype = ctypes.c_char_p


class MltError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, mlt_status_string(status), status))


# The usual case of a call (plain GPU tensors, an output given, no stream) goes through native code (csrc/fastcall.cpp), which returns
# None for everything else: the functions below then marshal, allocate or raise. A call that the library refuses raises there.
# (us per mlt_gemm call of 16 x 64 x 64 back to back: 7.5 without, 3.8 with; the library's and the runtime's own part is 3.1.)
# It is built against one torch, whose tensors it looks into; with another one, with a torch without ROCm, or where it has not been built,
# every call goes through the functions below.
class _PythonOnly:
    gemm = gemm_acc = gemm_bias_act = mha_fwd = paged_attn_decode = quant_fp8 = gemm_fp8 = paged_append = paged_attn_decode_fp8 = staticmethod(lambda *args: None)
    mha_packed_fwd = paged_attn_prompt = paged_attn_decode_prefix = gemm_w4 = gemm


_fast = _PythonOnly
try:
    from . import _fastcall
    if _fastcall.torch_version == torch.__version__:
        _fastcall.bind(MltError, *(ctypes.cast(getattr(_lib, _f), _p).value for _f in (
            "mlt_gemm", "mlt_gemm_bias_act", "mlt_gemm_acc", "mlt_mha_fwd", "mlt_paged_attn_decode", "mlt_quant_fp8", "mlt_gemm_fp8", "mlt_paged_append",
            "mlt_paged_append_fp8", "mlt_paged_attn_decode_fp8", "mlt_mha_packed_fwd", "mlt_paged_attn_prompt", "mlt_paged_attn_decode_prefix", "mlt_gemm_w4")))
        _fast = _fastcall
except ImportError:
    pass


def raw():
    """The ctypes library object, for tests that pass raw pointers (error paths)."""
    return _lib


def mlt_status_string(status: int) -> str:
    return _lib.mlt_status_string(status).decode()


def mlt_version() -> str:
    return _lib.mlt_version().decode()


def mlt_last_kernel() -> str:
    return _lib.mlt_last_kernel().decode()


def mlt_diag_force_variant(gemm: str | None = None, mha: str | None = None) -> None:
    """Force a GEMM and/or attention kernel variant for the whole process (None: leave as is,
    "auto": the library's own choice)."""
    rc = _lib.mlt_diag_force_variant(None if gemm is None else gemm.encode(),
                                     None if mha is None else mha.encode())
    if rc != MLT_OK:
        raise MltError(rc, "mlt_diag_force_variant")


def mlt_diag_force_k_parts(parts: int) -> None:
    """0: the library's choice; 1: no K split across workgroups; 2 / 4 / 8: that many parts."""
    rc = _lib.mlt_diag_force_k_parts(int(parts))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_diag_force_k_parts")


def mlt_diag_force_key_split(ranges: int) -> None:
    """Paged decode, and attention with "k2" or "k4" forced: 0 = the library's choice; 1..64 = key ranges."""
    rc = _lib.mlt_diag_force_key_split(int(ranges))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_diag_force_key_split")


def mlt_diag_set_persistent_grid(workgroups: int) -> None:
    rc = _lib.mlt_diag_set_persistent_grid(int(workgroups))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_diag_set_persistent_grid")


def mlt_paged_attn_decode(Q: torch.Tensor, Kc: torch.Tensor, Vc: torch.Tensor,
                          block_table: torch.Tensor, seq_lens: torch.Tensor, scale: float,
                          O: torch.Tensor = None) -> torch.Tensor:
    """Q [B,H,D]; Kc, Vc [num_blocks,H,block_size,D]; block_table int32 [B,max_blocks]; seq_lens
    int32 [B]; returns O [B,H,D]. All on the GPU, contiguous."""
    done = _fast.paged_attn_decode(Q, Kc, Vc, block_table, seq_lens, scale, O)
    if done is not None:
        return done
    B, H, D = Q.shape
    nb, Hc, bs, Dc = Kc.shape
    if (Hc, Dc) != (H, D) or Vc.shape != Kc.shape or Vc.dtype != Q.dtype or Kc.dtype != Q.dtype:
        raise ValueError("mlt_paged_attn_decode: cache shape/dtype does not match Q")
    if block_table.dtype != torch.int32 or seq_lens.dtype != torch.int32:
        raise ValueError("mlt_paged_attn_decode: block_table and seq_lens must be int32")
    if block_table.shape[0] != B or tuple(seq_lens.shape) != (B,):
        raise ValueError("mlt_paged_attn_decode: block_table / seq_lens shape")
    for t in (Q, Kc, Vc, block_table, seq_lens):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("mlt_paged_attn_decode: tensors must be contiguous GPU tensors")
    if O is None:
        O = torch.empty_like(Q)
    rc = _lib.mlt_paged_attn_decode(B, H, D, bs, block_table.shape[1], nb, Q.data_ptr(),
                                    Kc.data_ptr(), Vc.data_ptr(), block_table.data_ptr(),
                                    seq_lens.data_ptr(), O.data_ptr(), float(scale),
                                    _dtype_code(Q), _raw_stream(Q.device.index))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_paged_attn_decode")
    return O


def mlt_probe_mfma(iters: int, data: torch.Tensor, sink: torch.Tensor, mfma_size: int = 32) -> float:
    """Enqueue the register-only MFMA loop on the current stream; returns the flop it executes.
    `data`: at least 64 KiB of bf16 operand values on the GPU, `sink`: at least 4 bytes.
    mfma_size 32: 32x32x16 MFMAs (mlt_probe_mfma), 16: 16x16x32 (mlt_probe_mfma16)."""
    if not data.is_cuda or data.numel() * data.element_size() < 65536 or not data.is_contiguous():
        raise ValueError("mlt_probe_mfma: data must be a contiguous GPU tensor of at least 64 KiB")
    if mfma_size not in (16, 32):
        raise ValueError("mfma_size must be 16 or 32")
    fn = _lib.mlt_probe_mfma16 if mfma_size == 16 else _lib.mlt_probe_mfma
    flop = ctypes.c_double()
    rc = fn(int(iters), data.data_ptr(), sink.data_ptr(), ctypes.byref(flop),
            torch.cuda.current_stream(data.device).cuda_stream)
    if rc != MLT_OK:
        raise MltError(rc, "mlt_probe_mfma")
    return flop.value


def mlt_probe_mfma16(iters: int, data: torch.Tensor, sink: torch.Tensor) -> float:
    return mlt_probe_mfma(iters, data, sink, mfma_size=16)


def mlt_probe_hbm_read(data: torch.Tensor, sink: torch.Tensor) -> int:
    """Enqueue the read-only streaming kernel over `data` (contiguous GPU tensor, a multiple of 16
    bytes) on the current stream; returns the bytes it reads."""
    nbytes = data.numel() * data.element_size()
    if not data.is_cuda or not data.is_contiguous():
        raise ValueError("mlt_probe_hbm_read: data must be a contiguous GPU tensor")
    rc = _lib.mlt_probe_hbm_read(data.data_ptr(), nbytes, sink.data_ptr(),
                                 torch.cuda.current_stream(data.device).cuda_stream)
    if rc != MLT_OK:
        raise MltError(rc, "mlt_probe_hbm_read")
    return nbytes


def mlt_query_tiling(op: int, dims, dtype: int):
    d = (_i64 * 4)(*[int(x) for x in dims])
    out = (ctypes.c_int32 * 10)()
    rc = _lib.mlt_query_tiling(op, d, dtype, out)
    if rc != MLT_OK:
        raise MltError(rc, "mlt_query_tiling")
    return list(out)


def mlt_set_timing_events(start, stop) -> None:
    """start/stop: raw hipEvent_t handles as ints (or None)."""
    _lib.mlt_set_timing_events(start, stop)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return MLT_BF16
    if t.dtype == torch.float16:
        return MLT_FP16
    raise TypeError("mlt works on bfloat16 / float16 tensors, got %s" % t.dtype)


def _stream(stream, device) -> int:
    if stream is None:
        return _raw_stream(device.index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """An output that the call allocates itself: memory of the stream that the call goes to. The current stream's may still have an earlier tensor's
    work pending on it, and its next tensor may take it while the call is pending."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device) if int(stream) else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class _OtherDevice:
    """torch.cuda.device, entered only when `device` is not the current one: its enter and exit, and
    torch.cuda.current_stream() beside them, took 6 of the 11 us of a small call (2000 calls of
    16 x 64 x 64 back to back: 10.9 us each, 7.4 in this form; the library's own part is 3.7 to 4.6)."""
    __slots__ = ("guard",)

    def __init__(self, device):
        self.guard = None if device.index == _current_device() else torch.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)
        return False


def _rows_contiguous(t: torch.Tensor, name: str) -> int:
    if t.dim() != 2:
        raise ValueError("%s must be 2-D" % name)
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("%s must have contiguous rows" % name)
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _gemm_operands(name: str, A, B, C, transB: bool, c_dtype=None, stream=None):
    """Shapes, dtype code and leading dimensions of a GEMM call (C allocated when None): the
    marshalling every GEMM entry point shares."""
    if not (A.is_cuda and B.is_cuda and (C is None or C.is_cuda)):
        raise ValueError("%s needs GPU tensors" % name)
    dt = _dtype_code(A)
    if B.dtype != A.dtype:
        raise TypeError("A and B must share a dtype")
    M, K = A.shape
    N, Kb = (B.shape[0], B.shape[1]) if transB else (B.shape[1], B.shape[0])
    if K != Kb:
        raise ValueError("inner dimensions differ: %d vs %d" % (K, Kb))
    c_dtype = A.dtype if c_dtype is None else c_dtype
    if C is None:
        C = _empty((M, N), c_dtype, A.device, stream)
    elif C.dtype != c_dtype or tuple(C.shape) != (M, N):
        raise ValueError("C has the wrong dtype or shape")
    lda, ldb, ldc = _rows_contiguous(A, "A"), _rows_contiguous(B, "B"), _rows_contiguous(C, "C")
    return M, N, K, lda, ldb, ldc, dt, C


def mlt_gemm(A: torch.Tensor, B: torch.Tensor, C: torch.Tensor | None = None, transB: bool = False,
             stream=None) -> torch.Tensor:
    """C = A @ B (transB=False, B is [K, N]) or C = A @ B.T (transB=True, B is [N, K]).

    Row strides of A, B and C are passed through as lda/ldb/ldc, so row-sliced views work."""
    done = _fast.gemm(A, B, C, transB, stream)
    if done is not None:
        return done
    M, N, K, lda, ldb, ldc, dt, C = _gemm_operands("mlt_gemm", A, B, C, transB, stream=stream)
    with _OtherDevice(A.device):
        rc = _lib.mlt_gemm(M, N, K, A.data_ptr(), lda, B.data_ptr(), ldb, int(transB),
                           C.data_ptr(), ldc, dt, _stream(stream, A.device))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_gemm")
    return C


def mlt_gemm_noalloc(A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, transB: bool = False,
                     stream=None) -> torch.Tensor:
    """mlt_gemm through the entry point that allocates nothing: C must be given."""
    if C is None:
        raise ValueError("mlt_gemm_noalloc needs the C it writes (this wrapper allocates nothing)")
    M, N, K, lda, ldb, ldc, dt, C = _gemm_operands("mlt_gemm_noalloc", A, B, C, transB)
    with _OtherDevice(A.device):
        rc = _lib.mlt_gemm_noalloc(M, N, K, A.data_ptr(), lda, B.data_ptr(), ldb, int(transB),
                                   C.data_ptr(), ldc, dt, _stream(stream, A.device))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_gemm_noalloc")
    return C


ACT_NONE, ACT_RELU, ACT_GELU = 0, 1, 2
TILING_AUTO, TILING_HORIZONTAL, TILING_VERTICAL, TILING_SQUARE = 0, 1, 2, 3


def mlt_gemm_tiled(A: torch.Tensor, B: torch.Tensor, tiling: int, C: torch.Tensor | None = None,
                   transB: bool = False, stream=None) -> torch.Tensor:
    """mlt_gemm with the paper's tiling hint (TILING_AUTO / _HORIZONTAL / _VERTICAL / _SQUARE)."""
    M, N, K, lda, ldb, ldc, dt, C = _gemm_operands("mlt_gemm_tiled", A, B, C, transB, stream=stream)
    with _OtherDevice(A.device):
        rc = _lib.mlt_gemm_tiled(M, N, K, A.data_ptr(), lda, B.data_ptr(), ldb, int(transB),
                                 C.data_ptr(), ldc, dt, int(tiling), _stream(stream, A.device))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_gemm_tiled")
    return C


def mlt_gemm_bias_act(A: torch.Tensor, B: torch.Tensor, bias: torch.Tensor | None = None,
                      act: int = ACT_NONE, C: torch.Tensor | None = None, transB: bool = False,
                      stream=None) -> torch.Tensor:
    """C = act(A @ B + bias) (or A @ B.T), bias a contiguous [N] tensor of the input dtype or None,
    act one of ACT_NONE / ACT_RELU / ACT_GELU."""
    done = _fast.gemm_bias_act(A, B, bias, act, C, transB, stream)
    if done is not None:
        return done
    M, N, K, lda, ldb, ldc, dt, C = _gemm_operands("mlt_gemm_bias_act", A, B, C, transB, stream=stream)
    if bias is not None and (not bias.is_cuda or bias.dtype != A.dtype or tuple(bias.shape) != (N,)
                             or not bias.is_contiguous()):
        raise ValueError("bias must be a contiguous GPU tensor of N elements of the input dtype")
    with _OtherDevice(A.device):
        rc = _lib.mlt_gemm_bias_act(M, N, K, A.data_ptr(), lda, B.data_ptr(), ldb, int(transB),
                                    bias.data_ptr() if bias is not None else None, int(act),
                                    C.data_ptr(), ldc, dt, _stream(stream, A.device))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_gemm_bias_act")
    return C


def mlt_gemm_acc(A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, transB: bool = False,
                 stream=None) -> torch.Tensor:
    """C += A @ B (or A @ B.T) with C an fp32 [M, N] tensor that is read and written."""
    done = _fast.gemm_acc(A, B, C, transB, stream)
    if done is not None:
        return done
    if C is None:
        raise ValueError("mlt_gemm_acc needs the fp32 C it accumulates into")
    M, N, K, lda, ldb, ldc, dt, C = _gemm_operands("mlt_gemm_acc", A, B, C, transB, torch.float32)
    with _OtherDevice(A.device):
        rc = _lib.mlt_gemm_acc(M, N, K, A.data_ptr(), lda, B.data_ptr(), ldb, int(transB),
                               C.data_ptr(), ldc, dt, _stream(stream, A.device))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_gemm_acc")
    return C


def mlt_mha_fwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, scale: float,
                causal: bool = False, O: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """O = softmax(scale * Q K^T [+ causal mask]) V for contiguous [B, H, S, D] tensors."""
    done = _fast.mha_fwd(Q, K, V, scale, causal, O, stream)
    if done is not None:
        return done
    if not (Q.is_cuda and K.is_cuda and V.is_cuda):
        raise ValueError("mlt_mha_fwd needs GPU tensors")
    dt = _dtype_code(Q)
    if K.dtype != Q.dtype or V.dtype != Q.dtype:
        raise TypeError("Q, K and V must share a dtype")
    if Q.dim() != 4 or K.dim() != 4 or V.shape != K.shape:
        raise ValueError("expected Q [B,H,Sq,D], K and V [B,H,Sk,D]")
    B, H, Sq, D = Q.shape
    Sk = K.shape[2]
    if K.shape != (B, H, Sk, D):
        raise ValueError("K shape does not match Q")
    if not (Q.is_contiguous() and K.is_contiguous() and V.is_contiguous()):
        raise ValueError("Q, K and V must be contiguous")
    if O is None:
        O = _empty(Q.shape, Q.dtype, Q.device, stream)
    elif O.dtype != Q.dtype or O.shape != Q.shape or not O.is_contiguous():
        raise ValueError("O has the wrong dtype, shape or layout")
    with _OtherDevice(Q.device):
        rc = _lib.mlt_mha_fwd(B, H, Sq, Sk, D, Q.data_ptr(), K.data_ptr(), V.data_ptr(),
                              O.data_ptr(), float(scale), int(causal), dt, _stream(stream, Q.device))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_mha_fwd")
    return O


# ---- 8 bits: tensors of torch.float8_e4m3fn with fp32 scales

E4M3 = torch.float8_e4m3fn


def _gpu(name: str, *tensors) -> None:
    """All of them (None aside) on one GPU."""
    device = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("%s needs GPU tensors" % name)
        if device is None:
            device = t.device
        elif t.device != device:
            raise ValueError("%s: all tensors must be on one GPU" % name)


def _scales(t: torch.Tensor, shape, name: str) -> int:
    if t.dtype != torch.float32 or tuple(t.shape) != shape:
        raise ValueError("%s must be an fp32 tensor of shape %s" % (name, list(shape)))
    return _rows_contiguous(t, name)


def mlt_quant_fp8(X: torch.Tensor, block_rows: int = 1, Xq: torch.Tensor | None = None, S: torch.Tensor | None = None, stream=None):
    """Xq (e4m3 [M, K]) and S (fp32 [ceil(K/128), ceil(M/block_rows)]) of X [M, K]: a power of two as the scale of every
    block_rows x 128 block. block_rows: 1 (activations) or 128 (weights)."""
    done = _fast.quant_fp8(X, block_rows, Xq, S, stream)
    if done is not None:
        return done
    _gpu("mlt_quant_fp8", X, Xq, S)
    dt, ldx = _dtype_code(X), _rows_contiguous(X, "X")
    M, K = X.shape
    rows = int(block_rows)
    shape = (-(-K // 128), -(-M // rows) if rows > 0 else 0)
    if Xq is None:
        Xq = _empty((M, -(-K // 16) * 16), E4M3, X.device, stream)[:, :K]               # rows start on 16 bytes
    elif Xq.dtype != E4M3 or Xq.shape != X.shape:
        raise ValueError("Xq must be a float8_e4m3fn tensor of X's shape")
    if S is None:
        S = _empty(shape, torch.float32, X.device, stream)
    ldq, lds = _rows_contiguous(Xq, "Xq"), _scales(S, shape, "S")
    with _OtherDevice(X.device):
        rc = _lib.mlt_quant_fp8(M, K, X.data_ptr(), ldx, rows, Xq.data_ptr(), ldq, S.data_ptr(), lds, dt, _stream(stream, X.device))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_quant_fp8")
    return Xq, S


def mlt_gemm_fp8(A: torch.Tensor, Sa: torch.Tensor, B: torch.Tensor, Sb: torch.Tensor, C: torch.Tensor | None = None,
                 dtype: torch.dtype = torch.bfloat16, stream=None) -> torch.Tensor:
    """C = (A * Sa) @ (B * Sb).T: A [M, K], B [N, K] e4m3, Sa [ceil(K/128), M] and Sb [ceil(K/128), ceil(N/128)] fp32, as
    mlt_quant_fp8 makes them with block_rows 1 and 128. C (`dtype`, where it is not given) is bf16 or fp16 [M, N]."""
    done = _fast.gemm_fp8(A, Sa, B, Sb, C, stream)
    if done is not None:
        return done
    _gpu("mlt_gemm_fp8", A, Sa, B, Sb, C)
    if A.dtype != E4M3 or B.dtype != E4M3:
        raise TypeError("A and B must be float8_e4m3fn tensors")
    lda, ldb = _rows_contiguous(A, "A"), _rows_contiguous(B, "B")
    M, K = A.shape
    N = B.shape[0]
    if B.shape[1] != K:
        raise ValueError("inner dimensions differ: %d vs %d" % (K, B.shape[1]))
    kb = -(-K // 128)
    ldsa, ldsb = _scales(Sa, (kb, M), "Sa"), _scales(Sb, (kb, -(-N // 128)), "Sb")
    if C is None:
        C = _empty((M, N), dtype, A.device, stream)
    elif tuple(C.shape) != (M, N):
        raise ValueError("C has the wrong shape")
    dt, ldc = _dtype_code(C), _rows_contiguous(C, "C")
    with _OtherDevice(A.device):
        rc = _lib.mlt_gemm_fp8(M, N, K, A.data_ptr(), lda, Sa.data_ptr(), ldsa, B.data_ptr(), ldb, Sb.data_ptr(), ldsb, C.data_ptr(), ldc, dt,
                               _stream(stream, A.device))
    if rc != MLT_OK:
        raise MltError(rc, "mlt_gemm_fp8")
    return C


def _head_rows(t: torch.Tensor, T: int, D: int, dtype, name: str) -> int:
    """Row stride of [T, heads, D] whose heads lie side by side."""
    if t.dim() != 3 or t.shape[0] != T or t.shape[2] != D or t.dtype != dtype:
        raise ValueError("%s must be [%d, heads, %d] of K's type" % (name, T, D))
    if (D > 1 and t.stride(2) != 1) or (t.shape[1] > 1 and t.stride(1) != D):
        raise ValueError("%s: the heads of a token must lie side by side" % name)
    return t.stride(0) if T > 1 else t.shape[1] * D


def _append(name: str, Q, K, V, offsets, seq_lens, block_table, cos, sin, Kc, Vc, Ks, Vs, Qo, interleaved, stream):
    done = _fast.paged_append(Q, K, V, offsets, seq_lens, block_table, cos, sin, Kc, Vc, Ks, Vs, Qo, interleaved, stream)
    if done is not None:
        return done
    _gpu(name, K, V, Q, offsets, seq_lens, block_table, cos, sin, Kc, Vc, Ks, Vs, Qo)
    dt = _dtype_code(K)
    if K.dim() != 3:
        raise ValueError("%s: K must be [tokens, heads, D]" % name)
    T, H, D = K.shape
    ldk, ldv = _head_rows(K, T, D, K.dtype, "K"), _head_rows(V, T, D, K.dtype, "V")
    if V.shape != K.shape:
        raise ValueError("%s: K and V differ in shape" % name)
    Hq, ldq = 0, 0
    if Q is not None:
        Hq, ldq = Q.shape[1] if Q.dim() == 3 else 0, _head_rows(Q, T, D, K.dtype, "Q")
        if Qo is None:
            Qo = _empty((T, Hq, D), K.dtype, K.device, stream)
        elif Qo.dtype != K.dtype or Qo.shape != Q.shape or not Qo.is_contiguous():
            raise ValueError("%s: Qo must be contiguous, of Q's shape and type" % name)
    elif Qo is not None:
        raise ValueError("%s: Qo without Q" % name)
    if Kc.dim() != 4 or Kc.shape[1] != H or Kc.shape[3] != D or Vc.shape != Kc.shape:
        raise ValueError("%s: the cache must be [num_blocks, %d, block_size, %d]" % (name, H, D))
    want = K.dtype if Ks is None else E4M3
    if Kc.dtype != want or Vc.dtype != want:
        raise ValueError("%s: the cache must be of type %s" % (name, want))
    if block_table.dim() != 2 or seq_lens.dim() != 1:
        raise ValueError("%s: block_table / seq_lens shape" % name)
    B = seq_lens.shape[0]
    if any(t.dtype != torch.int32 for t in (offsets, seq_lens, block_table)):
        raise ValueError("%s: offsets, seq_lens and block_table must be int32" % name)
    if tuple(offsets.shape) != (B + 1,) or block_table.shape[0] != B:
        raise ValueError("%s: offsets / block_table shape" % name)
    rot, positions = 0, 0
    if (cos is None) != (sin is None):
        raise ValueError("%s: cos and sin come together" % name)
    if cos is not None:
        if cos.dim() != 2 or cos.shape != sin.shape or cos.dtype != torch.float32 or sin.dtype != torch.float32:
            raise ValueError("%s: cos and sin must be fp32 [positions, rot / 2]" % name)
        positions, rot = cos.shape[0], 2 * cos.shape[1]
    for s in (Ks, Vs):
        if s is not None and (s.dtype != torch.float32 or tuple(s.shape) != (Kc.shape[0], H)):
            raise ValueError("%s: Ks and Vs must be fp32 [num_blocks, %d]" % (name, H))
    for t in (offsets, seq_lens, block_table, cos, sin, Kc, Vc, Ks, Vs):
        if t is not None and not t.is_contiguous():
            raise ValueError("%s: offsets, seq_lens, block_table, cos, sin and the cache must be contiguous" % name)
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    head = (T, B, Hq, H, D, Kc.shape[2], block_table.shape[1], Kc.shape[0], ptr(Q), ldq, K.data_ptr(), ldk, V.data_ptr(), ldv, offsets.data_ptr(),
            seq_lens.data_ptr(), block_table.data_ptr(), ptr(cos), ptr(sin), rot, positions, int(bool(interleaved)), ptr(Qo), Kc.data_ptr(), Vc.data_ptr())
    with _OtherDevice(K.device):
        at = _stream(stream, K.device)
        rc = _lib.mlt_paged_append(*head, dt, at) if Ks is None else _lib.mlt_paged_append_fp8(*head, Ks.data_ptr(), Vs.data_ptr(), dt, at)
    if rc != MLT_OK:
        raise MltError(rc, name)
    return Qo


def mlt_paged_append(Q: torch.Tensor | None, K: torch.Tensor, V: torch.Tensor, offsets: torch.Tensor, seq_lens: torch.Tensor,
                     block_table: torch.Tensor, cos: torch.Tensor | None, sin: torch.Tensor | None, Kc: torch.Tensor, Vc: torch.Tensor,
                     Qo: torch.Tensor | None = None, interleaved: bool = False, stream=None) -> torch.Tensor | None:
    """The new tokens' keys (turned by their positions' angles) and values into the paged cache, in place; returns the turned
    queries. Q [T, Hq, D] (or None), K, V [T, H, D]: a token's heads side by side, any row stride; offsets int32 [B + 1]: the
    rows of each sequence; seq_lens int32 [B]: its tokens with the new ones; block_table int32 [B, max_blocks]; cos, sin fp32
    [positions, rot / 2] or None; Kc, Vc [num_blocks, H, block_size, D] of K's type."""
    return _append("mlt_paged_append", Q, K, V, offsets, seq_lens, block_table, cos, sin, Kc, Vc, None, None, Qo, interleaved, stream)


def mlt_paged_append_fp8(Q: torch.Tensor | None, K: torch.Tensor, V: torch.Tensor, offsets: torch.Tensor, seq_lens: torch.Tensor,
                         block_table: torch.Tensor, cos: torch.Tensor | None, sin: torch.Tensor | None, Kc: torch.Tensor, Vc: torch.Tensor,
                         Ks: torch.Tensor, Vs: torch.Tensor, Qo: torch.Tensor | None = None, interleaved: bool = False,
                         stream=None) -> torch.Tensor | None:
    """mlt_paged_append into an e4m3 cache with fp32 scales Ks, Vs [num_blocks, H], which are updated with it."""
    if Ks is None or Vs is None:
        raise ValueError("mlt_paged_append_fp8 needs the cache's scales")
    return _append("mlt_paged_append_fp8", Q, K, V, offsets, seq_lens, block_table, cos, sin, Kc, Vc, Ks, Vs, Qo, interleaved, stream)


def mlt_paged_attn_decode_fp8(Q: torch.Tensor, Kc: torch.Tensor, Vc: torch.Tensor, Ks: torch.Tensor, Vs: torch.Tensor,
                              block_table: torch.Tensor, seq_lens: torch.Tensor, scale: float, O: torch.Tensor | None = None,
                              stream=None) -> torch.Tensor:
    """Q [B, Hq, D]; Kc, Vc e4m3 [num_blocks, H, block_size, D] with Hq a multiple of H; Ks, Vs fp32 [num_blocks, H]; block_table
    int32 [B, max_blocks]; seq_lens int32 [B], 0 for a sequence without keys (zeros); returns O [B, Hq, D]."""
    name = "mlt_paged_attn_decode_fp8"
    done = _fast.paged_attn_decode_fp8(Q, Kc, Vc, Ks, Vs, block_table, seq_lens, scale, O, stream)
    if done is not None:
        return done
    _gpu(name, Q, Kc, Vc, Ks, Vs, block_table, seq_lens, O)
    dt = _dtype_code(Q)
    if Q.dim() != 3 or Kc.dim() != 4 or Vc.shape != Kc.shape or Kc.shape[3] != Q.shape[2]:
        raise ValueError("%s: cache shape does not match Q" % name)
    if Kc.dtype != E4M3 or Vc.dtype != E4M3:
        raise TypeError("%s: the cache must be of type float8_e4m3fn" % name)
    B, Hq, D = Q.shape
    nb, H, bs, _ = Kc.shape
    for s in (Ks, Vs):
        if s.dtype != torch.float32 or tuple(s.shape) != (nb, H):
            raise ValueError("%s: Ks and Vs must be fp32 [num_blocks, H]" % name)
    if block_table.dtype != torch.int32 or seq_lens.dtype != torch.int32:
        raise ValueError("%s: block_table and seq_lens must be int32" % name)
    if block_table.dim() != 2 or block_table.shape[0] != B or tuple(seq_lens.shape) != (B,):
        raise ValueError("%s: block_table / seq_lens shape" % name)
    if O is None:
        O = _empty(Q.shape, Q.dtype, Q.device, stream)
    elif O.dtype != Q.dtype or O.shape != Q.shape:
        raise ValueError("%s: O has the wrong dtype or shape" % name)
    for t in (Q, Kc, Vc, Ks, Vs, block_table, seq_lens, O):
        if not t.is_contiguous():
            raise ValueError("%s: tensors must be contiguous" % name)
    with _OtherDevice(Q.device):
        rc = _lib.mlt_paged_attn_decode_fp8(B, Hq, H, D, bs, block_table.shape[1], nb, Q.data_ptr(), Kc.data_ptr(), Vc.data_ptr(), Ks.data_ptr(),
                                            Vs.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), O.data_ptr(), float(scale), dt,
                                            _stream(stream, Q.device))
    if rc != MLT_OK:
        raise MltError(rc, name)
    return O


# ---- prompts, shared prefixes, 4-bit weights

def _offsets(name: str, t: torch.Tensor, B: int, what: str) -> None:
    if t.dtype != torch.int32 or tuple(t.shape) != (B + 1,) or not t.is_contiguous():
        raise ValueError("%s: %s must be a contiguous int32 tensor of %d elements" % (name, what, B + 1))


def _packed_queries(name: str, Q: torch.Tensor, O, stream):
    """dtype code, row strides and output (allocated when None) of packed queries [T, Hq, D]."""
    if Q.dim() != 3:
        raise ValueError("%s: Q must be [tokens, heads, D]" % name)
    T, Hq, D = Q.shape
    dt, ldq = _dtype_code(Q), _head_rows(Q, T, D, Q.dtype, "Q")
    if O is None:
        O = _empty(Q.shape, Q.dtype, Q.device, stream)
    elif O.shape != Q.shape:
        raise ValueError("%s: O has the wrong shape" % name)
    return dt, ldq, _head_rows(O, T, D, Q.dtype, "O"), O


def _paged_cache(name: str, Kc: torch.Tensor, Vc: torch.Tensor, D: int, dtype) -> None:
    if Kc.dim() != 4 or Vc.shape != Kc.shape or Kc.shape[3] != D:
        raise ValueError("%s: cache shape does not match Q" % name)
    if Kc.dtype != dtype or Vc.dtype != dtype:
        raise TypeError("%s: the cache must be of Q's type" % name)
    if not Kc.is_contiguous() or not Vc.is_contiguous():
        raise ValueError("%s: the cache must be contiguous" % name)


def _paged_tables(name: str, block_table: torch.Tensor, seq_lens: torch.Tensor) -> int:
    if block_table.dtype != torch.int32 or seq_lens.dtype != torch.int32:
        raise ValueError("%s: block_table and seq_lens must be int32" % name)
    if block_table.dim() != 2 or seq_lens.dim() != 1 or block_table.shape[0] != seq_lens.shape[0]:
        raise ValueError("%s: block_table / seq_lens shape" % name)
    if not block_table.is_contiguous() or not seq_lens.is_contiguous():
        raise ValueError("%s: block_table and seq_lens must be contiguous" % name)
    return seq_lens.shape[0]


def mlt_mha_packed_fwd(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, q_offsets: torch.Tensor, k_offsets: torch.Tensor | None, scale: float,
                       causal: bool = True, O: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Attention of packed sequences. Q [Tq, Hq, D], K, V [Tk, H, D] with Hq a multiple of H: a token's heads side by side, any row stride; q_offsets
    (k_offsets; None: the same) int32 [B + 1]: the rows of each sequence. causal: the last query of a sequence sees all its keys, the one before one
    less. Returns O [Tq, Hq, D]; rows of no sequence are left as they are."""
    name = "mlt_mha_packed_fwd"
    if k_offsets is None:
        k_offsets = q_offsets
    done = _fast.mha_packed_fwd(Q, K, V, q_offsets, k_offsets, scale, causal, O, stream)
    if done is not None:
        return done
    _gpu(name, Q, K, V, q_offsets, k_offsets, O)
    dt, ldq, ldo, O = _packed_queries(name, Q, O, stream)
    T, Hq, D = Q.shape
    if K.dim() != 3 or V.shape != K.shape:
        raise ValueError("%s: K and V must be [tokens, heads, D] of one shape" % name)
    Tk, H = K.shape[:2]
    ldk, ldv = _head_rows(K, Tk, D, Q.dtype, "K"), _head_rows(V, Tk, D, Q.dtype, "V")
    B = q_offsets.numel() - 1
    _offsets(name, q_offsets, B, "q_offsets")
    _offsets(name, k_offsets, B, "k_offsets")
    with _OtherDevice(Q.device):
        rc = _lib.mlt_mha_packed_fwd(T, Tk, B, Hq, H, D, Q.data_ptr(), ldq, K.data_ptr(), ldk, V.data_ptr(), ldv, q_offsets.data_ptr(), k_offsets.data_ptr(),
                                     O.data_ptr(), ldo, float(scale), int(bool(causal)), dt, _stream(stream, Q.device))
    if rc != MLT_OK:
        raise MltError(rc, name)
    return O


def mlt_paged_attn_prompt(Q: torch.Tensor, Kc: torch.Tensor, Vc: torch.Tensor, offsets: torch.Tensor, seq_lens: torch.Tensor, block_table: torch.Tensor,
                          scale: float, O: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Causal attention of the new tokens of sequences whose keys are in the paged cache (see mlt_paged_append). Q [T, Hq, D]; Kc, Vc [num_blocks, H,
    block_size, D] with Hq a multiple of H; offsets int32 [B + 1]: the rows of each sequence; seq_lens int32 [B]: its tokens with the new ones;
    block_table int32 [B, max_blocks]. Returns O [T, Hq, D]; rows of no sequence are left as they are."""
    name = "mlt_paged_attn_prompt"
    done = _fast.paged_attn_prompt(Q, Kc, Vc, offsets, seq_lens, block_table, scale, O, stream)
    if done is not None:
        return done
    _gpu(name, Q, Kc, Vc, offsets, seq_lens, block_table, O)
    dt, ldq, ldo, O = _packed_queries(name, Q, O, stream)
    T, Hq, D = Q.shape
    _paged_cache(name, Kc, Vc, D, Q.dtype)
    B = _paged_tables(name, block_table, seq_lens)
    _offsets(name, offsets, B, "offsets")
    nb, H, bs, _ = Kc.shape
    with _OtherDevice(Q.device):
        rc = _lib.mlt_paged_attn_prompt(T, B, Hq, H, D, bs, block_table.shape[1], nb, Q.data_ptr(), ldq, Kc.data_ptr(), Vc.data_ptr(), offsets.data_ptr(),
                                        seq_lens.data_ptr(), block_table.data_ptr(), O.data_ptr(), ldo, float(scale), dt, _stream(stream, Q.device))
    if rc != MLT_OK:
        raise MltError(rc, name)
    return O


def mlt_paged_attn_decode_prefix_work(B: int, Hq: int, H: int, D: int, block_size: int, max_blocks: int, prefix_len: int) -> int:
    """Bytes of `work` for a call of these sizes on the current GPU."""
    n = _lib.mlt_paged_attn_decode_prefix_work(B, Hq, H, D, block_size, max_blocks, prefix_len)
    if n < 0:
        raise MltError(n, "mlt_paged_attn_decode_prefix_work")
    return n


def mlt_paged_attn_decode_prefix(Q: torch.Tensor, Kc: torch.Tensor, Vc: torch.Tensor, prefix_table: torch.Tensor | None, prefix_len: int,
                                 block_table: torch.Tensor, seq_lens: torch.Tensor, scale: float, O: torch.Tensor | None = None,
                                 work: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """One query a sequence over a prefix that all share, read once, and its own keys. Q [B, Hq, D]; Kc, Vc [num_blocks, H, block_size, D] with Hq a
    multiple of H; prefix_table int32 [at least ceil(prefix_len / block_size)]: the prefix's blocks; block_table int32 [B, max_blocks] and seq_lens int32 [B]: as for
    mlt_paged_append, the prefix's tokens among a sequence's. work: uint8, mlt_paged_attn_decode_prefix_work bytes, for calls that are captured into
    a graph. Returns O [B, Hq, D]."""
    name = "mlt_paged_attn_decode_prefix"
    done = _fast.paged_attn_decode_prefix(Q, Kc, Vc, prefix_table, prefix_len, block_table, seq_lens, scale, O, work, stream)
    if done is not None:
        return done
    _gpu(name, Q, Kc, Vc, prefix_table, block_table, seq_lens, O, work)
    dt, P = _dtype_code(Q), int(prefix_len)
    if Q.dim() != 3:
        raise ValueError("%s: Q must be [sequences, heads, D]" % name)
    Bq, Hq, D = Q.shape
    _paged_cache(name, Kc, Vc, D, Q.dtype)
    B = _paged_tables(name, block_table, seq_lens)
    if B != Bq:
        raise ValueError("%s: block_table / seq_lens shape" % name)
    nb, H, bs, _ = Kc.shape
    if P > 0 and (prefix_table is None or prefix_table.dtype != torch.int32 or prefix_table.dim() != 1 or not prefix_table.is_contiguous()
                  or prefix_table.shape[0] * bs < P):
        raise ValueError("%s: prefix_table must be a contiguous int32 tensor with a block for every %d keys of the prefix" % (name, bs))
    if O is None:
        O = _empty(Q.shape, Q.dtype, Q.device, stream)
    elif O.dtype != Q.dtype or O.shape != Q.shape:
        raise ValueError("%s: O has the wrong dtype or shape" % name)
    if not Q.is_contiguous() or not O.is_contiguous():
        raise ValueError("%s: Q and O must be contiguous" % name)
    if work is not None and (work.dtype != torch.uint8 or not work.is_contiguous()):
        raise ValueError("%s: work must be a contiguous uint8 tensor" % name)
    with _OtherDevice(Q.device):
        rc = _lib.mlt_paged_attn_decode_prefix(B, Hq, H, D, bs, block_table.shape[1], nb, Q.data_ptr(), Kc.data_ptr(), Vc.data_ptr(),
                                               None if prefix_table is None else prefix_table.data_ptr(), P, block_table.data_ptr(), seq_lens.data_ptr(),
                                               O.data_ptr(), float(scale), None if work is None else work.data_ptr(), 0 if work is None else work.numel(),
                                               dt, _stream(stream, Q.device))
    if rc != MLT_OK:
        raise MltError(rc, name)
    return O


def mlt_gemm_w4(A: torch.Tensor, Wq: torch.Tensor, S: torch.Tensor, Z: torch.Tensor | None = None, group: int = 128, C: torch.Tensor | None = None,
                stream=None) -> torch.Tensor:
    """C = A @ W.T with 4-bit weights: A [M, K]; Wq uint8 [N, K / 2], element k in the low (even k) or high half of byte k / 2; S [ceil(K / group), N] of
    A's type; Z uint8 [ceil(K / group), N] or None (8): W[n, k] = S[k // group, n] * (q[n, k] - Z[k // group, n]). Returns C [M, N]."""
    name = "mlt_gemm_w4"
    done = _fast.gemm_w4(A, Wq, S, Z, group, C, stream)
    if done is not None:
        return done
    _gpu(name, A, Wq, S, Z, C)
    dt, g = _dtype_code(A), int(group)
    if Wq.dtype != torch.uint8 or (Z is not None and Z.dtype != torch.uint8) or S.dtype != A.dtype:
        raise TypeError("%s: Wq and Z must be uint8 tensors, S of A's type" % name)
    lda, ldw, lds = _rows_contiguous(A, "A"), _rows_contiguous(Wq, "Wq"), _rows_contiguous(S, "S")
    M, K = A.shape
    N = Wq.shape[0]
    shape = (-(-K // g) if g > 0 else 0, N)
    if 2 * Wq.shape[1] != K or (g > 0 and tuple(S.shape) != shape) or (Z is not None and Z.shape != S.shape):
        raise ValueError("%s: Wq must be [N, K / 2], S and Z [ceil(K / group), N]" % name)
    if C is None:
        C = _empty((M, N), A.dtype, A.device, stream)
    elif C.dtype != A.dtype or tuple(C.shape) != (M, N):
        raise ValueError("%s: C has the wrong dtype or shape" % name)
    with _OtherDevice(A.device):
        rc = _lib.mlt_gemm_w4(M, N, K, A.data_ptr(), lda, Wq.data_ptr(), ldw, g, S.data_ptr(), lds, None if Z is None else Z.data_ptr(),
                              0 if Z is None else _rows_contiguous(Z, "Z"), C.data_ptr(), _rows_contiguous(C, "C"), dt, _stream(stream, A.device))
    if rc != MLT_OK:
        raise MltError(rc, name)
    return C
