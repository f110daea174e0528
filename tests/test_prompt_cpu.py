"""Refusals of the operators for prompts, shared prefixes and 4-bit weights: the C entry points' checks (no device is touched) and the binding's."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2503_14985_amd import binding
    return binding


P, ODD, ODDER = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008), ctypes.c_void_p(0x10002)   # never dereferenced: validation comes first
BIG = 1 << 31


def _with(base, **changes):
    return list({**base, **changes}.values())


def _refuses(b, f, ok, invalid, unsupported):
    for bad in invalid:
        assert f(*_with(ok, **bad)) == b.MLT_ERR_INVALID_ARG, bad
    for bad in unsupported:
        assert f(*_with(ok, **bad)) == b.MLT_ERR_UNSUPPORTED, bad


def test_packed_refusals(b):
    ok = dict(Tq=9, Tk=9, B=2, Hq=4, H=2, D=64, Q=P, ldq=256, K=P, ldk=128, V=P, ldv=128, qo=P, ko=P, O=P, ldo=256, scale=0.1, causal=1, dtype=0, stream=None)
    f = b.raw().mlt_mha_packed_fwd
    _refuses(b, f, ok,
             [dict(dtype=2), dict(Tq=-1), dict(Tk=-1), dict(B=-1), dict(Hq=-4), dict(H=-2), dict(D=0), dict(scale=math.nan), dict(scale=math.inf), dict(H=0), dict(H=3), dict(Q=None),
              dict(K=None), dict(V=None), dict(qo=None), dict(ko=None), dict(O=None), dict(Q=ODD), dict(K=ODD), dict(V=ODD), dict(O=ODD), dict(qo=ODDER), dict(ko=ODDER),
              dict(ldq=248), dict(ldk=120), dict(ldv=120), dict(ldo=248)],
             [dict(D=96), dict(ldq=260), dict(ldk=132), dict(ldv=132), dict(ldo=260), dict(Tq=BIG), dict(Tk=BIG), dict(B=BIG), dict(ldk=1 << 23), dict(Tq=1 << 28, Hq=64, ldq=4096, ldo=4096)])
    for none in (dict(Tq=0, Q=None, O=None), dict(B=0, qo=None, ko=None), dict(Hq=0, Q=None)):
        assert f(*_with(ok, **none)) == b.MLT_OK


def test_prompt_refusals(b):
    ok = dict(T=9, B=2, Hq=4, H=2, D=128, bs=16, mb=4, nb=10, Q=P, ldq=512, Kc=P, Vc=P, offsets=P, lens=P, table=P, O=P, ldo=512, scale=0.1, dtype=1, stream=None)
    f = b.raw().mlt_paged_attn_prompt
    _refuses(b, f, ok,
             [dict(dtype=-1), dict(T=-1), dict(B=-1), dict(H=0), dict(H=3), dict(bs=0), dict(mb=0), dict(nb=0), dict(Q=None), dict(Kc=None), dict(Vc=None), dict(offsets=None),
              dict(lens=None), dict(table=None), dict(O=None), dict(Q=ODD), dict(Kc=ODD), dict(Vc=ODD), dict(O=ODD), dict(table=ODDER), dict(lens=ODDER), dict(ldq=504), dict(ldo=504),
              dict(scale=-math.inf)],
             [dict(D=80), dict(bs=24), dict(bs=2048), dict(ldq=516), dict(ldo=516), dict(mb=BIG), dict(nb=BIG), dict(mb=1 << 27)])
    assert f(*_with(ok, T=0, Q=None)) == b.MLT_OK


def test_prefix_refusals(b):
    ok = dict(B=2, Hq=4, H=2, D=128, bs=16, mb=4, nb=10, Q=P, Kc=P, Vc=P, prefix=P, P=30, table=P, lens=P, O=P, scale=0.1, work=P, bytes=0, dtype=1, stream=None)
    f = b.raw().mlt_paged_attn_decode_prefix
    _refuses(b, f, ok,
             [dict(dtype=5), dict(B=-1), dict(Hq=-1), dict(H=0), dict(H=3), dict(D=0), dict(bs=0), dict(mb=0), dict(nb=0), dict(P=-1), dict(P=65), dict(Q=None), dict(Kc=None),
              dict(Vc=None), dict(prefix=None), dict(table=None), dict(lens=None), dict(O=None), dict(Q=ODD), dict(Kc=ODD), dict(Vc=ODD), dict(work=ODD), dict(bytes=-1),
              dict(prefix=ODDER), dict(scale=math.nan)],
             [dict(D=256), dict(bs=8), dict(bs=1040), dict(nb=BIG), dict(mb=BIG), dict(B=1 << 30)])
    assert f(*_with(ok, B=0)) == b.MLT_OK and f(*_with(ok, Hq=0)) == b.MLT_OK
    w = b.raw().mlt_paged_attn_decode_prefix_work
    assert w(2, 4, 3, 128, 16, 4, 0) == b.MLT_ERR_INVALID_ARG and w(2, 4, 2, 32, 16, 4, 0) == b.MLT_ERR_UNSUPPORTED and w(0, 4, 2, 128, 16, 4, 0) == 0


def test_w4_refusals(b):
    ok = dict(M=4, N=8, K=128, A=P, lda=128, Wq=P, ldw=64, group=32, S=P, lds=8, Z=P, ldz=8, C=P, ldc=8, dtype=1, stream=None)
    f = b.raw().mlt_gemm_w4
    _refuses(b, f, ok,
             [dict(dtype=2), dict(M=-1), dict(N=-1), dict(K=-32), dict(group=0), dict(A=None), dict(Wq=None), dict(S=None), dict(C=None), dict(lda=120), dict(ldw=48), dict(lds=7),
              dict(ldz=7), dict(ldc=7), dict(A=ODD), dict(Wq=ODD), dict(S=ctypes.c_void_p(0x10001)), dict(C=ctypes.c_void_p(0x10001))],
             [dict(group=16), dict(group=256), dict(K=112), dict(lda=132), dict(ldw=72), dict(M=BIG), dict(N=BIG), dict(lda=1 << 26), dict(ldw=1 << 26), dict(lds=1 << 26), dict(ldz=1 << 26)])
    assert f(*_with(ok, M=0, A=None)) == b.MLT_OK and f(*_with(ok, N=0, C=None)) == b.MLT_OK


def test_binding_refusals(b):
    """Host tensors never reach the library."""
    q, k, off = torch.zeros((4, 4, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    cache, table = torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((1, 1), dtype=torch.int32)
    for call in (lambda: b.mlt_mha_packed_fwd(q, k, k, off, off, 0.1), lambda: b.mlt_paged_attn_prompt(q, cache, cache, off, off[:1], table, 0.1),
                 lambda: b.mlt_paged_attn_decode_prefix(q[:1], cache, cache, None, 0, table, off[:1], 0.1),
                 lambda: b.mlt_gemm_w4(q[0], torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((1, 8), dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            call()
