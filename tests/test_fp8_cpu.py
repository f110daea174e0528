"""Refusals of the 8-bit operators: the C entry points' checks (no device is touched) and the binding's. And the parity tests' own oracle."""
import ctypes

import numpy as np
import pytest
import torch

import fp8_util as u


@pytest.fixture(scope="module")
def b():
    from paper_2503_14985_amd import binding
    return binding


P, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)   # never dereferenced: validation comes first


def _with(base, **changes):
    return list({**base, **changes}.values())


def test_quant_refusals(b):
    ok = dict(M=4, K=128, X=P, ldx=128, rows=1, Xq=P, ldq=128, S=P, lds=4, dtype=0, stream=None)
    f = b.raw().mlt_quant_fp8
    for bad in (dict(dtype=2), dict(M=-1), dict(K=-8), dict(rows=0), dict(X=None), dict(Xq=None), dict(S=None), dict(ldx=120), dict(ldq=112), dict(lds=3),
                dict(X=ODD), dict(Xq=ODD), dict(S=ctypes.c_void_p(0x10002))):
        assert f(*_with(ok, **bad)) == b.MLT_ERR_INVALID_ARG, bad
    for bad in (dict(rows=2), dict(rows=64), dict(K=124), dict(ldx=132), dict(ldq=136), dict(M=1 << 32, lds=1 << 32)):
        assert f(*_with(ok, **bad)) == b.MLT_ERR_UNSUPPORTED, bad
    assert f(*_with(ok, M=0, X=None)) == b.MLT_OK and f(*_with(ok, K=0, Xq=None)) == b.MLT_OK


def test_gemm_refusals(b):
    ok = dict(M=4, N=8, K=128, A=P, lda=128, Sa=P, ldsa=4, B=P, ldb=128, Sb=P, ldsb=1, C=P, ldc=8, dtype=1, stream=None)
    f = b.raw().mlt_gemm_fp8
    for bad in (dict(dtype=-1), dict(M=-1), dict(N=-1), dict(K=-16), dict(A=None), dict(B=None), dict(Sa=None), dict(Sb=None), dict(C=None), dict(lda=112), dict(ldb=112),
                dict(ldsa=3), dict(ldsb=0), dict(ldc=7), dict(A=ODD), dict(B=ODD), dict(Sa=ctypes.c_void_p(0x10001)), dict(C=ctypes.c_void_p(0x10001))):
        assert f(*_with(ok, **bad)) == b.MLT_ERR_INVALID_ARG, bad
    for bad in (dict(K=120), dict(lda=136), dict(ldb=136), dict(lda=1 << 23), dict(ldb=1 << 23), dict(M=1 << 31, ldsa=1 << 31)):
        assert f(*_with(ok, **bad)) == b.MLT_ERR_UNSUPPORTED, bad
    assert f(*_with(ok, M=0, A=None)) == b.MLT_OK and f(*_with(ok, N=0, C=None)) == b.MLT_OK


APPEND = dict(T=3, B=2, Hq=4, H=2, D=64, block=16, max_blocks=2, num_blocks=4, Q=P, ldq=256, K=P, ldk=128, V=P, ldv=128, offsets=P, lens=P, table=P, cos=P, sin=P, rot=64,
              positions=10, interleaved=0, Qo=P, Kc=P, Vc=P)


@pytest.mark.parametrize("fp8", [False, True])
def test_append_refusals(b, fp8):
    ok = dict(APPEND, **(dict(Ks=P, Vs=P) if fp8 else {}), dtype=0, stream=None)
    f = b.raw().mlt_paged_append_fp8 if fp8 else b.raw().mlt_paged_append
    invalid = [dict(dtype=3), dict(T=-1), dict(B=-1), dict(Hq=-1), dict(H=-1), dict(block=0), dict(max_blocks=0), dict(num_blocks=0), dict(rot=-16), dict(rot=80), dict(Q=None),
               dict(K=None), dict(V=None), dict(offsets=None), dict(lens=None), dict(table=None), dict(cos=None), dict(sin=None), dict(positions=0), dict(Qo=None), dict(Kc=None),
               dict(Vc=None), dict(ldq=248), dict(ldk=120), dict(ldv=120), dict(Q=ODD), dict(K=ODD), dict(V=ODD), dict(Qo=ODD), dict(Kc=ODD), dict(Vc=ODD)]
    if fp8:
        invalid += [dict(Ks=None), dict(Vs=None), dict(Vs=ctypes.c_void_p(0x10002))]
    for bad in invalid:
        assert f(*_with(ok, **bad)) == b.MLT_ERR_INVALID_ARG, bad
    for bad in (dict(D=96, rot=0, ldq=384, ldk=192, ldv=192), dict(block=24), dict(block=1040), dict(rot=24), dict(ldq=260), dict(ldk=132), dict(ldv=132), dict(T=1 << 31),
                dict(max_blocks=1 << 28), dict(num_blocks=1 << 32), dict(positions=1 << 32)):
        assert f(*_with(ok, **bad)) == b.MLT_ERR_UNSUPPORTED, bad
    for none in (dict(T=0, K=None), dict(B=0, offsets=None), dict(Hq=0, H=0, Q=None, K=None)):
        assert f(*_with(ok, **none)) == b.MLT_OK, none


def test_attn_refusals(b):
    ok = dict(B=2, Hq=8, H=2, D=64, block=16, max_blocks=2, num_blocks=4, Q=P, Kc=P, Vc=P, Ks=P, Vs=P, table=P, lens=P, O=P, scale=0.1, dtype=0, stream=None)
    f = b.raw().mlt_paged_attn_decode_fp8
    for bad in (dict(dtype=9), dict(B=-1), dict(Hq=-8), dict(H=0), dict(H=3), dict(H=-2), dict(D=0), dict(block=0), dict(max_blocks=0), dict(num_blocks=0), dict(Q=None), dict(Kc=None),
                dict(Vc=None), dict(Ks=None), dict(Vs=None), dict(table=None), dict(lens=None), dict(O=None), dict(Q=ODD), dict(Kc=ODD), dict(Vc=ODD), dict(scale=float("nan")),
                dict(scale=float("inf"))):
        assert f(*_with(ok, **bad)) == b.MLT_ERR_INVALID_ARG, bad
    for bad in (dict(D=96), dict(block=24), dict(block=2048), dict(max_blocks=1 << 28), dict(num_blocks=1 << 31), dict(B=1 << 30)):
        assert f(*_with(ok, **bad)) == b.MLT_ERR_UNSUPPORTED, bad
    assert f(*_with(ok, B=0, Q=None)) == b.MLT_OK and f(*_with(ok, Hq=0, O=None)) == b.MLT_OK


def test_binding_takes_gpu_tensors_only(b):
    x, q8, s = torch.zeros((2, 128), dtype=torch.bfloat16), torch.zeros((2, 128)).to(u.F8), torch.ones((1, 2))
    i = torch.zeros(2, dtype=torch.int32)
    cache, sc = torch.zeros((2, 1, 16, 128)).to(u.F8), torch.ones((2, 1))
    k = x.reshape(2, 1, 128)
    for call in (lambda: b.mlt_quant_fp8(x), lambda: b.mlt_gemm_fp8(q8, s, q8, torch.ones((1, 1))),
                 lambda: b.mlt_paged_append(None, k, k, i, i[:1], i[:1].reshape(1, 1), None, None, cache.bfloat16(), cache.bfloat16()),
                 lambda: b.mlt_paged_append_fp8(None, k, k, i, i[:1], i[:1].reshape(1, 1), None, None, cache, cache, sc, sc),
                 lambda: b.mlt_paged_attn_decode_fp8(k, cache, cache, sc, sc, i.reshape(2, 1), i, 1.0)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_oracle_numbers():
    codes = torch.arange(127, dtype=torch.uint8).view(u.F8).double().numpy()
    assert np.array_equal(codes, u.E4M3)
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[(x.float().abs() <= 448)].double().numpy()
    assert np.array_equal(u.e4m3(x), torch.from_numpy(x).float().to(u.F8).double().numpy())
    assert u.scale_of(448.0) == 1.0 and u.scale_of(448.1) == 2.0 and u.scale_of(224.0) == 0.5 and u.scale_of(0.0) == 2.0 ** -100 == u.scale_of(1e-38)
    for top in np.exp(np.random.default_rng(0).uniform(-20, 20, 1000)):
        s = u.scale_of(top)
        assert top <= 448 * s and top > 224 * s


def test_oracle_against_torch():
    """The quantised product, the rotation and attention of the oracle against float64 compositions of another form."""
    g = np.random.default_rng(1)
    x = g.standard_normal((130, 200))
    q, s = u.quant(x, 128)
    back = q * np.repeat(np.repeat(s.T, 128, 0)[:130], 128, 1)[:, :200]
    assert (np.abs(back - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * s.max()).all()
    a, sa = u.quant(g.standard_normal((5, 200)), 1)
    c, mass, top = u.gemm(a, sa, q, s)
    assert (np.abs(c) <= mass * (1 + 1e-12)).all() and (top <= mass).all() and (mass <= 8 * top * (1 + 1e-12)).all()
    assert np.allclose(c, (a * np.repeat(sa.T, 128, 1)[:, :200]) @ back.T, rtol=1e-12, atol=1e-12)
    z = g.standard_normal((3, 2, 8))
    t = g.uniform(-3, 3, (3, 4))
    turned = (z[..., 0::2] + 1j * z[..., 1::2]) * np.exp(1j * t)[:, None]
    y = u.rotate(z, np.cos(t), np.sin(t), True)
    assert np.allclose(y[..., 0::2], turned.real) and np.allclose(y[..., 1::2], turned.imag)
    halves = np.concatenate([z[..., 0::2], z[..., 1::2]], -1)
    assert np.allclose(u.rotate(halves, np.cos(t), np.sin(t), False), np.concatenate([turned.real, turned.imag], -1))
    qv, k, v = g.standard_normal(8), g.standard_normal((11, 8)), g.standard_normal((11, 8))
    o = torch.softmax(torch.from_numpy(k @ qv) * 0.4, 0) @ torch.from_numpy(v)
    assert np.allclose(u.attn(qv, k, v, 0.4)[0], o.numpy())
