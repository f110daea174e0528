"""GPU parity of the 8-bit operators (mlt_quant_fp8, mlt_gemm_fp8, mlt_paged_append, mlt_paged_append_fp8, mlt_paged_attn_decode_fp8)
against their definitions in 64 bits (fp8_util), each alone and all of them as a decoder's attention layer uses them."""
import math

import numpy as np
import pytest
import torch

import fp8_util as u

pytestmark = pytest.mark.gpu
BF16, FP16, F8 = torch.bfloat16, torch.float16, u.F8


@pytest.fixture(autouse=True)
def _announce(request):
    print("\n[case] %s" % request.node.name, flush=True)
    yield


@pytest.fixture(scope="module")
def lib():
    from paper_2503_14985_amd import binding
    return binding


def dev():
    return torch.device("cuda:0")


def rand(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def f64(t):
    return t.detach().cpu().to(torch.float32).double().numpy() if t.dtype != torch.float64 else t.numpy()


def same(got, want):
    """Equal numbers, NaN in the same places."""
    return np.array_equal(np.asarray(got, np.float64), np.asarray(want, np.float64), equal_nan=True)


# ---- quantisation

@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K", [(1, 8), (1, 128), (3, 136), (16, 4096), (17, 512), (65, 648), (128, 256), (129, 1000), (300, 904)])
def test_quant(lib, dtype, rows, M, K):
    x = rand((M, K), dtype, M + K) * torch.exp(torch.randn(K, generator=torch.Generator().manual_seed(1)) * 3).to(dtype)
    wide = torch.full((M, K + 24), float("nan"), dtype=dtype)
    wide[:, 8:8 + K] = x
    view = wide.to(dev())[:, 8:8 + K]
    out = torch.full((M, (K + 31) // 16 * 16), 3.0, device=dev()).to(F8)
    s = torch.full((-(-K // 128), -(-M // rows) + 3), -1.0, device=dev())
    q, t = lib.mlt_quant_fp8(view, rows, Xq=out[:, :K], S=s[:, :-3])
    want_q, want_s = u.quant(f64(x), rows)
    assert same(f64(q), want_q) and same(f64(t), want_s)
    assert bool((out[:, K:].float() == 3.0).all()) and bool((s[:, -3:] == -1.0).all())      # what lies beside them
    q2, t2 = lib.mlt_quant_fp8(view, block_rows=rows)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(t2, t)       # (NaN, too, where fp16 has overflowed)


@pytest.mark.parametrize("rows", [1, 128])
def test_quant_edge_values(lib, rows):
    x = torch.zeros((256, 384), dtype=BF16)
    x[0, 0], x[1, 5], x[2, 130] = float("inf"), float("nan"), -float("inf")
    x[0, 7], x[130, 3] = 448.0, 450.0                       # the largest of a scale of 1, and the first past it
    x[3, 128:256] = torch.tensor(2.0 ** -130)               # below the smallest scale's reach
    x[4, 256:] = torch.finfo(BF16).max
    x[200, 256:260] = torch.tensor([2.0 ** -126, -0.0, 1.0, -2.0 ** -9])
    q, s = lib.mlt_quant_fp8(x.to(dev()), rows)
    want_q, want_s = u.quant(f64(x), rows)
    assert same(f64(q), want_q) and same(f64(s), want_s)
    assert np.isnan(f64(q)[0, 0]) and np.isnan(f64(q)[1, 5]) and np.isnan(f64(q)[2, 130]) and np.isfinite(f64(s)).all()


def test_quant_every_half_precision_number(lib):
    for dtype in (BF16, FP16):
        x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype).reshape(512, 128)
        q, s = lib.mlt_quant_fp8(x.to(dev()))
        want_q, want_s = u.quant(f64(x), 1)
        assert same(f64(q), want_q) and same(f64(s), want_s)


# ---- matrix product

def gemm_operands(M, N, K, seed):
    """e4m3 values over most of the format's range, scales that are no powers of two."""
    g = torch.Generator().manual_seed(seed)
    a, b = (torch.randn((r, K), generator=g).mul_(40).to(F8) for r in (M, N))
    kb = -(-K // 128)
    sa = torch.exp(torch.randn((kb, M), generator=g)) / 64
    sb = torch.exp(torch.randn((kb, -(-N // 128)), generator=g)) / 64
    return a, sa, b, sb


@pytest.mark.parametrize("rows,M,K", [(1, 1200000, 16), (128, 8500000, 8)])
def test_quant_many_rows(lib, rows, M, K):
    """More rows than a launch has in its second dimension. Small whole numbers times a power of two per row (per 128 rows): they come back exactly."""
    r = torch.arange(M, device=dev(), dtype=torch.int32)
    x = ((r[:, None] + torch.arange(K, device=dev(), dtype=torch.int32)) % 7 - 3).to(BF16) * torch.exp2((r // rows % 5).float()).to(BF16)[:, None]
    q, s = lib.mlt_quant_fp8(x, rows)
    assert torch.equal(q.to(BF16) * s[0].repeat_interleave(rows)[:M, None].to(BF16), x)


def gemm_check(C, a, sa, b, sb, dtype, K):
    ref, mass, top = u.gemm(f64(a), f64(sa), f64(b), f64(sb))
    tol = u.gemm_tolerance(ref, mass, top, K, sa.shape[0], dtype)
    if dtype == FP16:
        assert np.abs(ref).max() < 6e4
    err = np.abs(f64(C) - ref)
    assert np.isfinite(f64(C)).all() and (err <= tol).all(), float((err / tol).max())


GEMM_SHAPES = [(1, 1, 16), (1, 1024, 128), (2, 17, 144), (4, 2048, 512), (16, 4096, 1024), (17, 1030, 2048), (33, 1500, 1040), (64, 1024, 4096), (48, 300, 272),
               (65, 129, 128), (100, 257, 400), (128, 128, 256), (129, 640, 1152), (255, 384, 4096), (300, 777, 1008), (512, 512, 512), (257, 2050, 640),
               (520, 1100, 2064)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("M,N,K", GEMM_SHAPES)
def test_gemm(lib, dtype, M, N, K):
    a, sa, b, sb = gemm_operands(M, N, K, M + N + K)
    # rows in wider arrays, whose rest is NaN
    def wide(t, extra):
        w = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), device=dev()).to(t.dtype)
        w[:, :t.shape[1]].copy_(t.to(dev()))
        return w[:, :t.shape[1]]
    C = torch.full((M + 1, N + 5), -7.0, dtype=dtype, device=dev())
    out = C[:M, 2:2 + N]
    got = lib.mlt_gemm_fp8(wide(a, 32), wide(sa, 3), wide(b, 16), wide(sb, 1), C=out)
    print("   kernel=%s" % lib.mlt_last_kernel(), flush=True)
    assert got is out
    gemm_check(out, a, sa, b, sb, dtype, K)
    rest = C.clone()
    rest[:M, 2:2 + N] = -7.0
    assert bool((rest == -7.0).all())
    again = lib.mlt_gemm_fp8(a.to(dev()), sa.to(dev()), b.to(dev()), sb.to(dev()), dtype=dtype)
    gemm_check(again, a, sa, b, sb, dtype, K)                # (equal up to the order of the sums, which goes by B's alignment, too)


@pytest.fixture
def k_parts(lib):
    yield lib.mlt_diag_force_k_parts
    lib.mlt_diag_force_k_parts(0)


TILES = {"256pp16": "256x256_pp", "128pp16": "128x128_pp", "256x128kp": "256x128_kp", "224x128kp": "224x128_kp", "192x128kp": "192x128_kp", "128kp": "128x128_kp"}


@pytest.fixture
def variant(lib):
    yield lambda v: lib.mlt_diag_force_variant(gemm=v)
    lib.mlt_diag_force_variant(gemm="auto")


@pytest.mark.parametrize("name", sorted(TILES))
@pytest.mark.parametrize("M,N,K", [(1, 5, 128), (70, 200, 16), (129, 300, 272), (255, 129, 384), (256, 256, 512), (300, 777, 1040), (513, 640, 640), (900, 1030, 1296)])
def test_gemm_every_tile_kernel(lib, variant, name, M, N, K):
    """Tiles with rows and columns past the matrix, one K step, an odd and an even number of them, a step that K does not fill."""
    variant(name)
    a, sa, b, sb = gemm_operands(M, N, K, M + N + K)
    for dtype in (BF16, FP16):
        C = torch.full((M, N + 3), -7.0, dtype=dtype, device=dev())
        lib.mlt_gemm_fp8(a.to(dev()), sa.to(dev()), b.to(dev()), sb.to(dev()), C=C[:, :N])
        assert lib.mlt_last_kernel().startswith("gemm_fp8_" + TILES[name]), lib.mlt_last_kernel()
        gemm_check(C[:, :N], a, sa, b, sb, dtype, K)
        assert bool((C[:, N:] == -7.0).all())


def test_gemm_plan_follows_the_shape(lib):
    """The choice by itself: few rows stream B, a full grid takes the large tiles, few tiles against a long K its split, none of it under capture."""
    def name(M, N, K):
        a, b = (torch.zeros((r, K), device=dev()).to(F8) for r in (M, N))
        lib.mlt_gemm_fp8(a, torch.ones((-(-K // 128), M), device=dev()), b, torch.ones((-(-K // 128), -(-N // 128)), device=dev()))
        return lib.mlt_last_kernel()
    assert name(16, 4096, 4096) == "gemm_fp8_skinny"
    assert name(64, 512, 14336).startswith("gemm_fp8_skinny_splitk")
    assert name(512, 512, 1024) == "gemm_fp8_skinny"
    assert name(64, 28672, 14336) == "gemm_fp8_128x128_kp"
    assert name(4096, 4096, 4096) == "gemm_fp8_256x256_pp"
    assert name(2048, 4096, 1024) == "gemm_fp8_128x128_pp"
    assert name(512, 1024, 16384).startswith("gemm_fp8_128x128_kp_splitk")
    assert name(7, 9, 0) == "gemm_fp8_zero"
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = name(512, 1024, 16384)
    assert captured.startswith("gemm_fp8_") and "_splitk" not in captured


@pytest.mark.parametrize("parts", [2, 4, 8])
@pytest.mark.parametrize("name", [n for n in sorted(TILES) if n.endswith("kp")])
def test_gemm_tiles_with_k_in_parts(lib, variant, k_parts, name, parts):
    """Parts of one step and of several, of an odd number, the last one shorter; added in a fixed order."""
    variant(name)
    k_parts(parts)
    for M, N, K in ((100, 130, 1024), (300, 520, 3216), (257, 128, 128 * parts)):
        a, sa, b, sb = gemm_operands(M, N, K, M + N + K + parts)
        at = [t.to(dev()) for t in (a, sa, b, sb)]
        C = lib.mlt_gemm_fp8(*at)
        assert lib.mlt_last_kernel() == "gemm_fp8_%s_splitk%d" % (TILES[name], parts)
        gemm_check(C, a, sa, b, sb, BF16, K)
        for _ in range(3):
            assert torch.equal(lib.mlt_gemm_fp8(*at).view(torch.int16), C.view(torch.int16))


@pytest.mark.parametrize("parts", [2, 4, 8])
@pytest.mark.parametrize("M,N,K", [(1, 64, 128), (3, 1030, 2048), (16, 4096, 4112), (30, 520, 1040), (64, 2000, 2304), (50, 5000, 1024)])
def test_gemm_k_split_across_workgroups(lib, k_parts, variant, parts, M, N, K):
    """Few rows: parts of K by workgroups of their own, some of them empty, added by the last one; the same bits on every run."""
    k_parts(parts)
    variant("skinny")
    a, sa, b, sb = gemm_operands(M, N, K, M + N + K + parts)
    at = [t.to(dev()) for t in (a, sa, b, sb)]
    C = lib.mlt_gemm_fp8(*at)
    assert lib.mlt_last_kernel() == "gemm_fp8_skinny_splitk%d" % parts
    gemm_check(C, a, sa, b, sb, BF16, K)
    for _ in range(4):
        assert torch.equal(lib.mlt_gemm_fp8(*at).view(torch.int16), C.view(torch.int16))


@pytest.mark.parametrize("parts", [1, 2, 8])
@pytest.mark.parametrize("M", [65, 80, 129, 200, 333, 777, 1000, 1024, 1500, 4096])
def test_gemm_rows_shared_out(lib, k_parts, variant, parts, M):
    """More rows than one workgroup of the kernel for few rows takes: the last share ends inside a tile of 16 or before one; operands without a byte behind them."""
    k_parts(parts)
    variant("skinny")
    for N, K, dtype in ((1, 16, BF16), (150, 528, FP16), (40, 4112, BF16)):
        a, sa, b, sb = gemm_operands(M, N, K, M + N + K + parts)
        at = [t.to(dev()) for t in (a, sa, b, sb)]
        C = torch.full((M + 2, N), 7.0, dtype=dtype, device=dev())
        lib.mlt_gemm_fp8(*at, C=C[1:-1])
        assert lib.mlt_last_kernel() == "gemm_fp8_skinny" + ("_splitk%d" % parts if parts > 1 else "")
        assert bool((C[0] == 7).all()) and bool((C[-1] == 7).all())
        gemm_check(C[1:-1], a, sa, b, sb, dtype, K)


def test_gemm_large_sampled(lib):
    M, N, K = 2048, 4096, 4096
    a, sa, b, sb = gemm_operands(M, N, K, 5)
    C = lib.mlt_gemm_fp8(a.to(dev()), sa.to(dev()), b.to(dev()), sb.to(dev()))
    rows = np.unique(np.concatenate([np.arange(0, M, 61), [127, 128, 255, 256, M - 1]]))
    cols = np.unique(np.concatenate([np.arange(0, N // 128) * 128, [63, 64, 255, 256, N - 1]]))
    nb = torch.from_numpy(np.unique(cols // 128))
    full = np.concatenate([np.arange(128 * j, 128 * j + 128) for j in nb.tolist()])
    gemm_check(C[torch.from_numpy(rows).to(dev())][:, torch.from_numpy(full).to(dev())], a[rows].clone(), sa[:, rows], b[full].clone(), sb[:, nb], BF16, K)


def test_gemm_identity_and_scales(lib):
    """One 1 in each row of A picks a column of B: every position of K, row and column, exactly, with its own scales."""
    K, N = 512, 384
    a = torch.zeros((K, K)).to(F8)
    a.view(torch.uint8)[torch.arange(K), (torch.arange(K) * 37) % K] = 0x38                 # 1.0
    b = ((torch.arange(N)[:, None] * 7 + torch.arange(K)[None] * 3) % 15 - 7.0).to(F8)
    sa = (2.0 ** (torch.arange(4)[:, None] - torch.arange(K)[None] % 5)).float()
    sb = (2.0 ** (torch.arange(4)[:, None] * 2.0 - torch.arange(3)[None])).float()
    C = lib.mlt_gemm_fp8(a.to(dev()), sa.to(dev()), b.to(dev()), sb.to(dev()))
    assert same(f64(C), u.gemm(f64(a), f64(sa), f64(b), f64(sb))[0])


def test_gemm_empty(lib):
    e = lambda *s: torch.zeros(s, device=dev())  # noqa: E731
    C = torch.full((5, 7), 3.0, dtype=BF16, device=dev())
    lib.mlt_gemm_fp8(e(5, 0).to(F8), e(0, 5), e(7, 0).to(F8), e(0, 1), C=C)
    assert bool((C == 0).all())
    assert lib.mlt_gemm_fp8(e(0, 128).to(F8), e(1, 0), e(7, 128).to(F8), e(1, 1)).shape == (0, 7)
    assert lib.mlt_gemm_fp8(e(5, 128).to(F8), e(1, 5), e(0, 128).to(F8), e(1, 0)).shape == (5, 0)


# ---- the paged cache

def angles(positions, r, seed=None):
    p = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(r, dtype=torch.float64) / max(1, r))
    return p.cos().float(), p.sin().float()


def cache_state(B, lens, block, H, D, dtype, seed, extra=2):
    """Shuffled tables for the given lengths; a cache whose every slot holds something."""
    g = torch.Generator().manual_seed(seed)
    per = max(1, max(-(-max(1, n) // block) for n in lens))
    nb = B * per + extra
    table = torch.randperm(nb, generator=g)[:B * per].to(torch.int32).reshape(B, per)
    if dtype == F8:
        kc, vc = (torch.randn((nb, H, block, D), generator=g).mul_(60).to(F8) for _ in range(2))
        ks, vs = (torch.exp2(torch.randint(-8, -4, (nb, H), generator=g).float()) for _ in range(2))
    else:
        kc, vc = (torch.randn((nb, H, block, D), generator=g).to(dtype) for _ in range(2))
        ks = vs = None
    return table.contiguous(), kc, vc, ks, vs


def append_case(lib, new, before, Hq, H, D, block, rot, interleaved, dtype, fp8, seed, pad=0, gain=1.0, positions=None, tables=None, keep=False):
    B = len(new)
    T = sum(new) + pad
    lens = [n + p for n, p in zip(new, before)]
    offsets = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    table, kc, vc, ks, vs = cache_state(B, lens, block, H, D, F8 if fp8 else dtype, seed)
    if tables is not None:
        table = tables(table)
    rows = rand((T, (Hq + 2 * H) * D + 16), dtype, seed + 1, gain)
    if pad:
        rows[T - pad:] = float("nan")
    rows = rows.to(dev())
    q, k, v = (rows[:, a * D:(a + n) * D].unflatten(1, (n, D)) if n else None for a, n in ((0, Hq), (Hq, H), (Hq + H, H)))
    npos = positions or max(lens) + 1
    cos, sin = angles(npos, rot // 2) if rot else (None, None)
    args = [t.to(dev()) if t is not None else None for t in (torch.from_numpy(offsets), torch.tensor(lens, dtype=torch.int32), table, cos, sin, kc, vc)]
    Qo = torch.full((T, Hq, D), 9.0, dtype=dtype, device=dev()) if Hq else None
    Kc, Vc = args[5], args[6]
    if fp8:
        Ks, Vs = ks.to(dev()), vs.to(dev())
        out = lib.mlt_paged_append_fp8(q, k, v, *args, Ks, Vs, Qo=Qo, interleaved=interleaved)
    else:
        out = lib.mlt_paged_append(q, k, v, *args, Qo=Qo, interleaved=interleaved)
    torch.cuda.synchronize()
    assert out is Qo
    if keep:
        return dict(q=q, k=k, v=v, args=args, Ks=Ks if fp8 else None, Vs=Vs if fp8 else None, Qo=Qo)
    # expected, by rows that have a place
    spots = list(u.places(offsets.tolist(), lens, table.numpy(), block, kc.shape[0]))
    owner = np.zeros(T, int)
    pos = np.zeros(T, int)
    for b in range(B):
        for i in range(new[b]):
            owner[offsets[b] + i], pos[offsets[b] + i] = 1, lens[b] - new[b] + i
    at = np.clip(pos, 0, npos - 1)
    c64, s64 = (f64(cos)[at], f64(sin)[at]) if rot else (np.zeros((T, 0)), np.zeros((T, 0)))
    # two products and a sum in fp32, then the rounding to the type
    grow = lambda x: u.rotate(np.abs(x), np.abs(c64), -np.abs(s64), interleaved) + u.rotate(np.abs(x), np.abs(c64), np.abs(s64), interleaved)  # noqa: E731
    if Hq:
        q64 = np.nan_to_num(f64(q))
        want = u.rotate(q64, c64, s64, interleaved)
        got = f64(Qo)
        tol = u.HALF[dtype] * np.abs(want) + grow(q64) * 2.0 ** -22 + 2.0 ** -25
        assert (np.abs(got - want)[owner == 1] <= tol[owner == 1]).all()
        assert (got[owner == 0] == 9.0).all()                                # rows of no sequence stay as they were
    k64, v64 = np.nan_to_num(f64(k)), np.nan_to_num(f64(v))
    kr = u.rotate(k64, c64, s64, interleaved)
    if not fp8:
        for x, raw, cache, got in ((kr, k64, kc, Kc), (v64, v64, vc, Vc)):
            want, tol = f64(cache).copy(), np.zeros(cache.shape)
            allowed = u.HALF[dtype] * np.abs(x) + grow(raw) * 2.0 ** -22 + 2.0 ** -25
            for t, b, p, blk, slot in spots:
                want[blk, :, slot] = x[t]
                tol[blk, :, slot] = allowed[t]
            assert (np.abs(f64(got) - want) <= tol).all()
            assert cache is not vc or same(f64(got), want)                   # values are copied
        return
    for x, raw, cache, scales, got, gots in ((kr, k64, kc, ks, Kc, Ks), (v64, v64, vc, vs, Vc, Vs)):
        want, wants = u.append_fp8(x, f64(cache), f64(scales), spots)
        assert same(f64(gots), wants)
        if x is v64 or rot == 0:
            assert same(f64(got), want)
            continue
        # a turned key's fp32 error may take it over the middle between two numbers: then it is the other neighbour
        tol, have, slack = np.zeros(cache.shape), f64(got), grow(raw) * 2.0 ** -22
        for t, b, p, blk, slot in spots:
            s = wants[blk][:, None]
            tol[blk, :, slot] = 2 * u.HALF[F8] * np.abs(want[blk, :, slot]) + 2.0 ** -9
            off = np.abs(have[blk, :, slot] * s - x[t])
            assert (off <= u.HALF[F8] * np.abs(x[t]) * 1.0001 + s * 2.0 ** -10 * 1.0001 + slack[t]).all()
        diff = np.abs(have - want)
        assert (diff <= tol).all() and (diff > 0).mean() < 1e-4


APPENDS = [  # new, before, block
    ([1], [0], 16), ([1], [15], 16), ([1], [16], 16), ([1, 1, 1, 1, 1], [0, 3, 15, 16, 100], 16), ([0, 1, 0, 2], [5, 6, 0, 31], 16),
    ([37], [0], 16), ([5, 60, 1, 0, 33], [11, 4, 16, 9, 0], 16), ([70, 3], [29, 40], 32), ([200, 1], [7, 130], 64), ([300, 20], [3, 100], 128), ([50], [1000], 1024),
    ([1] * 150, list(range(150)), 16), ([2] * 70, [13] * 70, 48)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new,before,block", APPENDS)
def test_append(lib, fp8, new, before, block):
    many = len(new) > 20
    append_case(lib, new, before, 2 if many else 6, 2, 64 if many else 128, block, 32 if many else 128, False, BF16, fp8, 7, pad=3)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hq,H,D,rot", [(4, 1, 64, 64), (1, 1, 128, 16), (3, 3, 64, 48), (8, 2, 128, 64), (0, 2, 128, 128), (5, 5, 128, 112), (2, 1, 64, 0)])
def test_append_heads_and_rotations(lib, fp8, interleaved, Hq, H, D, rot):
    append_case(lib, [3, 20, 1], [14, 0, 40], Hq, H, D, 16, rot, interleaved, FP16, fp8, 11)


@pytest.mark.parametrize("gain", [1e-3, 30.0])
def test_append_fp8_scale_is_kept_or_grows(lib, gain):
    """Small new tokens keep a block's scale, large ones make its earlier tokens be rounded again."""
    append_case(lib, [1, 4, 30], [9, 30, 5], 2, 3, 128, 32, 64, False, BF16, True, 13, gain=gain)
    append_case(lib, [1, 4, 90], [9, 30, 5], 2, 2, 64, 64, 64, False, FP16, True, 17, gain=gain)


def test_append_bad_table_entries_and_positions(lib):
    """Blocks outside the cache are not written, positions past the tables of angles take the last row; all else is as ever."""
    def bad(t):
        t = t.clone()
        t[0, 0], t[1, 1] = -3, 1 << 30
        return t
    for fp8 in (False, True):
        append_case(lib, [20, 20, 20], [0, 0, 4], 2, 2, 64, 16, 64, False, BF16, fp8, 19, tables=bad)
        append_case(lib, [20, 3], [0, 30], 2, 2, 64, 16, 32, True, BF16, fp8, 23, positions=11)
        # a length that is shorter than the new tokens (the first ones lie in front of the sequence), or longer than the table
        B, T = 2, 40
        table, kc, vc, ks, vs = cache_state(B, [20, 20], 16, 1, 64, F8 if fp8 else BF16, 29)
        k = rand((T, 1, 64), BF16, 31).to(dev())
        for lens in ([4, -50], [1 << 30, 33], [-(1 << 31), (1 << 31) - 1]):
            K1, V1 = kc.to(dev()), vc.to(dev())
            args = (None, k, k, torch.tensor([0, 20, 40], dtype=torch.int32, device=dev()), torch.tensor(lens, dtype=torch.int32, device=dev()), table.to(dev()), None, None, K1, V1)
            if fp8:
                lib.mlt_paged_append_fp8(*args, ks.to(dev()), vs.to(dev()))
            else:
                lib.mlt_paged_append(*args)
                want = f64(vc).copy()
                for t, b, p, blk, slot in u.places([0, 20, 40], lens, table.numpy(), 16, kc.shape[0]):
                    want[blk, :, slot] = f64(k)[t]
                assert same(f64(V1), want)


def test_append_is_repeatable(lib):
    """The same tokens again change nothing more."""
    st = append_case(lib, [5, 60, 1], [11, 4, 16], 4, 2, 128, 16, 128, False, BF16, True, 37, gain=8.0, keep=True)
    a = st["args"]
    held = [t.clone() for t in (a[5].view(torch.uint8), a[6].view(torch.uint8), st["Ks"], st["Vs"], st["Qo"])]
    lib.mlt_paged_append_fp8(st["q"], st["k"], st["v"], *a, st["Ks"], st["Vs"], Qo=st["Qo"])
    for x, y in zip(held, (a[5].view(torch.uint8), a[6].view(torch.uint8), st["Ks"], st["Vs"], st["Qo"])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,block", [(64, 32), (128, 48), (64, 80), (128, 128), (64, 144), (128, 256), (64, 1024), (128, 1024)])
def test_append_block_sizes(lib, D, block, interleaved):
    """From one wavefront to sixteen for a (block, head): blocks filled at once, in pieces, over a border, and single tokens far into a block, with growing and falling scales."""
    for gain in (0.01, 20.0):
        append_case(lib, [2 * block + 5, 3, block - 1, 37], [0, block - 2, 1, block // 2], 2, 3, D, block, D // 2, interleaved, BF16, True, 51, gain=gain)
        append_case(lib, [1, 1, 1, 0], [block - 1, block // 2 + 1, 0, 7], 1, 2, D, block, D, interleaved, FP16, True, 53, gain=gain)


# ---- attention

def attn_case(lib, lens, Hq, H, D, block, dtype, seed, scale=None, poison=True, spread=True):
    B, scale = len(lens), 1.0 / math.sqrt(D) if scale is None else scale
    table, kc, vc, ks, vs = cache_state(B, lens, block, H, D, F8, seed)
    g = torch.Generator().manual_seed(seed + 1)
    if spread:                                              # scales that are no powers of two, apart by up to 2^6
        ks, vs = (torch.exp2(torch.rand(ks.shape, generator=g) * 2 - 8), torch.exp2(torch.rand(vs.shape, generator=g) * 6 - 9))
    q = rand((B, Hq, D), dtype, seed + 2)
    if poison:                                              # what no key holds: NaN behind the last one, in unused blocks and their scales
        used = torch.zeros(kc.shape[0], kc.shape[2], dtype=torch.bool)
        for b, n in enumerate(lens):
            for p in range(n):
                used[table[b, p // block], p % block] = True
        for c in (kc, vc):
            c.view(torch.uint8)[(~used)[:, None].expand(-1, H, -1)] = 0x7F
        ks[~used.any(1)] = float("nan")
        vs[~used.any(1)] = float("nan")
        for b, n in enumerate(lens):
            table[b, -(-n // block):] = 1 << 20
    O = torch.full((B, Hq, D), 5.0, dtype=dtype, device=dev())
    at = [t.to(dev()) for t in (q, kc, vc, ks, vs, table, torch.tensor(lens, dtype=torch.int32))]
    assert lib.mlt_paged_attn_decode_fp8(*at, scale, O=O) is O
    got = f64(O)
    assert np.isfinite(got).all()
    k64, v64 = f64(kc) * f64(ks)[..., None, None], f64(vc) * f64(vs)[..., None, None]
    G = Hq // H
    worst = 0.0
    for b, n in enumerate(lens):
        blocks = table[b, :-(-n // block)].long().numpy()
        for h in range(H):
            k, v = (x[blocks, h].reshape(-1, D)[:n] for x in (k64, v64))
            for j in range(G):
                o, mass, reach = u.attn(f64(q)[b, h * G + j], k, v, scale)
                tol = u.attn_tolerance(o, mass, reach, n, D, dtype, float(np.abs(v).max()) if n else 0.0)
                err = np.abs(got[b, h * G + j] - o)
                worst = max(worst, float((err / tol).max()))
                assert (err <= tol).all(), (b, h, j, float((err / tol).max()))
                if n == 0:
                    assert (got[b, h * G + j] == 0).all()
    print("   kernel=%s worst %.2f of the tolerance" % (lib.mlt_last_kernel(), worst), flush=True)
    return at, O


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block", [16, 48, 64])
def test_attn_ragged_lengths(lib, dtype, D, block):
    attn_case(lib, [1, 0, 2, 15, 16, 17, 31, 32, 33, 63, 65, 127, 129, 257, 1000, 4 * block], 6, 3, D, block, dtype, 41)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block", [80, 256, 1024])
def test_attn_large_blocks(lib, D, block):
    attn_case(lib, [1, block - 1, block, block + 1, 0, 2 * block + 17], 4, 2, D, block, BF16, 42)


@pytest.mark.parametrize("Hq,H", [(1, 1), (8, 8), (8, 1), (16, 1), (17, 1), (40, 2), (96, 3)])
def test_attn_head_groups(lib, Hq, H):
    attn_case(lib, [77, 0, 300, 1], Hq, H, 128, 16, BF16, 43)
    attn_case(lib, [77, 0, 300, 1], Hq, H, 64, 32, FP16, 44)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_attn_scale_edge_values(lib, scale):
    attn_case(lib, [5, 130, 700], 4, 2, 128, 32, BF16, 47, scale=scale)
    attn_case(lib, [5, 130, 700], 4, 2, 64, 16, FP16, 48, scale=scale)


@pytest.fixture
def key_split(lib):
    yield lib.mlt_diag_force_key_split
    lib.mlt_diag_force_key_split(0)


@pytest.mark.parametrize("nsplit", [1, 2, 3, 7, 8, 9, 33, 64])
@pytest.mark.parametrize("dtype,D", [(BF16, 128), (FP16, 64)])
def test_attn_key_split(lib, key_split, nsplit, dtype, D):
    key_split(nsplit)
    at, O = attn_case(lib, [1, 0, 2, 16, 33, 257, 1023, 2048, 3001], 6, 2, D, 16, dtype, 53)
    assert lib.mlt_last_kernel().endswith("_keysplit%d" % nsplit if nsplit > 1 else "_w8")
    for _ in range(3):
        assert torch.equal(lib.mlt_paged_attn_decode_fp8(*at, 1.0 / math.sqrt(D)), O)


def test_attn_long_and_batches(lib):
    attn_case(lib, [5000], 8, 8, 128, 16, BF16, 59, poison=False)
    assert "keysplit" in lib.mlt_last_kernel()
    attn_case(lib, [100 + 3 * i for i in range(70)], 8, 8, 64, 16, FP16, 61, poison=False)
    attn_case(lib, [1 + 40 * i for i in range(40)], 8, 2, 128, 32, BF16, 67, poison=False)


@pytest.mark.parametrize("H,Hq,D,top,nsplit", [(16, 16, 128, 1030, 1), (40, 40, 64, 2050, 1), (5, 90, 128, 2050, 2), (16, 16, 128, 1030, 3)])
def test_attn_mixed_batch_dealt_by_length(lib, key_split, H, Hq, D, top, nsplit):
    """Enough workgroups, and enough for each to read, for them to be dealt out by length: equal lengths, empty sequences and a negative length among them."""
    key_split(nsplit)
    lens = [0, 7, 1000, 7, 7, top, 0, 64, 65, 96, 96, 1, 500, 1000, 31, 33, 800, 0, 2]
    at, O = attn_case(lib, lens, Hq, H, D, 32, BF16, 79, poison=False)
    low = at[6].clone()
    low[low == 0] = -9
    for _ in range(3):
        assert torch.equal(lib.mlt_paged_attn_decode_fp8(*at[:6], low, 1.0 / math.sqrt(D)), O)


def test_attn_single_key_and_constant_values(lib):
    """One key: its value, rounded once. Constant values with one scale: they come back; block placement is irrelevant."""
    at, O = attn_case(lib, [1, 33, 200], 4, 2, 128, 16, BF16, 71, spread=False)
    vc, vs, table = at[2], at[4], at[5]
    first = int(table[0, 0])
    want = (f64(vc)[first, :, 0] * f64(vs)[first][:, None]).repeat(2, 0)
    assert same(f64(O)[0], f64(torch.from_numpy(want).to(BF16)))
    const = torch.full_like(vc.float(), -2.5).to(F8)
    O2 = lib.mlt_paged_attn_decode_fp8(at[0], at[1], const, at[3], torch.ones_like(vs), table, at[6], 0.1)
    assert (np.abs(f64(O2) + 2.5) <= 2.5 * 2.0 ** -8).all()
    perm = torch.randperm(vc.shape[0], generator=torch.Generator().manual_seed(3))
    inv = torch.argsort(perm).to(torch.int32)
    moved = [t.view(torch.uint8).cpu()[perm].to(dev()).view(F8) for t in (at[1], at[2])] + [t.cpu()[perm].to(dev()) for t in (at[3], at[4])]
    t2 = table.cpu().clone()
    ok = t2 < vc.shape[0]
    t2[ok] = inv[t2[ok].long()]
    O3 = lib.mlt_paged_attn_decode_fp8(at[0], *moved, t2.to(dev()), at[6], 1.0 / math.sqrt(128))
    assert torch.equal(O3, O)


def test_attn_peaked_rising_and_far_scales(lib):
    """Scores that rise all along the sequence (the reference moves again and again), and value scales that do."""
    n, H, D, block = 640, 2, 128, 16
    table = torch.arange(n // block, dtype=torch.int32).reshape(1, -1)
    g = torch.Generator().manual_seed(5)
    q = torch.ones((1, 4, D), dtype=BF16)
    kc = torch.full((n // block, H, block, D), 1.0)
    kc = (kc * (1 + torch.arange(block)[None, None, :, None] % 4)).to(F8)
    ks = (torch.arange(n // block).float() / 16 + 0.1)[:, None].repeat(1, H)
    vc = torch.randn((n // block, H, block, D), generator=g).mul_(50).to(F8)
    vs = torch.exp2(torch.arange(n // block).float() * 2 - 60)[:, None].repeat(1, H)
    for flip in (False, True):
        scales = vs.flip(0) if flip else vs
        O = lib.mlt_paged_attn_decode_fp8(*(t.contiguous().to(dev()) for t in (q, kc, vc, ks, scales, table)), torch.tensor([n], dtype=torch.int32, device=dev()), 0.3)
        k64, v64 = f64(kc) * f64(ks)[..., None, None], f64(vc) * f64(scales)[..., None, None]
        for h in range(H):
            o, mass, reach = u.attn(f64(q)[0, 0], k64[:, h].reshape(-1, D), v64[:, h].reshape(-1, D), 0.3)
            tol = u.attn_tolerance(o, mass, reach, n, D, BF16, np.abs(v64).max())
            assert (np.abs(f64(O)[0, 2 * h] - o) <= tol).all()


def test_attn_bad_lengths_and_blocks_stay_inside(lib):
    at, O = attn_case(lib, [40, 40, 40], 2, 2, 64, 16, BF16, 73, poison=False)
    t2, l2 = at[5].clone(), at[6].clone()
    t2[1, 1], t2[1, 2], l2[2] = 10 ** 6, -5, 1 << 30
    out = lib.mlt_paged_attn_decode_fp8(*at[:5], t2, l2, 1.0 / 8)
    assert torch.equal(out[0], O[0]) and bool(torch.isfinite(out.float()).all())
    l2[2] = -(1 << 31)
    assert bool((lib.mlt_paged_attn_decode_fp8(*at[:5], at[5], l2, 1.0 / 8)[2] == 0).all())


# ---- all of them

def layer(lib, w, x, state, Qo, stream=None):
    """A decoder's attention layer for a step's tokens: projection, rotation and append, attention, projection back."""
    xq, sx = lib.mlt_quant_fp8(x, stream=stream)
    qkv = lib.mlt_gemm_fp8(xq, sx, *w["in"], dtype=x.dtype, stream=stream)
    Hq, H, D = w["heads"]
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, H * D, H * D], 1))
    lib.mlt_paged_append_fp8(q, k, v, *state["where"], state["cos"], state["sin"], state["Kc"], state["Vc"], state["Ks"], state["Vs"], Qo=Qo, stream=stream)
    o = lib.mlt_paged_attn_decode_fp8(Qo, state["Kc"], state["Vc"], state["Ks"], state["Vs"], state["where"][2], state["where"][1], 1.0 / math.sqrt(D), stream=stream)
    oq, so = lib.mlt_quant_fp8(o.flatten(1), stream=stream)
    return lib.mlt_gemm_fp8(oq, so, *w["out"], dtype=x.dtype, stream=stream)


def layer_setup(lib, B, seed, dtype=BF16):
    Hq, H, D, hidden, block = 4, 2, 64, 384, 16
    w_in, w_out = rand(((Hq + 2 * H) * D, hidden), dtype, seed, 0.05), rand((hidden, Hq * D), dtype, seed + 1, 0.05)
    w = dict(heads=(Hq, H, D), **{"in": lib.mlt_quant_fp8(w_in.to(dev()), 128), "out": lib.mlt_quant_fp8(w_out.to(dev()), 128)})
    nb = B * 6
    st = dict(Kc=torch.zeros((nb, H, block, D), device=dev()).to(F8), Vc=torch.zeros((nb, H, block, D), device=dev()).to(F8),
              Ks=torch.ones((nb, H), device=dev()), Vs=torch.ones((nb, H), device=dev()))
    cos, sin = angles(96, D // 2)
    table = torch.randperm(nb, generator=torch.Generator().manual_seed(seed)).to(torch.int32).reshape(B, 6)
    st.update(cos=cos.to(dev()), sin=sin.to(dev()),
              where=[torch.arange(B + 1, dtype=torch.int32, device=dev()), torch.zeros(B, dtype=torch.int32, device=dev()), table.to(dev())])
    return w, st


def test_steps_of_a_layer(lib):
    """Forty decode steps of an attention layer against the same layer in 64 bits on the exact keys and values: the outputs differ by what 8 bits
    lose (each e4m3 operand is off by half a step, 2^-4 relative, at random: an rms of 2^-4 / sqrt(3) of it at most; three of
    them in a row (weight, activation, cache), their effect on the weights of the softmax of the same order)."""
    B, steps = 5, 40
    w, st = layer_setup(lib, B, 79)
    Hq, H, D = w["heads"]
    dq = lambda q, s, rows: f64(q) * np.repeat(np.repeat(f64(s).T, rows, 0)[:q.shape[0]], 128, 1)[:, :q.shape[1]]  # noqa: E731
    Wi, Wo = dq(*w["in"], 128), dq(*w["out"], 128)
    cos, sin = f64(st["cos"]), f64(st["sin"])
    keys, values = [[] for _ in range(B)], [[] for _ in range(B)]
    Qo = torch.empty((B, Hq, D), dtype=BF16, device=dev())
    off, size = 0.0, 0.0
    for i in range(steps):
        st["where"][1] += 1
        x = rand((B, 384), BF16, 1000 + i)
        y = f64(layer(lib, w, x.to(dev()), st, Qo))
        qkv = (f64(x) @ Wi.T).reshape(B, Hq + 2 * H, D)
        at = np.full(B, i)
        q, k = u.rotate(qkv[:, :Hq], cos[at], sin[at], False), u.rotate(qkv[:, Hq:Hq + H], cos[at], sin[at], False)
        want = np.empty((B, Hq * D))
        for b in range(B):
            keys[b].append(k[b])
            values[b].append(qkv[b, Hq + H:])
            for h in range(Hq):
                kk, vv = (np.stack(z)[:, h // (Hq // H)] for z in (keys[b], values[b]))
                want[b, h * D:(h + 1) * D] = u.attn(q[b, h], kk, vv, 1 / math.sqrt(D))[0]
        ref = want @ Wo.T
        off += ((y - ref) ** 2).sum()
        size += (ref ** 2).sum()
    rel = math.sqrt(off / size)
    print("   relative rms %.4f" % rel, flush=True)
    assert rel <= 4 * 2.0 ** -4 / math.sqrt(3)


def test_on_another_stream(lib):
    """Explicit stream and current stream: the work is enqueued there, behind what is on it."""
    B = 3
    w, st = layer_setup(lib, B, 83)
    w2, st2 = layer_setup(lib, B, 83)
    Qo, Qo2 = (torch.empty((B, 4, 64), dtype=BF16, device=dev()) for _ in range(2))
    side = torch.cuda.Stream()
    x = rand((B, 384), BF16, 89).to(dev())
    st["where"][1] += 1
    want = layer(lib, w, x * 2, st, Qo)
    side.wait_stream(torch.cuda.current_stream())
    for explicit in (True, False):
        with torch.cuda.stream(side):
            torch.cuda._sleep(5_000_000)
            x2 = x * 2
            st2["where"][1].fill_(1)
            if not explicit:
                y = layer(lib, w2, x2, st2, Qo2)
        if explicit:
            side.synchronize()
            y = layer(lib, w2, x2, st2, Qo2, stream=side)
        side.synchronize()
        assert torch.equal(y, want)


def test_split_calls_on_two_streams_at_once(lib):
    """Calls that spread one result over workgroups, on two streams that overlap: each stream has its own partial results and counters."""
    def product(M, N, K, seed):
        at = [t.to(dev()) for t in gemm_operands(M, N, K, seed)]
        return lambda stream: lib.mlt_gemm_fp8(*at, stream=stream)

    def attention(B, H, n, seed):
        g = torch.Generator(device=dev())
        g.manual_seed(seed)
        per = -(-n // 16)
        kc, vc = (torch.randn((B * per, H, 16, 128), generator=g, device=dev()).to(F8) for _ in range(2))
        ks, vs = (torch.rand((B * per, H), generator=g, device=dev()) + 0.1 for _ in range(2))
        table = torch.randperm(B * per, generator=g, device=dev()).to(torch.int32).reshape(B, per).contiguous()
        q = torch.randn((B, 2 * H, 128), generator=g, device=dev()).to(BF16)
        lens = torch.full((B,), n, dtype=torch.int32, device=dev())
        return lambda stream: lib.mlt_paged_attn_decode_fp8(q, kc, vc, ks, vs, table, lens, 0.1, stream=stream)

    calls = [product(512, 4096, 2048, 1), product(64, 512, 8192, 2), attention(4, 2, 3000, 3), attention(1, 2, 9000, 4), product(130, 2048, 8192, 5), attention(2, 8, 2100, 6)]
    want, names = [], []
    for c in calls:
        want.append(c(None).clone())
        names.append(lib.mlt_last_kernel())
    assert sum("split" in n for n in names) >= 4, names
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        got = [[c(s) for c in (calls if s is sides[0] else calls[::-1])] for s in sides]
        torch.cuda.synchronize()
        for a, b, w in zip(got[0], got[1][::-1], want):
            assert torch.equal(a, w) and torch.equal(b, w)


def test_captured_calls_that_would_split(lib):
    """Captured, nothing is spread over workgroups through scratch: replays between eager calls that are give the same bits each time, and those of the eager
    calls up to the order of the sums."""
    at = [t.to(dev()) for t in gemm_operands(512, 4096, 2048, 11)]
    eager = lib.mlt_gemm_fp8(*at)
    C = torch.empty_like(eager)
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.mlt_gemm_fp8(*at, C=C)
    C2 = torch.empty_like(eager)
    with torch.cuda.graph(other):
        lib.mlt_gemm_fp8(*at, C=C2)
    first = None
    for _ in range(5):
        graph.replay()
        again = lib.mlt_gemm_fp8(*at)
        other.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, eager) and torch.equal(C, C2)
        first = C.clone() if first is None else first
        assert torch.equal(C, first)
        C.zero_()
        C2.zero_()
    gemm_check(first[:64], at[0][:64].cpu(), at[1][:, :64].cpu(), at[2].cpu(), at[3].cpu(), BF16, 2048)


def test_captured_and_replayed(lib):
    """A graph of the layer, replayed with eager work between: every replay gives what the eager layer gives."""
    B = 4
    w, st = layer_setup(lib, B, 97)
    w2, st2 = layer_setup(lib, B, 97)
    Qo, Qo2 = (torch.empty((B, 4, 64), dtype=BF16, device=dev()) for _ in range(2))
    x = torch.zeros((B, 384), dtype=BF16, device=dev())
    layer(lib, w, x, st, Qo)                                # (lengths 0: nothing is appended, attention gives zeros)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st["where"][1].add_(1)
        y = layer(lib, w, x, st, Qo)
    for i in range(25):
        new = rand((B, 384), BF16, 2000 + i).to(dev())
        x.copy_(new)
        graph.replay()
        st2["where"][1] += 1
        want = layer(lib, w2, new, st2, Qo2)
        torch.cuda.synchronize()
        assert torch.equal(st["where"][1], st2["where"][1])
        assert torch.equal(y, want), i
        assert torch.equal(st["Kc"].view(torch.uint8), st2["Kc"].view(torch.uint8)) and torch.equal(st["Vs"], st2["Vs"])


def test_caches_past_4_gib(lib):
    """Blocks whose bytes lie past 2^32 in the cache."""
    H, D, block = 8, 128, 16
    nb = (1 << 32) // (H * D * block) + 70000
    kc = torch.zeros((nb, H, block, D), dtype=torch.uint8, device=dev()).view(F8)
    vc = torch.zeros((nb, H, block, D), dtype=torch.uint8, device=dev()).view(F8)
    ks, vs = torch.ones((nb, H), device=dev()), torch.ones((nb, H), device=dev())
    table = torch.tensor([[nb - 1, 3], [nb - 60000, nb - 2]], dtype=torch.int32, device=dev())
    lens = torch.tensor([20, 30], dtype=torch.int32, device=dev())
    k, v = rand((50, H, D), BF16, 101), rand((50, H, D), BF16, 103)
    off = torch.tensor([0, 20, 50], dtype=torch.int32, device=dev())
    lib.mlt_paged_append_fp8(None, k.to(dev()), v.to(dev()), off, lens, table, None, None, kc, vc, ks, vs)
    q = rand((2, H, D), BF16, 107)
    O = lib.mlt_paged_attn_decode_fp8(q.to(dev()), kc, vc, ks, vs, table, lens, 0.1)
    for b, (t0, t1) in enumerate(((0, 20), (20, 50))):
        rows = table[b].long()
        K64, V64 = (f64(c.view(torch.uint8)[rows].view(F8)) * f64(s[rows])[..., None, None] for c, s in ((kc, ks), (vc, vs)))
        for h in range(H):
            kk, vv = K64[:, h].reshape(-1, D)[:t1 - t0], V64[:, h].reshape(-1, D)[:t1 - t0]
            assert (np.abs(vv - f64(v)[t0:t1, h]) <= u.HALF[F8] * np.abs(f64(v)[t0:t1, h]) + 2.0 ** -6 * 2.0 ** -10).all()
            o, mass, reach = u.attn(f64(q)[b, h], kk, vv, 0.1)
            assert (np.abs(f64(O)[b, h] - o) <= u.attn_tolerance(o, mass, reach, t1 - t0, D, BF16, np.abs(vv).max())).all()


# ---- the binding's native call path

def test_native_and_python_paths_agree(lib, monkeypatch):
    """What the native path takes gives the bits of the step-by-step path; what it does not take (an output to allocate, a stream, a missing Q,
    another type) it leaves to that."""
    w, st = layer_setup(lib, 3, 109)
    x = rand((3, 384), BF16, 113).to(dev())
    f8 = lambda *s: torch.zeros(s, device=dev()).to(F8)  # noqa: E731
    q, s = f8(3, 384), torch.empty((3, 3), device=dev())
    lib.mlt_quant_fp8(x, Xq=q, S=s)
    rows = rand((3, 8, 64), BF16, 127).to(dev())
    st["where"][1] += 1
    wide = torch.empty((3, 400), dtype=BF16, device=dev())
    calls = {"quant_fp8": lambda: lib.mlt_quant_fp8(x, 1, Xq=f8(3, 384), S=torch.empty((3, 3), device=dev())),
             "gemm_fp8": lambda: lib.mlt_gemm_fp8(q, s, *w["in"], C=torch.empty((3, 512), dtype=FP16, device=dev())),
             "paged_append": lambda: lib.mlt_paged_append_fp8(rows[:, :4], rows[:, 4:6], rows[:, 6:], *st["where"], st["cos"], st["sin"], st["Kc"], st["Vc"], st["Ks"], st["Vs"],
                                                              Qo=torch.empty((3, 4, 64), dtype=BF16, device=dev())),
             "paged_attn_decode_fp8": lambda: lib.mlt_paged_attn_decode_fp8(rows[:, :4].contiguous(), st["Kc"], st["Vc"], st["Ks"], st["Vs"], st["where"][2], st["where"][1], 0.1,
                                                                            O=torch.empty((3, 4, 64), dtype=BF16, device=dev()))}
    sixteen = lambda: lib.mlt_paged_append(rows[:, :4], rows[:, 4:6], rows[:, 6:], *st["where"], st["cos"], st["sin"], torch.zeros((18, 2, 16, 64), dtype=BF16, device=dev()),  # noqa: E731
                                           torch.zeros((18, 2, 16, 64), dtype=BF16, device=dev()), Qo=torch.empty((3, 4, 64), dtype=BF16, device=dev()))
    taken = []
    native = {f: getattr(lib._fast, f) for f in calls}

    class Fast:
        def __getattr__(self, f):
            def call(*a):
                r = native[f](*a)
                taken.append(r is not None)
                return r
            return call

    class Off:
        def __getattr__(self, f):
            return lambda *a: None

    todo = list(calls.values()) + [sixteen]
    monkeypatch.setattr(lib, "_fast", Fast())
    got = [c() for c in todo]
    assert taken == [True] * len(todo)
    monkeypatch.setattr(lib, "_fast", Off())
    bits = lambda t: [i.contiguous().view(torch.uint8).clone() for i in (t if isinstance(t, tuple) else (t,))]  # noqa: E731
    for c, g in zip(todo, got):
        assert all(torch.equal(i, j) for i, j in zip(bits(c()), bits(g)))
    side = torch.cuda.Stream()
    z = st["where"]
    for f, args in (("quant_fp8", (x, 1, None, s, None)), ("quant_fp8", (x, 1, q, s, side)), ("quant_fp8", (x, 1.0, q, s, None)), ("quant_fp8", (x.float(), 1, q, s, None)),
                    ("quant_fp8", (x, 128, q, s, None)), ("quant_fp8", (x, 1, q, s.t().contiguous().t(), None)), ("gemm_fp8", (q, s, *w["in"], None, None)),
                    ("gemm_fp8", (q, s, *w["in"], wide, None)), ("gemm_fp8", (x, s, *w["in"], wide, None)), ("gemm_fp8", (q, s.half(), *w["in"], wide, None)),
                    ("paged_append", (None, rows, rows, *z, st["cos"], st["sin"], st["Kc"], st["Vc"], st["Ks"], st["Vs"], None, False, None)),
                    ("paged_append", (rows[:, :4], rows[:, 4:6], rows[:, 6:], z[0].long(), z[1], z[2], st["cos"], st["sin"], st["Kc"], st["Vc"], st["Ks"], st["Vs"], rows[:, :4].clone(), False, None)),
                    ("paged_append", (rows[:, :4], rows[:, 4:6], rows[:, 6:], *z, st["cos"], st["sin"], st["Kc"], st["Vc"], None, None, rows[:, :4].clone(), False, None)),
                    ("paged_attn_decode_fp8", (rows[:, :4], st["Kc"], st["Vc"], st["Ks"], st["Vs"], z[2], z[1], 0.1, rows[:, :4].clone(), None)),
                    ("paged_attn_decode_fp8", (rows, st["Kc"], st["Vc"], st["Ks"], st["Vs"], z[2], z[1], 1, rows.clone(), None))):
        assert native[f](*args) is None, f


def test_binding_refuses_what_does_not_fit(lib):
    w, st = layer_setup(lib, 3, 131)
    x = rand((3, 384), BF16, 137).to(dev())
    q, s = lib.mlt_quant_fp8(x)
    rows = rand((3, 2, 64), BF16, 139).to(dev())
    z, cs = st["where"], (st["cos"], st["sin"])
    cache = (st["Kc"], st["Vc"], st["Ks"], st["Vs"])
    for call in (lambda: lib.mlt_quant_fp8(x, Xq=q[:2]), lambda: lib.mlt_quant_fp8(x, S=s[:2]), lambda: lib.mlt_quant_fp8(x, S=s.double()), lambda: lib.mlt_quant_fp8(x.t()),
                 lambda: lib.mlt_gemm_fp8(q, s[:2], *w["in"]), lambda: lib.mlt_gemm_fp8(q, s, *w["out"]), lambda: lib.mlt_gemm_fp8(q, s, *w["in"], C=x),
                 lambda: lib.mlt_paged_append_fp8(None, rows, rows[:2], *z, *cs, *cache), lambda: lib.mlt_paged_append_fp8(None, rows, rows, z[0][:3], z[1], z[2], *cs, *cache),
                 lambda: lib.mlt_paged_append_fp8(None, rows, rows, *z, cs[0], None, *cache), lambda: lib.mlt_paged_append_fp8(None, rows, rows, *z, *cs, *cache[:2], None, None),
                 lambda: lib.mlt_paged_append_fp8(None, rows, rows, *z, *cs, cache[0], cache[1], cache[2][:3], cache[3]), lambda: lib.mlt_paged_append(None, rows, rows, *z, *cs, *cache[:2]),
                 lambda: lib.mlt_paged_append_fp8(None, rows.transpose(0, 1).contiguous().transpose(0, 1), rows, *z, *cs, *cache),
                 lambda: lib.mlt_paged_append_fp8(None, rows, rows, z[0].long(), z[1], z[2], *cs, *cache), lambda: lib.mlt_paged_append_fp8(None, rows, rows, *z, *cs, *cache, Qo=rows),
                 lambda: lib.mlt_paged_attn_decode_fp8(rows, *cache, z[2], z[1][:2], 0.1), lambda: lib.mlt_paged_attn_decode_fp8(rows[:, :, :32], *cache, z[2], z[1], 0.1),
                 lambda: lib.mlt_paged_attn_decode_fp8(rows, *cache[:2], cache[2].half(), cache[3], z[2], z[1], 0.1)):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(TypeError):
        lib.mlt_gemm_fp8(x, s, *w["in"])
    with pytest.raises(TypeError):
        lib.mlt_paged_attn_decode_fp8(rows, cache[0].float(), cache[1].float(), *cache[2:], z[2], z[1], 0.1)
    with pytest.raises(lib.MltError) as e:
        lib.mlt_paged_attn_decode_fp8(torch.cat([rows, rows[:, :1]], 1), *cache, z[2], z[1], 0.1)        # 3 query heads over 2
    assert e.value.status == lib.MLT_ERR_INVALID_ARG
    with pytest.raises(lib.MltError) as e:
        lib.mlt_paged_append_fp8(None, rows, rows, *z, cs[0][:, :4].contiguous(), cs[1][:, :4].contiguous(), *cache)       # 8 turned elements
    assert e.value.status == lib.MLT_ERR_UNSUPPORTED
    with pytest.raises(lib.MltError) as e:
        lib.mlt_quant_fp8(x, 64, Xq=torch.empty((3, 384), device=dev()).to(F8), S=torch.empty((3, 1), device=dev()))
    assert e.value.status == lib.MLT_ERR_UNSUPPORTED
