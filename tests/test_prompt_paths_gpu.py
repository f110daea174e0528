"""The operators for prompts, shared prefixes and 4-bit weights on the paths around their kernels: the binding's native call path, streams with pending work, two streams at once, captured
graphs that are replayed among other work, the debug build, and tensors beyond 4 GiB."""
import ctypes
import math
import os

import pytest
import torch

from prompt_util import HALF, attend, cache_of, check, check_packed, ends, ints, normal, rows_of, tolerance, w4_exact, w4_inputs, w4_tolerance

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DBG = os.path.join(ROOT, "paper_2503_14985_amd", "libmlt_dbg.so")


@pytest.fixture(autouse=True)
def _announce(request):
    print("\n[case] %s" % request.node.name, flush=True)
    yield


@pytest.fixture(scope="module")
def lib():
    from paper_2503_14985_amd import binding
    return binding


def cases(lib, seed=0, dtype=BF):
    """name -> (inputs, call(inputs, O, stream, work) -> O, shape of O). Splits of every kind among them."""
    out = {}
    D, H, Hq, block = 128, 2, 8, 32
    for name, batch in (("packed", [(65, 65), (1, 1), (130, 300)]), ("packed, keys split", [(20, 3000)])):
        cu, ku = ends([n for n, _ in batch]), ends([m for _, m in batch])
        t = [normal(seed + 1, (cu[-1], Hq, D), dtype), normal(seed + 2, (ku[-1], H, D), dtype), normal(seed + 3, (ku[-1], H, D), dtype), ints(cu), ints(ku)]
        out[name] = (t, lambda t, O, st, work: lib.mlt_mha_packed_fwd(*t, 0.1, O=O, stream=st), t[0].shape)
    for name, lens, new in (("prompt", [90, 33, 200], [40, 33, 7]), ("prompt, keys split", [2500], [30])):
        Kc, Vc, table = cache_of(seed + 4, lens, H, D, block, dtype)
        t = [normal(seed + 5, (sum(new), Hq, D), dtype), Kc, Vc, ints(ends(new)), ints(lens), table]
        out[name] = (t, lambda t, O, st, work: lib.mlt_paged_attn_prompt(*t, 0.1, O=O, stream=st), t[0].shape)
    for name, B, P, own in (("prefix, few", 3, 5700, 90), ("prefix, many", 70, 8500, 30), ("prefix, alone", 12, 500, 200), ("prefix, none", 4, 0, 1200)):
        lens = [P + own - b * own // 100 for b in range(B)]
        Kc, Vc, table = cache_of(seed + 6, lens, H, D, block, dtype)
        t = [normal(seed + 7, (B, Hq, D), dtype), Kc, Vc, table[0].contiguous(), table, ints(lens)]
        out[name] = (t, lambda t, O, st, work, P=P: lib.mlt_paged_attn_decode_prefix(t[0], t[1], t[2], t[3], P, t[4], t[5], 0.1, O=O, work=work, stream=st), t[0].shape)
    for name, M, N, K, group, zeros in (("4 bits, one row", 1, 500, 2048, 128, False), ("4 bits, rows, K in parts", 24, 512, 8192, 32, True), ("4 bits, tiles, K in parts", 57, 900, 4096, 64, True),
                                        ("4 bits, tiles", 100, 8200, 512, 128, False), ("4 bits, nothing to add", 3, 70, 0, 128, False)):
        A, Wq, S, Z, _ = w4_inputs(seed + 8, M, N, K, group, zeros, dtype) if K else [torch.zeros(s, dtype=d, device="cuda") for s, d in
                                                                                     (((M, 0), dtype), ((N, 0), torch.uint8), ((0, N), dtype))] + [None, None]
        t = [A, Wq, S] + ([Z] if zeros else [])
        out[name] = (t, lambda t, O, st, work, group=group: lib.mlt_gemm_w4(*t, group=group, C=O, stream=st), (M, N))
    return out


def run(case, dtype=BF, inputs=None, stream=None, work=None):
    t, call, shape = case
    O = torch.full(shape, 7.0, dtype=dtype, device="cuda")
    call(t if inputs is None else inputs, O, stream, work)
    return O


def test_native_and_python_paths_agree(lib, monkeypatch):
    names = ("mha_packed_fwd", "paged_attn_prompt", "paged_attn_decode_prefix", "gemm_w4")
    native, taken = {f: getattr(lib._fast, f) for f in names}, []

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

    for dtype in (BF, FP):
        everything = cases(lib, dtype=dtype)
        taken.clear()
        monkeypatch.setattr(lib, "_fast", Fast())
        got = {n: run(c, dtype) for n, c in everything.items()}
        assert taken == [True] * len(everything), dict(zip(everything, taken))
        monkeypatch.setattr(lib, "_fast", Off())
        for n, c in everything.items():
            assert torch.equal(run(c, dtype).view(torch.int16), got[n].view(torch.int16)), n
            t, call, shape = c
            O = call(t, None, None, None)                            # allocated by the call
            assert O.dtype == dtype and torch.equal(O.view(torch.int16), got[n].view(torch.int16)), n


@pytest.mark.parametrize("explicit", [True, False])
def test_calls_are_ordered_behind_the_streams_work(lib, explicit):
    side = torch.cuda.Stream()
    for name, case in cases(lib).items():
        print("[case] %s, %s" % (name, "stream given" if explicit else "current stream"), flush=True)
        late = case[0]
        want, kernel = run(case), lib.mlt_last_kernel()
        ready = [t.clone() for t in late]
        O = torch.full(case[2], 7.0, dtype=BF, device="cuda")
        before = [t.clone() for t in late] + [O.clone()]
        torch.cuda.synchronize()
        case[1](before[:-1], before[-1], side, None)                  # (its kernels and scratch are there: what follows does not wait for them)
        for t in late:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)
            for t, r in zip(late, ready):
                t.copy_(r, non_blocking=True)
            if not explicit:
                case[1](late, O, None, None)
        if explicit:
            case[1](late, O, side, None)
        pending = not side.query()
        side.synchronize()
        assert pending, "the stream was done before the call was made"
        assert lib.mlt_last_kernel() == kernel
        assert torch.equal(O.view(torch.int16), want.view(torch.int16)), name


def test_two_streams_at_once(lib):
    """Calls on two streams at a time, each with other inputs: partial results and counters of one are not the other's."""
    ones, others = cases(lib, 0), cases(lib, 50)
    for name in ones:
        a, b = ones[name], others[name]
        want = [run(c) for c in (a, b)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        outs = [[torch.full(c[2], 7.0, dtype=BF, device="cuda") for _ in range(20)] for c in (a, b)]
        torch.cuda.synchronize()
        for i in range(20):
            for c, s, o in zip((a, b), streams, outs):
                c[1](c[0], o[i], s, None)
        torch.cuda.synchronize()
        for w, o in zip(want, outs):
            for x in o:
                assert torch.equal(x.view(torch.int16), w.view(torch.int16)), name


def verify(name, t, O):
    """Against the definition in 64 bits."""
    if name.startswith("packed"):
        check_packed(O, t[0], t[1], t[2], t[3].tolist(), t[4].tolist(), 0.1, True, what=name)
    elif name.startswith("prompt"):
        cu, lens, block = t[3].tolist(), t[4].tolist(), t[1].shape[2]
        for b, m in enumerate(lens):
            K, V = (rows_of(c, t[5][b, :-(-m // block)], m) for c in t[1:3])
            check_packed(O[cu[b]:cu[b + 1]], t[0][cu[b]:cu[b + 1]], K, V, [0, cu[b + 1] - cu[b]], [0, m], 0.1, True, what=name)
    elif name.startswith("prefix"):
        P, block = {"few": 5700, "many": 8500, "alone": 500, "none": 0}[name.split()[1]], t[1].shape[2]
        for b, m in enumerate(t[5].tolist()):
            j = torch.arange(m, device="cuda")
            blk = torch.where(j < P, t[3][j // block], t[4][b][j // block]).long()
            K, V = (c[blk, :, j % block] for c in t[1:3])
            o, c = attend(t[0][b:b + 1], K, V, 0.1, [m])
            check(O[b:b + 1], o, tolerance(o, c, O.shape[2], O.dtype, HALF[O.dtype], moves=m // 32 + 40), name)
    elif t[0].shape[1]:
        group = {"one row": 128, "rows, K in parts": 32, "tiles, K in parts": 64, "tiles": 128}[name[len("4 bits, "):]]
        q = torch.stack([t[1] & 15, t[1] >> 4], -1).flatten(1)
        c, size = w4_exact(t[0], q, t[2], t[3] if len(t) > 3 else None, group)
        check(O, c, w4_tolerance(c, size, t[0].shape[1], group, O.dtype), name)
    else:
        assert bool((O == 0).all())


@pytest.mark.parametrize("with_work", [False, True], ids=["no_work", "work"])
def test_captured_and_replayed(lib, with_work):
    """Each call recorded into a graph of its own, replayed several times among eager calls of the same and other inputs on the same and another stream."""
    stream, others = torch.cuda.Stream(), cases(lib, 70)
    for name, case in cases(lib).items():
        if with_work and name not in ("prefix, few", "prefix, many"):
            continue
        t, call, shape = case
        other = others[name]
        works = None
        if with_work:
            B, Hq, D = t[0].shape
            P = 5700 if "few" in name else 8500
            need = lib.mlt_paged_attn_decode_prefix_work(B, Hq, t[1].shape[1], D, t[1].shape[2], t[4].shape[1], P)
            assert need > 0
            works = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
        ref = run(case)
        alt = run(other)
        inputs = [x.clone() for x in t]
        outs = [torch.zeros(shape, dtype=BF, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            call(inputs, outs[0], None, works[0] if works else None)  # warm: the stream has its scratch
        torch.cuda.synchronize()
        graphs = []
        for i in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call(inputs, outs[i], None, works[i] if works else None)
            graphs.append(g)
        side = torch.cuda.Stream()
        first = None
        for turn in range(4):
            for x, src in zip(inputs, t if turn % 2 == 0 else other[0]):
                x.copy_(src)
            for o in outs:
                o.fill_(3.0)
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                graphs[0].replay()
            with torch.cuda.stream(stream):
                graphs[1].replay()
                eager = run(case, stream=None)                       # on the stream whose scratch the graphs must not have
            torch.cuda.synchronize()
            assert torch.equal(eager.view(torch.int16), ref.view(torch.int16)), name
            want = ref if turn % 2 == 0 else alt
            for o in outs:
                if with_work:
                    assert torch.equal(o.view(torch.int16), want.view(torch.int16)), (name, turn)
                else:                                                # (nothing is split under capture: other orders of the same sums)
                    verify(name, inputs, o)
            assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16)), name
            if turn == 0:
                first = outs[0].clone()
            if turn == 2:
                assert torch.equal(first.view(torch.int16), outs[0].view(torch.int16)), name


def test_the_debug_build_agrees(lib):
    """libmlt_dbg.so waits for all loads and takes pipeline barriers twice: equal bits, or a tile was read before it had landed."""
    if not os.path.exists(DBG):
        pytest.skip("libmlt_dbg.so is not built (python -c 'import __graft_entry__ as g; g.build_debug_lib()')")
    dbg = ctypes.CDLL(DBG)
    dbg.mlt_last_kernel.restype = ctypes.c_char_p
    for f in ("mlt_mha_packed_fwd", "mlt_paged_attn_prompt", "mlt_paged_attn_decode_prefix", "mlt_gemm_w4"):
        getattr(dbg, f).argtypes = getattr(lib.raw(), f).argtypes
    p = lambda x: None if x is None else x.data_ptr()  # noqa: E731
    st = lambda: ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)  # noqa: E731
    for D in (64, 128):
        for dtype, code in ((BF, 0), (FP, 1)):
            Hq, H, block = 8, 2, 16
            for batch in ([(65, 65), (300, 300), (1, 700), (513, 900)], [(30, 5000)]):
                cu, ku = ends([n for n, _ in batch]), ends([m for _, m in batch])
                Q, K, V = normal(1, (cu[-1], Hq, D), dtype), normal(2, (ku[-1], H, D), dtype), normal(3, (ku[-1], H, D), dtype)
                for causal in (True, False):
                    want = lib.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), 0.1, causal=causal)
                    name, a, b = lib.mlt_last_kernel(), ints(cu), ints(ku)
                    for _ in range(3):
                        O = torch.full_like(want, math.nan)
                        assert dbg.mlt_mha_packed_fwd(cu[-1], ku[-1], len(batch), Hq, H, D, p(Q), Hq * D, p(K), H * D, p(V), H * D, p(a), p(b), p(O), Hq * D, 0.1, int(causal), code, st()) == 0
                        assert dbg.mlt_last_kernel().decode() == name and torch.equal(O.view(torch.int16), want.view(torch.int16)), name
                lens = [m for _, m in batch]
                Kc, Vc, table = cache_of(5, lens, H, D, block, dtype)
                want = lib.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), table, 0.1)
                name, n = lib.mlt_last_kernel(), ints(lens)
                for _ in range(3):
                    O = torch.full_like(want, math.nan)
                    assert dbg.mlt_paged_attn_prompt(cu[-1], len(batch), Hq, H, D, block, table.shape[1], Kc.shape[0], p(Q), Hq * D, p(Kc), p(Vc), p(a), p(n), p(table), p(O), Hq * D, 0.1, code, st()) == 0
                    assert dbg.mlt_last_kernel().decode() == name and torch.equal(O.view(torch.int16), want.view(torch.int16)), name
            for B, P, own in ((3, 6000, 300), (6, 5777, 90), (70, 9000, 20), (20, 500, 260), (5, 0, 900), (2, 0, 9000)):
                lens = [P + own - b * own // 100 for b in range(B)]
                Kc, Vc, table = cache_of(6, lens, H, D, block, dtype)
                Q, n, pre = normal(7, (B, Hq, D), dtype), ints(lens), table[0].contiguous()
                want = lib.mlt_paged_attn_decode_prefix(Q, Kc, Vc, pre, P, table, n, 0.1)
                name = lib.mlt_last_kernel()
                for _ in range(3):
                    O = torch.full_like(want, math.nan)
                    assert dbg.mlt_paged_attn_decode_prefix(B, Hq, H, D, block, table.shape[1], Kc.shape[0], p(Q), p(Kc), p(Vc), p(pre), P, p(table), p(n), p(O), 0.1, None, 0, code, st()) == 0
                    assert dbg.mlt_last_kernel().decode() == name and torch.equal(O.view(torch.int16), want.view(torch.int16)), name
    for dtype, code in ((BF, 0), (FP, 1)):
        for M, N, K in ((1, 1000, 4096), (16, 4100, 1056), (30, 700, 8192), (57, 1030, 4128), (128, 8200, 1024)):
            for group in (32, 64, 128):
                for zeros in (False, True):
                    A, Wq, S, Z, _ = w4_inputs(M, M, N, K, group, zeros, dtype)
                    want = lib.mlt_gemm_w4(A, Wq, S, Z, group=group)
                    name = lib.mlt_last_kernel()
                    for _ in range(2):
                        C = torch.full_like(want, math.nan)
                        assert dbg.mlt_gemm_w4(M, N, K, p(A), K, p(Wq), K // 2, group, p(S), N, p(Z), N, p(C), N, code, st()) == 0
                        assert dbg.mlt_last_kernel().decode() == name and torch.equal(C.view(torch.int16), want.view(torch.int16)), (name, M, N, K)


def _large(shape, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for i in range(0, shape[0], 4096):
        out[i:i + 4096] = torch.randn((min(4096, shape[0] - i),) + tuple(shape[1:]), generator=g, device="cuda", dtype=torch.float32).to(dtype)
    return out


def test_a_cache_beyond_4_gib(lib):
    nb, H, block, D, Hq = 70000, 16, 16, 128, 32                     # K and V caches of 4.6 GB each
    assert nb * H * block * D * 2 > 1 << 32
    Kc, Vc = (_large((nb, H, block, D), s, BF) for s in (1, 2))
    g = torch.Generator().manual_seed(3)
    place = torch.randperm(nb, generator=g).to(torch.int32).cuda()
    place[0], place[1] = nb - 1, 0
    lens, new = [900, 333, 5000], [100, 333, 9]
    table = torch.zeros((3, 320), dtype=torch.int32, device="cuda")
    for b in range(3):
        table[b] = place[b * 320:(b + 1) * 320]
    cu = ends(new)
    Q = normal(4, (cu[-1], Hq, D), BF)
    O = lib.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), table, 0.1)
    for b, m in enumerate(lens):
        K, V = (rows_of(c, table[b, :-(-m // block)], m) for c in (Kc, Vc))
        check_packed(O[cu[b]:cu[b + 1]], Q[cu[b]:cu[b + 1]], K, V, [0, new[b]], [0, m], 0.1, True, what="prompt %d" % b)
    P = 777
    for B in (2, 20):
        lens = [P + 400 - 11 * b for b in range(B)]
        own = place[1000:1000 + B * 74].reshape(B, 74).contiguous()
        prefix = place[:49].contiguous()
        Qd = normal(5, (B, Hq, D), BF)
        O = lib.mlt_paged_attn_decode_prefix(Qd, Kc, Vc, prefix, P, own, ints(lens), 0.1)
        for b in (0, B - 1):
            j = torch.arange(lens[b], device="cuda")
            blk = torch.where(j < P, torch.nn.functional.pad(prefix, (0, 74))[j // block], own[b][j // block]).long()
            K, V = (c[blk, :, j % block] for c in (Kc, Vc))
            o, c = attend(Qd[b:b + 1], K, V, 0.1, [lens[b]])
            check(O[b:b + 1], o, tolerance(o, c, D, BF, HALF[BF], moves=lens[b] // 32 + 40), "prefix %d of %d" % (b, B))
    del Kc, Vc
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M", [2, 40])
def test_weights_beyond_4_gib(lib, M):
    N, K, group = 1 << 19, 1 << 14, 128                              # 4.3 GB of weights
    Wq = torch.empty((N, K // 2), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(0, N, 1 << 16):
        Wq[i:i + (1 << 16)] = torch.randint(0, 256, (1 << 16, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    S = (torch.rand((K // group, N), generator=g, device="cuda") * 0.02 + 0.002).to(BF)
    A = normal(2, (M, K), BF)
    C = lib.mlt_gemm_w4(A, Wq, S, group=group)
    for cols in (slice(0, 40), slice(N // 2 - 20, N // 2 + 20), slice(N - 40, N)):
        w = Wq[cols]
        q = torch.stack([w & 15, w >> 4], -1).flatten(1)
        c, t = w4_exact(A, q, S[:, cols], None, group)
        check(C[:, cols], c, w4_tolerance(c, t, K, group, BF), "columns %s" % cols)
    del Wq, S, C
    torch.cuda.empty_cache()
