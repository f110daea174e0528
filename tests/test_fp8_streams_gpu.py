"""The 8-bit operators on a stream that still has the work in front of it that makes their inputs: the stream given to the call, and the current one. Nothing waits in
between, so a call that went to another stream would read what was there before."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def lib():
    from paper_2503_14985_amd import binding
    return binding


def dev():
    return torch.device("cuda:0")


def cases(lib):
    """name -> (inputs that are produced late, with what is there before; call(inputs, stream) -> outputs)"""
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g).to(dev())  # noqa: E731
    out = {}
    x = r(40, 512).to(BF16)
    xq, s = torch.empty((40, 512), dtype=F8, device=dev()), torch.empty((4, 40), device=dev())
    out["quant"] = ([x], lambda t, st: lib.mlt_quant_fp8(t[0], 1, Xq=xq, S=s, stream=st))
    wq, ws = torch.empty((40, 512), dtype=F8, device=dev()), torch.empty((4, 1), device=dev())
    out["quant of a weight"] = ([x], lambda t, st: lib.mlt_quant_fp8(t[0], 128, Xq=wq, S=ws, stream=st))
    for name, M, N, K in (("product, few rows", 16, 512, 1024), ("product, few rows, K in parts", 64, 512, 8192), ("product, tiles", 512, 1024, 1024), ("product, tiles, K in parts", 512, 4096, 2048),
                          ("product, nothing to add", 5, 7, 0)):
        kb = K // 128
        at = [r(M, K).to(F8), r(kb, M).abs(), r(N, K).to(F8), r(kb, -(-N // 128)).abs()]
        C = torch.empty((M, N), dtype=BF16, device=dev())
        out[name] = (at if K else [C], (lambda C: lambda t, st: lib.mlt_gemm_fp8(*t, C=C, stream=st))(C) if K else
                     (lambda C, at: lambda t, st: lib.mlt_gemm_fp8(*at, C=C, stream=st))(C, at))
    B, Hq, H, D, block = 3, 4, 2, 128, 16
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev())  # noqa: E731
    for name, fp8, new in (("append", False, [1, 20, 3]), ("append, 8 bits", True, [1, 20, 3]), ("append, 8 bits, single tokens", True, [1, 1, 1])):
        T = sum(new)
        rows = r(T, Hq + 2 * H, D).to(BF16)
        cum = [sum(new[:i]) for i in range(4)]
        angle = r(64, D // 2)
        kc, vc = (r(12, H, block, D).to(F8 if fp8 else BF16) for _ in range(2))
        ks, vs = (r(12, H).abs() + 0.01 for _ in range(2))
        table, Qo = i32([[0, 5, 2, 9], [11, 1, 3, 4], [6, 7, 8, 10]]), torch.empty((T, Hq, D), dtype=BF16, device=dev())
        late = [rows, i32(cum), i32([n + 9 for n in new]), angle.cos(), angle.sin(), kc, vc] + ([ks, vs] if fp8 else [])

        def call(t, st, fp8=fp8, table=table, Qo=Qo):
            q, k, v = t[0][:, :4], t[0][:, 4:6], t[0][:, 6:]
            if fp8:
                lib.mlt_paged_append_fp8(q, k, v, t[1], t[2], table, *t[3:], Qo=Qo, stream=st)
            else:
                lib.mlt_paged_append(q, k, v, t[1], t[2], table, *t[3:], Qo=Qo, stream=st)
            return [Qo] + t[5:]
        out[name] = (late, call)
    for name, B, n in (("attention", 3, 200), ("attention, keys in ranges", 2, 3000), ("attention, keys in many ranges", 1, 9000)):
        per = -(-n // 16)
        kc, vc = (r(B * per, H, 16, D).to(F8) for _ in range(2))
        ks, vs = (r(B * per, H).abs() + 0.01 for _ in range(2))
        table = torch.randperm(B * per, generator=g).to(torch.int32).reshape(B, per).to(dev())
        O = torch.empty((B, Hq, D), dtype=BF16, device=dev())
        out[name] = ([r(B, Hq, D).to(BF16), kc, vc, ks, vs, table, i32([n - 3 * b for b in range(B)])],
                     lambda t, st, O=O: lib.mlt_paged_attn_decode_fp8(*t, 1.0 / math.sqrt(D), O=O, stream=st))
    return out


def bits(t):
    return [x.contiguous().view(torch.uint8).clone() for x in (t if isinstance(t, (list, tuple)) else (t,))]


@pytest.mark.parametrize("explicit", [True, False])
def test_calls_are_ordered_behind_the_streams_work(lib, explicit):
    side = torch.cuda.Stream()
    for name, (late, call) in cases(lib).items():
        print("\n[case] %s, %s" % (name, "stream given" if explicit else "current stream"), flush=True)
        ready = [t.clone() for t in late]                                 # what the inputs hold in time
        want = bits(call([t.clone() for t in late], None))
        kernel = lib.mlt_last_kernel()
        before = [torch.zeros_like(t) for t in late]
        for t in late:
            t.zero_()
        stale = bits(call(before, None))
        call([t.clone() for t in ready], side)                            # (its kernels and scratch are there: what follows does not wait for them)
        for t in late:
            t.zero_()
        torch.cuda.synchronize()
        assert lib.mlt_last_kernel() == kernel
        if name != "product, nothing to add":
            assert any(not torch.equal(a, b) for a, b in zip(want, stale)), name
        with torch.cuda.stream(side):
            torch.cuda._sleep(200_000_000)
            for t, r in zip(late, ready):
                t.copy_(r, non_blocking=True)
            if not explicit:
                got = call(late, None)
        if explicit:
            got = call(late, side)
        pending = not side.query()
        side.synchronize()
        assert pending, "the stream was done before the call was made"
        assert lib.mlt_last_kernel() == kernel
        for a, b in zip(bits(got), want):
            assert torch.equal(a, b), name
