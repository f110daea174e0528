"""Decode attention over the 8-bit cache with more than 32 units of 32 keys to a wavefront, which looks the next 32 up (block numbers, scales) while it works on these.
Against 64 bits."""
import math

import pytest
import torch

import fp8_attn_util as a
from test_fp8_debug_gpu import _stream, both, dbg  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16
WEIGHT_HALF = 2.0 ** -22                                                  # the weights in the second product: 11 bits, and 11 of what they leave


@pytest.fixture(autouse=True)
def _announce(request):
    print("\n[case] %s" % request.node.name, flush=True)
    yield


@pytest.fixture(scope="module")
def lib():
    from paper_2503_14985_amd import binding
    return binding


@pytest.fixture
def key_split(lib):
    yield lib.mlt_diag_force_key_split
    lib.mlt_diag_force_key_split(0)


def dev():
    return torch.device("cuda:0")


def run(lib, c):
    return lib.mlt_paged_attn_decode_fp8(c["q"], c["kc"], c["vc"], c["ks"], c["vs"], c["table"], c["lens"], c["scale"])


def check(lib, c):
    O = run(lib, c)
    o, more = a.exact(**c)
    n, D = int(c["lens"].max()), o.shape[2]
    tol = a.tolerance(o, more, n, D, O.dtype, n // 128, WEIGHT_HALF)      # (units a wavefront, at most)
    err = (O.double() - o).abs()
    print("   kernel=%s worst %.2f of the tolerance" % (lib.mlt_last_kernel(), float((err / tol).max())), flush=True)
    assert bool(torch.isfinite(O.float()).all()) and bool((err <= tol).all()), float((err / tol).max())
    return O


def long_case(B, lens, Hq, H, D, block, dtype, seed):
    """Sequences over shuffled blocks; NaN in every slot and scale that no key has, and in the table numbers far outside."""
    g = torch.Generator(device=dev())
    g.manual_seed(seed)
    per = -(-max(lens) // block)
    nb = B * per + 3
    table = torch.randperm(nb, generator=g, device=dev())[:B * per].to(torch.int32).reshape(B, per).contiguous()
    kc, vc = (torch.randn((nb, H, block, D), generator=g, device=dev(), dtype=BF16).mul_(60).to(a.F8) for _ in range(2))
    ks, vs = (torch.exp2(torch.rand((nb, H), generator=g, device=dev()) * 3 - 8) for _ in range(2))
    used = torch.zeros((nb, block), dtype=torch.bool, device=dev())
    for b, n in enumerate(lens):
        p = torch.arange(n, device=dev())
        used[table[b, p // block].long(), p % block] = True
        table[b, -(-n // block):] = 1 << 20
    for c in (kc, vc):
        c.view(torch.uint8).masked_fill_(~used[:, None, :, None], 0x7F)
    for s in (ks, vs):
        s[~used.any(1)] = float("nan")
    q = torch.randn((B, Hq, D), generator=g, device=dev()).to(dtype)
    return dict(q=q, kc=kc, vc=vc, ks=ks, vs=vs, table=table, lens=torch.tensor(lens, dtype=torch.int32, device=dev()), scale=1.0 / math.sqrt(D))


LONG = [  # lengths, query heads, heads, D, block, split
    ([8192, 8193, 0, 8447, 8448, 8449, 1], 4, 2, 128, 16, 1),             # 32 units a wavefront, and one key more; the last of 33
    ([20000, 16384, 16385, 777], 2, 2, 64, 16, 1), ([33000], 8, 1, 128, 48, 1), ([24999, 50], 4, 2, 64, 1024, 1), ([49999], 2, 1, 128, 32, 2)]


@pytest.mark.parametrize("lens,Hq,H,D,block,split", LONG)
def test_more_than_32_units_a_wavefront(lib, key_split, lens, Hq, H, D, block, split):
    key_split(split)
    for dtype in (BF16, FP16):
        c = long_case(len(lens), lens, Hq, H, D, block, dtype, sum(lens))
        O = check(lib, c)
        for _ in range(2):
            assert torch.equal(run(lib, c), O)


def test_more_than_32_units_with_four_wavefronts(lib, key_split):
    key_split(1)
    lens = [9000 - 500 * i for i in range(9)]
    c = long_case(9, lens, 60, 60, 64, 16, BF16, 11)
    check(lib, c)
    assert lib.mlt_last_kernel() == "paged_decode_fp8_d64_w4"


def test_captured_long_sequence(lib):
    """While a stream records nothing is spread over workgroups: a sequence that is split otherwise goes through one workgroup a head."""
    c = long_case(1, [30000], 8, 2, 128, 16, BF16, 13)
    eager = run(lib, c)
    assert "keysplit" in lib.mlt_last_kernel()
    O = torch.empty_like(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.mlt_paged_attn_decode_fp8(c["q"], c["kc"], c["vc"], c["ks"], c["vs"], c["table"], c["lens"], c["scale"], O=O)
    assert "keysplit" not in lib.mlt_last_kernel()
    o, more = a.exact(**c)
    tol = a.tolerance(o, more, 30000, 128, BF16, 30000 // 128, WEIGHT_HALF)
    for _ in range(3):
        O.zero_()
        graph.replay()
        again = run(lib, c)
        torch.cuda.synchronize()
        assert torch.equal(again, eager) and bool(((O.double() - o).abs() <= tol).all())


@pytest.mark.parametrize("lens,Hq,H,D,block,split", LONG + [([9000 - 500 * i for i in range(9)], 60, 60, 64, 16, 1)])
def test_long_sequences_agree_with_the_debug_build(dbg, both, lens, Hq, H, D, block, split):  # noqa: F811
    """The loads that look the next 32 units up stand in the counted stream of the others: the same bits where every wait is one for all of them."""
    from paper_2503_14985_amd import binding
    both(split=split)
    for dtype, code in ((BF16, 0), (FP16, 1)):
        c = long_case(len(lens), lens, Hq, H, D, block, dtype, sum(lens) + 1)
        want = run(binding, c)
        name = binding.mlt_last_kernel()
        at = [c[x].data_ptr() for x in ("q", "kc", "vc", "ks", "vs", "table", "lens")]
        for _ in range(3):                                                # a race need not strike on the first launch
            got = torch.full_like(want, float("nan"))
            assert dbg.mlt_paged_attn_decode_fp8(len(lens), Hq, H, D, block, c["table"].shape[1], c["kc"].shape[0], *at, got.data_ptr(), c["scale"], code, _stream()) == 0
            assert dbg.mlt_last_kernel().decode() == name
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)), name


def mixed(B, s):
    """Lengths from s / 4 to s out of order, with empty sequences, single keys and equal lengths among them."""
    lens = [s // 4 + (s - s // 4) * i // (B - 1) for i in range(B)]
    lens = [lens[37 * i % B] if B % 37 else lens[i] for i in range(B)]
    lens[3], lens[B // 2], lens[5] = 0, 1, lens[6]
    return lens


@pytest.mark.parametrize("B,s,Hq,H,D,block", [(70, 4100, 16, 8, 128, 16), (70, 8192, 8, 8, 64, 32), (128, 1100, 8, 8, 128, 16), (250, 4096, 4, 4, 64, 64), (256, 2100, 3, 3, 128, 16),
                                              (300, 4097, 1, 1, 128, 16), (512, 8200, 1, 1, 64, 128)])
def test_large_mixed_batches_dealt_by_length(lib, dbg, both, B, s, Hq, H, D, block):  # noqa: F811
    """More sequences than a wavefront has lanes (up to one for each thread of a workgroup), the longest with more than 32 units to a wavefront; and the debug build's bits."""
    lens = mixed(B, s)
    c = long_case(B, lens, Hq, H, D, block, BF16, B + s)
    O = check(lib, c)
    assert bool((O[3] == 0).all())
    both(split=1)
    want = run(lib, c)
    at = [c[x].data_ptr() for x in ("q", "kc", "vc", "ks", "vs", "table", "lens")]
    for _ in range(2):
        got = torch.full_like(O, float("nan"))
        assert dbg.mlt_paged_attn_decode_fp8(B, Hq, H, D, block, c["table"].shape[1], c["kc"].shape[0], *at, got.data_ptr(), c["scale"], 0, _stream()) == 0
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
