"""Single-token attention behind a shared prefix against its definition in 64 bits: prefixes that end anywhere in a block, own keys from none to many, grouped heads,
sequences that end inside the prefix, work memory of the caller's."""
import math

import pytest
import torch

from prompt_util import HALF, attend, check, ints, normal, tolerance

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding as b
    return b


def make(seed, P, lens, H, D, block, dtype, poison=True):
    """A cache, the prefix's blocks and the sequences' table: the prefix's whole blocks are named by every row, its last keys are in each sequence's own block too."""
    g = torch.Generator().manual_seed(seed)
    shared, first = -(-P // block), P // block
    own = [max(0, -(-n // block) - first) for n in lens]
    nb = shared + sum(own) + 2
    place = torch.randperm(nb, generator=g).to(torch.int32)
    table = torch.full((len(lens), max([1, shared] + [first + x for x in own])), -9, dtype=torch.int32)
    at = shared
    for b, x in enumerate(own):
        table[b, first:first + x] = place[at:at + x]                 # (entries of the prefix's blocks are not read: -9)
        at += x
    Kc, Vc = (torch.randn((nb, H, block, D), generator=g).to(dtype) for _ in range(2))
    prefix = place[:shared].clone()
    if poison:                                                       # what nobody reads
        used = torch.zeros((nb, block), dtype=torch.bool)
        for j in range(P):
            used[prefix[j // block].long(), j % block] = True
        for b, n in enumerate(lens):
            for j in range(P, n):
                used[table[b, j // block].long(), j % block] = True
        for c in (Kc, Vc):
            c.transpose(1, 2)[~used] = math.nan
    return [x.cuda() for x in (Kc, Vc, prefix, table)]


def expect(Q, Kc, Vc, prefix, P, table, lens, scale):
    block = Kc.shape[2]
    for b, n in enumerate(lens):
        j = torch.arange(n, device=Q.device)
        blk = torch.where(j < P, torch.nn.functional.pad(prefix, (0, table.shape[1]))[j // block], table[b][j // block]).long()
        K, V = (c[blk, :, j % block] for c in (Kc, Vc))
        yield b, attend(Q[b:b + 1], K, V, scale, [n])


def verify(O, Q, Kc, Vc, prefix, P, table, lens, scale, what=""):
    for b, (o, c) in expect(Q, Kc, Vc, prefix, P, table, lens, scale):
        check(O[b:b + 1], o, tolerance(o, c, Q.shape[2], Q.dtype, HALF[Q.dtype], moves=lens[b] // 16 + 8), "%s sequence %d" % (what, b))


CASES = [
    # prefix, lengths, query and key/value heads, block
    (0, [1, 5, 0, 40], (8, 2), 16),
    (16, [17, 16, 30, 15], (4, 4), 16),
    (100, [100, 101, 0, 3, 150, 260], (8, 2), 16),
    (500, [513, 600, 500, 499], (6, 2), 48),
    (1024, [1500, 1025], (16, 1), 128),
    (2049, [2050 + 3 * i for i in range(9)], (8, 2), 64),
    (777, [800], (40, 1), 32),
    (640, [641 + i for i in range(70)], (4, 2), 32),
    (33, [34, 2000, 33, 700], (3, 3), 1024),
]


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_prefix(binding, case, D, dtype):
    P, lens, (Hq, H), block = CASES[case]
    Kc, Vc, prefix, table = make(case, P, lens, H, D, block, dtype)
    Q, scale = normal(case + 50, (len(lens), Hq, D), dtype), 1.0 / math.sqrt(D)
    O = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), scale)
    verify(O, Q, Kc, Vc, prefix, P, table, lens, scale, binding.mlt_last_kernel())
    for b, n in enumerate(lens):
        if n == 0:
            assert bool((O[b] == 0).all())
    assert torch.equal(O, binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), scale))


@pytest.mark.parametrize("case", [2, 5, 7])
def test_work_of_the_caller(binding, case):
    """The caller's work memory gives the bits of the library's own; too little of it still a right result."""
    P, lens, (Hq, H), block = CASES[case]
    D = 128
    Kc, Vc, prefix, table = make(case, P, lens, H, D, block, BF)
    Q = normal(3, (len(lens), Hq, D), BF)
    own = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), 0.1)
    need = binding.mlt_paged_attn_decode_prefix_work(len(lens), Hq, H, D, block, table.shape[1], P)
    work = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    O = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), 0.1, work=work[:need])
    assert torch.equal(O, own) and bool((work[need:] == 255).all())
    if need:
        O = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), 0.1, work=work[:need - 16])
        verify(O, Q, Kc, Vc, prefix, P, table, lens, 0.1)


def test_bad_tables(binding):
    P, lens, (Hq, H), block = CASES[2]
    Kc, Vc, prefix, table = make(2, P, lens, H, 64, block, BF, poison=False)
    Q = normal(3, (len(lens), Hq, 64), BF)
    good = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), 0.1)
    bad = table.clone()
    bad[5, 8:10] = torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    odd = list(lens)
    odd[2], odd[4] = -3, 2 ** 31 - 1
    O = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, bad, ints(odd), 0.1)
    for b in (0, 1, 2, 3):
        assert torch.equal(O[b], good[b]), b


@pytest.mark.parametrize("scale", [0.0, -0.1, 2.0])
def test_scales(binding, scale):
    P, lens, (Hq, H), block = CASES[3]
    Kc, Vc, prefix, table = make(2, P, lens, H, 128, block, FP)
    Q = normal(3, (len(lens), Hq, 128), FP)
    O = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), scale)
    verify(O, Q, Kc, Vc, prefix, P, table, lens, scale)


SHARED = {
    # long enough to be read once for all: up to 16 queries of a key head, up to 32, more
    "16": (6001, [6001, 6040, 0], (8, 2), 32),
    "32": (5008, [5008 + 30 * i for i in range(5)] + [77, 5100], (8, 2), 16),
    "256": (9003, [9003 + i % 50 for i in range(68)] + [0, 9002], (8, 2), 48),
}


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", list(SHARED))
def test_shared_reading(binding, rows, D, dtype):
    P, lens, (Hq, H), block = SHARED[rows]
    Kc, Vc, prefix, table = make(len(rows), P, lens, H, D, block, dtype)
    Q, scale = normal(60, (len(lens), Hq, D), dtype), 1.0 / math.sqrt(D)
    for s in (scale, -0.05):
        O = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), s)
        name = binding.mlt_last_kernel()
        assert "_%s_p" % rows in name, name
        verify(O, Q, Kc, Vc, prefix, P, table, lens, s, name)
    need = binding.mlt_paged_attn_decode_prefix_work(len(lens), Hq, H, D, block, table.shape[1], P)
    work = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    again = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), s, work=work[:need])
    assert need > 0 and torch.equal(O, again) and bool((work[need:] == 255).all())
    alone = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), s, work=work[:need - 16])
    assert "_p0_" in binding.mlt_last_kernel()
    verify(alone, Q, Kc, Vc, prefix, P, table, lens, s)
