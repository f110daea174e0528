"""Attention of packed sequences and of new tokens over the paged cache against their definition in 64 bits: lengths from none to long ones, grouped heads, strides,
rows that see nothing, and what must have no influence."""
import math

import pytest
import torch

from prompt_util import cache_of, check_packed, ends, ints, normal, rows_of

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding as b
    return b


# (queries, keys) of each sequence
BATCHES = {
    "one": [(1, 1)],
    "few": [(3, 3), (1, 1), (17, 17)],
    "ragged": [(65, 65), (0, 0), (1, 1), (130, 130), (64, 64), (300, 300)],
    "pieces": [(5, 69), (64, 200), (1, 333), (0, 40), (31, 31), (128, 129)],
    "empty_rows": [(20, 7), (9, 0), (70, 64), (2, 1)],
    "long": [(257, 1500), (1, 2049), (600, 600)],
}
HEADS = [(4, 4), (8, 2), (6, 2), (5, 1), (16, 1), (40, 1)]


def make(seed, batch, Hq, H, D, dtype, lead=0, trail=0):
    new, have = [n for n, _ in batch], [m for _, m in batch]
    cu, ku = ends(new, lead), ends(have, lead)
    return cu, ku, normal(seed, (cu[-1] + trail, Hq, D), dtype), normal(seed + 1, (ku[-1] + trail, H, D), dtype), normal(seed + 2, (ku[-1] + trail, H, D), dtype)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("name", list(BATCHES))
def test_packed_batches(binding, name, causal, D, dtype):
    cu, ku, Q, K, V = make(len(name), BATCHES[name], 8, 2, D, dtype)
    scale = 1.0 / math.sqrt(D)
    O = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), scale, causal=causal)
    check_packed(O, Q, K, V, cu, ku, scale, causal, what=binding.mlt_last_kernel())
    assert torch.equal(O, binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), scale, causal=causal))


@pytest.mark.parametrize("heads", HEADS, ids=["%dq%d" % x for x in HEADS])
@pytest.mark.parametrize("D", [64, 128])
def test_packed_heads(binding, D, heads):
    for causal in (True, False):
        for name in ("ragged", "pieces"):
            cu, ku, Q, K, V = make(7, BATCHES[name], *heads, D, BF)
            O = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), 0.11, causal=causal)
            check_packed(O, Q, K, V, cu, ku, 0.11, causal, what=binding.mlt_last_kernel())


def test_packed_same_offsets_and_strides(binding):
    """Parts of one fused projection's result, an output with gaps, rows in front of the first and behind the last sequence."""
    Hq, H, D = 6, 3, 128
    cu = ends([33, 1, 90], 5)
    rows = normal(3, (cu[-1] + 9, (Hq + 2 * H) * D + 16), BF)
    rows[:5] = math.nan
    rows[cu[-1]:] = math.nan
    Q, K, V = (x.unflatten(1, (-1, D)) for x in rows[:, :-16].split([Hq * D, H * D, H * D], 1))
    out = torch.full((cu[-1] + 9, Hq * D + 8), 7.0, dtype=BF, device="cuda")
    O = out[:, :-8].unflatten(1, (-1, D))
    got = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), None, 0.1, O=O)
    assert got.data_ptr() == O.data_ptr()
    check_packed(O, Q, K, V, cu, cu, 0.1, True)
    assert bool((out[:5] == 7).all()) and bool((out[cu[-1]:] == 7).all()) and bool((out[:, -8:] == 7).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.09, 3.0])
def test_packed_scales(binding, scale, D):
    cu, ku, Q, K, V = make(11, BATCHES["pieces"], 8, 2, D, FP)
    O = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), scale)
    check_packed(O, Q, K, V, cu, ku, scale, True)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_unseen_keys_have_no_influence(binding, dtype, D, bad):
    """A key or value that is not finite reaches the queries that see it and no others: not earlier ones of its sequence, not other sequences."""
    batch = [(40, 40), (150, 150), (40, 100), (70, 70)]
    Hq, H = 4, 2
    cu, ku, Q, K, V = make(5, batch, Hq, H, D, dtype)
    scale = 1.0 / math.sqrt(D)
    clean = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), scale)
    for at, b in ((ku[1] + 77, 1), (ku[2] + 90, 2), (ku[0] + 39, 0)):
        for which in (K, V):
            dirty = which.clone()
            dirty[at] = bad
            O = binding.mlt_mha_packed_fwd(Q, dirty if which is K else K, dirty if which is V else V, ints(cu), ints(ku), scale)
            first = cu[b] + max(0, at - ku[b] - (batch[b][1] - batch[b][0]))         # the first query that sees it
            assert torch.equal(O[:cu[b]], clean[:cu[b]]) and torch.equal(O[cu[b + 1]:], clean[cu[b + 1]:]), (at, which is K)
            n, m = first - cu[b], ku[b + 1] - ku[b] - (cu[b + 1] - first)            # the sequence as far as nothing has happened
            check_packed(O[cu[b]:first], Q[cu[b]:first], K[ku[b]:ku[b] + m], V[ku[b]:ku[b] + m], [0, n], [0, m], scale, True, what="key %d" % at)
            if which is V:
                want = torch.full_like(O[first:cu[b + 1]], bad)
                assert torch.equal(O[first:cu[b + 1]].nan_to_num(9.0, 8.0, 7.0), want.nan_to_num(9.0, 8.0, 7.0)), (at, bad)


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
def test_an_infinity_in_the_last_value(binding, causal):
    """Tiles that the keys do not fill repeat the last one: an infinity there is one in the output, not NaN."""
    cu, ku, Q, K, V = make(8, [(3, 3), (50, 70), (1, 200)], 4, 2, 64, BF)
    for b in range(3):
        dirty = V.clone()
        dirty[ku[b + 1] - 1] = -math.inf
        O = binding.mlt_mha_packed_fwd(Q, K, dirty, ints(cu), ints(ku), 0.1, causal=causal)
        assert bool(torch.isneginf(O[cu[b + 1] - 1 if causal else cu[b]:cu[b + 1]]).all())
        assert int(torch.isfinite(O).all(-1).all(-1).sum()) == (cu[-1] - 1 if causal else cu[-1] - (cu[b + 1] - cu[b]))


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block", [16, 48, 128])
@pytest.mark.parametrize("name", list(BATCHES))
def test_paged_batches(binding, name, block, D, dtype):
    batch = BATCHES[name]
    cu, _, Q, _, _ = make(len(name), batch, 8, 2, D, dtype)
    lens = [m for _, m in batch]
    Kc, Vc, table = cache_of(9, lens, 2, D, block, dtype)
    for b, m in enumerate(lens):                                     # slots behind a sequence's last key: anything
        if m % block:
            Kc[table[b, m // block].long(), :, m % block:] = math.nan
            Vc[table[b, m // block].long(), :, m % block:] = math.inf
    scale = 1.0 / math.sqrt(D)
    O = binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), table, scale)
    for b, (n, m) in enumerate(batch):
        K, V = (rows_of(c, table[b, :-(-m // block)], m) for c in (Kc, Vc))
        check_packed(O[cu[b]:cu[b + 1]], Q[cu[b]:cu[b + 1]], K, V, [0, n], [0, m], scale, True, what="%s %d" % (binding.mlt_last_kernel(), b))


@pytest.mark.parametrize("heads", HEADS, ids=["%dq%d" % x for x in HEADS])
def test_paged_heads_and_strides(binding, heads):
    Hq, H = heads
    D, block, batch = 128, 32, BATCHES["pieces"]
    lens = [m for _, m in batch]
    cu = ends([n for n, _ in batch], 3)
    wide = normal(1, (cu[-1] + 4, Hq * D + 24), BF)
    Q = wide[:, :Hq * D].unflatten(1, (Hq, D))
    Kc, Vc, table = cache_of(2, lens, H, D, block, BF)
    O = torch.full((cu[-1] + 4, Hq, D), 5.0, dtype=BF, device="cuda")
    binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), table, 0.1, O=O)
    assert bool((O[:3] == 5).all()) and bool((O[cu[-1]:] == 5).all())
    for b, (n, m) in enumerate(batch):
        K, V = (rows_of(c, table[b, :-(-m // block)], m) for c in (Kc, Vc))
        check_packed(O[cu[b]:cu[b + 1]], Q[cu[b]:cu[b + 1]], K, V, [0, n], [0, m], 0.1, True)


def test_paged_bad_table_and_lengths(binding):
    """Block numbers and lengths out of range are clamped by the kernel: a wrong result for their sequences, none for the others."""
    D, block, H = 64, 16, 2
    lens = [40, 90, 33]
    Kc, Vc, table = cache_of(4, lens, H, D, block, BF, spare=0)
    cu = ends([40, 20, 33])
    Q = normal(6, (cu[-1], 4, D), BF)
    good = binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), table, 0.1)
    bad = table.clone()
    bad[1, 2], bad[1, 3] = 2 ** 31 - 1, -2 ** 31
    for l1 in (90, -5, 2 ** 31 - 1):
        O = binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints([40, l1, 33]), bad, 0.1)
        assert torch.equal(O[:40], good[:40]) and torch.equal(O[60:], good[60:])
        if l1 < 0:
            assert bool((O[40:60] == 0).all())


def test_packed_bad_offsets(binding):
    """Key offsets out of their range or order: no access out of range, the other sequences as they are."""
    cu, ku, Q, K, V = make(2, [(20, 20), (30, 30), (25, 25)], 4, 2, 64, FP)
    good = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), 0.1)
    for bad in ([0, 20, -9, 75], [0, 20, 10 ** 9, 75], [0, 20, 50, 2 ** 31 - 1], [0, 20, 50, 49]):
        O = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(bad), 0.1)
        assert torch.equal(O[:20], good[:20]), bad
    # query offsets that fall or leave the rows: rows outside them keep what they hold
    O = torch.full_like(Q, 3.0)
    binding.mlt_mha_packed_fwd(Q, K, V, ints([0, 20, 10 ** 9, 75]), ints(ku), 0.1, O=O)
    assert torch.equal(O[:20], good[:20])


def test_many_sequences(binding):
    """More sequences than a workgroup has threads, most of them single tokens."""
    g = torch.Generator().manual_seed(0)
    new = torch.randint(0, 4, (700,), generator=g).tolist()
    have = [n + int(x) for n, x in zip(new, torch.randint(0, 90, (700,), generator=g))]
    new[333], have[333] = 150, 400
    cu, ku, Q, K, V = make(1, list(zip(new, have)), 4, 2, 64, BF)
    O = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), 0.125)
    check_packed(O, Q, K, V, cu, ku, 0.125, True)


def test_no_sequences_no_keys(binding):
    Q, K = normal(1, (5, 4, 64), BF), normal(2, (0, 2, 64), BF)
    O = torch.full_like(Q, 2.0)
    binding.mlt_mha_packed_fwd(Q, K, K, ints([0]), ints([0]), 0.1, O=O)
    assert bool((O == 2).all())
    binding.mlt_mha_packed_fwd(Q, K, K, ints([0, 3]), ints([0, 0]), 0.1, causal=False, O=O)
    assert bool((O[:3] == 0).all()) and bool((O[3:] == 2).all())


# Few rows and long keys: the keys are split over several workgroups
BEHIND = {
    "one": [(16, 4000)],
    "token": [(1, 8191)],
    "chunk": [(300, 2816)],
    "four": [(3, 1300), (40, 2600), (0, 700), (7, 7)],
    "empty_rows": [(20, 7), (9, 0), (70, 64), (2, 4000)],
}


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("how", ["causal", "full", "paged"])
@pytest.mark.parametrize("name", list(BEHIND))
def test_split_keys(binding, name, how, D, dtype):
    batch = BEHIND[name]
    cu, ku, Q, K, V = make(len(name), batch, 8, 2, D, dtype, lead=2, trail=3)
    O = torch.full_like(Q, 5.0)
    scale = 1.0 / math.sqrt(D)
    lens = [m for _, m in batch]
    if how == "paged":
        Kc, Vc, table = cache_of(9, lens, 2, D, 48, dtype)
        for b, m in enumerate(lens):                                 # slots behind a sequence's last key: anything
            if m % 48:
                Kc[table[b, m // 48].long(), :, m % 48:] = math.nan
                Vc[table[b, m // 48].long(), :, m % 48:] = math.inf
        for _ in range(2):
            binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), table, scale, O=O)
        K, V = (torch.cat([K[:2]] + [rows_of(c, table[b, :-(-m // 48)], m) for b, m in enumerate(lens)]) for c in (Kc, Vc))
    else:
        binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), scale, causal=how == "causal", O=O)
    assert "parts" in binding.mlt_last_kernel()
    assert bool((O[:2] == 5).all()) and bool((O[cu[-1]:] == 5).all())
    check_packed(O, Q, K, V, cu, ku, scale, how != "full", what=binding.mlt_last_kernel())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("D", [64, 128])
def test_split_unseen_keys_have_no_influence(binding, D, bad):
    batch = [(40, 2040), (30, 1500)]
    cu, ku, Q, K, V = make(5, batch, 4, 2, D, BF)
    scale = 1.0 / math.sqrt(D)
    for at, b in ((ku[0] + 2020, 0), (ku[0] + 2039, 0), (ku[1] + 1490, 1)):
        for which in (K, V):
            dirty = which.clone()
            dirty[at] = bad
            O = binding.mlt_mha_packed_fwd(Q, dirty if which is K else K, dirty if which is V else V, ints(cu), ints(ku), scale)
            assert "parts" in binding.mlt_last_kernel()
            first = cu[b] + at - ku[b] - (batch[b][1] - batch[b][0])             # the first query that sees it
            n, m = first - cu[b], at - ku[b]
            check_packed(O[cu[b]:first], Q[cu[b]:first], K[ku[b]:ku[b] + m], V[ku[b]:ku[b] + m], [0, n], [0, m], scale, True, what="key %d" % at)
            o = 1 - b
            check_packed(O[cu[o]:cu[o + 1]], Q[cu[o]:cu[o + 1]], K[ku[o]:ku[o + 1]], V[ku[o]:ku[o + 1]], [0, batch[o][0]], [0, batch[o][1]], scale, True)
            if which is V:
                assert not bool(torch.isfinite(O[first:cu[b + 1]]).any())
