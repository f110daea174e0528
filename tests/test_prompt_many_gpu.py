"""Attention of packed and paged prompts for batches of some hundred to thousands of sequences, which workgroups take in the batch's order: against the definition in 64 bits, rows of no sequence,
offsets out of order, and a time that grows with the sequences and not with their square."""
import math

import pytest
import torch

from prompt_util import attend, cache_of, check, check_packed, ends, ints, limits, normal, rows_of, tolerance, HALF

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding as b
    return b


def lengths(seed, B, most, extra):
    g = torch.Generator().manual_seed(seed)
    new = torch.randint(0, most + 1, (B,), generator=g).tolist()
    have = [n + int(x) for n, x in zip(new, torch.randint(0, extra + 1, (B,), generator=g))]
    new[B // 3], have[B // 3] = 300, 340                             # several tiles
    new[0], have[-1] = 0, max(0, new[-1] - 1)                        # none; a row that sees nothing
    return new, have


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("B", [127, 128, 129, 130, 260, 4100])
def test_packed(binding, B, causal):
    new, have = lengths(B, B, 5 if B < 1000 else 1, 70 if B < 1000 else 6)
    cu, ku = ends(new, 3), ends(have, 2)
    Q, K, V = normal(1, (cu[-1] + 4, 6, 64), BF), normal(2, (ku[-1] + 4, 2, 64), BF), normal(3, (ku[-1] + 4, 2, 64), BF)
    O = torch.full_like(Q, 5.0)
    binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), 0.125, causal=causal, O=O)
    assert bool((O[:3] == 5).all()) and bool((O[cu[-1]:] == 5).all())
    if B < 1000:
        check_packed(O, Q, K, V, cu, ku, 0.125, causal)
        return
    for b in [0, 1, B // 3 - 1, B // 3, B // 3 + 1, B - 2, B - 1] + list(range(5, B, 131)):
        n, m = new[b], have[b]
        o, c = attend(Q[cu[b]:cu[b + 1]], K[ku[b]:ku[b + 1]], V[ku[b]:ku[b + 1]], 0.125, limits(n, m, causal))
        check(O[cu[b]:cu[b + 1]], o, tolerance(o, c, 64, BF, HALF[BF], moves=m // 64 + 1), "sequence %d" % b)
    assert not bool((O[3:cu[-1]] == 5).all(-1).all(-1).any())        # every row is written


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_paged(binding, dtype):
    B, D, block = 200, 128, 16
    new, have = lengths(7, B, 9, 50)
    cu = ends(new)
    Kc, Vc, table = cache_of(3, have, 1, D, block, dtype)
    Q, scale = normal(4, (cu[-1], 40, D), dtype), 1.0 / math.sqrt(D)  # 40 heads: 6 tokens to a tile
    O = binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(have), table, scale)
    for b in range(0, B, 3):
        m = have[b]
        K, V = (rows_of(c, table[b, :-(-m // block)], m) for c in (Kc, Vc))
        check_packed(O[cu[b]:cu[b + 1]], Q[cu[b]:cu[b + 1]], K, V, [0, new[b]], [0, m], scale, True, what="sequence %d" % b)


def test_offsets_out_of_order(binding):
    """Wrong results for the sequences concerned, no access out of range; with key offsets alone out of order the other sequences are as they were."""
    B = 300
    new, have = lengths(9, B, 4, 30)
    cu, ku = ends(new), ends(have)
    Q, K, V = normal(1, (cu[-1], 4, 64), FP), normal(2, (ku[-1], 2, 64), FP), normal(3, (ku[-1], 2, 64), FP)
    good = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), 0.1)
    bad = list(ku)
    bad[150], bad[151] = -9, 2 ** 31 - 1
    O = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(bad), 0.1)
    assert torch.equal(O[:cu[149]], good[:cu[149]]) and torch.equal(O[cu[152]:], good[cu[152]:])
    for odd in ([cu[-1]] * (B + 1), [0] * (B + 1), list(reversed(cu)), [-5] * 100 + [2 ** 31 - 1] * (B - 99), [10 ** 9 * (-1) ** i for i in range(B + 1)]):
        O = torch.full((cu[-1] + 8, 4, 64), 5.0, dtype=FP, device="cuda")
        binding.mlt_mha_packed_fwd(Q, K, V, ints(odd), ints(ku), 0.1, O=O[:cu[-1]])
        assert bool((O[cu[-1]:] == 5).all())


def test_the_time_grows_with_the_sequences(binding):
    """8192 single tokens, 8 key/value heads: 65536 workgroups with one tile of one key each, 1.5 ms. With every workgroup looking at every sequence it was 48 ms, four times as much for twice as many."""
    B = 8192
    cu = ints(list(range(B + 1)))
    Q, K = normal(1, (B, 32, 128), BF), normal(2, (B, 8, 128), BF)
    O = binding.mlt_mha_packed_fwd(Q, K, K, cu, None, 0.1)
    assert torch.equal(O, K.repeat_interleave(4, 1))                 # one key: its value
    times = []
    for _ in range(3):
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        binding.mlt_mha_packed_fwd(Q, K, K, cu, None, 0.1, O=O)
        stop.record()
        torch.cuda.synchronize()
        times.append(start.elapsed_time(stop))
    assert min(times) < 12.0, times
