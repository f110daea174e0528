"""Attention of packed and paged prompts where all scores of a row are -inf: no key has a weight, the output is zero, whatever stands in the values that the row does not see."""
import math

import pytest
import torch

from prompt_util import cache_of, ints, normal

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding as b
    return b


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("paged", [False, True], ids=["packed", "paged"])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n, m", [(40, 40), (30, 2600)], ids=["whole", "keys_split"])
def test_rows_whose_scores_are_all_minus_infinity(binding, n, m, D, dtype, paged, bad):
    """Positive queries; the keys of the first i rows hold -inf (a score of -inf, not NaN), the value of the last key one that is not finite, seen by the last row alone."""
    Hq, H, block, none = 4, 2, 16, m - n + 11
    Q = normal(1, (n, Hq, D), dtype).abs() + 0.1
    V = normal(2, (m, H, D), dtype)
    K = normal(3, (m, H, D), dtype)
    K[:none] = -math.inf
    if paged:
        Kc, Vc, table = cache_of(4, [m], H, D, block, dtype)

        def call(v):
            for cache, rows in ((Kc, K), (Vc, v)):
                for i, blk in enumerate(table[0, :-(-m // block)].tolist()):
                    part = rows[i * block:(i + 1) * block]
                    cache[blk, :, :part.shape[0]] = part.transpose(0, 1)
            return binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints([0, n]), ints([m]), table, 0.1)
    else:
        def call(v):
            return binding.mlt_mha_packed_fwd(Q, K, v, ints([0, n]), ints([0, m]), 0.1)
    clean = call(V)
    assert ("parts" in binding.mlt_last_kernel()) == (m > 2000)
    assert bool((clean[:11] == 0).all()) and bool(torch.isfinite(clean).all())
    dirty = V.clone()
    dirty[-1] = bad
    O = call(dirty)
    assert bool((O[:11] == 0).all()), "%d of the rows without a weight are not zero" % int((O[:11] != 0).any(-1).any(-1).sum())
    assert bool(torch.isfinite(O[:-1]).all()) and not bool(torch.isfinite(O[-1]).any())
