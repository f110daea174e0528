"""Block tables as wide as a model's context, far wider than any sequence of the batch: prompts and single tokens behind a prefix are spread over workgroups that mostly have no keys, and right all the same."""
import math

import pytest
import torch

from prompt_util import cache_of, check_packed, ends, ints, normal, rows_of
from test_paged_prefix_gpu import make, verify

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding as b
    return b


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("batch", [[(33, 33)], [(1, 1)], [(3, 0)], [(128, 128), (100, 90), (0, 0), (60, 700)]], ids=["33", "1", "no_keys", "four"])
def test_prompts(binding, batch, D, dtype):
    block, Hq, H = 16, 8, 2
    cu, lens = ends([n for n, _ in batch]), [m for _, m in batch]
    Kc, Vc, table = cache_of(1, lens, H, D, block, dtype, spare=2048)
    Q, scale = normal(2, (cu[-1], Hq, D), dtype), 1.0 / math.sqrt(D)
    O = binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), table, scale)
    assert "parts" in binding.mlt_last_kernel()
    for b, (n, m) in enumerate(batch):
        K, V = (rows_of(c, table[b, :-(-m // block)], m) for c in (Kc, Vc))
        check_packed(O[cu[b]:cu[b + 1]], Q[cu[b]:cu[b + 1]], K, V, [0, n], [0, m], scale, True, what="%s %d" % (binding.mlt_last_kernel(), b))


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P, lens", [(0, [1, 70, 0]), (500, [513, 600, 500, 499, 3]), (1000, [1040, 1100]), (6001, [6001 + 5 * i for i in range(40)])], ids=["0", "500", "1000", "6001"])
def test_prefixes(binding, P, lens, D, dtype):
    Hq, H, block = 8, 2, 16
    Kc, Vc, prefix, table = make(3, P, lens, H, D, block, dtype)
    table = torch.nn.functional.pad(table, (0, 2048), value=-9).contiguous()
    Q, scale = normal(4, (len(lens), Hq, D), dtype), 1.0 / math.sqrt(D)
    O = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), scale)
    verify(O, Q, Kc, Vc, prefix, P, table, lens, scale, binding.mlt_last_kernel())
    assert torch.equal(O, binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), scale))
