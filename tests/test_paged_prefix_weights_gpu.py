"""Single-token attention behind a shared prefix keeps the weights of own keys, and of a prefix read for up to 32 queries of a key head or by every sequence itself, to about 16 bits (bf16) or
22 (fp16), although the matrix units take 16-bit operands of 8 or 11 bits.

Two kinds of keys, with values +v and -v: kind A has the largest score and a weight of 1, kind B a weight r that lies between two numbers of the type, in such a number that the output is small. Rounding
r to the type would move the output by up to 2^-9 or 2^-12 of |v|, many times what is allowed here.

What is allowed. Scores are one product each, exact; times c = scale log2(e) <= 1, against the reference, plus a gain of 6: 4 roundings of numbers up to 8 in the exponent, 32 2^-24 ln 2 < 2^-19 in the
weight; exp2 2^-22; all references are the same number, so joins multiply by 1. A weight as the sum of two numbers of the type: 2^-16 (2^-22), and half of fp16's smallest step, 2^-25, against 64.
fp32 sums: no more than 32 keys in a product, 4 of those in a wavefront, 8 wavefronts and 64 parts one after the other, below 256 additions, 2^-16, of numerator and sum. The output's rounding."""
import math

import pytest
import torch

from prompt_util import HALF, SMALL, ints
from test_paged_prefix_gpu import make

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16

# prefix, lengths, query and key/value heads, block, what the kernel's name has
CASES = {
    "own": (0, [320, 32, 0, 640, 96], (8, 2), 16, "_p0_"),
    "alone": (96, [160, 96, 256, 128, 224, 192], (8, 2), 32, "_p0_"),
    "shared_16": (6016, [6080, 6112, 6016], (8, 2), 32, "_16_p"),
    "shared_32": (6016, [6048 + 32 * (i % 3) for i in range(6)], (8, 2), 16, "_32_p"),
}


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", list(CASES))
def test_weights_keep_their_bits(case, D, dtype):
    from paper_2503_14985_amd import binding
    P, lens, (Hq, H), block, kind = CASES[case]
    r = 155.45 / 256 if dtype == BF else 1243.45 / 2048               # between two numbers of the type, nearly in the middle
    scale = -math.log(r)
    Kc, Vc, prefix, table = make(1, P, lens, H, D, block, dtype, poison=False)
    is_a = torch.tensor([(7 * j + j // 32) % 32 < 12 for j in range(max(lens))], device="cuda")       # 12 of every 32
    v = (1 + torch.arange(D, device="cuda") % 8 / 8).to(dtype)
    Kc.zero_()
    for b, n in enumerate(lens):
        for j0 in range(0, n, block):
            blk = prefix[j0 // block] if j0 + block <= P else table[b, j0 // block]
            a = is_a[j0:j0 + block]
            Kc[blk.long(), :, :a.shape[0], 0] = a.to(dtype)
            Vc[blk.long(), :, :a.shape[0]] = torch.where(a[:, None], v, -v)
    Q = torch.zeros((len(lens), Hq, D), dtype=dtype, device="cuda")
    Q[..., 0] = 1
    O = binding.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, P, table, ints(lens), scale)
    assert kind in binding.mlt_last_kernel(), binding.mlt_last_kernel()

    def definition(weight, n):
        na = int(is_a[:n].sum())
        return v.double() * (na - (n - na) * weight) / max(1e-300, na + (n - na) * r)

    for b, n in enumerate(lens):
        if n == 0:
            assert bool((O[b] == 0).all())
            continue
        o = definition(r, n)
        tol = HALF[dtype] * o.abs() + v.double() * ((2.0 ** -16 if dtype == BF else 2.0 ** -22 + 2.0 ** -31) + 2 * (2.0 ** -19 + 2.0 ** -22 + 2.0 ** -16)) + SMALL[dtype]
        rounded = definition(float(torch.tensor(r, dtype=torch.float64).to(dtype)), n)
        assert bool(((rounded - o).abs() > 1.5 * tol).all()), "weights of the type's own bits would pass"
        off = (O[b].double() - o).abs()
        assert bool((off <= tol).all()), "sequence %d: %.3g of the bound (plainly rounded weights: %.3g)" % (b, float((off / tol).max()), float(((rounded - o).abs() / tol).min()))
