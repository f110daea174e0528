"""The operators as a serving program runs them, one after the other on one stream: a layer's products with 4-bit weights, the new tokens appended to the paged cache, attention of prompts
in pieces over it, then single tokens behind the prefix that the sequences share. Each step is checked in 64 bits against what the one before it left."""
import math

import pytest
import torch

from prompt_util import HALF, attend, check, check_packed, ends, ints, normal, tolerance, w4_exact, w4_inputs, w4_tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_then_tokens(dtype, D):
    from paper_2503_14985_amd import binding as lib
    Hq, H, block, hidden, group = 8, 2, 16, 512, 64
    shared, pieces = 75, [[20, 33, 1], [7, 1, 50]]                   # the prefix's tokens; each sequence's in two steps
    B, steps = 3, 2
    scale = 1.0 / math.sqrt(D)
    weights = w4_inputs(1, 1, (Hq + 2 * H) * D, hidden, group, True, dtype)
    out_w = w4_inputs(2, 1, hidden, Hq * D, group, False, dtype)
    total = [shared + sum(p[b] for p in pieces) + steps for b in range(B)]
    first = shared // block                                          # blocks that are whole: every sequence's; the last one is copied for each
    per = [-(-n // block) for n in total]
    nb = -(-shared // block) + sum(n - first for n in per) + 1
    place = torch.randperm(nb, generator=torch.Generator().manual_seed(3)).to(torch.int32)
    prefix = place[:-(-shared // block)].cuda()
    table = torch.zeros((B, max(per)), dtype=torch.int32)
    at = len(prefix)
    for b in range(B):
        table[b, :first] = place[:first]
        table[b, first:per[b]] = place[at:at + per[b] - first]
        at += per[b] - first
    table = table.cuda()
    Kc, Vc = (torch.zeros((nb, H, block, D), dtype=dtype, device="cuda") for _ in range(2))
    angle = torch.arange(256, device="cuda")[:, None] * 10000.0 ** -(torch.arange(D // 2, device="cuda") / (D // 2))
    cos, sin = angle.cos().float().contiguous(), angle.sin().float().contiguous()

    def project(x):
        A, Wq, S, Z, q = weights
        y = lib.mlt_gemm_w4(x, Wq, S, Z, group=group)
        c, t = w4_exact(x, q, S, Z, group)
        check(y, c, w4_tolerance(c, t, hidden, group, dtype), lib.mlt_last_kernel())
        return y.unflatten(1, (Hq + 2 * H, D))

    def keys(row, n):
        j = torch.arange(n, device="cuda")
        blk = row[j // block].long()
        return Kc[blk, :, j % block], Vc[blk, :, j % block]

    def prompt(x, new, lens, tab):
        y = project(x)
        cu = ends(new)
        Q = torch.empty((cu[-1], Hq, D), dtype=dtype, device="cuda")
        lib.mlt_paged_append(y[:, :Hq], y[:, Hq:Hq + H], y[:, Hq + H:], ints(cu), ints(lens), tab, cos, sin, Kc, Vc, Qo=Q)
        O = lib.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), tab, scale)
        for b, (n, m) in enumerate(zip(new, lens)):
            K, V = keys(tab[b], m)
            if n:
                assert torch.equal(V[m - n:], y[cu[b]:cu[b + 1], Hq + H:])   # the cache holds the new tokens
            check_packed(O[cu[b]:cu[b + 1]], Q[cu[b]:cu[b + 1]], K, V, [0, n], [0, m], scale, True, what="%s %d" % (lib.mlt_last_kernel(), b))
        A, Wq, S, Z, q = out_w
        z = lib.mlt_gemm_w4(O.flatten(1), Wq, S, group=group)
        c, t = w4_exact(O.flatten(1), q, S, None, group)
        check(z, c, w4_tolerance(c, t, Hq * D, group, dtype), lib.mlt_last_kernel())
        return O

    # the prefix, once; its last, partly filled block goes to each sequence
    x = normal(10, (shared, hidden), dtype)
    prompt(x, [shared], [shared], prefix[None].contiguous())
    if shared % block:
        for c in (Kc, Vc):
            c[table[:, first].long()] = c[prefix[first].long()].clone()
    # the sequences' own prompts, a piece of each at a time
    have = [shared] * B
    for i, new in enumerate(pieces):
        have = [n + m for n, m in zip(have, new)]
        prompt(normal(20 + i, (sum(new), hidden), dtype), new, have, table)
    # single tokens
    for i in range(steps):
        have = [n + 1 for n in have]
        y = project(normal(30 + i, (B, hidden), dtype))
        Q = torch.empty((B, Hq, D), dtype=dtype, device="cuda")
        lib.mlt_paged_append(y[:, :Hq], y[:, Hq:Hq + H], y[:, Hq + H:], ints(ends([1] * B)), ints(have), table, cos, sin, Kc, Vc, Qo=Q)
        lens = ints(have)
        O = lib.mlt_paged_attn_decode_prefix(Q, Kc, Vc, prefix, shared, table, lens, scale)
        for b, m in enumerate(have):
            K, V = keys(table[b], m)
            o, c = attend(Q[b:b + 1], K, V, scale, [m])
            check(O[b:b + 1], o, tolerance(o, c, D, dtype, HALF[dtype], moves=m // 32 + 40), "%s %d" % (lib.mlt_last_kernel(), b))
        # the same tokens as pieces of one: the prompts' attention, and every sequence by itself
        P = lib.mlt_paged_attn_prompt(Q, Kc, Vc, ints(ends([1] * B)), lens, table, scale)
        size = 4 * HALF[dtype] * Vc.abs().max().double()             # each is within 2 HALF of the largest value of the truth
        assert bool(((P.double() - O.double()).abs() <= size).all())
