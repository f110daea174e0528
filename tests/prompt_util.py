"""What the tests of the operators for prompts, shared prefixes and 4-bit weights share: inputs, results by the definitions in 64 bits, and what a kernel may be off."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}        # half a step, relative
SMALL = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}     # half of the smallest step
LOG2E = 1.4426950408889634


def ints(x, device="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=device)


def ends(new, first=0):
    """Offsets of sequences of these lengths that begin at row `first`."""
    out = [first]
    for n in new:
        out.append(out[-1] + n)
    return out


def attend(q, k, v, scale, limit):
    """q [n, Hq, D], k and v [m, H, D]; query i sees the keys 0 .. limit[i] - 1. In 64 bits: (o [n, Hq, D], what the error's bound needs)."""
    n, Hq, D = q.shape
    m, H = k.shape[:2]
    o = torch.zeros((n, Hq, D), dtype=torch.float64, device=q.device)
    c = dict(mass=torch.zeros_like(o), reach=torch.zeros((n, Hq, 1), dtype=torch.float64, device=q.device), big=torch.zeros((1, Hq, D), dtype=torch.float64, device=q.device),
             keys=max([0] + limit))
    if m == 0 or n == 0:
        return o, c
    lim = torch.tensor(limit, device=q.device)
    seen = torch.arange(m, device=q.device)[None] < lim[:, None]
    q64 = q.double()
    for h in range(Hq):
        any_row = seen.any(0)[:, None]
        kh, vh = (torch.where(any_row, x[:, h * H // Hq].double(), 0.0) for x in (k, v))
        s = q64[:, h] @ kh.t().contiguous() * scale
        s = torch.where(seen, s, -math.inf)
        top = s.amax(1, keepdim=True).clamp(min=-1e300)
        w = torch.exp(s - top)
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
        w = torch.where(seen, w, 0.0)
        o[:, h], c["mass"][:, h] = w @ vh, w @ vh.abs()
        c["reach"][:, h, 0] = torch.where(seen, q64[:, h].abs() @ kh.abs().t().contiguous(), 0.0).amax(1) * abs(scale)
        c["big"][0, h] = vh.abs().amax(0)
    return o, c


def tolerance(o, c, D, dtype, weight_half, moves=0):
    """|O - o| of a kernel at most.
    A score is a sum of D products in fp32, times the scale: reach (D + 4) 2^-24 off. In the exponent it stands against a reference of the same size: a = 2 reach log2(e) + 16 at
    most, off by 3 a 2^-24; exp2 by 2^-22. So is each of the `moves` factors by which a changed reference multiplies. Weights are rounded by weight_half, relative, for the product and
    for their sum or not; fp16's smallest step is 2^-24, half of it 2^-25, where the largest weight is 1 or more. The fp32 sums over the keys, and the output's rounding."""
    a = 2 * c["reach"] * LOG2E + 16
    one = c["reach"] * (D + 4) * 2.0 ** -24 + (moves + 2) * (3 * a * 2.0 ** -24 + 2.0 ** -22) + (c["keys"] + 64) * 2.0 ** -24
    under = 2 * c["keys"] * 2.0 ** -25 * c["big"] if dtype == torch.float16 else 0.0
    return HALF[dtype] * o.abs() + c["mass"] * (2 * weight_half + 2 * one) * 1.02 + under + SMALL[dtype]


def limits(n, m, causal):
    return [max(0, m - n + i + 1) if causal else m for i in range(n)]


def check(O, o, tol, what=""):
    off = (O.double() - o).abs()
    bad = ~(off <= tol)                                              # (a NaN is bad)
    assert not bool(bad.any()), "%s: %d of %d values off, worst %.3g of the bound, first at %s" % (
        what, int(bad.sum()), bad.numel(), float((off / tol).nan_to_num(math.inf).max()), bad.nonzero()[0].tolist())


def check_packed(O, Q, K, V, cu, ku, scale, causal, weight_half=None, what=""):
    """Every sequence of a packed batch (cu, ku: lists of offsets)."""
    D, dtype = Q.shape[2], Q.dtype
    for b in range(len(cu) - 1):
        n, m = cu[b + 1] - cu[b], ku[b + 1] - ku[b]
        o, c = attend(Q[cu[b]:cu[b + 1]], K[ku[b]:ku[b + 1]], V[ku[b]:ku[b + 1]], scale, limits(n, m, causal))
        check(O[cu[b]:cu[b + 1]], o, tolerance(o, c, D, dtype, HALF[dtype] if weight_half is None else weight_half, moves=m // 64 + 1), "%s sequence %d" % (what, b))


def rows_of(cache, blocks, n):
    """Keys 0 .. n - 1 of a sequence as [n, H, D] from a cache [num_blocks, H, block, D]."""
    return cache[blocks.long()].transpose(1, 2).flatten(0, 1)[:n]


def cache_of(seed, lens, H, D, block, dtype, extra_blocks=3, spare=1, device="cuda"):
    """A shuffled paged cache: Kc, Vc, block_table (with `spare` more columns than the longest sequence needs; entries that no key uses hold -7)."""
    g = torch.Generator().manual_seed(seed)
    per = [-(-n // block) for n in lens]
    nb = sum(per) + extra_blocks
    place = torch.randperm(nb, generator=g)
    table = torch.full((len(lens), max([1] + per) + spare), -7, dtype=torch.int32)
    at = 0
    for b, p in enumerate(per):
        table[b, :p] = place[at:at + p].to(torch.int32)
        at += p
    Kc, Vc = (torch.randn((nb, H, block, D), generator=g).to(dtype).to(device) for _ in range(2))
    return Kc, Vc, table.to(device)


def normal(seed, shape, dtype, device="cuda"):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(device)


# ---- 4-bit weights

def w4_inputs(seed, M, N, K, group, zeros, dtype, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    groups = -(-K // group)
    q = torch.randint(0, 16, (N, K), generator=g, dtype=torch.uint8)
    A = torch.randn((M, K), generator=g).to(dtype)
    S = (torch.rand((groups, N), generator=g) * 0.02 + 0.002).to(dtype)
    Z = torch.randint(0, 16, (groups, N), generator=g, dtype=torch.uint8) if zeros else None
    Wq = q[:, 0::2] | (q[:, 1::2] << 4)
    return [None if x is None else x.to(device) for x in (A, Wq, S, Z)] + [q.to(device)]


def w4_exact(A, q, S, Z, group):
    """C and a bound's size, sum over k of |a| |scale|, in 64 bits."""
    K = q.shape[1]
    spread = lambda x: x.double().t().repeat_interleave(group, 1)[:, :K]  # noqa: E731
    s = spread(S)
    w = (q.double() - (8.0 if Z is None else spread(Z))) * s
    return A.double() @ w.t().contiguous(), A.double().abs() @ s.abs().t().contiguous()


def w4_tolerance(c, size, K, group, dtype):
    """Products of |a| with numbers of up to 31 (a weight and 16, and a zero point and 16, of which the difference counts), two such sums over a group in fp32: 62 |a| times
    group + 4 roundings; the scaled sums over the groups, and what several parts of K add; the output's rounding."""
    return HALF[dtype] * c.abs() + 62 * size * (group + -(-K // group) + 24) * 2.0 ** -24 + SMALL[dtype]
