"""Decode attention over the 8-bit cache where its running references have to move: cases whose scores and value scales change from one unit of 32 keys to
the next one of the same wavefront, their result in 64 bits, a bound of the kernel's error, and the kernel's arithmetic in numpy (to see on the CPU that a
wrong rescaling would pass the bound)."""
import math

import numpy as np
import torch

F8 = torch.float8_e4m3fn
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative
UNIT, LAZY, GAIN = 32, 8.0, 6.0
LOG2E = 1.4426950408889634


def units_case(kind, step, waves, rounds, D, dtype, seed, H=2, G=2):
    """One sequence of `rounds` units of 32 keys for each of `waves` wavefronts, in blocks of 32 keys. All values are positive, so a result has the size of the sum that it is.
    kind: "rise" / "fall": scores of a round are `step` (log2) above / below the last round's; "scales_rise" / "scales_fall": the value scales are, at equal scores;
    "across": scores rise by `step` and the scales fall by 2 more; "light_first" / "light_last": the first (last) round has value scales 2^step times the others' and
    scores so far below that its part of the result is 2^-12 or less."""
    g = torch.Generator().manual_seed(seed)
    units = rounds * waves
    r = torch.arange(units) // waves                                     # the round of a unit
    s = torch.zeros(units)
    e = torch.full((units,), -8.0)
    if kind in ("rise", "fall"):
        s = step * (r if kind == "rise" else rounds - 1 - r).float()
    elif kind in ("scales_rise", "scales_fall"):
        e = 2.0 - step * (rounds - 1) + step * (r if kind == "scales_rise" else rounds - 1 - r).float()
    elif kind == "across":
        s, e = step * r.float(), step * (rounds - 1) - (step + 2) * r.float()
    else:
        light = r == (0 if kind == "light_first" else rounds - 1)
        s = torch.where(light, 0.0, step + 12.0)
        e = torch.where(light, step - 8.0, -8.0)
    q = (torch.rand((1, H * G, D), generator=g) * 0.5 + 0.75).to(dtype)
    k = (torch.rand((units, H, UNIT, D), generator=g) * 0.25 + 0.875).to(F8)
    v = (torch.rand((units, H, UNIT, D), generator=g) * 200 + 100).to(F8)
    scale = 1.0 / math.sqrt(D)
    # a key scale of (s + 1) / (log2(e) scale D) makes a score of about s + 1; per head a little off
    off = 1 + torch.arange(H).float() / 64
    ks = (s[:, None] + 1.0) / (LOG2E * scale * D) * off
    vs = torch.exp2(e)[:, None] * (1 + torch.rand((units, H), generator=g))
    table = torch.randperm(units, generator=g)
    where = torch.argsort(table)                                         # unit -> its block
    put = lambda x: x[table].contiguous()  # noqa: E731   block b holds unit table[b]
    lens = torch.tensor([units * UNIT - 5], dtype=torch.int32)
    return dict(q=q, kc=put(k), vc=put(v), ks=put(ks.float()), vs=put(vs.float()), table=where.to(torch.int32).reshape(1, -1).contiguous(), lens=lens, scale=scale)


def exact(q, kc, vc, ks, vs, table, lens, scale):
    """(o, what the error's bound needs) in 64 bits on the tensors' device: per query the sum of weight * |value|, the largest weight * value scale, the largest
    |scale| * sum |q k| and the largest |log2 of a value scale|."""
    B, Hq, D = q.shape
    H, block = kc.shape[1], kc.shape[2]
    G = Hq // H
    o = torch.zeros((B, Hq, D), dtype=torch.float64, device=q.device)
    mass, most = torch.zeros_like(o), torch.zeros((B, Hq, 1), dtype=torch.float64, device=q.device)
    reach, span = torch.zeros_like(most), torch.zeros_like(most)
    for b, n in enumerate(lens.tolist()):
        if n == 0:
            continue
        at = table[b, :-(-n // block)].long()

        def rows(c):                                                     # [H, n, D]
            return c.view(torch.uint8)[at].view(F8).double().transpose(0, 1).reshape(H, -1, D)[:, :n].contiguous()

        def spread(s):                                                   # [H, n]
            return s[at].double().t().repeat_interleave(block, 1)[:, :n].contiguous()
        sv = spread(vs)
        k, v = rows(kc) * spread(ks)[..., None], rows(vc) * sv[..., None]
        x = q[b].double().reshape(H, G, D)
        s = torch.matmul(x, k.transpose(1, 2).contiguous()) * scale
        w = torch.softmax(s, -1)
        o[b] = torch.matmul(w, v).reshape(Hq, D)
        mass[b] = torch.matmul(w, v.abs()).reshape(Hq, D)
        most[b] = (w * sv[:, None]).amax(-1).reshape(Hq, 1)
        reach[b] = (torch.matmul(x.abs(), k.abs().transpose(1, 2).contiguous()).amax(-1) * abs(scale)).reshape(Hq, 1)
        span[b] = torch.log2(sv).abs().amax(-1).repeat_interleave(G).reshape(Hq, 1)
    return o, dict(mass=mass, most=most, reach=reach, span=span)


def half_step(x, dtype):
    """Half the distance of x's neighbours in `dtype` (normal numbers): what rounding costs at most."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -14)))) * HALF[dtype]


def tolerance(o, c, n, D, dtype, rounds, weight_half):
    """|O - o| of the kernel at most.
    A score is a sum of D products in fp32, times the scales: reach (D + 4) 2^-24, and its rounding against a reference, which adds the references' size: an
    exponent of at most a = 2 reach log2(e) + 2 span + 16 in size is off by 3 a 2^-24. So is each factor by which a moved reference multiplies (one a round at most),
    and every exp2 by 2^-22. That counts for the weights and for their sum. `weight_half`: the weights' rounding for the second product, relative; fp16's smallest step is 2^-24,
    so half of it is 2^-25, against a reference of 2^GAIN times the largest weight * scale (rounded down to a power of two: half): 2^-30 of that for each key, times a value of up to 448.
    Then the fp32 sums over n keys, and the output's rounding with half of fp16's smallest step."""
    a = 2 * c["reach"] * LOG2E + 2 * c["span"] + 16
    one = (rounds + 2) * (3 * a * 2.0 ** -24 + 2.0 ** -22)
    rel = weight_half + 2 * (c["reach"] * (D + 4) * 2.0 ** -24 + one + n * 2.0 ** -24)
    return HALF[dtype] * o.abs() + c["mass"] * rel * 1.01 + n * 2.0 ** -30 * c["most"] * 448 + 2.0 ** -25


CASES = [("rise", 3.0), ("rise", 12.0), ("fall", 12.0), ("scales_rise", 3.0), ("scales_rise", 13.0), ("scales_fall", 13.0), ("across", 3.0), ("across", 11.0),
         ("light_first", 20.0), ("light_first", 28.0), ("light_first", 40.0), ("light_last", 28.0), ("light_last", 40.0)]


def two_halves(p):
    """p as the kernel multiplies with it: rounded to fp16, and what that left, rounded."""
    hi = np.float16(p).astype(float)
    return hi + np.float16(p - hi).astype(float)


def emulate(q, k, ks, v, vs, scale, waves, n, wrong=""):
    """The kernel's way for one query: q [D], k, v [units, 32, D], ks, vs [units]. wrong: a mistake to make."""
    parts = []
    for w in range(waves):
        m, top = np.float32(-math.inf), np.float32(0)                    # top is relative to m
        l, o = 0.0, np.zeros(q.shape[0])
        for u in range(w, k.shape[0], waves):
            mant, ex = np.frexp(vs[u])
            if wrong == "scale reference":                               # P against the largest value scale met, whatever its keys weigh
                ex = 0
            s = np.float32((k[u] @ q) * (ks[u] * scale * LOG2E))
            s[np.arange(32) + 32 * u >= n] = -math.inf
            mx = s.max()
            if mx > m + LAZY or mx - m + ex > top + LAZY:
                now = max(m, mx)
                down, most = m - now, np.float32(mx - now + ex)
                top_now = max(top + down, most) if m > -math.inf else most
                if wrong != "sum kept":
                    l *= 2.0 ** down
                if wrong != "outputs kept":
                    o *= 2.0 ** (down + (top - top_now))
                m, top = now, top_now
            if wrong == "scale reference":
                big = np.maximum.accumulate(vs[w:u + 1:waves])
                if len(big) > 1:
                    o *= big[-2] / big[-1]
                o = o + np.float16(2.0 ** (s - m - top + GAIN) * (vs[u] / big[-1])).astype(float) @ v[u]
            else:
                o = o + two_halves(2.0 ** np.float64(s - m + np.float32(ex + (GAIN - top))) * mant) @ v[u]
            l += (2.0 ** np.float64(s - m)).sum()
        last = np.max(vs[w::waves]) if wrong == "scale reference" else 1.0
        parts.append((float(m), l, o * last * 2.0 ** (float(top) - GAIN)))
    M = max(p[0] for p in parts)
    L = sum(p[1] * 2.0 ** (p[0] - M) for p in parts)
    return sum(p[2] * 2.0 ** (p[0] - M) for p in parts) / L
