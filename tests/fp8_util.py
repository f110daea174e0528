"""The 8-bit operators in 64 bits on the CPU, from their definitions, for the parity tests: numbers of e4m3, scales of blocks,
the scaled product, the rotation and the paged cache. Written apart from the library and from the measured cases' plain forms."""
import math

import numpy as np
import torch

F8 = torch.float8_e4m3fn
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, F8: 2.0 ** -4}     # half a step, relative
# every non-negative number of e4m3 in order: code c stands for E4M3[c], up to 448 (code 126)
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def e4m3(x):
    """x (float64) rounded to the nearest e4m3 number, ties to the even code; not finite or past the largest: NaN."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    with np.errstate(invalid="ignore"):
        hi = np.clip(np.searchsorted(E4M3, np.nan_to_num(a, nan=0.0, posinf=0.0)), 1, 126)
        lo = hi - 1
        d = (a - E4M3[lo]) - (E4M3[hi] - a)
        code = np.where(d < 0, lo, np.where(d > 0, hi, np.where(lo % 2 == 0, lo, hi)))
        v = np.copysign(E4M3[code], x)
    return np.where(np.isfinite(x) & (a < 464.0), v, np.nan)


def scale_of(top):
    """The smallest power of two s >= 2^-100 with top <= 448 s."""
    s = 2.0 ** max(-100, math.floor(math.log2(top)) - 10) if top > 0 else 2.0 ** -100
    while top > 448.0 * s:
        s *= 2
    return s


def scales_of(tops):
    return np.vectorize(scale_of, otypes=[np.float64])(tops)


def finite_top(x, axis):
    return np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=axis)


def quant(x, rows):
    """(values, scales [k blocks, row blocks]) of x (float64 [M, K])."""
    M, K = x.shape
    q, s = np.empty_like(x), np.empty((-(-K // 128), -(-M // rows)))
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            at = (slice(rows * j, rows * j + rows), slice(128 * i, 128 * i + 128))
            s[i, j] = scale_of(finite_top(x[at], None))
            q[at] = e4m3(x[at] / s[i, j])
    return q, s


def gemm(a, sa, b, sb):
    """(C, sum of |products|, sum over groups of 8 k of the largest |product|), float64 [M, N], of e4m3 values a [M, K], b [N, K] and
    scales [k blocks, ...]."""
    M, N = a.shape[0], b.shape[0]
    c, t, top = np.zeros((M, N)), np.zeros((M, N)), np.zeros((M, N))
    for i in range(sa.shape[0]):
        k = slice(128 * i, 128 * i + 128)
        s = np.outer(sa[i], np.repeat(sb[i], 128)[:N])
        aa, bb = np.abs(a[:, k]), np.abs(b[:, k])
        c += (a[:, k] @ b[:, k].T) * s
        t += (aa @ bb.T) * np.abs(s)
        part = np.zeros((M, N))
        for j in range(0, aa.shape[1], 8):
            most = np.zeros((M, N))
            for e in range(j, min(j + 8, aa.shape[1])):
                np.maximum(most, np.outer(aa[:, e], bb[:, e]), out=most)
            part += most
        top += part * np.abs(s)
    return c, t, top


def gemm_tolerance(ref, mass, top, K, blocks, dtype):
    """|C - ref| of the kernels at most.
    The MFMA on e4m3 adds the 8 products of 8 neighbouring k in a fixed-point sum whose last place is 2^-13 of the largest one's
    power of two (the product of the two leading ones); what lies below is cut off. (Measured: beside a product of 2^16 a
    product of 2^3 in the same group of 8 is kept, one of 7.03 is not, nor seven of them; in another group all are kept
    down to 2^-7, fp32's last place.) The other 7 products of a group lose less than one such place each, and the largest product is at
    least its power of two: less than 7 * 2^-13 of the largest product of each group, together 7 * 2^-13 * top.
    Beyond it K fp32 additions, and a scale's product, the scaled block's and its addition for each block: 2^-24 of the sum of
    magnitudes each. Then the output's rounding, and half of fp16's smallest step."""
    return HALF[dtype] * np.abs(ref) + (7 * 2.0 ** -13 * top + mass * (K + 4 * blocks) * 2.0 ** -24) * 1.01 + 2.0 ** -25


def rotate(x, cos, sin, interleaved):
    """x [T, heads, D] float64, cos, sin [T, r]: the leading 2 r elements of each head turned."""
    y, r = x.copy(), cos.shape[1]
    for i in range(r):
        i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
        c, s = cos[:, None, i], sin[:, None, i]
        y[..., i1] = x[..., i1] * c - x[..., i2] * s
        y[..., i2] = x[..., i2] * c + x[..., i1] * s
    return y


def places(offsets, lens, table, block, num_blocks):
    """(row, sequence, position, block, slot) of every new token that has a place in the cache."""
    for b in range(len(lens)):
        n = offsets[b + 1] - offsets[b]
        for i in range(n):
            p = lens[b] - n + i
            if 0 <= p < table.shape[1] * block and 0 <= table[b, p // block] < num_blocks:
                yield offsets[b] + i, b, p, int(table[b, p // block]), p % block


def append_fp8(x, cache, scales, spots):
    """New rows x [T, H, D] into a cache of e4m3 values (float64) with scales; returns both anew."""
    cache, scales = cache.copy(), scales.copy()
    by_block = {}
    for t, _, _, blk, slot in spots:
        by_block.setdefault(blk, []).append((t, slot))
    for blk, rows in by_block.items():
        first = min(s for _, s in rows)
        for h in range(x.shape[1]):
            s = scale_of(finite_top(np.stack([x[t, h] for t, _ in rows]), None))
            old = scales[blk, h]
            if first > 0:
                s = max(s, 2.0 ** math.ceil(math.log2(old)))
                if s != old:
                    cache[blk, h, :first] = e4m3(cache[blk, h, :first] * old / s)
            scales[blk, h] = s
            for t, slot in rows:
                cache[blk, h, slot] = e4m3(x[t, h] / s)
    return cache, scales


def attn(q, k, v, scale):
    """(o, sum of weight * |v|, bound of |scale * q.k| with every product positive) of q [D], k, v [n, D], float64."""
    if len(k) == 0:
        return np.zeros_like(q), np.zeros_like(q), 0.0
    s = k @ q * scale
    w = np.exp(s - s.max())
    w /= w.sum()
    return w @ v, w @ np.abs(v), float((np.abs(k) @ np.abs(q)).max() * abs(scale))


def attn_tolerance(o, mass, reach, n, D, dtype, top):
    """|O - o| of the kernel at most: the output's rounding; the weights' rounding to 11 bits and their error from a score's, which
    is a sum of D products in fp32 (D 2^-24 of the sum of their magnitudes) times scale and the key scale (2^-23 each); exp2 and
    the fp32 sums over n keys; fp16's smallest step on weights with a gain of 64, relative to a sum of at least 1, against
    values up to `top`."""
    score = reach * (D + 4) * 2.0 ** -24
    return HALF[dtype] * np.abs(o) + mass * (2.0 ** -11 + 2 * score + 2.0 ** -21 + n * 2.0 ** -24) * 1.01 + n * 2.0 ** -31 * top + 2.0 ** -25
