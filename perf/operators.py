"""The 8-bit serving operators as measured cases, beside their plain forms.

What a serving program does between two matrix products with 8-bit weights and an 8-bit key/value cache:
  quant     mlt_quant_fp8:              rows (or a weight's 128 x 128 squares) to e4m3, a power of two as scale of each block of 128
  gemm      mlt_gemm_fp8:               e4m3 x e4m3 -> bf16 / fp16 with those scales
  append    mlt_paged_append(_fp8):     positions rotated into queries and keys, keys and values into the paged cache
  attn      mlt_paged_attn_decode_fp8:  one query a sequence over the 8-bit paged cache, shared key/value heads

`listed()` holds the fixed cases, `draw(rng)` gives further ones of the same ranges, `prepare(case, seed)` makes what a program
holds before the call, `run(state)` is the call, `work(case)` the bytes and flops that no implementation can do without and
`exact(case, seed)` the result by the operator's definition in 64 bits. With `own` false, `run` computes the plain form in
elementary torch operations in 32 bits; with `own` true it calls the library.

A case is a dict of plain values. `op` is one of the names above; `dtype` is the 16-bit type of what is not 8-bit.
  quant   m, k, rows (1: a scale per row and 128 columns; 128: per 128 x 128)
  gemm    m, n, k
  append  b sequences, up to s tokens each in the cache, n new tokens in all ("decode": one each), hq query and h key/value heads,
          d, rot (rotated leading elements of a head), interleaved (pairs of neighbours instead of halves), block, cache ("fp8" / "same")
  attn    b, s (longest sequence), hq, h, d, block, idle (the first sequence of the batch has no keys)
"""
import math

import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}
_F8 = torch.float8_e4m3fn
_F8_MAX = 448.0


def listed():
    return [
        # The activations of a batch of 16 next tokens in front of an 8-bit product: the smallest call, latency alone.
        dict(name="quant_decode", op="quant", m=16, k=4096, rows=1, dtype="bf16"),
        # The activations of a prefill of 8192 tokens into a feed-forward layer's second product.
        dict(name="quant_prefill", op="quant", m=8192, k=14336, rows=1, dtype="bf16"),
        # A feed-forward weight laid out in 8 bits when a model is loaded; fp16, as a checkpoint may be.
        dict(name="quant_weight", op="quant", m=14336, k=4096, rows=128, dtype="fp16"),
        # Next-token decode, an attention projection: a batch of 16 against a 4096 x 4096 weight.
        dict(name="gemm_decode", op="gemm", m=16, n=4096, k=4096, dtype="bf16"),
        # Next-token decode, a feed-forward weight, a batch that does not fill its tile.
        dict(name="gemm_ffn_decode", op="gemm", m=24, n=14336, k=4096, dtype="fp16"),
        # A prompt of ragged length through a feed-forward layer's second product.
        dict(name="gemm_prefill", op="gemm", m=777, n=4096, k=14336, dtype="bf16"),
        # The largest: a prefill of many prompts at once, the benchmark's GEMM in 8 bits.
        dict(name="gemm_8192", op="gemm", m=8192, n=8192, k=8192, dtype="bf16"),
        # A decode step's append: a token each for 64 sequences, four query heads to a key/value head, 8-bit cache.
        dict(name="append_decode", op="append", b=64, s=4096, n=64, decode=True, hq=32, h=8, d=128, rot=128, interleaved=False,
             block=16, cache="fp8", dtype="bf16"),
        # A prefill step's append: prompts and pieces of prompts of ragged length, most of them starting inside a block.
        dict(name="append_prefill", op="append", b=13, s=4096, n=8191, decode=False, hq=32, h=8, d=128, rot=128, interleaved=False,
             block=16, cache="fp8", dtype="bf16"),
        # The same into a 16-bit cache of the library's older layout (as many key/value heads as query heads), neighbours rotated, half a head.
        dict(name="append_16bit", op="append", b=7, s=2048, n=4096, decode=False, hq=32, h=32, d=64, rot=32, interleaved=True,
             block=32, cache="same", dtype="fp16"),
        # A serving batch of mixed lengths over a shuffled cache of 16-key blocks, grouped heads, one slot of the batch idle.
        dict(name="attn_batch", op="attn", b=64, s=4096, hq=32, h=8, d=128, block=16, idle=True, dtype="bf16"),
        # One long sequence with few heads: too few (sequence, head) pairs to fill the chip.
        dict(name="attn_long", op="attn", b=1, s=32768, hq=8, h=8, d=128, block=16, idle=False, dtype="fp16"),
    ]


def _log(rng, lo, hi, mult=1):
    """An integer of [lo, hi], even over its logarithm, a multiple of `mult`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))
    return max(lo, min(hi, int(v) // mult * mult))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    kind = rng.choice(["quant", "gemm", "gemm", "gemm_few", "append", "append_decode", "attn", "attn", "attn_few"])
    if kind == "quant":
        while True:
            m, k = _log(rng, 1, 14336), _log(rng, 128, 14336, 16)
            if m * k <= 8192 * 14336:
                return dict(op="quant", m=m, k=k, rows=rng.choice([1, 1, 128]), dtype=dtype)
    if kind == "gemm":
        while True:
            m, n, k = _log(rng, 65, 8192), _log(rng, 257, 14336), _log(rng, 256, 14336, 16)
            if m * n * k <= 8192 ** 3:
                break
        if rng.random() < 0.7:                  # most layers' sizes are multiples of 128, some of a block's 128 no multiple
            n, k = max(128, n // 128 * 128), max(128, k // 128 * 128)
        return dict(op="gemm", m=m, n=n, k=k, dtype=dtype)
    if kind == "gemm_few":
        return dict(op="gemm", m=_log(rng, 1, 64), n=_log(rng, 1024, 28672, 8), k=_log(rng, 1024, 14336, 128), dtype=dtype)
    d, h, block = rng.choice([64, 128, 128]), rng.choice([1, 4, 8, 8, 16]), rng.choice([16, 16, 32, 64, 128])
    hq = h * rng.choice([1, 2, 4, 8])
    rot = rng.choice([d, d, d // 2])
    if kind == "append_decode":
        b = _log(rng, 1, 256)
        return dict(op="append", b=b, s=_log(rng, 64, 4096), n=b, decode=True, hq=hq, h=h, d=d, rot=rot, interleaved=rng.random() < 0.3,
                    block=block, cache=rng.choice(["fp8", "fp8", "same"]), dtype=dtype)
    if kind == "append":
        b = _log(rng, 1, 64)
        return dict(op="append", b=b, s=2048, n=_log(rng, b, 8191), decode=False, hq=hq, h=h, d=d, rot=rot, interleaved=rng.random() < 0.3,
                    block=block, cache=rng.choice(["fp8", "fp8", "same"]), dtype=dtype)
    if kind == "attn_few":
        return dict(op="attn", b=_log(rng, 1, 4), s=_log(rng, 1, 32768), hq=hq, h=h, d=d, block=block, idle=False, dtype=dtype)
    while True:
        b, s = _log(rng, 2, 256), _log(rng, 64, 16384)
        if b * s * h * d <= 64 * 4096 * 8 * 128:
            return dict(op="attn", b=b, s=s, hq=hq, h=h, d=d, block=block, idle=rng.random() < 0.3, dtype=dtype)


# ---- what the plain forms share

def _two_to(e, real):
    """2^e for whole e, by the format's exponent field (a power function may be off in its last place)."""
    return ((e.long() + 127) << 23).to(torch.int32).view(torch.float32) if real == torch.float32 else ((e.long() + 1023) << 52).view(torch.float64)


def _pow2_scale(amax):
    """The smallest power of two s with amax <= 448 s, at least 2^-100."""
    m, e = torch.frexp(amax)                                    # amax = m 2^e, m in [1/2, 1); 448 = 7/8 * 2^9
    e = (e - 9 + (m > 0.875)).clamp(min=-100)
    return _two_to(torch.where(amax > 0, e, -100), amax.dtype)


def _pow2_ceil(s):
    """The smallest power of two >= s, at least 2^-100."""
    m, e = torch.frexp(s)
    return _two_to((e - (m == 0.5).to(e.dtype)).clamp(min=-100), s.dtype)


def _blocked_amax(x, rows):
    """[k blocks, row blocks] maxima of |x| over `rows` x 128."""
    m, k = x.shape
    kb, mb = -(-k // 128), -(-m // rows)
    a = torch.nn.functional.pad(x.abs(), (0, kb * 128 - k, 0, mb * rows - m))
    return a.reshape(mb, rows, kb, 128).amax(dim=(1, 3)).t().contiguous()


def _spread(s, rows, m, k):
    """A scale of each element from the [k blocks, row blocks] scales."""
    return s.t().repeat_interleave(rows, 0)[:m].repeat_interleave(128, 1)[:, :k]


def _plain_quant(x, rows, real=torch.float32):
    x = x.to(real)
    s = _pow2_scale(_blocked_amax(x, rows))
    return (x / _spread(s, rows, *x.shape)).to(_F8), s.float()


def _plain_gemm(st, real=torch.float32):
    a = st["A"].to(real) * _spread(st["Sa"].to(real), 1, *st["A"].shape)
    b = st["B"].to(real) * _spread(st["Sb"].to(real), 128, *st["B"].shape)
    return a @ b.t()


def _token_places(st):
    """Of each new token: its sequence, its position, its cache block and the slot in it; all of one type."""
    cu, lens, table, block = st["offsets"].long(), st["lens"].long(), st["table"].long(), st["Kc"].shape[2]
    t = torch.arange(st["K"].shape[0], device=cu.device)
    b = torch.searchsorted(cu[1:], t, right=True)
    pos = lens[b] - cu[b + 1] + t
    return b, pos, table[b, pos // block], pos % block


def _rotated(x, cos, sin, interleaved):
    """The leading 2 r elements of every head turned by the token's angles (cos, sin: [tokens, r])."""
    r = cos.shape[1]
    c, s = cos[:, None], sin[:, None]
    x1, x2 = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if interleaved else (x[..., :r], x[..., r:2 * r])
    y1, y2 = x1 * c - x2 * s, x2 * c + x1 * s
    y = torch.stack((y1, y2), -1).flatten(-2) if interleaved else torch.cat((y1, y2), -1)
    return torch.cat((y, x[..., 2 * r:]), -1)


def _plain_append(st, real=torch.float32):
    """Queries rotated, and the two caches (and, in 8 bits, their scales) with the new tokens in them, in place."""
    b, pos, blk, slot = _token_places(st)
    cos, sin = st["cos"][pos].to(real), st["sin"][pos].to(real)
    q = _rotated(st["Q"].to(real), cos, sin, st["interleaved"])
    k, v = _rotated(st["K"].to(real), cos, sin, st["interleaved"]), st["V"].to(real)
    out = [q]
    if st["Ks"] is None:
        for x, cache in ((k, st["Kc"]), (v, st["Vc"])):
            cache[blk, :, slot] = x.to(cache.dtype)
            out.append(cache)
        return out
    # 8 bits. Only the block that a sequence's first new token goes to can hold earlier tokens of it.
    cu, lens, block = st["offsets"].long(), st["lens"].long(), st["Kc"].shape[2]
    start = lens - cu[1:] + cu[:-1]
    blk0, first = st["table"].long()[torch.arange(lens.shape[0], device=lens.device), start // block], start % block
    old_slot = (torch.arange(block, device=lens.device) < first[:, None])[:, None, :, None]
    for x, cache, scales in ((k, st["Kc"], st["Ks"]), (v, st["Vc"], st["Vs"])):
        amax = torch.zeros(scales.shape, dtype=real, device=x.device)
        amax.scatter_reduce_(0, blk[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
        new = _pow2_scale(amax)
        old = scales[blk0].to(real)
        kept = torch.where((first > 0)[:, None], torch.maximum(new[blk0], _pow2_ceil(old)), new[blk0])
        new[blk0] = kept
        raw = cache.view(torch.uint8)
        again = (cache[blk0].to(real) * (old / kept)[:, :, None, None]).to(_F8).view(torch.uint8)
        raw[blk0] = torch.where(old_slot, again, raw[blk0])
        raw[blk, :, slot] = (x / new[blk][..., None]).to(_F8).view(torch.uint8)
        scales[blk] = new[blk].float()
        out += [cache, scales]
    return out


def _plain_attn(st, real=torch.float32):
    q, table = st["Q"].to(real), st["table"].long()
    bq, hq, d = q.shape
    block, h = st["Kc"].shape[2], st["Kc"].shape[1]
    keys = table.shape[1] * block

    def dense(cache, scales):                   # [b, h, keys, d]
        x = cache.view(torch.uint8)[table].view(_F8).to(real) * scales[table].to(real)[..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(bq, h, keys, d)

    qt = q.reshape(bq, h, hq // h, d).transpose(2, 3).contiguous()
    s = torch.matmul(dense(st["Kc"], st["Ks"]), qt) * st["scale"]                       # [b, h, keys, group]
    seen = (torch.arange(keys, device=q.device) < st["lens"].long()[:, None])[:, None, :, None]
    s = torch.where(seen, s, -math.inf)
    top = s.amax(2, keepdim=True).clamp(min=torch.finfo(real).min)
    p = torch.exp(s - top)
    total = p.sum(2)                                                                    # [b, h, group]
    o = torch.matmul(p.transpose(2, 3).contiguous(), dense(st["Vc"], st["Vs"]))
    o = torch.where((total > 0)[..., None], o / total.clamp(min=1e-30)[..., None], 0.0)
    return o.reshape(bq, hq, d)


# ---- the state of a case

def _append_lengths(case):
    """New tokens of each sequence and tokens that it has with them. Before the batch is shuffled: shares of n that
    grow evenly (at least one token each), and what was in the cache from nothing to what is left of s, in turn."""
    b, n, s = case["b"], case["n"], case["s"]
    if case["decode"]:
        new = [1] * b
        return new, [max(1, s // 4 + (s - s // 4) * (i + 1) // b) for i in range(b)]
    edges = [b + (n - b) * (i * (i + 1)) // (b * (b + 1)) - b + i for i in range(b + 1)]
    new = [edges[i + 1] - edges[i] for i in range(b)]
    have = [(s * (i % 4) // 5 + 7 * (i % 4) + (3 * i) % 5 * (i % 2)) for i in range(b)]
    return new, [x + y for x, y in zip(new, have)]


def _attn_lengths(case):
    """Evenly from s/4 to s; the first one nothing where the batch has an idle slot."""
    b, s = case["b"], case["s"]
    lo = max(1, s // 4)
    lens = [s - (s - lo) * i // max(1, b - 1) for i in range(b)]
    return ([0] + lens[1:]) if case["idle"] else lens


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dtype = _DTYPE[case["dtype"]]

    def normal(shape, std=1.0, dt=dtype):
        t = torch.randn(shape, generator=gen, device=dev, dtype=dt)
        return t if std == 1.0 else t.mul_(std)

    def e4m3(shape):                            # N(0, 1) in steps of the middle scale below
        return normal(shape, 64.0, torch.bfloat16).to(_F8)

    def cache_scales(shape):
        return _two_to(torch.randint(-7, -4, shape, generator=gen, device=dev), torch.float32)

    op = case["op"]
    if op == "quant":
        m, k, rows = case["m"], case["k"], case["rows"]
        x = normal((m, k), 1.0 if rows == 1 else 0.02)
        x.mul_(torch.exp(torch.randn((k,), generator=gen, device=dev)).to(dtype))       # channels differ, as activations' do
        return dict(op=op, X=x, rows=rows, Xq=torch.empty((m, k), dtype=_F8, device=dev),
                    S=torch.empty((-(-k // 128), -(-m // rows)), device=dev))
    if op == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        a, sa = _plain_quant(normal((m, k)), 1)
        b, sb = _plain_quant(normal((n, k), 0.02), 128)
        sb = sb * (0.5 + 0.5 * torch.rand(sb.shape, generator=gen, device=dev))         # a checkpoint's scales are any numbers
        return dict(op=op, A=a, Sa=sa, B=b, Sb=sb, C=torch.empty((m, n), dtype=dtype, device=dev))
    b, h, hq, d, block = case["b"], case["h"], case["hq"], case["d"], case["block"]
    order = torch.randperm(b, generator=gen, device=dev)
    if op == "append":
        new, lens = (torch.tensor(x, dtype=torch.int32, device=dev)[order] for x in _append_lengths(case))
        per_seq = -(-(max(_append_lengths(case)[1])) // block)
        n = case["n"]
        # a fused projection's result: query, key and value heads side by side in a row
        rows = normal((n, (hq + 2 * h) * d))
        q, k, v = (t.unflatten(1, (-1, d)) for t in rows.split([hq * d, h * d, h * d], 1))
        r = case["rot"] // 2
        turn = torch.arange(per_seq * block, device=dev, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(r, device=dev, dtype=torch.float64) / r)
        st = dict(op=op, Q=q, K=k, V=v, cos=turn.cos().float(), sin=turn.sin().float(), interleaved=case["interleaved"],
                  offsets=torch.nn.functional.pad(new.cumsum(0), (1, 0)).to(torch.int32), lens=lens.contiguous(),
                  Qo=torch.empty((n, hq, d), dtype=dtype, device=dev), Ks=None, Vs=None)
        shape = (b * per_seq, h, block, d)
        if case["cache"] == "fp8":
            st.update(Kc=e4m3(shape), Vc=e4m3(shape), Ks=cache_scales(shape[:2]), Vs=cache_scales(shape[:2]))
        else:
            st.update(Kc=normal(shape), Vc=normal(shape))
        st["table"] = torch.randperm(b * per_seq, generator=gen, device=dev).to(torch.int32).reshape(b, per_seq).contiguous()
        return st
    lens = torch.tensor(_attn_lengths(case), dtype=torch.int32, device=dev)[order].contiguous()
    per_seq = -(-case["s"] // block)
    nb = b * per_seq
    table = torch.randperm(nb, generator=gen, device=dev).to(torch.int32).reshape(b, per_seq).contiguous()
    q = normal((b, hq, d))
    return dict(op=op, Q=q, Kc=e4m3((nb, h, block, d)), Vc=e4m3((nb, h, block, d)), Ks=cache_scales((nb, h)), Vs=cache_scales((nb, h)),
                table=table, lens=lens, O=torch.empty_like(q), scale=1.0 / math.sqrt(d))


def run(st):
    op = st["op"]
    if own:
        from paper_2503_14985_amd import binding
        if op == "quant":
            return binding.mlt_quant_fp8(st["X"], st["rows"], Xq=st["Xq"], S=st["S"])
        if op == "gemm":
            return binding.mlt_gemm_fp8(st["A"], st["Sa"], st["B"], st["Sb"], C=st["C"])
        if op == "append":
            at = (st["Q"], st["K"], st["V"], st["offsets"], st["lens"], st["table"], st["cos"], st["sin"], st["Kc"], st["Vc"])
            if st["Ks"] is None:
                q = binding.mlt_paged_append(*at, Qo=st["Qo"], interleaved=st["interleaved"])
                return [q, st["Kc"], st["Vc"]]
            q = binding.mlt_paged_append_fp8(*at, st["Ks"], st["Vs"], Qo=st["Qo"], interleaved=st["interleaved"])
            return [q, st["Kc"], st["Ks"], st["Vc"], st["Vs"]]
        return binding.mlt_paged_attn_decode_fp8(st["Q"], st["Kc"], st["Vc"], st["Ks"], st["Vs"], st["table"], st["lens"], st["scale"], O=st["O"])
    if op == "quant":
        return _plain_quant(st["X"], st["rows"])
    if op == "gemm":
        return _plain_gemm(st).to(st["C"].dtype)
    if op == "append":
        out = _plain_append(st)
        return [out[0].to(st["Q"].dtype)] + out[1:]
    return _plain_attn(st).to(st["Q"].dtype)


def work(case):
    op = case["op"]
    if op == "quant":
        m, k = case["m"], case["k"]
        return dict(bytes=3 * m * k + 4 * -(-k // 128) * -(-m // case["rows"]), flops=2.0 * m * k)
    if op == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // 128)
        return dict(bytes=(m + n) * k + 4 * kb * (m + -(-n // 128)) + 2 * m * n, flops=2.0 * m * n * k)
    b, h, hq, d, block = (case[x] for x in ("b", "h", "hq", "d", "block"))
    if op == "append":
        n, elem = case["n"], 1 if case["cache"] == "fp8" else 2
        new, lens = _append_lengths(case)
        blocks = sum((e - 1) // block - (e - x) // block + 1 for x, e in zip(new, lens))
        # rows read, queries and cache rows written, an angle's cosine and sine for each token, block numbers, scales read and written
        return dict(bytes=2 * n * d * (2 * hq + 2 * h) + 2 * n * h * d * elem + 4 * n * case["rot"] + 4 * blocks + 8 * b
                    + (8 * blocks * h if elem == 1 else 0), flops=3.0 * n * case["rot"] * (hq + h))
    lens = _attn_lengths(case)
    keys, blocks = sum(lens), sum(-(-x // block) for x in lens)
    return dict(bytes=2 * keys * h * d + 8 * blocks * h + 4 * b * hq * d + 4 * (b + blocks), flops=4.0 * keys * hq * d)


# ---- by the definitions, in 64 bits

def _power(e):
    """2.0 ** e of whole numbers held as doubles, from a table."""
    return torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device=e.device)[e.long() + 200]


def _least_scale(top):
    """The smallest power of two s >= 2^-100 with top <= 448 s; the logarithm is put right where it rounded."""
    e = torch.ceil(torch.log2(top / _F8_MAX)).clamp(-100, 199)
    e = torch.where(_F8_MAX * _power(e) < top, e + 1, e)
    e = torch.where((_F8_MAX * _power(e - 1) >= top) & (e > -100), e - 1, e)
    return _power(e)


def _e4m3_value(x):
    """x rounded to the nearest number of e4m3 (ties to even), as a double."""
    _, e = torch.frexp(x)
    step = _power((e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_quant(st):
    x, rows = st["X"].double(), st["rows"]
    m, k = x.shape
    q, scales = torch.empty_like(x), torch.empty(st["S"].shape, dtype=torch.float64, device=x.device)
    for i in range(scales.shape[0]):            # a strip of 128 columns at a time
        strip = x[:, 128 * i:128 * i + 128]
        top = torch.stack([p.abs().max() for p in strip.split(rows)]) if rows > 1 else strip.abs().amax(1)
        s = _least_scale(top)
        scales[i] = s
        each = s if rows == 1 else s.repeat_interleave(rows)[:m]
        q[:, 128 * i:128 * i + 128] = _e4m3_value(strip / each[:, None])
    return [q, scales]


def _exact_gemm(st):
    a, b, sa, sb = st["A"].double(), st["B"].double(), st["Sa"].double(), st["Sb"].double()
    c = torch.zeros((a.shape[0], b.shape[0]), dtype=torch.float64, device=a.device)
    for i in range(sa.shape[0]):
        part = a[:, 128 * i:128 * i + 128] @ b[:, 128 * i:128 * i + 128].t().contiguous()
        c += part * sa[i][:, None] * sb[i].repeat_interleave(128)[None, :b.shape[0]]
    return c


def _exact_append(st):
    cu, lens, table = (st[x].tolist() for x in ("offsets", "lens", "table"))
    block, pairs = st["Kc"].shape[2], st["cos"].shape[1]
    where = [(s, p) for s in range(len(lens)) for p in range(lens[s] - cu[s + 1] + cu[s], lens[s])]
    pos = torch.tensor([p for _, p in where], device=st["Q"].device)
    unit = torch.complex(st["cos"].double()[pos], st["sin"].double()[pos])[:, None]

    def turned(x):
        x = x.double().clone()
        lead = x[..., :2 * pairs]
        z = torch.view_as_complex(lead.unflatten(-1, (pairs, 2)).contiguous()) if st["interleaved"] else torch.complex(lead[..., :pairs].contiguous(), lead[..., pairs:].contiguous())
        z = z * unit
        x[..., :2 * pairs] = torch.stack((z.real, z.imag), -1 if st["interleaved"] else -2).flatten(-2)
        return x

    out = [turned(st["Q"])]
    blk = torch.tensor([table[s][p // block] for s, p in where], device=pos.device)
    for x, cache, scales in ((turned(st["K"]), st["Kc"], st["Ks"]), (st["V"].double(), st["Vc"], st["Vs"])):
        held = cache.double()
        if scales is None:
            held[blk, :, pos % block] = x
            out.append(held)
            continue
        tops = torch.zeros(scales.shape, dtype=torch.float64, device=x.device).index_reduce_(0, blk, x.abs().amax(-1), "amax")
        s = _least_scale(tops)
        now = scales.double()
        touched = torch.zeros(scales.shape[0], dtype=torch.bool, device=x.device)
        touched[blk] = True
        for b in range(len(lens)):              # the block that the first new token shares with earlier ones
            begin = lens[b] - cu[b + 1] + cu[b]
            j, used = table[b][begin // block], begin % block
            if used:
                s[j] = torch.maximum(s[j], _least_scale(now[j] * _F8_MAX))
                held[j, :, :used] = _e4m3_value(held[j, :, :used] * (now[j] / s[j])[:, None, None])
        held[blk, :, pos % block] = _e4m3_value(x / s[blk][..., None])
        out += [held, torch.where(touched[:, None], s, now)]
    return out


def _exact_attn(st):
    lens, block = st["lens"].tolist(), st["Kc"].shape[2]
    out = torch.zeros(st["Q"].shape, dtype=torch.float64, device=st["Q"].device)
    h = st["Kc"].shape[1]
    for b, n in enumerate(lens):
        if n == 0:
            continue
        blocks = st["table"][b, :-(-n // block)].long()

        def rows(cache, scales):                # [h, n, d]
            x = cache.view(torch.uint8)[blocks].view(_F8).double() * scales[blocks].double()[:, :, None, None]
            return x.transpose(0, 1).reshape(h, -1, x.shape[3])[:, :n]

        q = st["Q"][b].double().unflatten(0, (h, -1))
        w = torch.softmax(torch.matmul(q, rows(st["Kc"], st["Ks"]).transpose(1, 2).contiguous()) * st["scale"], -1)
        out[b] = torch.matmul(w, rows(st["Vc"], st["Vs"])).flatten(0, 1)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"quant": _exact_quant, "gemm": _exact_gemm, "append": _exact_append, "attn": _exact_attn}[st["op"]](st)
