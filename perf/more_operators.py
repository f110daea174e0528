"""Operators of serving prompts as measured cases, beside their plain forms.

What a serving program calls between the products of a layer, and for those products when the weights are in 4 bits:
  packed   mlt_mha_packed_fwd:            attention of packed sequences of different lengths, grouped heads, causal or not
  prompt   mlt_paged_attn_prompt:         the same for the newest tokens of sequences whose keys are in the paged cache
  decode   mlt_paged_attn_decode_prefix:  one query a sequence, over a prefix that all share and keys of its own, both in the paged cache
  w4       mlt_gemm_w4:                   few rows times a matrix of 4-bit weights with a scale for every group

`listed()` holds the fixed cases, `draw(rng)` gives further ones of the same ranges, `prepare(case, seed)` makes what a program
holds before the call, `run(state)` is the call, `work(case)` the bytes and flops that no implementation can do without and
`exact(case, seed)` the result by the operator's definition in 64 bits. With `own` false, `run` computes the plain form in
elementary torch operations in 32 bits; with `own` true it calls the library.

A case is a dict of plain values. `op` is one of the names above; `dtype` is the type of the 16-bit tensors.
  packed   b sequences, t query tokens in all, up to s keys of each sequence in front of its queries' own, hq query and h key/value heads of d, causal
  prompt   b sequences, t new tokens in all (mixed: one sequence has all but one each for the others), up to s tokens of each in the cache
           before them, hq, h, d, block (slots of a cache block)
  decode   b sequences, p tokens of prefix, up to s of their own behind it, hq, h, d, block, idle (the first one of the batch is empty)
  w4       m, n, k, group, zeros (a zero point for every group instead of 8)
"""
import math

import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # One short question: the smallest call of a prompt's attention, latency alone.
        dict(name="packed_short", op="packed", b=1, t=33, s=0, hq=32, h=8, d=128, causal=True, dtype="bf16"),
        # A prefill step: prompts of ragged length side by side, four query heads to a key/value head.
        dict(name="packed_batch", op="packed", b=13, t=8191, s=0, hq=32, h=8, d=128, causal=True, dtype="bf16"),
        # A batch of passages through an encoder: no mask, as many key/value heads as query heads.
        dict(name="packed_encoder", op="packed", b=24, t=6000, s=0, hq=16, h=16, d=64, causal=False, dtype="fp16"),
        # One long prompt whose keys have just been appended to the cache: the largest.
        dict(name="prompt_long", op="prompt", b=1, t=8192, s=0, mixed=False, hq=32, h=8, d=128, block=16, dtype="bf16"),
        # Prompts in pieces: the next pieces of four prompts over what the cache has of them already.
        dict(name="prompt_pieces", op="prompt", b=4, t=2048, s=8192, mixed=False, hq=32, h=8, d=128, block=32, dtype="fp16"),
        # A mixed step: a piece of one prompt and the next tokens of 31 other sequences in one call.
        dict(name="prompt_mixed", op="prompt", b=32, t=543, s=4096, mixed=True, hq=32, h=8, d=128, block=16, dtype="bf16"),
        # A few continuations of one short shared prompt: latency.
        dict(name="decode_few", op="decode", b=4, p=1000, s=100, hq=16, h=16, d=64, block=16, idle=False, dtype="fp16"),
        # A serving batch behind one long system prompt, one slot of the batch idle.
        dict(name="decode_batch", op="decode", b=64, p=8192, s=512, hq=32, h=8, d=128, block=16, idle=True, dtype="bf16"),
        # Many samples of one long document: almost all keys are shared.
        dict(name="decode_samples", op="decode", b=250, p=32001, s=128, hq=32, h=8, d=128, block=64, idle=False, dtype="bf16"),
        # The next token of one sequence through an attention projection: latency, and the weight once.
        dict(name="w4_token", op="w4", m=1, n=4096, k=4096, group=128, zeros=False, dtype="bf16"),
        # Next tokens of a batch through a large feed-forward weight.
        dict(name="w4_ffn", op="w4", m=16, n=28672, k=8192, group=128, zeros=False, dtype="bf16"),
        # A larger batch against a narrow matrix with fine groups and zero points, a number of rows that does not fill its tile.
        dict(name="w4_batch", op="w4", m=57, n=4100, k=14336, group=32, zeros=True, dtype="fp16"),
    ]


def _log(rng, lo, hi, mult=1):
    """An integer of [lo, hi], even over its logarithm, a multiple of `mult`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))
    return max(lo, min(hi, int(v) // mult * mult))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    op = rng.choice(["packed", "packed", "prompt", "prompt", "decode", "decode", "w4", "w4"])
    if op == "w4":
        while True:
            m, n, k = _log(rng, 1, 64), _log(rng, 256, 28672), _log(rng, 256, 14336, 32)
            if n * k <= 28672 * 8192:
                break
        if rng.random() < 0.6:                   # most layers' sizes are multiples of 128
            n, k = max(256, n // 128 * 128), max(256, k // 128 * 128)
        return dict(op=op, m=m, n=n, k=k, group=rng.choice([32, 64, 128, 128]), zeros=rng.random() < 0.4, dtype=dtype)
    d, h = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8, 8, 16])
    hq = h * rng.choice([1, 2, 3, 4, 4, 8])
    block = rng.choice([16, 16, 32, 48, 64, 128])
    if op == "decode":
        while True:
            b, p, s = _log(rng, 1, 256), _log(rng, 16, 32768), _log(rng, 1, 4096)
            if b * (p + s) * hq * d <= 250 * 32129 * 32 * 128 and b * s * h * d <= 64 * 4096 * 8 * 128:
                return dict(op=op, b=b, p=p, s=s, hq=hq, h=h, d=d, block=block, idle=rng.random() < 0.2, dtype=dtype)
    while True:
        b, t, s = _log(rng, 1, 64), _log(rng, 1, 8192), rng.choice([0, 0, _log(rng, 16, 8192)])
        mixed = op == "prompt" and rng.random() < 0.3
        case = dict(op=op, b=b, t=max(t, b), s=s, hq=hq, h=h, d=d, dtype=dtype)
        case.update(dict(mixed=mixed, block=block) if op == "prompt" else dict(causal=rng.random() < 0.7))
        new, lens = _prompt_lengths(case)
        pairs = sum(x * (y if not case.get("causal", True) else y - x / 2) for x, y in zip(new, lens))
        if pairs * hq * d <= 8192 * 4096 * 32 * 128 and b * max(new) * max(lens) * hq <= 4e9 and sum(lens) * h * d <= 1 << 28:
            return case


# ---- lengths

def _prompt_lengths(case):
    """Query tokens of each sequence and the keys that it has with them. Shares of t that grow evenly (or, mixed, all but one each for the others),
    at least one token each; in front of them from nothing to s keys, in turn."""
    b, t, s = case["b"], case["t"], case["s"]
    if case.get("mixed"):
        new = [1] * (b - 1) + [t - (b - 1)]
    else:
        edges = [(t - b) * (i * (i + 1)) // (b * (b + 1)) + i for i in range(b + 1)]
        new = [edges[i + 1] - edges[i] for i in range(b)]
    have = [s - s * ((5 * i) % 7) // 7 for i in range(b)]
    return new, [x + y for x, y in zip(new, have)]


def _decode_lengths(case):
    """Keys of each sequence: the prefix and from s/4 to s of its own, evenly; the first one nothing where the batch has an idle slot."""
    b, p, s = case["b"], case["p"], case["s"]
    lo = max(1, s // 4)
    lens = [p + s - (s - lo) * i // max(1, b - 1) for i in range(b)]
    return ([0] + lens[1:]) if case["idle"] else lens


# ---- the state of a case

def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dtype = _DTYPE[case["dtype"]]

    def normal(shape, dt=dtype):
        return torch.randn(shape, generator=gen, device=dev, dtype=dt)

    op = case["op"]
    if op == "w4":
        m, n, k, group = case["m"], case["n"], case["k"], case["group"]
        groups = -(-k // group)
        st = dict(op=op, A=normal((m, k)), group=group, Z=None, C=torch.empty((m, n), dtype=dtype, device=dev))
        w = torch.nn.functional.pad(normal((n, k), torch.float32).mul_(0.02), (0, groups * group - k)).view(n, groups, group)
        if case["zeros"]:                        # a checkpoint's asymmetric groups: from the smallest to the largest weight
            lo, hi = w.amin(2).clamp(max=0.0), w.amax(2).clamp(min=0.0)
            s = ((hi - lo) / 15).to(dtype)
            z = (-lo / s.float()).round().clamp(0, 15)
            st["Z"] = z.t().to(torch.uint8).contiguous()
        else:
            s = (w.abs().amax(2) / 7).to(dtype)
            z = torch.full_like(s, 8.0, dtype=torch.float32)
        q = (w / s.float()[..., None]).round_().add_(z[..., None]).clamp_(0, 15).to(torch.uint8).view(n, -1)[:, :k]
        st["Wq"] = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()
        st["S"] = s.t().contiguous()
        return st
    b, hq, h, d = case["b"], case["hq"], case["h"], case["d"]
    order = torch.randperm(b, generator=gen, device=dev)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    def ends(x):
        return torch.nn.functional.pad(x.cumsum(0), (1, 0)).to(torch.int32)

    scale = 1.0 / math.sqrt(d)
    if op == "decode":
        p, block = case["p"], case["block"]
        lens = _decode_lengths(case)
        first, per_seq = p // block, -(-max(lens) // block)          # blocks that are the prefix's alone; blocks of the longest sequence
        mine = per_seq - first                                      # of which each sequence has these for itself (the prefix's last keys in a copy)
        shared = -(-p // block)
        nb = shared + b * mine
        place = torch.randperm(nb, generator=gen, device=dev).to(torch.int32)
        table = torch.cat((place[:first].expand(b, first), place[shared:].view(b, mine)), 1).contiguous()
        q = normal((b, hq, d))
        return dict(op=op, Q=q, Kc=normal((nb, h, block, d)), Vc=normal((nb, h, block, d)), prefix=place[:shared].contiguous(), p=p, table=table,
                    lens=ints(lens)[order].contiguous(), longest=max(lens), scale=scale, O=torch.empty_like(q))
    new, lens = _prompt_lengths(case)
    st = dict(op=op, mq=max(new), mk=max(lens), scale=scale, causal=case.get("causal", True))
    new, lens = ints(new)[order], ints(lens)[order].contiguous()
    st.update(offsets=ends(new), lens=lens)
    t = case["t"]
    if op == "packed":
        if case["s"] == 0:                       # a fused projection's result: query, key and value heads side by side in a row
            rows = normal((t, (hq + 2 * h) * d))
            st["Q"], st["K"], st["V"] = (x.unflatten(1, (-1, d)) for x in rows.split([hq * d, h * d, h * d], 1))
            st["k_offsets"] = st["offsets"]
        else:
            total = sum(_prompt_lengths(case)[1])
            st["Q"], st["K"], st["V"] = normal((t, hq, d)), normal((total, h, d)), normal((total, h, d))
            st["k_offsets"] = ends(lens)
    else:
        block = case["block"]
        per_seq = -(-st["mk"] // block)
        st["Q"] = normal((t, hq, d))
        st["Kc"], st["Vc"] = normal((b * per_seq, h, block, d)), normal((b * per_seq, h, block, d))
        st["table"] = torch.randperm(b * per_seq, generator=gen, device=dev).to(torch.int32).reshape(b, per_seq).contiguous()
    st["O"] = torch.empty((t, hq, d), dtype=dtype, device=dev)
    return st


# ---- the plain forms, in 32 bits

def _attend(q, k, v, seen, scale):
    """q [b, h, rows, d], k and v [b, h, keys, d], seen [b, 1, rows, keys]; rows that see nothing give zeros."""
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).masked_fill_(~seen, -math.inf)
    s = s.sub_(s.amax(3, keepdim=True).clamp(min=torch.finfo(s.dtype).min)).exp_()
    total = s.sum(3, keepdim=True)
    o = torch.matmul(s, torch.where(seen.any(2)[..., None], v, 0.0))
    return torch.where(total > 0, o / total.clamp(min=1e-30), 0.0)


def _plain_prompt(st):
    cu, lens = st["offsets"].long(), st["lens"].long()
    q = st["Q"].float()
    t, hq, d = q.shape
    b, mq, mk = lens.shape[0], st["mq"], st["mk"]
    dev = q.device
    i, j = torch.arange(mq, device=dev), torch.arange(mk, device=dev)
    n = cu[1:] - cu[:-1]
    rows = (cu[:-1, None] + i).clamp(max=t - 1)                                         # [b, mq]
    if st["op"] == "packed":
        at = (st["k_offsets"].long()[:-1, None] + j).clamp(max=st["K"].shape[0] - 1)
        k, v = (st[x].float()[at].transpose(1, 2) for x in ("K", "V"))                  # [b, h, mk, d]
    else:
        block = st["Kc"].shape[2]
        blk = st["table"].long()[:, j // block]
        k, v = (st[x].float()[blk, :, (j % block)[None]].transpose(1, 2) for x in ("Kc", "Vc"))
    h = k.shape[1]
    g = hq // h
    qd = q[rows].view(b, mq, h, g, d).permute(0, 2, 3, 1, 4).reshape(b, h, g * mq, d)
    seen = (j < lens[:, None])[:, None, :].expand(b, mq, mk)
    if st["causal"]:
        seen = seen & (j <= (lens - n)[:, None, None] + i[None, :, None])
    o = _attend(qd, k, v, seen[:, None].expand(b, g, mq, mk).reshape(b, 1, g * mq, mk), st["scale"])
    o = o.view(b, h, g, mq, d).permute(0, 3, 1, 2, 4).reshape(b, mq, hq, d)
    which = torch.searchsorted(cu[1:], torch.arange(t, device=dev), right=True)
    return o[which, torch.arange(t, device=dev) - cu[which]]


def _plain_decode(st):
    """The prefix with the queries of all sequences as rows, then each sequence's own keys; one softmax over both."""
    q, lens, p, block = st["Q"].float(), st["lens"].long(), st["p"], st["Kc"].shape[2]
    b, hq, d = q.shape
    h = st["Kc"].shape[1]
    g = hq // h
    dev = q.device
    j = torch.arange(p, device=dev)
    kp, vp = (st[x][st["prefix"].long()[j // block], :, j % block].float().transpose(0, 1).contiguous() for x in ("Kc", "Vc"))     # [h, p, d]
    j = torch.arange(p, st["longest"], device=dev)
    ko, vo = (st[x][st["table"].long()[:, j // block], :, (j % block)[None]].float().transpose(1, 2) for x in ("Kc", "Vc"))         # [b, h, own, d]
    qg = q.view(b, h, g, d)
    sp = torch.matmul(qg.transpose(0, 1).reshape(h, b * g, d), kp.transpose(1, 2).contiguous()).view(h, b, g, p).transpose(0, 1)
    so = torch.matmul(qg, ko.transpose(2, 3).contiguous())
    seen = (torch.arange(st["longest"], device=dev) < lens[:, None])[:, None, None]
    s = torch.cat((sp, so), 3).mul_(st["scale"]).masked_fill_(~seen, -math.inf)
    s = s.sub_(s.amax(3, keepdim=True).clamp(min=torch.finfo(s.dtype).min)).exp_()
    total = s.sum(3, keepdim=True)
    wp = s[..., :p].transpose(0, 1).reshape(h, b * g, p)
    o = torch.matmul(wp, vp).view(h, b, g, d).transpose(0, 1) + torch.matmul(s[..., p:], vo)
    return torch.where(total > 0, o / total.clamp(min=1e-30), 0.0).reshape(b, hq, d)


def _plain_w4(st):
    q = torch.stack((st["Wq"] & 15, st["Wq"] >> 4), 2).flatten(1).float()
    k, group = q.shape[1], st["group"]

    def spread(x):
        return x.float().t().repeat_interleave(group, 1)[:, :k]

    return st["A"].float() @ ((q - (8.0 if st["Z"] is None else spread(st["Z"]))) * spread(st["S"])).t()


def run(st):
    op = st["op"]
    if own:
        from paper_2503_14985_amd import binding
        if op == "packed":
            return binding.mlt_mha_packed_fwd(st["Q"], st["K"], st["V"], st["offsets"], st["k_offsets"], st["scale"], causal=st["causal"], O=st["O"])
        if op == "prompt":
            return binding.mlt_paged_attn_prompt(st["Q"], st["Kc"], st["Vc"], st["offsets"], st["lens"], st["table"], st["scale"], O=st["O"])
        if op == "decode":
            return binding.mlt_paged_attn_decode_prefix(st["Q"], st["Kc"], st["Vc"], st["prefix"], st["p"], st["table"], st["lens"], st["scale"], O=st["O"])
        return binding.mlt_gemm_w4(st["A"], st["Wq"], st["S"], st["Z"], group=st["group"], C=st["C"])
    if op == "w4":
        return _plain_w4(st).to(st["C"].dtype)
    return (_plain_decode(st) if op == "decode" else _plain_prompt(st)).to(st["O"].dtype)


def work(case):
    op = case["op"]
    if op == "w4":
        m, n, k = case["m"], case["n"], case["k"]
        groups = -(-k // case["group"])
        return dict(bytes=n * k / 2 + groups * n * (3 if case["zeros"] else 2) + 2 * m * k + 2 * m * n, flops=2.0 * m * n * k)
    b, hq, h, d = (case[x] for x in ("b", "hq", "h", "d"))
    if op == "decode":
        lens, p, block = _decode_lengths(case), case["p"], case["block"]
        mine = sum(max(0, x - p) for x in lens)
        blocks = -(-p // block) + sum(-(-x // block) - p // block for x in lens if x > p)
        return dict(bytes=4 * (p + mine) * h * d + 4 * b * hq * d + 4 * (b + blocks), flops=4.0 * d * hq * sum(lens))
    new, lens = _prompt_lengths(case)
    pairs = sum(x * y - (x * (x - 1) // 2 if case.get("causal", True) else 0) for x, y in zip(new, lens))
    blocks = sum(-(-x // case["block"]) for x in lens) if op == "prompt" else 0
    return dict(bytes=4 * case["t"] * hq * d + 4 * sum(lens) * h * d + 4 * (2 * b + 2 + blocks), flops=4.0 * d * hq * pairs)


# ---- by the definitions, in 64 bits

def _softmax_rows(q, k, v, scale, limit):
    """q [n, d], k and v [m, d]: row i over the keys 0 .. limit[i] - 1."""
    out = torch.zeros((q.shape[0], v.shape[1]), dtype=torch.float64, device=q.device)
    for r in range(0, q.shape[0], 2048):
        lim = limit[r:r + 2048]
        top = int(lim.max()) if lim.numel() else 0
        if top <= 0:
            continue
        x = (q[r:r + 2048].double() @ k[:top].double().t().contiguous()) * scale
        gone = torch.arange(top, device=q.device)[None, :] >= lim[:, None]
        w = torch.softmax(x.masked_fill(gone, -1e300), 1).masked_fill(gone, 0.0)
        out[r:r + 2048] = w @ v[:top].double()
    return out


def _exact_attention(st):
    cu, lens = st["offsets"].tolist(), st["lens"].tolist()
    hq = st["Q"].shape[1]
    out = torch.zeros(st["Q"].shape, dtype=torch.float64, device=st["Q"].device)
    for b, m in enumerate(lens):
        n = cu[b + 1] - cu[b]
        if st["op"] == "packed":
            k0 = st["k_offsets"].tolist()[b]
            k, v = (st[x][k0:k0 + m] for x in ("K", "V"))
        else:
            blocks = st["table"][b, :-(-m // st["Kc"].shape[2])].long()
            k, v = (st[x][blocks].transpose(1, 2).flatten(0, 1)[:m] for x in ("Kc", "Vc"))
        limit = torch.arange(m - n + 1, m + 1, device=out.device) if st["causal"] else torch.full((n,), m, device=out.device)
        for q in range(hq):
            kv = q * k.shape[1] // hq
            out[cu[b]:cu[b + 1], q] = _softmax_rows(st["Q"][cu[b]:cu[b + 1], q], k[:, kv], v[:, kv], st["scale"], limit)
    return out


def _exact_decode(st):
    block, p, h = st["Kc"].shape[2], st["p"], st["Kc"].shape[1]
    out = torch.zeros(st["Q"].shape, dtype=torch.float64, device=st["Q"].device)

    def rows(cache, blocks, lo, hi):            # [h, hi - lo, d]
        return cache[blocks.long()].transpose(0, 1).flatten(1, 2)[:, lo:hi].double()

    shared = [rows(st[x], st["prefix"], 0, p) for x in ("Kc", "Vc")]
    for b, n in enumerate(st["lens"].tolist()):
        if n == 0:
            continue
        at = p // block
        mine = [rows(st[x], st["table"][b, at:-(-n // block)], p - at * block, n - at * block) for x in ("Kc", "Vc")]
        k, v = (torch.cat((x, y), 1) for x, y in zip(shared, mine))
        q = st["Q"][b].double().unflatten(0, (h, -1))
        w = torch.softmax(torch.matmul(q, k.transpose(1, 2).contiguous()) * st["scale"], -1)
        out[b] = torch.matmul(w, v).flatten(0, 1)
    return out


def _exact_w4(st):
    a, wq, group = st["A"].double(), st["Wq"], st["group"]
    c = torch.zeros((a.shape[0], wq.shape[0]), dtype=torch.float64, device=a.device)
    for i in range(st["S"].shape[0]):           # a group of columns of the weight at a time
        part = wq[:, i * group // 2:(i + 1) * group // 2].int()
        z = 8 if st["Z"] is None else st["Z"][i].int()[:, None]
        even, odd = ((part % 16) - z).double(), ((part // 16) - z).double()
        ai = a[:, i * group:(i + 1) * group]
        c += (ai[:, 0::2] @ even.t().contiguous() + ai[:, 1::2] @ odd.t().contiguous()) * st["S"][i].double()
    return c


def exact(case, seed):
    st = prepare(case, seed)
    return {"packed": _exact_attention, "prompt": _exact_attention, "decode": _exact_decode, "w4": _exact_w4}[st["op"]](st)
