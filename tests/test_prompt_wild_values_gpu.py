"""Attention of packed and paged prompts over many values that are not finite: every element is what the values that its row sees make of it (an infinity, NaN, or a finite number), and a call
takes a time of its usual order, not one that working out row after row by itself would take."""
import math

import pytest
import torch

from prompt_util import HALF, attend, cache_of, check, ends, ints, limits, normal, tolerance

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16
HOW = {"channel": "one element of every value +inf", "all": "all +inf", "some": "here and there +inf, -inf and NaN", "late": "NaN in the last value", "signs": "+inf and -inf in turn in some elements"}


@pytest.fixture(scope="module")
def binding():
    from paper_2503_14985_amd import binding as b
    return b


def spoil(V, how, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if how == "channel":
        V[..., 5] = math.inf
    elif how == "all":
        V[:] = math.inf
    elif how == "some":
        u = torch.rand(V.shape, generator=g, device="cuda")
        V[u < 0.004] = math.inf
        V[u > 0.996] = -math.inf
        V[(u > 0.5) & (u < 0.501)] = math.nan
    elif how == "late":
        V[-1] = math.nan
    else:
        V[0::2, :, 7] = math.inf
        V[1::2, :, 7] = -math.inf
        V[::5, :, 9] = -math.inf


def verify(O, Q, K, V, scale, limit, what):
    """Finite elements against the definition in 64 bits, the others by the kinds of values seen."""
    H, Hq = K.shape[1], Q.shape[1]
    seen = torch.arange(K.shape[0], device="cuda")[None] < torch.tensor(limit, device="cuda")[:, None]
    o, c = attend(Q, K, torch.where(torch.isfinite(V), V, 0), scale, limit)
    has = {}
    for name, at in (("pos", V == math.inf), ("neg", V == -math.inf), ("nan", V.isnan())):
        has[name] = torch.stack([(seen.float() @ at[:, h * H // Hq].float()) > 0 for h in range(Hq)], 1)
    bad = has["nan"] | (has["pos"] & has["neg"])
    any_wild = bad | has["pos"] | has["neg"]
    assert torch.equal(O.isnan(), bad), what + ": NaN where %d, should be %d" % (int(O.isnan().sum()), int(bad.sum()))
    assert torch.equal(O == math.inf, has["pos"] & ~bad) and torch.equal(O == -math.inf, has["neg"] & ~bad), what
    tol = tolerance(o, c, Q.shape[2], Q.dtype, HALF[Q.dtype], moves=K.shape[0] // 64 + 1)
    check(torch.where(any_wild, torch.zeros_like(O), O), torch.where(any_wild, 0.0, o), tol + (any_wild * 1.0), what)


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["causal", "full", "paged"])
@pytest.mark.parametrize("how", list(HOW))
def test_every_element(binding, how, kind, D, dtype):
    Hq, H, block = 8, 2, 16
    for batch in ([(40, 40), (150, 150), (1, 70), (90, 200), (20, 7)], [(30, 2600)]):
        new, lens = [n for n, _ in batch], [m for _, m in batch]
        cu, ku = ends(new), ends(lens)
        Q, K, V = normal(1, (cu[-1], Hq, D), dtype), normal(2, (ku[-1], H, D), dtype), normal(3, (ku[-1], H, D), dtype)
        for b in range(len(batch)):
            spoil(V[ku[b]:ku[b + 1]], how, b)
        scale = 1.0 / math.sqrt(D)
        if kind == "paged":
            Kc, Vc, table = cache_of(4, lens, H, D, block, dtype)
            for b, m in enumerate(lens):
                for i, blk in enumerate(table[b, :-(-m // block)].tolist()):
                    for cache, rows in ((Kc, K), (Vc, V)):
                        part = rows[ku[b] + i * block:min(ku[b] + (i + 1) * block, ku[b + 1])]
                        cache[blk, :, :part.shape[0]] = part.transpose(0, 1)
            O = binding.mlt_paged_attn_prompt(Q, Kc, Vc, ints(cu), ints(lens), table, scale)
        else:
            O = binding.mlt_mha_packed_fwd(Q, K, V, ints(cu), ints(ku), scale, causal=kind != "full")
        assert ("parts" in binding.mlt_last_kernel()) == (len(batch) == 1)
        for b, (n, m) in enumerate(batch):
            verify(O[cu[b]:cu[b + 1]], Q[cu[b]:cu[b + 1]], K[ku[b]:ku[b + 1]], V[ku[b]:ku[b + 1]], scale, limits(n, m, kind != "full"), "%s, %s, sequence %d" % (HOW[how], kind, b))


@pytest.mark.parametrize("n, m", [(100, 100), (30, 2600)], ids=["whole", "keys_split"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_are_not_finite(binding, D, n, m):
    """A NaN among the keys that a row sees makes all of the row NaN, also beside infinities that it sees and others that it does not."""
    K, V, Q = normal(1, (m, 2, D), BF), normal(2, (m, 2, D), BF), normal(3, (n, 4, D), BF)
    at = m - n + 20
    K[at] = math.nan
    V[..., 3] = math.inf
    O = binding.mlt_mha_packed_fwd(Q, K, V, ints([0, n]), ints([0, m]), 0.1)
    assert bool(O[20:].isnan().all())
    assert bool((O[:20, :, 3] == math.inf).all()) and int(torch.isfinite(O[:20]).sum()) == 20 * 4 * (D - 1)


def test_time(binding):
    """4096 tokens: 0.15 ms of finite values. One channel of infinities took 106 ms with every row worked out again."""
    T = 4096
    Q, K, V = normal(1, (T, 32, 128), FP), normal(2, (T, 8, 128), FP), normal(3, (T, 8, 128), FP)
    V[..., 3] = math.inf
    times = []
    for _ in range(3):
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        O = binding.mlt_mha_packed_fwd(Q, K, V, ints([0, T]), None, 0.1)
        stop.record()
        torch.cuda.synchronize()
        times.append(start.elapsed_time(stop))
    assert bool((O[..., 3] == math.inf).all()) and int(torch.isfinite(O).sum()) == T * 32 * 127
    assert min(times) < 20.0, times
