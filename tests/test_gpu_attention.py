"""The paged cache and attention over it, against their formulas in 64 bits on the CPU.

Tolerances, with u = 2^-24.  A value rounded to bfloat16 is off by 2^-8 of itself at most.

Rotation: the fraction of a turn is rounded to fp32 (off by 2^-26 of a turn at most, and the positions here, times frequencies up to 1, add nothing in 64 bits), which is
2 pi 2^-26 < 2^-23 in the sine and cosine, whose own error is below 2^-22; two products and a sum add 2 u of them each.  In all less than 2^-20 (|a| + |b|),
before the rounding to bfloat16.

Attention: a score is a sum of d exact products in fp32, in any order off by 2 d u of the sum of their sizes (2 u: adders that cut off), times the scale, which adds 2 u of
the score, and log2 e another; taking off the maximum and the exponential add 4 u of the score's size, which is at most that sum, and 4 u.  So a weight is off
by E = (2 d + 12) u S + 4 u of itself, S the largest scaled sum of sizes, and it is rounded to bfloat16 (2^-8) for the product with the values.  The sums over n keys
are off by 2 n u of the sums of sizes; scaling them to another maximum adds u each time, less than n u in all.  The output is a quotient of two such sums: off by
(2 E (1 + E) + 2^-8 + 8 n u + 16 u) A, A the weighted mean of |v|, and its own rounding, 2^-8 of itself.

That bound is loose where many keys are seen.  So what is seen is tested with queries of zeros: all weights are 1, and the output is the mean of whole numbers, whose
sum is exact: off by the reciprocal's rounding and a product's (4 u), and the rounding to bfloat16.
"""
import math

import numpy as np
import pytest
import torch

from paper_2504_02692_amd import binding as B
from tests.test_gpu_serving import bf16, f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = 2.0 ** -8 * (1 + 2.0 ** -6)
TINY = 2.0 ** -133


class Cache:
    """Random sequences, (new tokens, tokens before them) each, in pages anywhere; everything that no sequence has is NaN."""

    def __init__(self, pairs, kv_heads, d, page, seed=0, wider=1, missing=(), spare=3):
        self.r = r = np.random.default_rng([seed, kv_heads, d, page, len(pairs)])
        self.pairs, self.kv, self.d, self.page = pairs, kv_heads, d, page
        used = [-(-max(c + b, 0) // page) for c, b in pairs]
        pages = sum(used) + spare
        ids = r.permutation(pages)
        self.table = np.full((len(pairs), max(used + [0]) + wider), -1, np.int32)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = ids[at:at + u]
            at += u
        self.table[:, max(used + [0]):] = 2 ** 31 - 1                # (behind every sequence: never looked at, or no page)
        for s, i in missing:
            self.table[s, i] = -1 if i % 2 else pages
        self.starts = np.concatenate([[0], np.cumsum([c for c, _ in pairs])]).astype(np.int32)
        self.lengths = np.array([c + b for c, b in pairs], np.int32)
        self.tokens = int(self.starts[-1])
        self.pages = pages
        self.k = [self.values((max(c + b, 0), kv_heads, d)) for c, b in pairs]
        self.v = [self.values((max(c + b, 0), kv_heads, d)) for c, b in pairs]

    def values(self, shape):
        return torch.from_numpy(self.r.standard_normal(shape)).to(torch.bfloat16).double().numpy()

    def arrays(self):
        """(keys, values) as 64-bit arrays, NaN where there is nothing."""
        page, d = self.page, self.d
        keys = np.full((self.pages, self.kv, d // 8, page, 8), np.nan)
        values = np.full((self.pages, self.kv, page // 8, d, 8), np.nan)
        for s in range(len(self.pairs)):
            for p in range(len(self.k[s])):
                id = self.table[s, p // page]
                if 0 <= id < self.pages:
                    keys[id, :, :, p % page] = self.k[s][p].reshape(self.kv, d // 8, 8)
                    values[id, :, p % page // 8, :, p % 8] = self.v[s][p]
        return keys, values

    def device(self):
        keys, values = self.arrays()
        return dict(keys=bf16(keys), values=bf16(values), table=torch.from_numpy(self.table).cuda(), starts=torch.from_numpy(self.starts).cuda(),
                    lengths=torch.from_numpy(self.lengths).cuda())

    def here(self, s):
        """Whether the positions of sequence s have a page."""
        ids = self.table[s][np.arange(len(self.k[s])) // self.page] if len(self.k[s]) else np.zeros(0, int)
        return (ids >= 0) & (ids < self.pages)


def seen(c, s, window, sinks):
    """(new tokens x positions) truth values."""
    count, before = c.pairs[s]
    p, j = np.arange(before, before + count)[:, None], np.arange(len(c.k[s]))[None, :]
    see = (j <= p) & c.here(s)[None, :]
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def workspace(tokens, seqs, heads, kv, d):
    ws = B.workspace(B.gptaq_attention_workspace_bytes(tokens, seqs, heads, kv, d))
    ws.fill_(255)                                                    # (NaN)
    return ws


def queries(c, heads, d, scale=2.0, extra=0):
    q = bf16(c.r.standard_normal((c.tokens, heads, d)) * scale)
    if not extra:
        return q
    rows = torch.full((c.tokens + 1, heads * d + extra), float("nan"), dtype=torch.bfloat16, device="cuda")
    v = rows.view(-1)[extra // 2:extra // 2 + c.tokens * (heads * d + extra)].view(c.tokens, -1)[:, :heads * d].view(c.tokens, heads, d)
    v.copy_(q)
    return v


def check(got, c, q, heads, window, sinks, scale=None):
    d, group = c.d, heads // c.kv
    scale = d ** -0.5 if scale is None else scale
    got, q = f64(got), f64(q)
    worst = 0.0
    for s, (count, before) in enumerate(c.pairs):
        rows = slice(c.starts[s], c.starts[s + 1])
        see = seen(c, s, window, sinks)
        n = see.shape[1]
        for h in range(heads):
            k, v = c.k[s][:, h // group], c.v[s][:, h // group]
            logit = np.where(see, q[rows, h] @ k.T * scale, -np.inf)
            top = logit.max(1, initial=-np.inf, keepdims=True)
            w = np.exp(logit - np.where(np.isfinite(top), top, 0.0))
            total = np.maximum(w.sum(1, keepdims=True), 1e-300)
            want, size = w @ v / total, w @ np.abs(v) / total
            S = (np.where(see, np.abs(q[rows, h]) @ np.abs(k).T, 0.0) * abs(scale)).max(1, initial=0.0, keepdims=True)
            E = (2 * d + 12) * U * S + 4 * U
            tol = (2 * E * (1 + E) + HALF + 8 * n * U + 16 * U) * size * (1 + 2.0 ** -5) + np.abs(want) * HALF + TINY
            err = np.abs(got[rows, h] - want)
            assert np.all(err <= tol), (s, h, float(np.nanmax(err / tol)), np.argwhere(~(err <= tol))[:4].tolist())
            worst = max(worst, float((err / tol).max(initial=0.0)))
    return worst


def run(pairs, heads, kv, d, page, window=0, sinks=0, extra=0, scale=None, **more):
    print("attention", pairs, heads, kv, d, page, window, sinks, extra, more, flush=True)
    c = Cache(pairs, kv, d, page, **more)
    q = queries(c, heads, d, extra=extra)
    dev = c.device()
    ws = workspace(c.tokens, len(pairs), heads, kv, d)
    whole = torch.full((c.tokens + 2, heads + 1, d + extra), 7.0, dtype=torch.bfloat16, device="cuda")
    out = whole[1:-1, :heads, :d]
    y = B.gptaq_attention(q, **dev, ws=ws, window=window, sinks=sinks, scale=scale, out=out)
    check(y, c, q, heads, window, sinks, scale)
    assert torch.all(whole[0] == 7.0) and torch.all(whole[-1] == 7.0) and torch.all(whole[:, heads:] == 7.0) and torch.all(whole[:, :, d:] == 7.0)
    # what is seen: the mean of whole numbers
    for s in range(len(pairs)):
        c.v[s] = 2.0 * c.r.integers(-8, 8, c.v[s].shape) + 1.0
    dev = c.device()
    y = f64(B.gptaq_attention(torch.zeros_like(q), **dev, ws=ws, window=window, sinks=sinks, scale=scale))
    for s in range(len(pairs)):
        see = seen(c, s, window, sinks).astype(np.float64)
        for h in range(heads):
            want = see @ c.v[s][:, h // (heads // kv)] / np.maximum(see.sum(1, keepdims=True), 1.0)
            err = np.abs(y[c.starts[s]:c.starts[s + 1], h] - want)
            tol = np.abs(want) * (HALF + 4 * U)
            assert np.all(err <= tol), (s, h, np.argwhere(~(err <= tol))[:4].tolist())


STEPS = [  # (new, before) of the sequences, heads, kv_heads, window, sinks
    ([(1, 0)], 1, 1, 0, 0), ([(1, 1)], 4, 4, 0, 0), ([(1, 15), (1, 16), (1, 17)], 8, 2, 0, 0), ([(1, 62), (1, 63), (1, 64), (1, 65)], 8, 1, 0, 0),
    ([(1, 500), (1, 3), (0, 40), (1, 129)], 6, 2, 0, 0), ([(1, 700)], 32, 32, 100, 4), ([(1, 700), (1, 90), (1, 2)], 8, 2, 64, 0), ([(1, 300)], 3, 1, 1, 0),
    ([(1, 300)], 3, 1, 1, 1), ([(1, 900)], 16, 2, 65, 130), ([(1, 900)], 16, 1, 200, 900), ([(0, 0), (1, 5), (0, 0)], 2, 1, 0, 0),
    ([(3, 200), (1, 0), (5, 77)], 8, 2, 0, 0), ([(2, 200), (4, 30)], 24, 1, 40, 7), ([(1, 3000)], 8, 8, 0, 0), ([(1, 2500), (1, 40)], 40, 1, 0, 0),
]


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("pairs,heads,kv,window,sinks", STEPS)
def test_steps(pairs, heads, kv, window, sinks, d, page):
    run(pairs, heads, kv, d, page, window, sinks)


PROMPTS = [
    ([(2, 0)], 1, 1, 0, 0), ([(17, 0)], 2, 2, 0, 0), ([(64, 0), (65, 0)], 4, 1, 0, 0), ([(130, 0), (1, 0), (31, 0)], 3, 1, 0, 0), ([(300, 0)], 2, 1, 50, 0),
    ([(257, 100), (40, 33)], 8, 2, 64, 3), ([(200, 500)], 4, 4, 128, 70), ([(333, 0), (0, 9), (90, 1), (5, 700)], 6, 2, 100, 4), ([(513, 0)], 1, 1, 0, 0),
    ([(256, 256)], 8, 1, 1, 0), ([(600, 3)], 2, 2, 1, 64), ([(129, 1000)], 5, 1, 0, 0), ([(400, 0)], 4, 2, 399, 1),
]


@pytest.mark.parametrize("page", [32, 128])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("pairs,heads,kv,window,sinks", PROMPTS)
def test_prompts(pairs, heads, kv, window, sinks, d, page):
    run(pairs, heads, kv, d, page, window, sinks)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("pairs", [[(1, 260), (1, 7)], [(150, 60), (33, 0)]])
def test_pages_and_strides(pairs, page):
    run(pairs, 4, 2, 64, page, extra=8)
    run(pairs, 4, 2, 96, page, 70, 5, extra=3)                       # rows that start at any element
    run(pairs, 6, 1, 128, page, extra=1, scale=-0.3, wider=0)


@pytest.mark.parametrize("pairs", [[(1, 260), (1, 100)], [(150, 60), (33, 100)]])
def test_pages_that_are_not_there(pairs):
    """Given back: nothing there is seen, and what lies in page 0 or in others is not read for it."""
    run(pairs, 4, 2, 64, 16, missing=[(0, 0), (0, 3), (1, 2)])
    run(pairs, 4, 2, 128, 32, missing=[(0, 0), (0, 1), (1, 0)])
    run(pairs, 4, 2, 96, 64, 20, 3, missing=[(0, 0)])
    run(pairs, 2, 2, 64, 256, missing=[(0, 0), (1, 0)])              # nothing at all


def test_lengths_that_are_less_than_the_new_tokens():
    """Tokens with positions below 0 see nothing; those of no sequence are left alone."""
    c = Cache([(5, -2), (4, -4), (3, 10)], 1, 64, 16)
    q = queries(c, 2, 64)
    out = torch.full((c.tokens, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    B.gptaq_attention(q, **c.device(), ws=workspace(c.tokens, 3, 2, 1, 64), out=out)
    check(out, c, q, 2, 0, 0)
    assert torch.all(out[:2] == 0) and torch.all(out[5:9] == 0)
    dev = c.device()
    dev["starts"] = torch.tensor([1, 4, 4, 6], dtype=torch.int32, device="cuda")
    out.fill_(7.0)
    B.gptaq_attention(q, **dev, ws=workspace(c.tokens, 3, 2, 1, 64), out=out)
    assert torch.all(out[0] == 7.0) and torch.all(out[6:] == 7.0) and not torch.any(out[1:6] == 7.0)


@pytest.mark.parametrize("starts,lengths", [([0, 9, 4], [9, 9]), ([-5, 3, 1 << 30], [1 << 30, -7]), ([4, 2, 0], [2 ** 31 - 1, 2 ** 31 - 1]), ([7, 7, 7], [0, 0])])
def test_arrays_that_make_no_sense_stay_inside(starts, lengths):
    """Positions and rows are bounded by the kernels themselves, whatever the arrays on the device hold: the calls end, and write nothing but their outputs."""
    c = Cache([(4, 30), (3, 50)], 2, 64, 16)
    dev = c.device()
    dev["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    dev["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    for many in (1, 40):
        q = bf16(np.ones((7 * many, 4, 64)))
        B.gptaq_attention(q, **dev, ws=workspace(7 * many, 2, 4, 2, 64))
        kv = bf16(np.ones((7 * many, 2, 64)))
        B.gptaq_cache_append(q, kv, kv, **dev, freqs=None)
        torch.cuda.synchronize()


def plain_from(dev, c, q, heads, window=0, sinks=0):
    """The formula on the cache as it is on the device, in 64 bits, with what it says of infinities and NaN."""
    keys, values = f64(dev["keys"]), f64(dev["values"])
    group, out = heads // c.kv, np.zeros((c.tokens, heads, c.d))
    q = f64(q)
    for s in range(len(c.pairs)):
        see = seen(c, s, window, sinks)
        for t in range(c.pairs[s][0]):
            js = np.flatnonzero(see[t])
            ids, slots = c.table[s][js // c.page], js % c.page
            for h in range(heads):
                k = keys[ids, h // group, :, slots].reshape(len(js), c.d)
                v = values[ids, h // group, slots // 8, :, slots % 8]
                with np.errstate(invalid="ignore"):
                    logit = k @ q[c.starts[s] + t, h] * c.d ** -0.5
                    w = np.exp(logit - logit.max())
                    out[c.starts[s] + t, h] = (w[:, None] * v).sum(0) / w.sum()
    return out


@pytest.mark.parametrize("pairs", [[(3, 150)], [(200, 37)], [(90, 0), (1, 200)]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 3)])
def test_infinities_and_nan_reach_those_who_see_them(pairs, window, sinks):
    """A value of a position, or an entry of its key, that is not finite: tokens that see it have what the formula says, the others' outputs do not change."""
    c = Cache(pairs, 2, 64, 16, seed=5)
    q = queries(c, 4, 64, scale=0.5)
    clean = c.device()
    ws = workspace(c.tokens, len(pairs), 4, 2, 64)
    base = B.gptaq_attention(q, **clean, ws=ws, window=window, sinks=sinks)
    count, before = pairs[0]
    n = count + before
    for kind, bad in (("values", float("inf")), ("values", -float("inf")), ("values", float("nan")), ("keys", float("nan"))):
        for j in sorted({1, n // 2, n - 20, n - 2, n - 1}):
            dev = {k: v.clone() for k, v in clean.items()}
            id, slot = int(c.table[0, j // 16]), j % 16
            if kind == "values":
                dev["values"][id, 1, slot // 8, 5, slot % 8] = bad
                if j == n - 2:                                       # both infinities seen by the last token alone
                    dev["values"][id if (n - 1) // 16 == j // 16 else int(c.table[0, (n - 1) // 16]), 1, (n - 1) % 16 // 8, 5, (n - 1) % 8] = -bad
            else:
                dev["keys"][id, 1, 2, slot, 3] = bad
            y = B.gptaq_attention(q, **dev, ws=ws, window=window, sinks=sinks)
            want = plain_from(dev, c, q, 4, window, sinks)
            got = f64(y)
            odd = ~np.isfinite(want)
            assert np.array_equal(got[odd], want[odd], equal_nan=True), (kind, bad, j)
            same = torch.from_numpy(~odd).cuda()
            assert torch.equal(y[same], base[same]), (kind, bad, j)


def test_large_scores():
    """Scores that differ by thousands, with either sign, in whatever order: no overflow, and no part of a row is lost."""
    for pairs in ([(1, 400)], [(80, 200)]):
        c = Cache(pairs, 1, 64, 16, seed=9)
        for s in range(len(pairs)):
            grow = c.r.permutation(np.linspace(-300, 300, len(c.k[s])))
            c.k[s] = torch.from_numpy(c.k[s] * 0.01 + grow[:, None, None] / 8).to(torch.bfloat16).double().numpy()
        for sign in (1.0, -1.0, 50.0):
            q = bf16(np.full((c.tokens, 2, 64), sign))
            got = B.gptaq_attention(q, **c.device(), ws=workspace(c.tokens, 1, 2, 1, 64))
            check(got, c, q, 2, 0, 0)


@pytest.mark.parametrize("pairs", [[(1, 300)], [(150, 150)]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 3)])
def test_a_scale_of_zero_weighs_all_alike(pairs, window, sinks):
    """Whatever the sums of products are (2^123 here, of either sign): each key that is seen has the same weight."""
    c = Cache(pairs, 1, 64, 16, seed=11)
    c.k[0][:] = np.where(np.arange(len(c.k[0])) % 3 == 0, 2.0 ** 62, -(2.0 ** 62))[:, None, None]
    c.v[0] = 2.0 * c.r.integers(-8, 8, c.v[0].shape) + 1.0
    q = bf16(np.full((c.tokens, 2, 64), 2.0 ** 55))
    see = seen(c, 0, window, sinks).astype(np.float64)
    want = see @ c.v[0][:, 0] / see.sum(1, keepdims=True)
    for scale in (0.0, -0.0, 2.0 ** -149):               # (the last: exponents of 2^-26, weights within as much of 1, values up to 15)
        got = f64(B.gptaq_attention(q, **c.device(), ws=workspace(c.tokens, 1, 2, 1, 64), window=window, sinks=sinks, scale=scale))
        tol = np.abs(want) * (HALF + 4 * U) + 32 * 2.0 ** -26 * (scale != 0.0)
        assert np.all(np.abs(got[:, 0] - want) <= tol) and np.array_equal(got[:, 0], got[:, 1]), scale


@pytest.mark.parametrize("pairs", [[(1, 300)], [(150, 150)]])
def test_scores_near_the_ends_of_fp32(pairs):
    """Scores of 1e33 and more, of either sign: one key that stands out has all the weight, and equal scores have equal weights."""
    c = Cache(pairs, 1, 64, 16, seed=10)
    n = len(c.k[0])
    c.k[0][:] = -(2.0 ** 53)
    for s in range(len(pairs)):
        c.v[s] = 2.0 * c.r.integers(-8, 8, c.v[s].shape) + 1.0
    q = bf16(np.full((c.tokens, 2, 64), 2.0 ** 53))
    ws = workspace(c.tokens, 1, 2, 1, 64)
    see = seen(c, 0, 0, 0).astype(np.float64)
    got = f64(B.gptaq_attention(q, **c.device(), ws=ws))
    want = see @ c.v[0][:, 0] / see.sum(1, keepdims=True)
    assert np.all(np.abs(got[:, 0] - want) <= np.abs(want) * (HALF + 4 * U)) and np.array_equal(got[:, 0], got[:, 1])
    c.k[0][37] = 2.0 ** 53
    got = f64(B.gptaq_attention(q, **c.device(), ws=ws))
    assert np.array_equal(got[see[:, 37] > 0], np.broadcast_to(c.v[0][37], got[see[:, 37] > 0].shape))


@pytest.mark.parametrize("pairs", [[(1, 120), (1, 70)], [(120, 100), (100, 33)]])
def test_shared_pages_and_tables_in_wider_arrays(pairs):
    """Sequences with the same first pages, and a table whose rows are parts of longer ones."""
    c = Cache(pairs, 2, 64, 16, seed=12)
    shared = min(before for _, before in pairs) // 16                # (whole pages in front of the new tokens)
    c.table[1, :shared] = c.table[0, :shared]
    c.k[1][:shared * 16], c.v[1][:shared * 16] = c.k[0][:shared * 16], c.v[0][:shared * 16]
    dev = c.device()
    wide = torch.full((2, c.table.shape[1] + 9), -1, dtype=torch.int32, device="cuda")
    dev["table"] = wide[:, 4:4 + c.table.shape[1]]
    dev["table"].copy_(torch.from_numpy(c.table))
    q = queries(c, 4, 64)
    ws = workspace(c.tokens, 2, 4, 2, 64)
    check(B.gptaq_attention(q, **dev, ws=ws), c, q, 4, 0, 0)
    k = bf16(c.r.standard_normal((c.tokens, 2, 64)))
    before = dev["keys"].clone()
    B.gptaq_cache_append(q, k, k, **dev, freqs=None)                  # (new tokens are behind the shared pages)
    for s, (count, first) in enumerate(c.pairs):
        p = first + count - 1
        id = int(c.table[s, p // 16])
        assert torch.equal(dev["keys"][id, :, :, p % 16].reshape(2, 64), k[c.starts[s + 1] - 1])
    for id in c.table[0, :shared]:
        assert torch.equal(dev["keys"][id].view(torch.int16), before[id].view(torch.int16))


@pytest.mark.parametrize("tokens", [1, 300])
def test_no_pages_and_no_table(tokens):
    empty = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    one = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    q = bf16(np.ones((tokens, 4, 64)))
    ws = workspace(tokens, 1, 4, 2, 64)
    table = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    for keys, values, t in ((empty(0, 2, 8, 16, 8), empty(0, 2, 2, 64, 8), table), (empty(5, 2, 8, 16, 8), empty(5, 2, 2, 64, 8), table[:, :0])):
        y = B.gptaq_attention(q, keys, values, t, one(0, tokens), one(tokens), ws)
        assert torch.all(y == 0)
        assert torch.equal(B.gptaq_cache_append(q, q[:, :2], q[:, 2:], keys, values, t, one(0, tokens), one(tokens), None), q)
    assert B.gptaq_attention(q, keys, values, table[:0], one(0), table[0, :0], ws).shape == q.shape


def test_two_graphs_that_share_a_workspace():
    """A prompt's and a step's attention, captured with one workspace and replayed in turn with eager calls between."""
    cases = []
    ws = workspace(300, 2, 8, 2, 128)
    for pairs in ([(200, 700), (100, 5)], [(1, 900), (1, 77)]):
        c = Cache(pairs, 2, 128, 16, seed=len(cases))
        q, out = queries(c, 8, 128), torch.empty((c.tokens, 8, 128), dtype=torch.bfloat16, device="cuda")
        dev = c.device()
        B.gptaq_attention(q, **dev, ws=ws, out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.gptaq_attention(q, **dev, ws=ws, out=out)
        cases.append((c, q, dev, out, graph))
    for k in range(3):
        for c, q, dev, out, graph in cases:
            q.copy_(queries(c, 8, 128))
            graph.replay()
        torch.cuda.synchronize()
        for c, q, dev, out, graph in cases:
            got = out.clone()
            assert torch.equal(B.gptaq_attention(q, **dev, ws=ws), got), k
            check(got, c, q, 8, 0, 0)


def test_many_sequences():
    """More than a wavefront tries at once, empty ones among them."""
    r = np.random.default_rng(11)
    pairs = [(int(r.integers(0, 3)), int(r.integers(0, 60))) for _ in range(300)]
    run(pairs, 4, 2, 64, 16)
    run([(0, 3)] * 70 + [(1, 5)] + [(0, 0)] * 130 + [(2, 90)], 2, 1, 64, 32, 8, 2)


def test_offsets_past_32_bits():
    """A cache of 5 GiB, its sequence in the last pages and the first."""
    page, kv, d = 256, 8, 128
    pages = 5 * 2 ** 30 // (page * kv * d * 2)
    c = Cache([(1, 700), (30, 520)], kv, d, page, spare=0)
    keys, values = (bf16(a) for a in c.arrays())
    big_k = torch.empty((pages, kv, d // 8, page, 8), dtype=torch.bfloat16, device="cuda")
    big_v = torch.empty((pages, kv, page // 8, d, 8), dtype=torch.bfloat16, device="cuda")
    where = [pages - 1, 0, pages - 2, 1, pages // 2, pages - 7][:c.pages]
    for i, w in enumerate(where):
        big_k[w], big_v[w] = keys[i], values[i]
    dev = c.device()
    table = torch.full_like(dev["table"], -1)
    for i, w in enumerate(where):
        table[dev["table"] == i] = w
    dev.update(keys=big_k, values=big_v, table=table)
    q = queries(c, 8, d)
    check(B.gptaq_attention(q, **dev, ws=workspace(c.tokens, 2, 8, kv, d)), c, q, 8, 0, 0)
    k, v = (bf16(c.r.standard_normal((c.tokens, kv, d))) for _ in range(2))
    B.gptaq_cache_append(q, k, v, **dev, freqs=None)
    for s, (count, before) in enumerate(c.pairs):
        for t in (0, count - 1):
            p = before + t
            id = int(table[s, p // page])
            assert torch.equal(big_k[id, :, :, p % page].reshape(kv, d), k[c.starts[s] + t]) and torch.equal(big_v[id, :, p % page // 8, :, p % 8], v[c.starts[s] + t])


# ---- the cache

def turned(x, positions, freqs, interleaved):
    """(rotated, |a| + |b| of each entry's pair)."""
    half = len(freqs)
    y, size = x.copy(), np.zeros_like(x)
    ang = positions[:, None, None].astype(np.float64) * freqs
    cos, sin = np.cos(ang), np.sin(ang)
    i, j = (np.arange(half) * 2, np.arange(half) * 2 + 1) if interleaved else (np.arange(half), half + np.arange(half))
    a, b = x[..., i], x[..., j]
    y[..., i], y[..., j] = a * cos - b * sin, b * cos + a * sin
    size[..., i] = size[..., j] = np.abs(a) + np.abs(b)
    return y, size


def append_case(pairs, heads, kv, d, page, pairs_of=None, interleaved=False, one_row=False, missing=(), in_place=False, far=0, wider=1):
    print("append", pairs, heads, kv, d, page, pairs_of, interleaved, one_row, missing, in_place, flush=True)
    half = d // 2 if pairs_of is None else pairs_of
    c = Cache(pairs, kv, d, page, missing=missing, wider=wider)
    dev = c.device()
    freqs = 10000.0 ** (-np.arange(half) / max(half, 1))
    rows = bf16(c.r.standard_normal((c.tokens + 1, (heads + 2 * kv) * d + (5 if one_row else 0))))[:c.tokens]
    q, k, v = (rows[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    if not one_row:
        q, k, v = q.contiguous(), k.contiguous(), v.transpose(0, 1).contiguous().transpose(0, 1)
    before_q, before_k, before_v = f64(q), f64(k), f64(v)
    keys, values = dev["keys"].view(torch.int16).cpu().numpy().copy(), dev["values"].view(torch.int16).cpu().numpy().copy()
    out = q if in_place else None
    y = B.gptaq_cache_append(q, k, v, **dev, freqs=torch.from_numpy(freqs).cuda() if half else None, interleaved=interleaved, out=out)
    assert not in_place or y is q
    got_k, got_v = f64(dev["keys"]), f64(dev["values"])
    y = f64(y)
    touched_k, touched_v = np.zeros(keys.shape, bool), np.zeros(values.shape, bool)
    for s, (count, before) in enumerate(pairs):
        p = np.arange(before, before + count)
        here = slice(c.starts[s], c.starts[s + 1])
        want, size = turned(before_q[here], p, freqs, interleaved)
        ok = p >= 0
        assert np.all(np.abs(y[here] - want)[ok] <= (size * 2.0 ** -20 + np.abs(want) * HALF)[ok])
        want, size = turned(before_k[here], p, freqs, interleaved)
        for t in np.flatnonzero(ok):
            id = c.table[s, p[t] // page]
            if not 0 <= id < c.pages:
                continue
            slot = p[t] % page
            assert np.all(np.abs(got_k[id, :, :, slot].reshape(kv, d) - want[t]) <= size[t] * 2.0 ** -20 + np.abs(want[t]) * HALF)
            assert np.array_equal(got_v[id, :, slot // 8, :, slot % 8], before_v[here][t])
            touched_k[id, :, :, slot] = touched_v[id, :, slot // 8, :, slot % 8] = True
    assert np.array_equal(dev["keys"].view(torch.int16).cpu().numpy()[~touched_k], keys[~touched_k])
    assert np.array_equal(dev["values"].view(torch.int16).cpu().numpy()[~touched_v], values[~touched_v])


@pytest.mark.parametrize("one_row", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pairs,heads,kv,d,page,half", [
    ([(1, 0)], 1, 1, 16, 16, None), ([(1, 5), (1, 7), (1, 8), (1, 200)], 8, 2, 64, 16, None), ([(7, 0), (9, 3), (0, 5), (16, 8)], 3, 1, 96, 16, 24),
    ([(40, 13), (1, 0)], 4, 4, 128, 32, 32), ([(300, 70)], 2, 2, 128, 64, None), ([(65, 0), (33, 31)], 6, 2, 64, 256, 8), ([(20, 3)], 2, 1, 256, 128, None),
    ([(20, 3)], 2, 1, 80, 16, 0), ([(1, 4000), (1, 100)], 64, 8, 128, 16, None), ([(5, -2), (4, -4), (3, 10)], 2, 1, 64, 16, None)])
def test_append(pairs, heads, kv, d, page, half, interleaved, one_row):
    append_case(pairs, heads, kv, d, page, half, interleaved, one_row)


def test_append_in_place_and_where_pages_are_missing():
    append_case([(33, 20), (1, 60)], 4, 2, 64, 16, in_place=True, one_row=True)
    append_case([(33, 20), (1, 60)], 4, 2, 64, 16, missing=[(0, 2), (1, 3)])
    append_case([(33, 20)], 4, 2, 64, 16, wider=0)


def test_append_of_many_sequences():
    r = np.random.default_rng(12)
    append_case([(int(r.integers(0, 4)), int(r.integers(0, 30))) for _ in range(200)], 2, 1, 32, 16)


def test_far_positions():
    """Angles of far positions keep their fraction of a turn."""
    page, d = 256, 64
    table_pages = 4096
    positions = np.array([1048575, 1000003, 262144, 77777])
    keys = torch.zeros((4, 1, d // 8, page, 8), dtype=torch.bfloat16, device="cuda")
    values = torch.zeros((4, 1, page // 8, d, 8), dtype=torch.bfloat16, device="cuda")
    table = torch.full((4, table_pages), -1, dtype=torch.int32, device="cuda")
    for s, p in enumerate(positions):
        table[s, p // page] = s
    r = np.random.default_rng(2)
    q, k, v = bf16(r.standard_normal((4, 2, d))), bf16(r.standard_normal((4, 1, d))), bf16(r.standard_normal((4, 1, d)))
    freqs = 1.0 * 10000.0 ** (-np.arange(32) / 32)
    y = B.gptaq_cache_append(q, k, v, keys, values, table, torch.arange(5, dtype=torch.int32, device="cuda"), torch.from_numpy((positions + 1).astype(np.int32)).cuda(),
                             torch.from_numpy(freqs).cuda())
    want, size = turned(f64(q), positions, freqs, False)
    assert np.all(np.abs(f64(y) - want) <= size * 2.0 ** -20 + np.abs(want) * HALF)
    want, size = turned(f64(k), positions, freqs, False)
    for s, p in enumerate(positions):
        assert np.all(np.abs(f64(keys[s, 0, :, p % page]).reshape(d) - want[s, 0]) <= size[s, 0] * 2.0 ** -20 + np.abs(want[s, 0]) * HALF)


def test_captured_steps_on_a_stream_of_their_own():
    """Append and attention of a growing cache, captured once and replayed while lengths grow, against eager calls on copies."""
    heads, kv, d, page, seqs, width = 4, 2, 64, 16, 3, 20
    r = np.random.default_rng(8)
    keys = torch.zeros((seqs * width, kv, d // 8, page, 8), dtype=torch.bfloat16, device="cuda")
    values = torch.zeros((seqs * width, kv, page // 8, d, 8), dtype=torch.bfloat16, device="cuda")
    table = torch.from_numpy(r.permutation(seqs * width).reshape(seqs, width).astype(np.int32)).cuda()
    starts = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    lengths = torch.tensor([1, 40, 200], dtype=torch.int32, device="cuda")
    freqs = torch.from_numpy(10000.0 ** (-np.arange(d // 2) / (d // 2))).cuda()
    rows = torch.zeros((seqs, (heads + 2 * kv) * d), dtype=torch.bfloat16, device="cuda")
    parts = [rows[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv))]
    ws = workspace(seqs, seqs, heads, kv, d)
    out, turned_q = torch.empty((seqs, heads, d), dtype=torch.bfloat16, device="cuda"), torch.empty((seqs, heads, d), dtype=torch.bfloat16, device="cuda")

    def step(keys, values, ws, out, turned_q):
        B.gptaq_cache_append(*parts, keys, values, table, starts, lengths, freqs, out=turned_q)
        return B.gptaq_attention(turned_q, keys, values, table, starts, lengths, ws, window=64, sinks=4, out=out)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(keys, values, ws, out, turned_q)
    torch.cuda.synchronize()
    eager = keys.clone(), values.clone(), workspace(seqs, seqs, heads, kv, d), torch.empty_like(out), torch.empty_like(out)
    for _ in range(5):
        rows.copy_(bf16(r.standard_normal(rows.shape)))
        graph.replay()
        torch.cuda.synchronize()
        want = step(*eager)
        assert torch.equal(out, want) and torch.equal(keys, eager[0]) and torch.equal(values, eager[1])
        lengths += torch.tensor([17, 1, 3], dtype=torch.int32, device="cuda")


def test_the_same_bits_every_time():
    for pairs, heads, kv in (([(1, 3000), (1, 90)], 8, 2), ([(300, 700), (20, 0)], 8, 2)):
        c = Cache(pairs, kv, 128, 16)
        q = queries(c, heads, 128)
        dev, ws = c.device(), workspace(c.tokens, 2, heads, kv, 128)
        first = B.gptaq_attention(q, **dev, ws=ws)
        for _ in range(3):
            ws.fill_(255)
            assert torch.equal(B.gptaq_attention(q, **dev, ws=ws), first)
    assert B.gptaq_attention(q[:0], **dict(dev, starts=dev["starts"] * 0), ws=ws).shape == (0, heads, 128)


def test_thousands_of_sequences():
    """More than two searches of 64 find: most of them empty or of a token, in whatever order."""
    r = np.random.default_rng(17)
    for seqs, busy in ((4097, 60), (5000, 200), (10000, 90)):
        pairs = [(0, 0)] * seqs
        for s in {0, seqs - 1, *r.choice(seqs, busy, replace=False).tolist()}:
            pairs[s] = (int(r.integers(0, 3)), int(r.integers(0, 70)))
        pairs[seqs - 2] = (9, 40)
        run(pairs, 2, 1, 64, 16)
        append_case(pairs, 2, 1, 32, 16)
    run([(1, int(b)) for b in r.integers(0, 20, 4500)], 2, 1, 64, 16)
    append_case([(1, int(b)) for b in r.integers(0, 20, 4500)], 2, 1, 16, 16)


def test_the_output_may_be_the_queries_memory():
    """With parts and a join, without, and in rows that are parts of longer ones."""
    for pairs, heads, kv, extra in (([(1, 3000), (1, 5)], 8, 2, 0), ([(1, 30), (2, 20), (0, 3)], 8, 2, 6), ([(40, 100), (1, 7)], 6, 2, 0)):
        c = Cache(pairs, kv, 64, 16)
        q, dev, ws = queries(c, heads, 64, extra=extra), c.device(), workspace(c.tokens, len(pairs), heads, kv, 64)
        want = B.gptaq_attention(q, **dev, ws=ws)
        assert B.gptaq_attention(q, **dev, ws=ws, out=q) is q and torch.equal(q, want)


@pytest.mark.parametrize("pairs", [[(1, 300), (3, 20)], [(150, 150)]])
def test_scores_of_minus_infinity_weigh_nothing(pairs):
    """Where a token sees no others, zeros, as for one that sees nothing.  One of infinity makes NaN."""
    c = Cache(pairs, 2, 64, 16, seed=14)
    for s in range(len(pairs)):
        c.k[s][::3, 0, 7] = -np.inf
        c.k[s][:, 1, 9] = -np.inf
    q = queries(c, 4, 64)
    q[..., 7] = q[..., 9] = 1.0
    dev, ws = c.device(), workspace(c.tokens, len(pairs), 4, 2, 64)
    y = B.gptaq_attention(q, **dev, ws=ws)
    assert torch.all(y[:, 2:] == 0)
    for s in range(len(pairs)):                                      # scores so low that they weigh nothing
        c.k[s][::3, 0] = np.where(np.arange(64) == 7, -(2.0 ** 40), 0.0)
        c.k[s][:, 1] = 0.0
    see = f64(B.gptaq_attention(q, **c.device(), ws=ws))
    assert np.array_equal(f64(y)[:, :2], see[:, :2])
    c.k[0][0, 0, 7] = np.inf
    y = B.gptaq_attention(q, **c.device(), ws=ws)
    assert torch.all(torch.isnan(y[:c.pairs[0][0], :2])) and not torch.any(torch.isnan(y[c.pairs[0][0]:])) and not torch.any(torch.isnan(y[:, 2:]))


@pytest.mark.parametrize("pairs", [[(1, 8000), (1, 30)], [(150, 300)]])
def test_values_of_2_to_the_100(pairs):
    """Sums of weights of up to 2^8 a key stay inside fp32 for them."""
    c = Cache(pairs, 2, 64, 16, seed=15)
    for s in range(len(pairs)):
        c.v[s] = c.v[s] * 2.0 ** 100
    q = queries(c, 4, 64, scale=8.0)
    check(B.gptaq_attention(q, **c.device(), ws=workspace(c.tokens, len(pairs), 4, 2, 64)), c, q, 4, 0, 0)
