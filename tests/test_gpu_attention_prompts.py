"""Attention with enough heads that calls take blocks of many rows, at the sizes, masks and pages where these can go wrong; tolerances as in test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from paper_2504_02692_amd import binding as B
from tests.test_gpu_attention import HALF, PROMPTS, U, Cache, bf16, check, f64, queries, run, seen, workspace

pytestmark = pytest.mark.gpu


def times(pairs, heads, kv, page, window=0, sinks=0, wider=1, table_pages=None):
    """How often the heads have to be there for blocks of many rows: the blocks of 16 rows, times their tiles and nine, pass 22000."""
    tokens, group = sum(c for c, _ in pairs), heads // kv
    assert tokens * group > 16 * len(pairs)
    width = max(-(-(c + b) // page) for c, b in pairs) + wider if table_pages is None else table_pages
    tiles = -(-width * page // 64)
    if window:
        tiles = min(tiles, window // 64 + sinks // 64 + 4)
    return 22000 // (max(-(-tokens * group // 16), len(pairs)) * kv * (tiles + 9)) + 1


def run_many(pairs, heads, kv, d, page, window=0, sinks=0, wider=1, **more):
    m = times(pairs, heads, kv, page, window, sinks, wider)
    run(pairs, heads * m, kv * m, d, page, window, sinks, wider=wider, **more)


@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 128), (128, 16)])
@pytest.mark.parametrize("pairs,heads,kv,window,sinks", [p for p in PROMPTS if sum(c for c, _ in p[0]) * (p[1] // p[2]) > 16 * len(p[0])])
def test_prompts(pairs, heads, kv, window, sinks, d, page):
    run_many(pairs, heads, kv, d, page, window, sinks)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_pages_and_strides(page):
    pairs = [(150, 60), (33, 0)]
    run_many(pairs, 4, 2, 64, page, extra=8)
    run_many(pairs, 4, 2, 96, page, 70, 5, extra=3)                  # rows that start at any element
    run_many(pairs, 6, 1, 128, page, extra=1, scale=-0.3, wider=0)


def test_pages_that_are_not_there():
    pairs = [(150, 60), (33, 100)]
    run_many(pairs, 4, 2, 64, 16, missing=[(0, 0), (0, 3), (1, 2)])
    run_many(pairs, 4, 2, 128, 32, missing=[(0, 0), (0, 1), (1, 0)])
    run_many(pairs, 4, 2, 96, 64, 20, 3, missing=[(0, 0)])
    run_many(pairs, 2, 2, 64, 256, missing=[(0, 0), (1, 0)])         # nothing at all


def test_long_rows_in_parts():
    """Few blocks of many rows: their keys are taken in parts, and joined."""
    for pairs, heads, kv, d, page, window, sinks in (([(128, 9000)], 20, 20, 64, 64, 0, 0), ([(100, 6000), (60, 100)], 24, 12, 128, 16, 0, 0),
                                                    ([(128, 6000)], 60, 30, 96, 32, 3000, 700)):
        assert times(pairs, heads, kv, page, window, sinks) == 1
        run(pairs, heads, kv, d, page, window, sinks)


def test_lengths_that_are_less_than_the_new_tokens():
    """Tokens with positions below 0 see nothing; those of no sequence are left alone."""
    pairs = [(50, -20), (40, -40), (60, 100)]
    m = times(pairs, 2, 1, 16)
    c = Cache(pairs, m, 64, 16)
    q = queries(c, 2 * m, 64)
    out = torch.full((c.tokens, 2 * m, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    dev, ws = c.device(), workspace(c.tokens, 3, 2 * m, m, 64)
    B.gptaq_attention(q, **dev, ws=ws, out=out)
    check(out, c, q, 2 * m, 0, 0)
    assert torch.all(out[:20] == 0) and torch.all(out[50:90] == 0)
    dev["starts"] = torch.tensor([1, 50, 50, 149], dtype=torch.int32, device="cuda")
    out.fill_(7.0)
    B.gptaq_attention(q, **dev, ws=ws, out=out)
    assert torch.all(out[0] == 7.0) and torch.all(out[149:] == 7.0) and not torch.any(out[1:149] == 7.0)


@pytest.mark.parametrize("starts,lengths", [([0, 90, 40], [90, 90]), ([-5, 30, 1 << 30], [1 << 30, -7]), ([280, 2, 0], [2 ** 31 - 1, 2 ** 31 - 1]), ([280, 280, 280], [0, 0])])
def test_arrays_that_make_no_sense_stay_inside(starts, lengths):
    """Positions and rows are bounded by the kernels themselves, whatever the arrays on the device hold: the calls end, and write nothing but their outputs."""
    m = times([(280, 0), (0, 0)], 4, 2, 16, table_pages=5)
    c = Cache([(4, 30), (3, 50)], 2 * m, 64, 16)
    dev = c.device()
    dev["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    dev["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = bf16(np.ones((280, 4 * m, 64)))
    B.gptaq_attention(q, **dev, ws=workspace(280, 2, 4 * m, 2 * m, 64))
    torch.cuda.synchronize()
    wide = torch.full((2, 800), -1, dtype=torch.int32, device="cuda")        # steps beside prompts
    wide[:, :dev["table"].shape[1]] = dev["table"]
    B.gptaq_attention(q[:, :16], **dict(dev, table=wide, keys=dev["keys"][:, :8].contiguous(), values=dev["values"][:, :8].contiguous()), ws=workspace(280, 2, 16, 8, 64))
    torch.cuda.synchronize()


def test_many_sequences():
    r = np.random.default_rng(13)
    pairs = [(int(r.integers(0, 40)), int(r.integers(0, 60))) for _ in range(300)]
    assert sum(c for c, _ in pairs) > 16 * len(pairs)
    run_many(pairs, 16, 4, 64, 16)
    run_many([(0, 3)] * 70 + [(200, 5)] + [(0, 0)] * 30 + [(60, 90), (1, 1)], 16, 1, 64, 32, 8, 2)


def plain_head(dev, c, q, h, kv_head, window, sinks):
    """The formula for a head on the cache as it is on the device, in 64 bits, with what it says of infinities and NaN."""
    keys, values, q = f64(dev["keys"][:, kv_head]), f64(dev["values"][:, kv_head]), f64(q[:, h])
    out = np.zeros((c.tokens, c.d))
    for s in range(len(c.pairs)):
        see = seen(c, s, window, sinks)
        for t in range(c.pairs[s][0]):
            js = np.flatnonzero(see[t])
            ids, slots = c.table[s][js // c.page], js % c.page
            with np.errstate(invalid="ignore"):
                logit = keys[ids, :, slots].reshape(len(js), c.d) @ q[c.starts[s] + t] * c.d ** -0.5
                w = np.exp(logit - logit.max())
                out[c.starts[s] + t] = (w[:, None] * values[ids, slots // 8, :, slots % 8]).sum(0) / w.sum()
    return out


@pytest.mark.parametrize("pairs", [[(200, 37)], [(90, 0), (40, 200)]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 3)])
def test_infinities_and_nan_reach_those_who_see_them(pairs, window, sinks):
    m = times(pairs, 4, 2, 16, window, sinks)
    c = Cache(pairs, 2 * m, 64, 16, seed=5)
    q = queries(c, 4 * m, 64, scale=0.5)
    clean = c.device()
    ws = workspace(c.tokens, len(pairs), 4 * m, 2 * m, 64)
    base = B.gptaq_attention(q, **clean, ws=ws, window=window, sinks=sinks)
    n = sum(pairs[0])
    for kind, bad in (("values", float("inf")), ("values", -float("inf")), ("values", float("nan")), ("keys", float("nan"))):
        for j in sorted({1, n // 2, n - 20, n - 2, n - 1}):
            dev = {k: v.clone() for k, v in clean.items()}
            id, slot = int(c.table[0, j // 16]), j % 16
            if kind == "values":
                dev["values"][id, 1, slot // 8, 5, slot % 8] = bad
                if j == n - 2:                                       # both infinities seen by the last token alone
                    dev["values"][int(c.table[0, (n - 1) // 16]), 1, (n - 1) % 16 // 8, 5, (n - 1) % 8] = -bad
            else:
                dev["keys"][id, 1, 2, slot, 3] = bad
            y = B.gptaq_attention(q, **dev, ws=ws, window=window, sinks=sinks)
            assert torch.equal(y[:, :2], base[:, :2]) and torch.equal(y[:, 4:], base[:, 4:]), (kind, bad, j)
            for h in (2, 3):
                want, got = plain_head(dev, c, q, h, 1, window, sinks), f64(y[:, h])
                odd = ~np.isfinite(want)
                assert odd.any() and np.array_equal(got[odd], want[odd], equal_nan=True), (kind, bad, j, h)
                same = torch.from_numpy(~odd).cuda()
                assert torch.equal(y[:, h][same], base[:, h][same]), (kind, bad, j, h)


def test_large_scores():
    """Scores that differ by thousands, with either sign, in whatever order: no overflow, and no part of a row is lost."""
    pairs = [(80, 200)]
    m = times(pairs, 2, 1, 16)
    c = Cache(pairs, m, 64, 16, seed=9)
    grow = c.r.permutation(np.linspace(-300, 300, len(c.k[0])))
    c.k[0] = torch.from_numpy(c.k[0] * 0.01 + grow[:, None, None] / 8).to(torch.bfloat16).double().numpy()
    for sign in (1.0, -1.0, 50.0):
        q = bf16(np.full((c.tokens, 2 * m, 64), sign))
        check(B.gptaq_attention(q, **c.device(), ws=workspace(c.tokens, 1, 2 * m, m, 64)), c, q, 2 * m, 0, 0)


@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 3)])
def test_scores_near_the_ends_of_fp32_and_a_scale_of_zero(window, sinks):
    """One key that stands out has all the weight, equal scores have equal weights, and with a scale of zero all have."""
    pairs = [(150, 150)]
    m = times(pairs, 2, 1, 16, window, sinks)
    c = Cache(pairs, m, 64, 16, seed=10)
    c.k[0][:] = -(2.0 ** 53)
    c.v[0] = 2.0 * c.r.integers(-8, 8, c.v[0].shape) + 1.0
    q = bf16(np.full((c.tokens, 2 * m, 64), 2.0 ** 53))
    ws = workspace(c.tokens, 1, 2 * m, m, 64)
    see = seen(c, 0, window, sinks).astype(np.float64)
    mean = np.stack([see @ c.v[0][:, h // 2] / see.sum(1, keepdims=True) for h in range(2 * m)], 1)
    tol = np.abs(mean) * (HALF + 4 * U)
    call = lambda **more: f64(B.gptaq_attention(q, **c.device(), ws=ws, window=window, sinks=sinks, **more))
    assert np.all(np.abs(call() - mean) <= tol)
    c.k[0][2] = c.k[0][170] = 2.0 ** 53                              # (one that all see with no window or with sinks, one in the middle)
    assert np.all(np.abs(call(scale=0.0) - mean) <= tol) and np.all(np.abs(call(scale=-0.0) - mean) <= tol)
    one = (see[:, 170] > 0) & (see[:, 2] == 0)
    got, c.k[0][2] = call(), -(2.0 ** 53)
    for row in np.flatnonzero(one):
        assert np.array_equal(got[row], np.repeat(c.v[0][170], 2, 0))
    got = call()
    for row in np.flatnonzero(see[:, 170] > 0):
        assert np.array_equal(got[row], np.repeat(c.v[0][170], 2, 0))


def test_graphs_that_share_a_workspace_and_the_same_bits_every_time():
    """Prompts in blocks of many rows and of few, captured with one workspace and replayed in turn with eager calls between."""
    cases = []
    ws = workspace(400, 2, 96, 24, 128)
    for pairs, heads, kv in (([(200, 700), (100, 5)], 96, 24), ([(100, 900), (77, 77)], 8, 2), ([(300, 100)], 96, 24)):
        assert (times(pairs, heads, kv, 16) == 1) == (heads == 96)
        c = Cache(pairs, kv, 128, 16, seed=len(cases))
        q, out = queries(c, heads, 128), torch.empty((c.tokens, heads, 128), dtype=torch.bfloat16, device="cuda")
        dev = c.device()
        B.gptaq_attention(q, **dev, ws=ws, out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.gptaq_attention(q, **dev, ws=ws, out=out)
        cases.append((c, q, dev, out, graph, heads))
    for k in range(3):
        for c, q, dev, out, graph, heads in cases:
            q.copy_(queries(c, heads, 128))
            graph.replay()
        torch.cuda.synchronize()
        for c, q, dev, out, graph, heads in cases:
            got = out.clone()
            ws.fill_(255)
            assert torch.equal(B.gptaq_attention(q, **dev, ws=ws), got), k
            if k == 0:
                check(got, c, q, heads, 0, 0)


def test_shared_pages_and_offsets_past_32_bits():
    """Sequences with the same first pages, in a cache of 5 GiB of which they have the last pages and the first."""
    page, kv, d = 256, 8, 128
    pages = 5 * 2 ** 30 // (page * kv * d * 2)
    pairs = [(130, 700), (200, 520)]
    heads = 8 * kv
    assert times(pairs, heads, kv, page) == 1
    c = Cache(pairs, kv, d, page, spare=0)
    c.table[1, :2] = c.table[0, :2]
    c.k[1][:512], c.v[1][:512] = c.k[0][:512], c.v[0][:512]
    keys, values = (bf16(a) for a in c.arrays())
    big_k = torch.empty((pages, kv, d // 8, page, 8), dtype=torch.bfloat16, device="cuda")
    big_v = torch.empty((pages, kv, page // 8, d, 8), dtype=torch.bfloat16, device="cuda")
    where = [pages - 1, 0, pages - 2, 1, pages // 2, pages - 7, pages - 9, 3][:c.pages]
    assert len(where) == c.pages
    for i, w in enumerate(where):
        big_k[w], big_v[w] = keys[i], values[i]
    dev = c.device()
    table = torch.full_like(dev["table"], -1)
    for i, w in enumerate(where):
        table[dev["table"] == i] = w
    dev.update(keys=big_k, values=big_v, table=table)
    q = queries(c, heads, d)
    check(B.gptaq_attention(q, **dev, ws=workspace(c.tokens, 2, heads, kv, d)), c, q, heads, 0, 0)


MIXED = [  # steps beside prompts: (new, before) of the sequences, heads, kv_heads, d, page, window, sinks
    ([(1, 3000), (300, 0), (1, 40), (0, 9), (2, 500), (1, 0)], 32, 8, 128, 16, 0, 0), ([(500, 20), (1, 700), (1, 2000)], 40, 20, 64, 64, 0, 0),
    ([(16, 50), (17, 50), (15, 3), (400, 10), (1, 1000)], 48, 48, 96, 32, 0, 0), ([(1, 8600), (1, 77), (400, 6900), (1, 900)], 32, 16, 128, 16, 6100, 70),
    ([(1, 5000)] * 3 + [(150, 4000)], 24, 24, 64, 128, 0, 0), ([(1, 900), (600, 0), (1, 3)], 32, 1, 128, 16, 0, 0), ([(1, 60)] * 40 + [(700, 0)] + [(1, 300)] * 25, 32, 8, 64, 16, 0, 0),
    ([(2, 7500), (3, 1500), (500, 0), (1, 6500)], 32, 4, 96, 16, 6097, 10),
]


@pytest.mark.parametrize("pairs,heads,kv,d,page,window,sinks", MIXED)
def test_steps_beside_prompts(pairs, heads, kv, d, page, window, sinks):
    """In tables with room for 12800 positions: steps are blocks of few rows, and prompts of many."""
    tokens, width = sum(c for c, _ in pairs), max(-(-(c + b) // page) for c, b in pairs)
    tiles = min(200, window // 64 + sinks // 64 + 4 if window else 200)
    assert len(pairs) > 1 and tiles > 96 and tiles * 4 > len(pairs) * kv and -(-(tokens - len(pairs) + 1) * (heads // kv) // 16) * kv * (tiles + 9) > 22000
    run(pairs, heads, kv, d, page, window, sinks, wider=12800 // page - width)


def test_captured_steps_beside_prompts():
    """The sequences that are steps and those that are prompts change places, and lengths grow, between replays of one graph; the workspace holds what other calls left."""
    heads, kv, d, page = 32, 8, 64, 16
    shapes = [[(1, 2000), (300, 0), (4, 900)], [(300, 33), (1, 7), (4, 1200)], [(4, 500), (1, 2222), (300, 1000)], [(100, 0), (100, 700), (105, 90)]]
    assert all(sum(c for c, _ in p) == 305 for p in shapes)
    caches = [Cache(p, kv, d, page, seed=k) for k, p in enumerate(shapes)]
    width, pages = 800, max(c.pages for c in caches)                 # (12800 positions)
    keys, values = torch.zeros((pages, kv, d // 8, page, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((pages, kv, page // 8, d, 8), dtype=torch.bfloat16, device="cuda")
    table = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    starts, lengths = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    q, out = (torch.zeros((305, heads, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = workspace(305, 3, heads, kv, d)

    def put(c):
        dev = c.device()
        keys[:c.pages], values[:c.pages] = dev["keys"], dev["values"]
        table.fill_(-1)
        table[:, :c.table.shape[1]] = dev["table"]
        starts.copy_(dev["starts"]); lengths.copy_(dev["lengths"]); q.copy_(queries(c, heads, d))

    call = lambda ws, out: B.gptaq_attention(q, keys, values, table, starts, lengths, ws, out=out)
    put(caches[0])
    call(ws, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ws, out)
    for c in [*caches, caches[0]]:
        put(c)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(call(workspace(305, 3, heads, kv, d), torch.empty_like(out)), got)
        check(got, c, q, heads, 0, 0)


def test_thousands_of_sequences():
    """A lane's run of sequences is longer than a wavefront: prompts among empty sequences, alone and with steps beside them."""
    r = np.random.default_rng(18)
    for seqs in (4200, 10000):
        pairs = [(0, 0)] * seqs
        for s in (0, 63, 64, seqs // 64 + 1, seqs // 2, seqs - 1):
            pairs[s] = (130, int(r.integers(0, 50)))
        tokens = 6 * 130
        for s in r.permutation(seqs).tolist():                       # (more tokens than sequences: as far as the host can tell one long prompt)
            if tokens < seqs + 4500 and pairs[s][0] == 0:
                pairs[s] = (int(r.integers(1, 100)), int(r.integers(0, 50)))
                tokens += pairs[s][0]
        width = max(-(-(c + b) // 16) for c, b in pairs) + 1
        assert -(-(tokens - seqs + 1) // 16) * 8 * (-(-width * 16 // 64) + 9) > 22000
        run(pairs, 8, 8, 64, 16)
    pairs = [(0, 0)] * 4303
    for s in r.choice(4303, 100, replace=False).tolist():
        pairs[s] = (int(r.integers(1, 4)), int(r.integers(0, 900)))
    pairs[0], pairs[70], pairs[2000], pairs[4302] = (1500, 0), (1, 2000), (1600, 100), (1500, 20)
    width = max(-(-(c + b) // 64) for c, b in pairs)
    assert 1300 * 4 > 4303 and -(-(sum(c for c, _ in pairs) - 4302) * 8 // 16) * 1309 > 22000
    run(pairs, 8, 1, 64, 64, wider=1300 - width)


def test_infinities_and_nan_in_steps_beside_prompts():
    """Planted in a prompt's, a step's and two tokens' keys and values: those who see them have what the formula says, the others' outputs do not change."""
    pairs, heads, kv = [(1, 500), (200, 37), (2, 90)], 64, 8
    c = Cache(pairs, kv, 64, 16, seed=6, wider=800 - 32)             # (room for 12800 positions)
    assert c.table.shape[1] == 800 and (203 - 3 + 1) * 8 // 16 * kv * 209 > 22000
    q = queries(c, heads, 64, scale=0.5)
    clean = c.device()
    ws = workspace(c.tokens, 3, heads, kv, 64)
    base = B.gptaq_attention(q, **clean, ws=ws)
    check(base, c, q, heads, 0, 0)
    for s, positions in ((0, (0, 250, 500)), (1, (3, 120, 236)), (2, (20, 90, 91))):
        for j in positions:
            for kind, bad in (("values", float("inf")), ("values", float("nan")), ("keys", float("nan"))):
                dev = {k: v.clone() for k, v in clean.items()}
                id, slot = int(c.table[s, j // 16]), j % 16
                if kind == "values":
                    dev["values"][id, 1, slot // 8, 5, slot % 8] = bad
                else:
                    dev["keys"][id, 1, 2, slot, 3] = bad
                y = B.gptaq_attention(q, **dev, ws=ws)
                assert torch.equal(y[:, :8], base[:, :8]) and torch.equal(y[:, 16:], base[:, 16:]), (s, j, kind, bad)
                for h in (8, 15):
                    want, got = plain_head(dev, c, q, h, 1, 0, 0), f64(y[:, h])
                    odd = ~np.isfinite(want)
                    assert odd.any() and np.array_equal(got[odd], want[odd], equal_nan=True), (s, j, kind, bad, h)
                    same = torch.from_numpy(~odd).cuda()
                    assert torch.equal(y[:, h][same], base[:, h][same]), (s, j, kind, bad, h)


def test_the_output_may_be_the_queries_memory():
    """In blocks of many rows, with parts and without, and with steps beside prompts."""
    for pairs, heads, kv, d, wider in (([(150, 60), (33, 0)], 4, 2, 64, 1), ([(100, 6000), (60, 100)], 24, 12, 128, 1), ([(1, 500), (200, 37), (2, 90)], 64, 8, 64, 766)):
        m = times(pairs, heads, kv, 16, wider=wider)
        c = Cache(pairs, kv * m, d, 16, wider=wider)
        q, dev, ws = queries(c, heads * m, d), c.device(), workspace(c.tokens, len(pairs), heads * m, kv * m, d)
        want = B.gptaq_attention(q, **dev, ws=ws)
        assert B.gptaq_attention(q, **dev, ws=ws, out=q) is q and torch.equal(q, want)


def test_scores_of_minus_infinity_weigh_nothing():
    """Where a token sees no others, zeros, as for one that sees nothing."""
    pairs = [(150, 150)]
    m = times(pairs, 2, 1, 16)
    c = Cache(pairs, m, 64, 16, seed=14)
    c.k[0][::3, 0, 7] = -np.inf
    c.k[0][:, 1, 9] = -np.inf
    q = queries(c, 2 * m, 64)
    q[..., 7] = q[..., 9] = 1.0
    ws = workspace(c.tokens, 1, 2 * m, m, 64)
    y = B.gptaq_attention(q, **c.device(), ws=ws)
    assert torch.all(y[:, 2:4] == 0) and not torch.any(torch.isnan(y))
    c.k[0][::3, 0] = np.where(np.arange(64) == 7, -(2.0 ** 40), 0.0)
    assert torch.equal(y[:, :2], B.gptaq_attention(q, **c.device(), ws=ws)[:, :2])


def test_values_of_2_to_the_100():
    """Sums of weights of up to 2^8 a key stay inside fp32 for them."""
    pairs = [(150, 3000)]
    m = times(pairs, 2, 1, 16)
    c = Cache(pairs, m, 64, 16, seed=15)
    c.v[0] = c.v[0] * 2.0 ** 100
    q = queries(c, 2 * m, 64, scale=8.0)
    check(B.gptaq_attention(q, **c.device(), ws=workspace(c.tokens, 1, 2 * m, m, 64)), c, q, 2 * m, 0, 0)
