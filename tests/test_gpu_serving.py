"""The operators that run quantised layers, against their formulas in 64 bits on the CPU.

Tolerances, with u = 2^-24: a value rounded to bfloat16 is off by 2^-8 of itself at most.  A sum of n products taken in fp32 in any
order is off by n * 2u of the sum of the products' absolute values (2u for adders that cut off instead of rounding).  The sum of
squares of n values is therefore off by 2 n u, its root by n u, and a few operations add 16 u.  The fast exponential of -g is off by
|g| 2u + 4u.  A code is the nearest to a quotient that is off by what its value and its scale are off.
"""
import numpy as np
import pytest
import torch

from paper_2504_02692_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -133                                     # half the distance of bfloat16's smallest values


def rng(*key):
    return np.random.default_rng([abs(hash(k)) if isinstance(k, str) else int(k) for k in key])


def bf16(a, device="cuda"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).to(device)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def padded(t, extra, shift=0):
    """The same values as a view with rows `extra` elements longer, its start `shift` elements behind an aligned address; what lies
    around them is NaN (or 77)."""
    rows, n = t.shape
    fill = float("nan") if t.dtype.is_floating_point else 77
    flat = torch.full((rows * (n + extra) + shift + 64,), fill, dtype=t.dtype, device=t.device)
    v = flat[shift:shift + rows * (n + extra)].view(rows, n + extra)[:, :n]
    v.copy_(t)
    return v


# ---- products

def quantised(m, n, bits, group, sym, r):
    """Codes, scales, zeros with every value that the solve may return."""
    G = n // group if group > 0 else 1
    codes = r.integers(0, 2 ** bits, (m, n)).astype(np.uint8)
    scales = (0.002 + 0.01 * r.random((m, G))).astype(np.float32)
    zeros = np.full((m, G), 2.0 ** (bits - 1)) if sym else r.integers(0, 2 ** bits, (m, G)).astype(float)
    return codes, scales, zeros.astype(np.float32)


def dequantised(codes, scales, zeros, group):
    m, n = codes.shape
    c = codes.astype(np.float64).reshape(m, -1, group if group > 0 else n)
    return ((c - zeros.astype(np.float64)[:, :, None]) * scales.astype(np.float64)[:, :, None]).reshape(m, n)


def pack(codes, scales, zeros, group, perm=None, bias=None):
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    w = B.gptaq_linear_pack(dev(codes), dev(scales), dev(zeros), group, perm=dev(perm), bias=dev(bias))
    assert w.info.item() == 0
    return w


def linear_case(tokens, m, n, bits, group, i8, sym=False, perm=False, bias=False, f32=False, extra=0, shift=0):
    print("linear", tokens, m, n, bits, group, i8, sym, perm, bias, f32, extra, shift, flush=True)
    r = rng(tokens, m, n, bits, group + 1, i8)
    codes, scales, zeros = quantised(m, n, bits, group, sym, r)
    p = r.permutation(n).astype(np.int32) if perm else None
    b = r.standard_normal(m).astype(np.float32) if bias else None
    w = pack(codes, scales, zeros, group, p, b)
    W = dequantised(codes, scales, zeros, group)
    ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
    ws.fill_(255)                                                  # (NaN as bf16)
    dtype = torch.float32 if f32 else torch.bfloat16
    if i8:
        q = r.integers(-127, 128, (tokens, n)).astype(np.int8)
        xs = (0.01 + 0.1 * r.random(tokens)).astype(np.float32)
        x = q.astype(np.float64) * xs.astype(np.float64)[:, None]
        Y = B.gptaq_linear_i8(padded(torch.from_numpy(q).cuda(), extra, shift), torch.from_numpy(xs).cuda(), w, ws, dtype=dtype)
    else:
        X = bf16(r.standard_normal((tokens, n)) * np.where(r.random(n) < 0.02, 20.0, 1.0))
        x = f64(X)
        Y = B.gptaq_linear(padded(X, extra, shift), w, ws, dtype=dtype)
    if perm:
        x = x[:, p]
    assert Y.shape == (tokens, m) and Y.dtype == dtype
    want = x @ W.T + (b if bias else 0.0)
    size = np.abs(x) @ np.abs(W).T + (np.abs(b) if bias else 0.0)
    tol = (n + 16) * 2 * U * size + (0.0 if f32 else np.abs(want) * 2.0 ** -8 * (1 + 2.0 ** -6))
    err = np.abs(f64(Y) - want)
    assert np.all(err <= tol), (float(np.max(err / np.maximum(tol, 1e-300))), np.argwhere(err > tol)[:4].tolist())


SHAPES = [                                             # tokens, m, n, group
    (1, 1, 1, 0), (1, 16, 32, 32), (1, 17, 128, 128), (2, 5, 96, 32), (3, 33, 192, 64), (1, 257, 1000, 0), (16, 48, 640, 128),
    (17, 64, 384, 64), (15, 100, 136, 0), (33, 129, 256, 32), (64, 128, 1024, 128), (65, 80, 520, 0), (130, 272, 512, 64),
    (1, 2048, 11008, 128), (300, 512, 768, 128), (257, 515, 1024, 0), (700, 1040, 384, 32), (520, 256, 2736, 0),
    # around the lines between kernels and tiles, and sums taken in parts of the columns
    (16, 8200, 256, 128), (9, 16400, 128, 32), (8, 16390, 256, 64), (17, 30, 2048, 128), (32, 500, 1536, 32), (33, 260, 2176, 64), (64, 129, 4096, 0), (65, 1000, 2944, 128),
    (128, 60, 8192, 128), (129, 300, 5000, 0), (300, 258, 3968, 128), (18, 1, 16384, 64),
]


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m,n,group", SHAPES)
def test_linear_is_the_formula(tokens, m, n, group, i8):
    linear_case(tokens, m, n, 4, group, i8)


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens", [1, 9, 70, 400])
@pytest.mark.parametrize("bits,group,sym,perm,bias,f32", [(2, 64, False, True, False, True), (3, 128, True, False, True, False), (4, 0, True, True, True, True),
                                                         (4, 32, False, True, True, False)])
def test_linear_forms(tokens, bits, group, sym, perm, bias, f32, i8):
    linear_case(tokens, 144, 512, bits, group, i8, sym, perm, bias, f32)


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens", [1, 20, 200])
@pytest.mark.parametrize("extra,shift", [(16, 0), (3, 0), (0, 1), (8, 8), (7, 5)])
def test_linear_strides_and_alignment(tokens, extra, shift, i8):
    linear_case(tokens, 96, 256, 4, 64, i8, extra=extra, shift=shift)
    linear_case(tokens, 40, 1003, 4, 0, i8, extra=extra, shift=shift)


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m,n,group", [(1, 64, 512, 128), (5, 40, 1024, 32), (40, 112, 768, 64), (260, 300, 640, 128), (600, 520, 512, 0), (12, 16, 2048, 0)])
def test_linear_is_exact_where_the_sums_are(tokens, m, n, group, i8):
    """Whole activations and scales that are powers of two: every sum is a float, so every entry is equal, in any order."""
    r = rng(tokens, m, n, group, 5)
    codes, scales, zeros = quantised(m, n, 4, group, False, r)
    scales = (2.0 ** r.integers(-3, 3, scales.shape)).astype(np.float32)
    w = pack(codes, scales, zeros, group)
    x = r.integers(-8, 9, (tokens, n)).astype(np.float64)
    want = x @ dequantised(codes, scales, zeros, group).T
    ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
    if i8:
        Y = B.gptaq_linear_i8(torch.from_numpy(x.astype(np.int8)).cuda(), torch.ones(tokens, device="cuda"), w, ws, dtype=torch.float32)
    else:
        Y = B.gptaq_linear(bf16(x), w, ws, dtype=torch.float32)
    assert np.array_equal(f64(Y), want)


@pytest.mark.parametrize("tokens", [1, 40, 300])
@pytest.mark.parametrize("i8", [False, True])
def test_linear_extremes_of_8_bits(tokens, i8):
    """The largest codes of either sign against the largest differences of either sign: no sum wraps."""
    m, n = 32, 16384
    for group in (0, 128):
        G = n // group if group else 1
        for c, z in ((15, 0), (0, 15)):
            w = pack(np.full((m, n), c, np.uint8), np.ones((m, G), np.float32), np.full((m, G), z, np.float32), group)
            ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
            for v in (127, -128):
                if i8:
                    Y = B.gptaq_linear_i8(torch.full((tokens, n), v, dtype=torch.int8, device="cuda"), torch.ones(tokens, device="cuda"), w, ws,
                                          dtype=torch.float32)
                else:
                    Y = B.gptaq_linear(torch.full((tokens, n), float(v), dtype=torch.bfloat16, device="cuda"), w, ws, dtype=torch.float32)
                assert torch.all(Y == float(v * (c - z) * n)), (group, c, z, v, Y[0, 0].item())


@pytest.mark.parametrize("tokens", [1, 7, 16, 30, 40, 300])
def test_linear_keeps_tokens_apart_and_passes_on_what_is_not_finite(tokens):
    """A token with an infinity or a NaN spoils its own outputs alone; an infinity meets weights of either sign."""
    m, n, group = 48, 256, 64
    r = rng(tokens, 8)
    codes, scales, zeros = quantised(m, n, 4, group, False, r)
    w = pack(codes, scales, zeros, group)
    W = dequantised(codes, scales, zeros, group)
    X = r.standard_normal((tokens, n)).astype(np.float32)
    clean = bf16(X)
    bad = clean.clone()
    bad[0, 37] = float("inf")
    if tokens > 20:
        bad[17, 3] = float("nan")
        bad[tokens - 1, n - 1] = float("-inf")
    ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
    a, b = B.gptaq_linear(clean, w, ws, dtype=torch.float32), B.gptaq_linear(bad, w, ws, dtype=torch.float32)
    fine = [t for t in range(tokens) if t not in (0, 17, tokens - 1)]
    assert torch.equal(a[fine], b[fine])
    got = b[0].cpu().numpy()
    col = W[:, 37]
    assert np.all(np.isposinf(got[col > 0])) and np.all(np.isneginf(got[col < 0])) and np.all(np.isnan(got[col == 0]))
    if tokens > 20:
        assert torch.isnan(b[17]).all() and not torch.isfinite(b[tokens - 1]).any()


def test_linear_skips_what_a_permutation_should_not_have():
    m, n = 16, 128
    codes, scales, zeros = quantised(m, n, 4, 32, False, rng(3))
    perm = np.arange(n, dtype=np.int32)
    perm[5], perm[77] = -1, 2 ** 31 - 1
    w = pack(codes, scales, zeros, 32, perm)
    x = rng(4).integers(-3, 4, (2, n)).astype(np.float64)
    Y = B.gptaq_linear(bf16(x), w, B.workspace(B.gptaq_linear_workspace_bytes(2, m, n)), dtype=torch.float32)
    x[:, [5, 77]] = 0.0
    want = x @ dequantised(codes, scales, zeros, 32).T
    assert np.all(np.abs(f64(Y) - want) <= (n + 16) * 2 * U * (np.abs(x) @ np.abs(dequantised(codes, scales, zeros, 32)).T))


def test_pack_reports_what_does_not_fit():
    codes, scales, zeros = quantised(40, 256, 4, 64, False, rng(9))
    dev = lambda a: torch.from_numpy(a).cuda()
    for row, what, value in ((7, "code", 16), (39, "code", 255), (12, "zero", 16.0), (0, "zero", 2.5), (3, "zero", -1.0), (30, "zero", float("nan"))):
        c, z = codes.copy(), zeros.copy()
        (c if what == "code" else z)[row, -1] = value
        assert B.gptaq_linear_pack(dev(c), dev(scales), dev(z), 64).info.item() == row + 1
    wide = torch.full((40, 300), 255, dtype=torch.uint8, device="cuda")           # what lies behind the columns is not looked at
    wide[:, :256] = dev(codes)
    w = B.gptaq_linear_pack(wide[:, :256], dev(scales), dev(zeros), 64)
    assert w.info.item() == 0 and torch.equal(w.data, B.gptaq_linear_pack(dev(codes), dev(scales), dev(zeros), 64).data)


def test_linear_rows_far_apart():
    """Rows of activations and outputs more than 2^31 elements from the first."""
    m, n, ld = 48, 256, (1 << 30) + 64
    codes, scales, zeros = quantised(m, n, 4, 64, False, rng(10))
    w = pack(codes, scales, zeros, 64)
    x = rng(11).integers(-8, 9, (4, n)).astype(np.float64)
    X = torch.empty(3 * ld + n, dtype=torch.bfloat16, device="cuda").as_strided((4, n), (ld, 1))
    Y = torch.empty(3 * ld + m, dtype=torch.bfloat16, device="cuda").as_strided((4, m), (ld, 1))
    X.copy_(bf16(x))
    ws = B.workspace(B.gptaq_linear_workspace_bytes(4, m, n))
    B.gptaq_linear(X, w, ws, out=Y)
    assert torch.equal(Y, B.gptaq_linear(bf16(x), w, ws))


# ---- rows

def norm_reference(x, res, w, eps):
    h = (x.float() + res.float()) if res is not None else x.float()
    h64 = f64(x) + (f64(res) if res is not None else 0.0)
    y = h64 / np.sqrt(np.mean(h64 * h64, 1, keepdims=True) + eps) * (f64(w) if w is not None else 1.0)
    return h.to(torch.bfloat16), y


def check_codes(codes, scales, y, rel, clip, extra=0.0):
    """rel: how far the values may be off, as a share of each; extra: as a share of each, an array."""
    top = np.abs(y).max(1)
    s = clip * top / 127.0
    got = f64(scales)
    assert np.all(np.abs(got - s) <= (rel + np.max(extra)) * s + 2.0 ** -148), float(np.max(np.abs(got - s) / np.maximum(s, 1e-300)))
    ideal = np.clip(np.divide(y, s[:, None], out=np.zeros_like(y), where=s[:, None] > 0), -127.0, 127.0)
    off = np.abs(f64(codes) - ideal)
    assert np.all(off <= 0.5 + 128.0 * (2 * rel + 2 * np.max(extra))), float(off.max())


ROWS = [(1, 1), (2, 7), (3, 8), (5, 9), (1, 64), (4, 513), (9, 1000), (1, 4096), (37, 4099), (3, 8192), (2, 16383), (2, 32768), (2, 33001), (1, 70000), (300, 520)]


@pytest.mark.parametrize("residual,weight", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("tokens,n", ROWS)
def test_rms_norm(tokens, n, residual, weight):
    print("norm", tokens, n, residual, weight, flush=True)
    r = rng(tokens, n, residual, weight)
    x, res = bf16(r.standard_normal((tokens, n))), bf16(3.0 * r.standard_normal((tokens, n))) if residual else None
    w = bf16(1.0 + 0.2 * r.standard_normal((1, n)))[0].contiguous() if weight else None
    h, y = norm_reference(x, res, w, 1e-5)
    rel = (n + 16) * U
    got, total = B.gptaq_rms_norm(x, w, 1e-5, residual=res)
    if residual:
        assert torch.equal(total, h)
    else:
        assert total is None
    assert np.all(np.abs(f64(got) - y) <= np.abs(y) * (2.0 ** -8 * (1 + 2.0 ** -6) + rel) + TINY)
    for clip in (1.0, 0.9):
        codes, scales, total = B.gptaq_rms_norm_i8(x, w, 1e-5, residual=res, clip=clip)
        check_codes(codes, scales, y, rel, clip)
        assert total is None or torch.equal(total, h)


@pytest.mark.parametrize("tokens,n", ROWS)
def test_silu_mul(tokens, n):
    print("silu", tokens, n, flush=True)
    r = rng(tokens, n, 77)
    g, u = bf16(4.0 * r.standard_normal((tokens, n))), bf16(r.standard_normal((tokens, n)))
    g64 = f64(g)
    y = g64 / (1.0 + np.exp(-g64)) * f64(u)
    rel, extra = 16 * U, np.abs(g64) * 2 * U
    assert np.all(np.abs(f64(B.gptaq_silu_mul(g, u)) - y) <= np.abs(y) * (2.0 ** -8 * (1 + 2.0 ** -6) + rel + extra) + TINY)
    for clip in (1.0, 0.9):
        check_codes(*B.gptaq_silu_mul_i8(g, u, clip=clip), y, rel, clip, extra)


def test_silu_mul_far_out():
    """Gates whose exponential leaves fp32's range."""
    g = torch.tensor([[-3e38, -1e4, -200.0, -100.0, -88.0, -50.0, 0.0, -0.0, 50.0, 200.0, 1e4, 3e38]], dtype=torch.bfloat16, device="cuda")
    u = torch.full_like(g, 2.0)
    g64 = f64(g)
    with np.errstate(over="ignore"):
        y = g64 / (1.0 + np.exp(-g64)) * 2.0
    got = f64(B.gptaq_silu_mul(g, u))
    assert np.isposinf(got[0, -1]) and np.all(np.isfinite(got[0, :-1]))
    y, got = y[:, :-1], got[:, :-1]
    assert np.all(np.abs(got - y) <= np.abs(y) * (2.0 ** -8 + np.abs(g64[:, :-1]) * 2 * U) + 2.0 ** -125)      # (below that fp32's own range ends)


@pytest.mark.parametrize("n", [72, 1001, 8192])
@pytest.mark.parametrize("extra,shift", [(0, 1), (5, 0), (8, 8), (3, 7)])
def test_rows_with_strides(n, extra, shift):
    r = rng(n, extra, shift)
    x, res, g = (bf16(r.standard_normal((6, n))) for _ in range(3))
    w = bf16(r.standard_normal((1, n)))[0].contiguous()
    wv = padded(w[None], 0, shift)[0]
    xv, rv, gv = padded(x, extra, shift), padded(res, extra + 1, shift), padded(g, extra + 2, shift + 1)
    y, total = B.gptaq_rms_norm(x, w, 1e-6, residual=res)
    out, tot = padded(torch.zeros_like(x), extra, shift), padded(torch.zeros_like(x), extra + 3, shift)
    B.gptaq_rms_norm(xv, wv, 1e-6, residual=rv, total=tot, out=out)
    assert torch.equal(out, y) and torch.equal(tot, total)
    if extra:
        behind = out.as_strided((5, extra), (out.stride(0), 1), out.storage_offset() + n)
        assert torch.isnan(behind).all()                          # nothing is written behind a row
    c, s, _ = B.gptaq_rms_norm_i8(x, w, 1e-6, residual=res)
    cv, sv, _ = B.gptaq_rms_norm_i8(xv, wv, 1e-6, residual=rv)
    assert torch.equal(c, cv) and torch.equal(s, sv)
    assert torch.equal(B.gptaq_silu_mul(gv, xv), B.gptaq_silu_mul(g, x))
    for a, b in zip(B.gptaq_silu_mul_i8(gv, xv), B.gptaq_silu_mul_i8(g, x)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n", [100, 4096, 40001])
def test_norm_in_place(n):
    r = rng(n, 6)
    x, res = bf16(r.standard_normal((5, n))), bf16(r.standard_normal((5, n)))
    w = bf16(r.standard_normal((1, n)))[0].contiguous()
    y, total = B.gptaq_rms_norm(x, w, 1e-5, residual=res)
    x2, res2 = x.clone(), res.clone()
    got, tot = B.gptaq_rms_norm(x2, w, 1e-5, residual=res2, total=res2, out=x2)
    assert tot is res2 and got is x2 and torch.equal(res2, total) and torch.equal(x2, y)
    c, s, t = B.gptaq_rms_norm_i8(x, w, 1e-5, residual=res)
    res2 = res.clone()
    c2, s2, _ = B.gptaq_rms_norm_i8(x, w, 1e-5, residual=res2, total=res2)
    assert torch.equal(c, c2) and torch.equal(s, s2) and torch.equal(res2, t)
    g = x.clone()
    want = B.gptaq_silu_mul(x, res)
    assert torch.equal(B.gptaq_silu_mul(g, res, out=g), want)


@pytest.mark.parametrize("n", [40, 1000, 4096, 33000])
def test_rows_of_zeros_and_rows_that_are_not_finite(n):
    x = bf16(rng(n, 12).standard_normal((6, n)))
    x[1] = 0.0
    x[2, n // 2] = float("nan")
    x[3, n - 1] = float("inf")
    x[4] = torch.finfo(torch.bfloat16).tiny                        # a scale without a reciprocal in fp32 after the gate
    clean = bf16(rng(n, 12).standard_normal((6, n)))
    y, _ = B.gptaq_rms_norm(x, None, 1e-5)
    c, s, _ = B.gptaq_rms_norm_i8(x, None, 1e-5)
    yc, _ = B.gptaq_rms_norm(clean, None, 1e-5)
    cc, sc, _ = B.gptaq_rms_norm_i8(clean, None, 1e-5)
    for k in (0, 5):                                               # rows do not touch each other
        assert torch.equal(y[k], yc[k]) and torch.equal(c[k], cc[k]) and s[k] == sc[k]
    assert torch.all(y[1] == 0) and torch.all(c[1] == 0) and s[1] == 0
    assert torch.isnan(y[2]).all() and torch.isnan(s[2]) and torch.isnan(s[3])
    assert torch.isfinite(s[4]) and torch.all(c[4] == 127)
    u = torch.ones_like(x)
    u[4] = 1e-3
    c, s = B.gptaq_silu_mul_i8(x, u)
    assert s[1] == 0 and torch.all(c[1] == 0) and torch.isnan(s[2]) and torch.isnan(s[3])
    assert torch.isfinite(s[4]) and torch.all(c[4] >= 0)


def test_rows_far_apart():
    n, ld = 300, (1 << 30) + 64
    x = bf16(rng(13).standard_normal((4, n)))
    X = torch.empty(3 * ld + n, dtype=torch.bfloat16, device="cuda").as_strided((4, n), (ld, 1))
    Y = torch.empty(3 * ld + n, dtype=torch.bfloat16, device="cuda").as_strided((4, n), (ld, 1))
    X.copy_(x)
    B.gptaq_rms_norm(X, None, 1e-5, out=Y)
    assert torch.equal(Y, B.gptaq_rms_norm(x, None, 1e-5)[0])
    B.gptaq_silu_mul(X, X, out=Y)
    assert torch.equal(Y, B.gptaq_silu_mul(x, x))


# ---- how they are used

def test_no_tokens():
    w = pack(*quantised(16, 64, 4, 32, False, rng(1)), 32)
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    ws = B.workspace(0)
    assert B.gptaq_linear(x, w, ws).shape == (0, 16)
    c, s, t = B.gptaq_rms_norm_i8(x, None, 1e-5, residual=x)
    assert c.shape == (0, 64) and s.shape == (0,) and t.shape == (0, 64)
    assert B.gptaq_linear_i8(c, s, w, ws, dtype=torch.float32).shape == (0, 16)
    assert B.gptaq_silu_mul(x, x).shape == (0, 64)


def test_binding_refusals():
    w = pack(*quantised(16, 64, 4, 32, False, rng(1)), 32)
    ws = B.workspace(B.gptaq_linear_workspace_bytes(4, 16, 64))
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    q, s = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda")
    for call in (lambda: B.gptaq_linear(x.float(), w, ws), lambda: B.gptaq_linear(x.cpu(), w, ws), lambda: B.gptaq_linear(x[:, :32], w, ws),
                 lambda: B.gptaq_linear(x, w, ws[:256]), lambda: B.gptaq_linear(x, w, ws, dtype=torch.float16),
                 lambda: B.gptaq_linear(x, w, ws, out=torch.zeros((4, 15), device="cuda")),
                 lambda: B.gptaq_linear(x, w, ws, out=torch.zeros((4, 16), dtype=torch.float16, device="cuda")),
                 lambda: B.gptaq_linear_i8(q, s[:3], w, ws), lambda: B.gptaq_linear_i8(x, s, w, ws),
                 lambda: B.gptaq_rms_norm(x, x[0, :32], 1e-5), lambda: B.gptaq_rms_norm(x, None, 1e-5, residual=x[:, :32]),
                 lambda: B.gptaq_rms_norm(x, None, -1.0), lambda: B.gptaq_rms_norm_i8(x, None, 1e-5, clip=0.0),
                 lambda: B.gptaq_silu_mul(x, x[:2]), lambda: B.gptaq_silu_mul(x.t(), x.t()),
                 lambda: B.gptaq_linear_pack(q.to(torch.uint8), torch.ones((4, 2), device="cuda"), torch.ones((4, 1), device="cuda"), 32),
                 lambda: B.gptaq_linear_pack(q.to(torch.uint8), torch.ones((4, 4), device="cuda"), torch.ones((4, 4), device="cuda"), 16)):
        with pytest.raises(B.GptaqError):
            call()


@pytest.mark.parametrize("tokens", [1, 130])
def test_another_stream_and_a_graph(tokens):
    """The calls run on the caller's current stream, wait for nothing and allocate nothing in the library: captured once and replayed on
    new inputs, with other work between the replays, they give what the plain calls give."""
    hidden, inner, group = 256, 384, 64
    up = pack(*quantised(2 * inner, hidden, 4, group, False, rng(20)), group, rng(22).permutation(hidden).astype(np.int32))
    down = pack(*quantised(hidden, inner, 4, group, False, rng(21)), group)
    ws = B.workspace(max(B.gptaq_linear_workspace_bytes(tokens, 2 * inner, hidden), B.gptaq_linear_workspace_bytes(tokens, hidden, inner)))
    x, res = (torch.zeros((tokens, hidden), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def block():
        c, s, total = B.gptaq_rms_norm_i8(x, None, 1e-5, residual=res)
        both = B.gptaq_linear_i8(c, s, up, ws)
        c, s = B.gptaq_silu_mul_i8(both[:, :inner], both[:, inner:])
        y = B.gptaq_linear_i8(c, s, down, ws)
        z, _ = B.gptaq_rms_norm(y, None, 1e-5)
        both = B.gptaq_linear(z, up, ws)
        return y, total, B.gptaq_linear(B.gptaq_silu_mul(both[:, :inner], both[:, inner:]), down, ws, dtype=torch.float32)

    def inputs(k):
        r = rng(tokens, k, 30)
        x.copy_(bf16(r.standard_normal((tokens, hidden))))
        res.copy_(bf16(r.standard_normal((tokens, hidden))))

    inputs(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = [t.clone() for t in block()]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, block()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = block()
    for k in range(4):
        inputs(k)
        graph.replay()
        got = [t.clone() for t in held]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, block())), k
        ws.fill_(k)


def test_rows_of_many_tokens_far_apart():
    """The same for the kernels that take more than 16 tokens."""
    m, n, ld = 40, 256, (1 << 27) + 64
    codes, scales, zeros = quantised(m, n, 4, 64, False, rng(14))
    w = pack(codes, scales, zeros, 64)
    x = rng(15).integers(-8, 9, (20, n)).astype(np.float64)
    X = torch.empty(19 * ld + n, dtype=torch.bfloat16, device="cuda").as_strided((20, n), (ld, 1))
    Y = torch.empty(19 * ld + m, dtype=torch.bfloat16, device="cuda").as_strided((20, m), (ld, 1))
    X.copy_(bf16(x))
    ws = B.workspace(B.gptaq_linear_workspace_bytes(20, m, n))
    B.gptaq_linear(X, w, ws, out=Y)
    assert torch.equal(Y, B.gptaq_linear(bf16(x), w, ws))


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m,n,group", [(1, 100, 512, 128), (17, 130, 4096, 32), (40, 500, 2048, 0), (70, 260, 4096, 64), (300, 77, 8192, 128), (140, 8200, 1024, 128)])
def test_linear_keeps_to_its_memory(tokens, m, n, group, i8):
    """A workspace of just the size that is asked for, and outputs with a gap behind each row: nothing around them changes."""
    r = rng(tokens, m, 40)
    w = pack(*quantised(m, n, 4, group, False, r), group, perm=r.permutation(n).astype(np.int32))
    size = B.gptaq_linear_workspace_bytes(tokens, m, n)
    buf = torch.full((size + 65536,), 85, dtype=torch.uint8, device="cuda")
    out = padded(torch.zeros((tokens, m), device="cuda"), 7, 3)
    if i8:
        q = torch.from_numpy(r.integers(-127, 128, (tokens, n)).astype(np.int8)).cuda()
        xs = torch.full((tokens,), 0.03, device="cuda")
        call = lambda o, ws: B.gptaq_linear_i8(q, xs, w, ws, out=o)
    else:
        x = bf16(r.standard_normal((tokens, n)))
        call = lambda o, ws: B.gptaq_linear(x, w, ws, out=o)
    call(out, buf[:size])
    assert torch.all(buf[size:] == 85)
    if tokens > 1:
        assert torch.isnan(out.as_strided((tokens - 1, 7), (out.stride(0), 1), out.storage_offset() + m)).all()
    plain = torch.empty((tokens, m), device="cuda")
    call(plain, B.workspace(size + 1024))
    assert torch.equal(out, plain)                                 # and the same bits from call to call


@pytest.mark.parametrize("group,act_order", [(64, False), (128, True), (0, True)])
def test_mlp_from_solve_to_answers(group, act_order):
    """The example at small sizes, against the formulas with the solve's dequantised weights in fp32: the outputs pass three roundings to
    bfloat16 (2^-8 each at most) and, with 8 bits, two to steps of 1/127 of a row's largest value, half a step off and about 4 of its
    deviations large: 1.6 % of a deviation at most, divided by sqrt(3) on average over a row."""
    from paper_2504_02692_amd import quantized_mlp as Q
    hidden, inner = 256, 384
    mlp, full, quant = Q.calibrate(hidden, inner, 2048, group=group, act_order=act_order)
    for tokens in (1, 5, 33, 200):
        x, residual = bf16(rng(tokens, 50).standard_normal((tokens, hidden))), bf16(rng(tokens, 51).standard_normal((tokens, hidden)))
        want = Q.full_precision(x, residual, mlp.norm, *quant)
        for eight_bits, most in ((False, 3 * 2.0 ** -8), (True, 3 * 2.0 ** -8 + 2 * 0.016)):
            y, total = mlp(x, residual, mlp.workspace(tokens), eight_bits)
            assert torch.equal(total, (x.float() + residual.float()).to(torch.bfloat16))
            assert (y.float() - want).norm().item() <= most * want.norm().item()
        # 4-bit weights keep most of the signal
        ref = Q.full_precision(x, residual, mlp.norm, *full)
        assert (y.float() - ref).norm().item() <= 0.35 * ref.norm().item()


# The kernel of many tokens starts where the work is more than a few workgroups': tiles of 64 and of 128 tokens, with and without parts.
MANY = [(40, 1100, 16384, 128), (70, 2100, 16384, 0), (130, 4100, 4224, 32), (300, 2050, 8192, 64), (600, 2050, 11008, 128), (1030, 4100, 1024, 0),
        (1100, 2100, 512, 32), (2050, 4097, 256, 128), (129, 20500, 1280, 64)]


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m,n,group", MANY)
def test_linear_many_is_the_formula(tokens, m, n, group, i8):
    linear_case(tokens, m, n, 4, group, i8)


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m", [(1100, 2100), (1030, 4100)])
@pytest.mark.parametrize("bits,group,sym,perm,bias,f32,extra,shift", [(2, 64, False, True, False, True, 0, 0), (3, 128, True, False, True, False, 3, 0),
                                                                     (4, 0, True, True, True, True, 16, 5), (4, 32, False, False, False, False, 0, 1)])
def test_linear_many_forms(tokens, m, bits, group, sym, perm, bias, f32, extra, shift, i8):
    linear_case(tokens, m, 512, bits, group, i8, sym, perm, bias, f32, extra, shift)


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m,n", [(700, 2100, 2048), (2050, 4100, 1024), (200, 2100, 8192)])
def test_linear_many_is_exact_where_the_sums_are(tokens, m, n, i8):
    test_linear_is_exact_where_the_sums_are(tokens, m, n, 64, i8)
    for c, z, v in ((15, 0, 127), (0, 15, -128)):
        w = pack(np.full((m, n), c, np.uint8), np.ones((m, 1), np.float32), np.full((m, 1), z, np.float32), 0)
        ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
        if i8:
            Y = B.gptaq_linear_i8(torch.full((tokens, n), v, dtype=torch.int8, device="cuda"), torch.ones(tokens, device="cuda"), w, ws, dtype=torch.float32)
        else:
            Y = B.gptaq_linear(torch.full((tokens, n), float(v), dtype=torch.bfloat16, device="cuda"), w, ws, dtype=torch.float32)
        assert torch.all(Y == float(v * (c - z) * n))


@pytest.mark.parametrize("tokens,m,n", [(400, 2100, 256), (2050, 4100, 256), (200, 2100, 8192)])
def test_linear_many_keeps_tokens_apart(tokens, m, n):
    codes, scales, zeros = quantised(m, n, 4, 64, False, rng(60))
    w = pack(codes, scales, zeros, 64)
    col = dequantised(codes, scales, zeros, 64)[:, 37]
    clean = bf16(rng(61).standard_normal((tokens, n)))
    bad = clean.clone()
    bad[0, 37], bad[17, 3], bad[tokens - 1, n - 1] = float("inf"), float("nan"), float("-inf")
    ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
    a, b = B.gptaq_linear(clean, w, ws, dtype=torch.float32), B.gptaq_linear(bad, w, ws, dtype=torch.float32)
    fine = [t for t in range(tokens) if t not in (0, 17, tokens - 1)]
    assert torch.equal(a[fine], b[fine])
    got = b[0].cpu().numpy()
    assert np.all(np.isposinf(got[col > 0])) and np.all(np.isneginf(got[col < 0])) and np.all(np.isnan(got[col == 0]))
    assert torch.isnan(b[17]).all() and not torch.isfinite(b[tokens - 1]).any()


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m,n,group", [(200, 2100, 8192, 128), (1030, 4100, 384, 64), (40, 1100, 16384, 32)])
def test_linear_many_keeps_to_its_memory(tokens, m, n, group, i8):
    test_linear_keeps_to_its_memory(tokens, m, n, group, i8)


def test_linear_in_parts_in_a_graph():
    """Sums in parts of the columns and their join, replayed on new activations."""
    tokens, m, n = 200, 2100, 8192
    w = pack(*quantised(m, n, 4, 128, False, rng(70)), 128)
    ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
    x = bf16(rng(71).standard_normal((tokens, n)))
    B.gptaq_linear(x, w, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = B.gptaq_linear(x, w, ws)
    for k in range(4):
        x.copy_(bf16(rng(72, k).standard_normal((tokens, n))))
        graph.replay()
        got = y.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, B.gptaq_linear(x, w, ws)), k
        ws.fill_(k)


def test_linear_weights_are_fixed_and_read_where_they_are():
    """What a layer's weights were checked with cannot be exchanged; a bias whose memory is another by the time of the call is read there."""
    g = torch.Generator(device="cuda").manual_seed(3)
    codes = torch.randint(0, 16, (48, 128), dtype=torch.uint8, device="cuda", generator=g)
    scales, zeros = torch.full((48, 1), 0.5, device="cuda"), torch.full((48, 1), 8.0, device="cuda")
    bias = torch.zeros(48, device="cuda")
    w = B.gptaq_linear_pack(codes, scales, zeros, 0, bias=bias)
    with pytest.raises(AttributeError):
        w.bias = torch.zeros(3, device="cuda")
    ws = B.workspace(B.gptaq_linear_workspace_bytes(4, 48, 128))
    X = torch.zeros((4, 128), dtype=torch.bfloat16, device="cuda")
    bias.data = torch.arange(48, device="cuda").float()
    assert torch.equal(B.gptaq_linear(X, w, ws, dtype=torch.float32), bias.expand(4, 48))
