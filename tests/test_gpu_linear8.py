"""Products with weights of up to 8 bits and 8-bit activations, and rows as 8-bit codes, against their formulas in 64 bits on the CPU.

Tolerances, with u = 2^-24: a sum of whole products is exact.  It is rounded to fp32 (u), multiplied by the product of two scales (u), and the result with the
bias is rounded (u of the result, at most u (|sum scales| + |bias|)): 3 u of |sum scales| + |bias| and second-order terms, 4 u in all.  A value
rounded to bfloat16 is off by 2^-8 of itself at most.  Codes are compared for equality: the formula is taken in fp32 by numpy, operation for operation.
"""
import numpy as np
import pytest
import torch

from paper_2504_02692_amd import binding as B
from tests.test_gpu_serving import bf16, f64, padded

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def layer(m, n, bits, sym, r):
    codes = r.integers(0, 2 ** bits, (m, n)).astype(np.uint8)
    scales = (0.0005 + 0.01 * r.random((m, 1))).astype(np.float32)
    zeros = np.full((m, 1), 2.0 ** (bits - 1)) if sym else r.integers(0, 2 ** bits, (m, 1)).astype(float)
    return codes, scales, zeros.astype(np.float32)


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def case(tokens, m, n, bits=8, sym=False, perm=False, bias=False, f32=False, extra=0, shift=0, extremes=False):
    print("linear8", tokens, m, n, bits, sym, perm, bias, f32, extra, shift, extremes, flush=True)
    r = np.random.default_rng([tokens, m, n, bits])
    codes, scales, zeros = layer(m, n, bits, sym, r)
    x = r.integers(-127, 128, (tokens, n)).astype(np.int8)
    if extremes:                                                   # the largest sums there are
        x[:] = -128
        codes[:], zeros[:] = 0, 255
        codes[1::2], zeros[1::2] = 255, 0
    xs = (0.01 + 0.1 * r.random(tokens)).astype(np.float32)
    p = r.permutation(n).astype(np.int32) if perm else None
    b = r.standard_normal(m).astype(np.float32) if bias else None
    w = B.gptaq_linear8_pack(padded(dev(codes), extra % 7, shift), dev(scales), dev(zeros), perm=dev(p), bias=dev(b))
    assert w.info.item() == 0
    ws = B.workspace(B.gptaq_linear8_workspace_bytes(tokens, m, n))
    ws.fill_(77)
    dtype = torch.float32 if f32 else torch.bfloat16
    whole = torch.full((tokens + 2, m + extra + 1), 7.0, dtype=dtype, device="cuda")
    out = whole[1:-1, :m]
    Y = B.gptaq_linear8_i8(padded(dev(x), extra, shift), dev(xs), w, ws, out=out)
    assert Y is out
    xp = (x[:, p] if perm else x).astype(np.float64)
    want = (xp @ (codes.astype(np.float64) - zeros).T) * xs.astype(np.float64)[:, None] * scales.astype(np.float64)[:, 0]
    size = np.abs(want) + (np.abs(b) if bias else 0.0)
    want = want + (b.astype(np.float64) if bias else 0.0)
    tol = 4 * U * size + (0.0 if f32 else np.abs(want) * 2.0 ** -8 * (1 + 2.0 ** -6))
    err = np.abs(f64(Y) - want)
    assert np.all(err <= tol), (float(np.max(err / np.maximum(tol, 1e-300))), np.argwhere(err > tol)[:4].tolist())
    assert torch.all(whole[0] == 7.0) and torch.all(whole[-1] == 7.0) and torch.all(whole[:, m:] == 7.0)      # nothing beside the outputs


SHAPES = [(1, 1, 1), (1, 16, 64), (1, 17, 128), (2, 5, 96), (3, 33, 192), (1, 257, 1000), (16, 48, 640), (17, 64, 384), (15, 100, 136), (33, 129, 256), (64, 128, 1024),
          (65, 80, 520), (130, 272, 512), (1, 2048, 11008), (300, 512, 768), (257, 515, 1024), (700, 1040, 384), (520, 256, 2736), (16, 8200, 256), (9, 16400, 128),
          (17, 30, 2048), (32, 500, 1536), (33, 260, 2176), (64, 129, 4096), (65, 1000, 2944), (128, 60, 8192), (129, 300, 5000), (300, 258, 3968), (18, 1, 16384),
          (1000, 700, 130), (513, 2050, 127), (48, 4096, 384), (1030, 1100, 1280)]


@pytest.mark.parametrize("tokens,m,n", SHAPES)
def test_linear8_is_the_formula(tokens, m, n):
    case(tokens, m, n, f32=True)


@pytest.mark.parametrize("tokens", [1, 9, 33, 70, 400, 1100])
@pytest.mark.parametrize("bits,sym,perm,bias,f32", [(5, False, True, False, True), (6, True, False, True, False), (8, True, True, True, True), (8, False, True, True, False),
                                                   (3, False, False, False, True)])
def test_linear8_forms(tokens, bits, sym, perm, bias, f32):
    case(tokens, 144, 512, bits, sym, perm, bias, f32)
    case(tokens, 530, 333, bits, sym, perm, bias, f32)


@pytest.mark.parametrize("tokens", [1, 20, 200, 600])
@pytest.mark.parametrize("extra,shift", [(16, 0), (3, 0), (0, 1), (16, 16), (7, 5)])
def test_linear8_strides_and_alignment(tokens, extra, shift):
    case(tokens, 96, 256, extra=extra, shift=shift)
    case(tokens, 300, 1003, extra=extra, shift=shift, f32=True)


@pytest.mark.parametrize("tokens", [1, 40, 300])
@pytest.mark.parametrize("n", [65536, 65535, 11008])
def test_linear8_holds_the_largest_sums(tokens, n):
    case(tokens, 34, n, extremes=True, f32=True)


def test_pack_says_what_is_wrong():
    r = np.random.default_rng(3)
    codes, scales, zeros = layer(40, 300, 8, False, r)
    for row, bad in ((0, -1.0), (39, 256.0), (17, 3.5), (5, float("nan"))):
        z = zeros.copy()
        z[row] = bad
        assert B.gptaq_linear8_pack(dev(codes), dev(scales), dev(z)).info.item() == 1 + row
    for change, column in ((lambda p: p.__setitem__(9, p[10]), 9), (lambda p: p.__setitem__(0, 300), 0), (lambda p: p.__setitem__(299, -1), 299)):
        p = r.permutation(300).astype(np.int32)
        named = p[column]
        change(p)
        assert B.gptaq_linear8_pack(dev(codes), dev(scales), dev(zeros), perm=dev(p)).info.item() == -1 - named


def test_linear8_refuses_what_does_not_fit():
    r = np.random.default_rng(4)
    codes, scales, zeros = (dev(a) for a in layer(32, 128, 8, False, r))
    w = B.gptaq_linear8_pack(codes, scales, zeros)
    x, xs, ws = torch.zeros((4, 128), dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda"), B.workspace(1 << 20)
    for wrong in (lambda: B.gptaq_linear8_i8(x[:, :64], xs, w, ws), lambda: B.gptaq_linear8_i8(x, xs[:3], w, ws), lambda: B.gptaq_linear8_i8(x, xs, w, ws, dtype=torch.float16),
                  lambda: B.gptaq_linear8_i8(x, xs, w, ws[:256]), lambda: B.gptaq_linear8_i8(x, xs, w, ws.cpu()), lambda: B.gptaq_linear8_i8(x.float(), xs, w, ws),
                  lambda: B.gptaq_linear8_i8(x, xs, w, ws, out=torch.empty((4, 31), device="cuda")), lambda: B.gptaq_linear8_pack(codes, scales[:5], zeros),
                  lambda: B.gptaq_linear8_pack(codes, scales.expand(32, 2), zeros), lambda: B.gptaq_linear8_pack(codes.float(), scales, zeros),
                  lambda: B.gptaq_linear8_pack(codes, scales, zeros, perm=torch.zeros(5, dtype=torch.int32, device="cuda")),
                  lambda: B.gptaq_linear8_pack(codes, scales, zeros, bias=torch.zeros(5, device="cuda")), lambda: B.gptaq_linear8_i8(x, xs, w, ws, out=torch.empty((4, 32)))):
        with pytest.raises(B.GptaqError):
            wrong()
    assert B.gptaq_linear8_i8(x[:0], xs[:0], w, ws).shape == (0, 32)


def test_linear8_captured_and_replayed():
    """Two graphs that share a workspace, replayed in turn on new inputs, against eager calls."""
    r = np.random.default_rng(6)
    codes, scales, zeros = (dev(a) for a in layer(600, 1000, 8, False, r))
    w = B.gptaq_linear8_pack(codes, scales, zeros)
    ws = B.workspace(B.gptaq_linear8_workspace_bytes(300, 600, 1000))
    inputs = [(torch.zeros((t, 1000), dtype=torch.int8, device="cuda"), torch.zeros(t, device="cuda"), torch.empty((t, 600), device="cuda")) for t in (5, 300)]
    graphs = []
    for x, xs, y in inputs:
        B.gptaq_linear8_i8(x, xs, w, ws, out=y)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.gptaq_linear8_i8(x, xs, w, ws, out=y)
        graphs.append(g)
    for _ in range(3):
        for (x, xs, y), g in zip(inputs, graphs):
            x.copy_(dev(r.integers(-127, 128, x.shape).astype(np.int8)))
            xs.copy_(dev(r.random(len(xs)).astype(np.float32)))
            g.replay()
        torch.cuda.synchronize()
        for x, xs, y in inputs:
            got = y.clone()
            assert torch.equal(B.gptaq_linear8_i8(x, xs, w, ws, dtype=torch.float32), got)


# ---- codes

def codes_of(x, clip):
    """The formula in fp32."""
    top = np.abs(x).max(1)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        scale = top * (np.float32(clip) / np.float32(127))
        q = np.where(scale[:, None] > 0, np.rint(x / scale[:, None]), np.float32(0))
    return np.clip(q, -127, 127).astype(np.int8), scale


@pytest.mark.parametrize("clip", [1.0, 0.9, 0.03])
@pytest.mark.parametrize("tokens,n,extra,shift", [(1, 1, 0, 0), (1, 7, 0, 1), (3, 64, 0, 0), (5, 511, 2, 3), (2, 4096, 8, 0), (600, 1000, 0, 0), (513, 8192, 0, 0), (1, 28672, 0, 0),
                                                  (530, 11008, 3, 1), (2, 40001, 0, 1)])
def test_codes_are_the_formula(tokens, n, extra, shift, clip):
    r = np.random.default_rng([tokens, n])
    X = bf16(r.standard_normal((tokens, n)) * np.where(r.random(n) < 0.02, 20.0, 1.0) * 2.0 ** r.integers(-60, 60, (tokens, 1)))
    codes, scales = B.gptaq_quant_activations_i8(padded(X, extra, shift), clip)
    want, scale = codes_of(X.float().cpu().numpy(), clip)
    assert np.array_equal(scales.cpu().numpy(), scale)
    assert np.array_equal(codes.cpu().numpy(), want)


def test_codes_at_ties_and_ends():
    """Quotients exactly between two codes go to the even one; rows of zeros, tiny rows, the largest rows, and rows that are not finite."""
    half = np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 63.5, -62.5, 126.5, 0.0]])
    X = bf16(np.concatenate([half, half * 2.0 ** 100, half * 2.0 ** -130, np.zeros((1, 10)), np.full((1, 10), 3.3e38), half * 2.0 ** -133]))
    codes, scales = B.gptaq_quant_activations_i8(X)
    want, scale = codes_of(X.float().cpu().numpy(), 1.0)
    assert np.array_equal(codes.cpu().numpy()[:5], want[:5]) and np.array_equal(scales.cpu().numpy()[:5], scale[:5])
    assert codes[0].tolist() == [127, 0, 2, 2, 0, -2, 64, -62, 126, 0] and scales[3].item() == 0.0 and codes[3].abs().max().item() == 0
    for bad in (float("inf"), -float("inf"), float("nan")):
        Y = X[:2].clone()
        Y[1, 4] = bad
        codes, scales = B.gptaq_quant_activations_i8(Y)
        assert torch.isnan(scales[1]) and not torch.isnan(scales[0]) and np.array_equal(codes[0].cpu().numpy(), want[0])
    assert B.gptaq_quant_activations_i8(X[:0])[0].shape == (0, 10)
    for wrong in (lambda: B.gptaq_quant_activations_i8(X, 0.0), lambda: B.gptaq_quant_activations_i8(X.float()), lambda: B.gptaq_quant_activations_i8(X.cpu())):
        with pytest.raises(B.GptaqError):
            wrong()


# ---- many tokens: every tile of linear8_many_kernel, and the columns in parts

def many_plan(tokens, m, n):
    """(tile, parts) of a call, or None where it takes the kernel of few tokens: the rule as launch_linear8 and many8_plan have it."""
    mt, kt, blocks = -(-m // 16), -(-n // 128), -(-tokens // 32)
    if blocks == 1 or (blocks * mt <= 2048 and blocks * mt * kt <= 57344):
        return None
    tiles = [-(-tokens // t) * -(-m // r) for t, r in ((64, 128), (128, 128), (256, 256))]
    t0, t1 = tiles[0] / 256, tiles[1] / 256
    times = [kt * (max(0.5, 0.38 * t0) if t0 <= 2 else max(1.0, 0.37 * t0)), kt * (0.7 if t1 <= 1 else max(1.15, 0.69 * t1)),
             kt * (1.6 if tiles[2] <= 128 else 1.9 * -(-tiles[2] // 256))]
    read = m * kt * 128 / 5e6
    best, least = (times.index(min(times)), 1), max(min(times), read)
    for parts in range(2, min(kt // 4, 512 // tiles[0]) + 1):
        us = max(read, kt / parts * max(0.5, 0.36 * t0 * parts)) + 4 + parts * tokens * m * 8 / 2.5e6
        if us < least:
            best, least = (0, parts), us
    return best


MANY = [  # tile and parts, tokens, m, n, what else of `case`
    ((0, 1), 97, 8200, 130, dict(bias=True)), ((0, 1), 257, 4097, 128, dict(bias=True, perm=True)), ((0, 1), 1030, 1000, 100, dict(bits=5)),
    ((0, 1), 257, 4097, 384, dict(sym=True, f32=True, bias=True, extra=3, shift=1)),
    ((0, 2), 65, 8200, 5003, dict(bias=True)), ((0, 2), 3000, 260, 5003, dict(f32=True, perm=True)), ((0, 3), 33, 8200, 8192, dict(bias=True, bits=6)),
    ((0, 3), 1500, 515, 5003, dict(bias=True, f32=True)), ((0, 4), 257, 2050, 8192, dict(perm=True, extra=16)), ((0, 5), 200, 2050, 8192, dict(bias=True, shift=5)),
    ((0, 6), 700, 515, 11008, dict(sym=True)),
    ((1, 1), 3000, 2050, 100, dict(bias=True)), ((1, 1), 1030, 6000, 130, dict(f32=True, bits=7)), ((1, 1), 3000, 2050, 384, dict(perm=True, bias=True, extra=7)),
    ((1, 1), 1030, 6001, 640, dict(sym=True, f32=True, bias=True)),
    ((2, 1), 1500, 8200, 100, dict(bias=True)), ((2, 1), 4097, 3001, 130, dict(f32=True, bias=True)), ((2, 1), 1500, 8200, 384, dict(perm=True, shift=1)),
    ((2, 1), 2100, 6001, 640, dict(bits=5, bias=True, extra=16)),
]


@pytest.mark.parametrize("plan,tokens,m,n,form", MANY)
def test_many_tokens_in_every_tile_and_in_parts(plan, tokens, m, n, form):
    assert many_plan(tokens, m, n) == plan
    case(tokens, m, n, **form)


@pytest.mark.parametrize("tokens,m,n,plan", [(200, 260, 65536, (0, 30)), (3000, 2050, 384, (1, 1)), (1500, 8200, 384, (2, 1))])
def test_many_tokens_hold_the_largest_sums(tokens, m, n, plan):
    assert many_plan(tokens, m, n) == plan
    case(tokens, m, n, extremes=True, f32=True)


def test_parts_captured_and_replayed():
    """Graphs of calls whose columns are in parts, and of others, that share a workspace, replayed in turn on new inputs, against eager calls."""
    r = np.random.default_rng(16)
    m, n = 2050, 8192
    codes, scales, zeros = (dev(a) for a in layer(m, n, 8, False, r))
    w = B.gptaq_linear8_pack(codes, scales, zeros)
    tokens = (257, 9, 200)
    assert [many_plan(t, m, n) for t in tokens] == [(0, 4), None, (0, 5)]
    ws = B.workspace(B.gptaq_linear8_workspace_bytes(max(tokens), m, n))
    inputs = [(torch.zeros((t, n), dtype=torch.int8, device="cuda"), torch.zeros(t, device="cuda"), torch.empty((t, m), device="cuda")) for t in tokens]
    graphs = []
    for x, xs, y in inputs:
        B.gptaq_linear8_i8(x, xs, w, ws, out=y)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.gptaq_linear8_i8(x, xs, w, ws, out=y)
        graphs.append(g)
    for _ in range(3):
        for (x, xs, y), g in zip(inputs, graphs):
            x.copy_(dev(r.integers(-127, 128, x.shape).astype(np.int8)))
            xs.copy_(dev(r.random(len(xs)).astype(np.float32)))
            g.replay()
        torch.cuda.synchronize()
        for x, xs, y in inputs:
            got = y.clone()
            ws.fill_(255)
            assert torch.equal(B.gptaq_linear8_i8(x, xs, w, ws, dtype=torch.float32), got)
            want = torch.matmul(x.double(), (codes.double() - zeros).t().contiguous()) * xs.double()[:, None] * scales[:, 0].double()
            assert torch.all((got.double() - want).abs() <= 4 * U * want.abs())


@pytest.mark.parametrize("clip", [1.0, 0.5])
def test_codes_of_rows_whose_scale_is_subnormal(clip):
    """Scales that have few bits left, and no reciprocal in fp32: scale and codes are still those of the formula; so are rows of the smallest values there are."""
    half = np.array([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 63.5, -62.5, 126.5, 0.0])
    X = bf16(np.stack([half * 2.0 ** -k for k in (120, 126, 127, 129, 130, 132, 133)] + [np.r_[2.0 ** -133, -(2.0 ** -133), np.zeros(8)], np.full(10, -(2.0 ** -126))]))
    codes, scales = B.gptaq_quant_activations_i8(X, clip)
    want, scale = codes_of(X.float().cpu().numpy(), clip)
    assert np.all(scale > 0) and np.any(scale < 2.0 ** -130)
    assert np.array_equal(scales.cpu().numpy(), scale) and np.array_equal(codes.cpu().numpy(), want)
