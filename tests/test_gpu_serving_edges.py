"""The operators that run quantised layers where their sums, their memory or their arguments could go wrong.

Where every partial sum, in any order, is a whole number of the smallest unit below 2^24 of these, fp32 holds all of them exactly, and
outputs are equal: in fp32 to the sum, in bfloat16 to the sum rounded to nearest even.
"""
import numpy as np
import pytest
import torch

from paper_2504_02692_amd import binding as B
from tests.test_gpu_serving import bf16, dequantised, f64, pack, padded, quantised, rng

pytestmark = pytest.mark.gpu


def rounded(want, dtype):
    """fp64 values that fp32 holds, as the outputs hold them."""
    assert np.array_equal(want.astype(np.float32).astype(np.float64), want)
    return torch.from_numpy(want.astype(np.float32)).to(dtype)


# ---- sums

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,m,n", [(1, 48, 98304), (20, 48, 98304), (600, 48, 98304), (1, 8200, 32768), (16, 8200, 32768), (5, 16400, 16384),
                                        (16, 16400, 16384), (32, 16400, 16384)])
def test_sums_of_one_sign_in_a_group_as_long_as_a_row(tokens, m, n, dtype):
    """code - zero is -1, 0 or 1 and the activations are whole numbers of 8 bits, all positive: the sums of these products stay below 2^24, those of
    16 + code, over the columns that one wavefront takes, far above."""
    g = torch.Generator(device="cuda").manual_seed(tokens + n)
    codes = torch.randint(13, 16, (m, n), dtype=torch.uint8, device="cuda", generator=g)
    zeros, scales = torch.full((m, 1), 14.0, device="cuda"), 2.0 ** torch.randint(-3, 3, (m, 1), device="cuda", generator=g).float()
    x = 2.0 * torch.randint(64, 128, (tokens, n), device="cuda", generator=g) + 1.0
    diff = codes.double() - 14.0
    assert torch.matmul(x.double(), diff.abs().t()).max().item() < 2 ** 24
    want = torch.matmul(x.double(), diff.t()) * scales.double()[:, 0]
    w = B.gptaq_linear_pack(codes, scales, zeros, 0)
    got = B.gptaq_linear(x.to(torch.bfloat16), w, B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n)), dtype=dtype)
    assert torch.equal(got.cpu(), rounded(want.cpu().numpy(), dtype))


@pytest.mark.parametrize("m", [80, 8200, 16400])
@pytest.mark.parametrize("tokens", [1, 5, 20, 300])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
def test_fp32_outputs_keep_small_activations_beside_a_large_one(tokens, group, m):
    """An outlier in each 128 columns, some 2^16 times the others, on whole numbers: exact in sums of code - zero."""
    n = 1024
    r = rng(tokens, group, 81)
    codes, zeros = r.integers(14, 16, (m, n)).astype(np.uint8), np.full((m, n // group if group else 1), 15.0, np.float32)
    scales = np.full(zeros.shape, 0.25, np.float32)
    x = 2.0 * r.integers(0, 8, (tokens, n)) + 1.0
    x[:, ::128] = 4096.0 * (2.0 * r.integers(64, 128, (tokens, n // 128)) + 1.0)
    assert x.sum(1).max() < 2 ** 24
    w = pack(codes, scales, zeros, group)
    ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
    got = B.gptaq_linear(bf16(x), w, ws, dtype=torch.float32)
    assert np.array_equal(f64(got), x @ dequantised(codes, scales, zeros, group).T)


def whole(tokens, m, n, group, perm=False, bias=False):
    """Activations of at most two bits and a sign, all codes and zeros, scales of 1/2 and 1: sums below 2^24 halves, and (16 + code) x likewise.
    Returns (weights, activations as fp64, outputs in fp64), on the GPU."""
    assert 2 * 31 * 3 * n < 2 ** 24
    g = torch.Generator(device="cuda").manual_seed(tokens + 7 * m + 11 * n + group)
    rand = lambda hi, *shape: torch.randint(0, hi, shape, device="cuda", generator=g)
    G = n // group if group else 1
    codes, zeros, scales = rand(16, m, n).to(torch.uint8), rand(16, m, G).float(), 0.5 * (1 + rand(2, m, G)).float()
    x = (rand(7, tokens, n) - 3).double()
    p = torch.randperm(n, device="cuda", generator=g).to(torch.int32) if perm else None
    b = (rand(64, m) - 32).float() if bias else None
    w = B.gptaq_linear_pack(codes, scales, zeros, group, perm=p, bias=b)
    assert w.info.item() == 0
    W = ((codes.view(m, G, -1).double() - zeros.double()[:, :, None]) * scales.double()[:, :, None]).view(m, n)
    want = torch.matmul(x[:, p.long()] if perm else x, W.t())
    return w, x, want + b.double() if bias else want


def product(x, w, dtype, i8, ws=None, out=None):
    ws = B.workspace(B.gptaq_linear_workspace_bytes(x.shape[0], w.m, w.n)) if ws is None else ws
    if i8:
        return B.gptaq_linear_i8(x.to(torch.int8), torch.ones(x.shape[0], device="cuda"), w, ws, dtype=dtype, out=out)
    return B.gptaq_linear(x.to(torch.bfloat16), w, ws, dtype=dtype, out=out)


def check_whole(tokens, m, n, group, i8, **other):
    print("whole", tokens, m, n, group, i8, other, flush=True)
    w, x, want = whole(tokens, m, n, group, **other)
    assert torch.equal(want.float().double(), want)
    for dtype in (torch.float32, torch.bfloat16):
        y = product(x, w, dtype, i8)
        assert torch.equal(y, want.float().to(dtype)), (dtype, (y.double() - want).abs().max().item())


# Rows in their hundreds of tiles, not a whole number of 32 or 64: a workgroup of the kernel of few tokens takes two tiles of them, then four.  Columns: several
# tiles to each wavefront and a remainder.
@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("m,n", [(8200, 2176), (8200, 8320), (16400, 2176), (16400, 8320)])
@pytest.mark.parametrize("tokens", [1, 9, 16, 17, 32])
def test_few_tokens_of_large_layers_are_exact(tokens, m, n, group, i8):
    check_whole(tokens, m, n, group, i8)


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m,n,perm", [(1, 8200, 2100, False), (16, 16400, 2100, True), (20, 8200, 1700, True), (32, 16400, 2100, False)])
def test_few_tokens_of_large_layers_of_any_width_are_exact(tokens, m, n, perm, i8):
    check_whole(tokens, m, n, 0, i8, perm=perm, bias=True)


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("tokens,m,n", [(1, 100, 16384), (16, 100, 16384), (30, 100, 16384), (200, 2100, 8320), (700, 2100, 16384), (1100, 4100, 8192)])
def test_long_rows_are_exact(tokens, m, n, group, i8):
    check_whole(tokens, m, n, group, i8)


@pytest.mark.parametrize("group", [0, 64, 128])
@pytest.mark.parametrize("tokens,m", [(5, 8200), (16, 8200), (1, 16400), (16, 16400)])
def test_large_layers_pass_on_what_is_not_finite(tokens, m, group):
    """An infinity or a NaN spoils its own token alone.  An activation that overflows times 16 + code, but meets codes equal to their zeros, spoils nothing."""
    n = 2176
    w, x, want = whole(tokens, m, n, group)
    G = n // group if group else 1
    W = torch.empty((m, n), dtype=torch.float64, device="cuda")
    for lo in range(0, n, 16):                                     # the weights' columns, by the products themselves
        unit = torch.zeros((16, n), dtype=torch.float64, device="cuda")
        unit[torch.arange(16), torch.arange(lo, lo + 16)] = 1.0
        W[:, lo:lo + 16] = product(unit, w, torch.float32, False).t()
    assert torch.equal(torch.matmul(x, W.t()), want)
    ws = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n))
    for at, value in ((37, float("inf")), (n - 1, float("-inf")), (5, float("nan"))):
        bad = x.clone()
        bad[0, at] = value
        y = product(bad, w, torch.bfloat16, False, ws)
        assert torch.equal(y[1:], want[1:].float().to(torch.bfloat16))
        col = W[:, at]
        if value == value:
            sign = col if value > 0 else -col
            assert torch.all(torch.isposinf(y[0][sign > 0])) and torch.all(torch.isneginf(y[0][sign < 0])) and torch.all(torch.isnan(y[0][sign == 0]))
        else:
            assert torch.isnan(y[0]).all()
    codes = torch.randint(0, 16, (m, n), dtype=torch.uint8, device="cuda")
    codes[:, 41] = 7
    v = B.gptaq_linear_pack(codes, torch.ones((m, G), device="cuda"), torch.full((m, G), 7.0, device="cuda"), group)
    huge = x.clone()
    huge[:, 41] = 0.0
    plain = product(huge, v, torch.bfloat16, False, ws)
    huge[0, 41], huge[tokens - 1, 41] = 2.0 ** 127, -2.0 ** 127
    assert torch.equal(product(huge, v, torch.bfloat16, False, ws), plain)


@pytest.mark.parametrize("i8", [False, True])
@pytest.mark.parametrize("tokens,m,n,group", [(700, 2100, 2048, 64), (1030, 4100, 1024, 0), (200, 2100, 8192, 128), (40, 1100, 16384, 32), (33, 8200, 256, 128)])
def test_many_tokens_with_rows_apart_are_read_in_place(tokens, m, n, group, i8):
    """Rows that start at 16 bytes but do not follow each other; what lies between them is NaN or 77."""
    w, x, _ = whole(tokens, m, n, group)
    x = x.to(torch.int8 if i8 else torch.bfloat16)
    apart = padded(x, 48)
    assert apart.data_ptr() % 16 == 0 and apart.stride(0) == n + 48
    ws, ones = B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n)), torch.ones(tokens, device="cuda")
    call = (lambda t: B.gptaq_linear_i8(t, ones, w, ws)) if i8 else (lambda t: B.gptaq_linear(t, w, ws))
    assert torch.equal(call(apart), call(x))


@pytest.mark.parametrize("ldx", [(1 << 23) - 8, 1 << 23])
def test_many_tokens_with_rows_far_apart(ldx):
    """As far as the kernel of many tokens reads them in place, and farther; outputs more than 2^32 elements from the first."""
    tokens, m, n, ldy = 300, 2100, 256, 1 << 24
    w, x, want = whole(tokens, m, n, 64)
    X = torch.empty((tokens - 1) * ldx + n, dtype=torch.bfloat16, device="cuda").as_strided((tokens, n), (ldx, 1))
    Y = torch.empty((tokens - 1) * ldy + m, dtype=torch.bfloat16, device="cuda").as_strided((tokens, m), (ldy, 1))
    X.copy_(x)
    B.gptaq_linear(X, w, B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n)), out=Y)
    assert torch.equal(Y, want.float().to(torch.bfloat16))


def test_more_tokens_than_one_launch_takes():
    """The most rows that a layer may have: 4096 tokens to a launch, the rest to another."""
    tokens, m, n = 4100, 1 << 20, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    codes = torch.randint(0, 16, (m, n), dtype=torch.uint8, device="cuda", generator=g)
    w = B.gptaq_linear_pack(codes, torch.ones((m, 1), device="cuda"), torch.full((m, 1), 8.0, device="cuda"), 128)
    x = (torch.randint(0, 7, (tokens, n), device="cuda", generator=g) - 3).float()
    y = B.gptaq_linear(x.to(torch.bfloat16), w, B.workspace(B.gptaq_linear_workspace_bytes(tokens, m, n)))
    for lo in range(0, m, 1 << 17):
        want = torch.matmul(x, (codes[lo:lo + (1 << 17)].float() - 8.0).t())
        assert torch.equal(y[:, lo:lo + (1 << 17)], want.to(torch.bfloat16)), lo


# ---- rows

def test_more_rows_than_one_launch_takes():
    tokens, n = (1 << 21) + 5, 8
    x = torch.randn((tokens, n), device="cuda", generator=torch.Generator(device="cuda").manual_seed(6)).to(torch.bfloat16)
    y, _ = B.gptaq_rms_norm(x, None, 1e-5)
    codes, scales = B.gptaq_silu_mul_i8(x, x)
    for part in (slice(0, 100), slice((1 << 21) - 50, tokens)):
        assert torch.equal(y[part], B.gptaq_rms_norm(x[part].clone(), None, 1e-5)[0])
        c, s = B.gptaq_silu_mul_i8(x[part].clone(), x[part].clone())
        assert torch.equal(codes[part], c) and torch.equal(scales[part], s)


@pytest.mark.parametrize("n", [40, 4096, 33000])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_rows_of_zeros_are_zeros_with_any_eps(n, eps):
    """h / sqrt(mean(h^2) + eps) of a row of zeros is 0 for every eps above 0, and so for eps = 0; other rows follow the formula there too."""
    x = bf16(rng(n, 90).standard_normal((5, n)))
    x[1], x[3] = 0.0, -0.0
    w = bf16(1.0 + rng(n, 91).standard_normal((1, n)))[0].contiguous()
    y, _ = B.gptaq_rms_norm(x, w, eps)
    codes, scales, total = B.gptaq_rms_norm_i8(x, w, eps, residual=torch.zeros_like(x))
    for k in (1, 3):
        assert torch.all(y[k] == 0) and torch.all(codes[k] == 0) and scales[k] == 0 and torch.all(total[k] == 0)
    h = f64(x)[[0, 2, 4]]
    want = h / np.sqrt(np.mean(h * h, 1, keepdims=True) + eps) * f64(w)
    rel = (n + 16) * 2.0 ** -24
    assert np.all(np.abs(f64(y)[[0, 2, 4]] - want) <= np.abs(want) * (2.0 ** -8 * (1 + 2.0 ** -6) + rel) + 2.0 ** -133)
    s = np.abs(want).max(1) / 127.0
    assert np.all(np.abs(f64(scales)[[0, 2, 4]] - s) <= rel * s)


# ---- arguments

def test_memory_of_another_device_is_refused(monkeypatch):
    """Tensors in host memory, or on a GPU that is not the current one, are refused by every call before anything is launched."""
    w = pack(*quantised(16, 64, 4, 32, False, rng(1)), 32, perm=np.arange(64, dtype=np.int32), bias=np.zeros(16, np.float32))
    ws = B.workspace(B.gptaq_linear_workspace_bytes(4, 16, 64))
    x, row = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda"), torch.ones(64, dtype=torch.bfloat16, device="cuda")
    q, s = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda")
    y = torch.zeros((4, 16), dtype=torch.bfloat16, device="cuda")
    host = lambda **other: B.LinearWeights(**{**{k: getattr(w, k) for k in ("data", "m", "n", "group", "perm", "bias", "info")}, **other})
    calls = [lambda: B.gptaq_linear(x, w, ws.cpu()), lambda: B.gptaq_linear_i8(q, s, w, ws.cpu()), lambda: B.gptaq_linear(x, w, ws, out=y.cpu()),
             lambda: B.gptaq_linear(x, host(data=w.data.cpu()), ws), lambda: B.gptaq_linear(x, host(perm=w.perm.cpu()), ws),
             lambda: B.gptaq_linear_i8(q, s, host(bias=w.bias.cpu()), ws), lambda: B.gptaq_linear_i8(q, s.cpu(), w, ws),
             lambda: B.gptaq_rms_norm(x, row.cpu(), 1e-5), lambda: B.gptaq_rms_norm(x, row, 1e-5, residual=x.cpu()),
             lambda: B.gptaq_rms_norm_i8(x, row, 1e-5, total=x.cpu()), lambda: B.gptaq_silu_mul(x, x.cpu()),
             lambda: B.gptaq_silu_mul(x, x, out=x.cpu()), lambda: B.gptaq_silu_mul_i8(x.cpu(), x),
             lambda: B.gptaq_accumulate(x, x, torch.zeros((64, 64), device="cuda"), torch.zeros((64, 64), device="cuda"), torch.empty(1 << 20, dtype=torch.uint8)),
             lambda: B.gptaq_prepare(torch.eye(64, device="cuda"), torch.zeros((64, 64), device="cuda"), 0.01, torch.empty(1 << 20, dtype=torch.uint8))]
    for k, call in enumerate(calls):
        with pytest.raises(B.GptaqError):
            call()
            pytest.fail(f"call {k} was taken")
    here = torch.cuda.current_device()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: here + 1)
    for k, call in enumerate([lambda: B.gptaq_linear(x, w, ws), lambda: B.gptaq_linear_i8(q, s, w, ws), lambda: B.gptaq_rms_norm(x, row, 1e-5),
                              lambda: B.gptaq_rms_norm_i8(x, row, 1e-5), lambda: B.gptaq_silu_mul(x, x), lambda: B.gptaq_silu_mul_i8(x, x)]):
        with pytest.raises(B.GptaqError):
            call()
            pytest.fail(f"call {k} was taken")


def test_stored_weights_run_as_before(tmp_path):
    w = pack(*quantised(40, 96, 4, 32, False, rng(2)), 32, perm=rng(3).permutation(96).astype(np.int32), bias=np.ones(40, np.float32))
    x, ws = bf16(rng(4).standard_normal((3, 96))), B.workspace(B.gptaq_linear_workspace_bytes(3, 40, 96))
    torch.save(w, tmp_path / "layer.pt")
    with torch.serialization.safe_globals([B.LinearWeights]):
        again = torch.load(tmp_path / "layer.pt", weights_only=True)
    assert torch.equal(B.gptaq_linear(x, again, ws), B.gptaq_linear(x, w, ws))


def test_one_row_or_one_column_with_any_stride():
    """A row alone is row-major whatever its stride is, and so is a column alone: torch says contiguous, and so do the calls."""
    n, m = 96, 40
    lone = lambda t: t.reshape(-1, 1).clone().t()                                 # (1, n), strides (1, 1)
    x, res, g = (bf16(rng(k, 95).standard_normal((1, n))) for k in range(3))
    assert lone(x).stride(0) == 1 and lone(x).is_contiguous()
    codes, scales, zeros = quantised(m, n, 4, 32, False, rng(96))
    w, ws = pack(codes, scales, zeros, 32), B.workspace(B.gptaq_linear_workspace_bytes(4, m, n))
    y = B.gptaq_linear(x, w, ws)
    assert torch.equal(B.gptaq_linear(lone(x), w, ws), y) and torch.equal(B.gptaq_linear(x.expand(4, n)[:1], w, ws, out=lone(y)), y)
    c, s, total = B.gptaq_rms_norm_i8(x, None, 1e-5, residual=res)
    assert all(torch.equal(a, b) for a, b in zip(B.gptaq_rms_norm_i8(lone(x), None, 1e-5, residual=lone(res), total=lone(x)), (c, s, total)))
    assert torch.equal(B.gptaq_linear_i8(lone(c), s, w, ws), B.gptaq_linear_i8(c, s, w, ws))
    h, _ = B.gptaq_rms_norm(x, None, 1e-5)
    assert torch.equal(B.gptaq_rms_norm(lone(x), None, 1e-5, out=lone(x))[0], h)
    assert torch.equal(B.gptaq_silu_mul(lone(g), lone(x), out=lone(x)), B.gptaq_silu_mul(g, x))
    assert all(torch.equal(a, b) for a, b in zip(B.gptaq_silu_mul_i8(lone(g), lone(x)), B.gptaq_silu_mul_i8(g, x)))
    one = [torch.from_numpy(a[:1].copy()).cuda() for a in (codes, scales, zeros)]
    v = B.gptaq_linear_pack(lone(one[0]), one[1], one[2], 32)
    assert torch.equal(B.gptaq_linear(x, v, ws), y[:, :1])
    column = bf16(rng(97).standard_normal((1, 3))).t()                            # (3, 1), strides (1, 3)
    assert column.stride(1) == 3
    assert torch.equal(B.gptaq_silu_mul(column, column), B.gptaq_silu_mul(column.contiguous().clone(), column.clone()))
    wide = torch.zeros((3, 8), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.GptaqError):
        B.gptaq_silu_mul(wide[:, ::2], wide[:, ::2])
