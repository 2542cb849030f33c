"""The operators between a norm and o_proj as a program runs them, prompts first and then a token at a time: each stage against its formula in 64 bits, from
what the stage before it returned, with the tolerances of that stage's own tests; and the module that runs them against these calls, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2504_02692_amd import binding as B
from paper_2504_02692_amd import quantized_attention as A
from paper_2504_02692_amd import quantized_mlp as M
from tests.test_gpu_attention import Cache, check, turned
from tests.test_gpu_linear8 import U
from tests.test_gpu_serving import bf16, f64

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8 * (1 + 2.0 ** -6)


class View(Cache):
    """What a cache on the device holds, as the checks of attention take it."""

    def __init__(self, cache, counts, kv, d):
        self.kv, self.d, self.page, self.pages = kv, d, cache.page, cache.keys.shape[0]
        self.table, self.starts, self.lengths = (t.cpu().numpy() for t in (cache.table, cache.starts, cache.lengths))
        self.tokens = int(self.starts[-1])
        self.pairs = [(c, int(n) - c) for c, n in zip(counts, self.lengths)]
        keys, values = f64(cache.keys), f64(cache.values)
        self.k, self.v = [], []
        for s, n in enumerate(self.lengths):
            p = np.arange(n)
            ids, slots = self.table[s][p // self.page], p % self.page
            self.k.append(keys[ids, :, :, slots].reshape(n, kv, d))
            self.v.append(values[ids, :, slots // 8, :, slots % 8].reshape(n, kv, d))


def product_is(got, codes, scales, weights):
    x = f64(codes) * f64(scales)[:, None]
    w = f64(weights)
    want = x @ w.T
    err = np.abs(f64(got) - want)
    # the weights here are the dequantised ones, rounded to fp32 each; the sums are taken of exact ones
    n = x.shape[1]
    assert np.all(err <= (n + 16) * 2 * U * (np.abs(x) @ np.abs(w).T) + np.abs(want) * HALF)


@pytest.mark.parametrize("bits,group,act_order,window,sinks,kv", [(8, 0, False, 0, 0, 2), (8, 0, True, 48, 4, 4), (6, 0, False, 0, 0, 1), (4, 64, False, 20, 0, 2)])
def test_prompts_and_steps(bits, group, act_order, window, sinks, kv):
    heads, d, hidden = 4, 64, 192
    block, _, (qkv_q, o_q) = A.calibrate(hidden, heads, kv, d, 4, 150, bits, group, act_order, window, sinks)
    cache, twin = (A.PagedCache(3, 60, kv, d, 16, 200) for _ in range(2))
    ws = block.workspace(200, 3)
    ws.fill_(255)
    r = np.random.default_rng(4)
    for counts in ([70, 0, 33], [1, 1, 1], [0, 90, 1], [1, 1, 1], [2, 1, 1]):
        tokens = sum(counts)
        x, residual = bf16(r.standard_normal((tokens, hidden))), bf16(r.standard_normal((tokens, hidden)))
        cache.grow(counts)
        twin.grow(counts)
        y, total = block(x, residual, twin, ws)
        assert torch.equal(total, (x.float() + residual.float()).to(torch.bfloat16))

        codes, scales, _ = B.gptaq_rms_norm_i8(x, block.norm, M.EPS, residual=residual)
        both = M.product(codes, scales, block.qkv, ws)
        product_is(both, codes, scales, qkv_q)
        q, k, v = (both[:, a * d:b * d].view(tokens, b - a, d) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
        turned_q = B.gptaq_cache_append(q, k, v, cache.keys, cache.values, cache.table, cache.starts, cache.lengths, block.freqs)
        view = View(cache, counts, kv, d)
        freqs = f64(block.freqs)
        for s, (count, before) in enumerate(view.pairs):
            here, at = slice(view.starts[s], view.starts[s + 1]), np.arange(before, before + count)
            for got, given in ((f64(turned_q)[here], q), (view.k[s][before:], k)):
                want, size = turned(f64(given)[here], at, freqs, False)
                assert np.all(np.abs(got - want) <= size * 2.0 ** -20 + np.abs(want) * HALF)
            assert np.array_equal(view.v[s][before:], f64(v)[here])
        attended = B.gptaq_attention(turned_q, cache.keys, cache.values, cache.table, cache.starts, cache.lengths, ws, window=window, sinks=sinks)
        check(attended, view, turned_q, heads, window, sinks)
        codes, scales = B.gptaq_quant_activations_i8(attended.view(tokens, heads * d))
        out = M.product(codes, scales, block.o, ws)
        product_is(out, codes, scales, o_q)
        assert torch.equal(y, out) and torch.equal(cache.keys, twin.keys) and torch.equal(cache.values, twin.values)


def test_an_mlp_of_8_bits():
    mlp, _, (gate_up_q, down_q) = M.calibrate(128, 320, 600, bits=8, group=0)
    r = np.random.default_rng(5)
    x, residual = bf16(r.standard_normal((70, 128))), bf16(r.standard_normal((70, 128)))
    ws = mlp.workspace(70)
    y, _ = mlp(x, residual, ws)
    codes, scales, _ = B.gptaq_rms_norm_i8(x, mlp.norm, M.EPS, residual=residual)
    both = M.product(codes, scales, mlp.gate_up, ws)
    product_is(both, codes, scales, gate_up_q)
    codes, scales = B.gptaq_silu_mul_i8(both[:, :320], both[:, 320:])
    out = M.product(codes, scales, mlp.down, ws)
    product_is(out, codes, scales, down_q)
    assert torch.equal(y, out)
