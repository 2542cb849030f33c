"""From calibration to answers: the attention of a decoder block, its two layers solved by the library and then run from their codes over a paged cache.

    python -m paper_2504_02692_amd.quantized_attention [--hidden 4096 --heads 32 --kv-heads 32 --prompt 2048 --bits 8]

Calibration follows Algorithm 2 of the paper: o_proj's input is the output of attention behind the quantised qkv product, and of the full-precision block.
Afterwards a pass is norm, qkv, the rotation and the cache, attention, 8-bit codes, o_proj; a prompt is one pass, each later token another.  Weights and
inputs are random; the output says how far the quantised block is from the full one.
"""
from __future__ import annotations

import argparse
import math
import time
from typing import NamedTuple, Optional

import torch

from paper_2504_02692_amd import binding as B
from paper_2504_02692_amd.quantized_mlp import EPS, product, product_workspace_bytes, solve

BASE = 10000.0


class PagedCache:
    """Keys and values of `seqs` sequences, `page` positions to a page, and which pages are whose.  Pages are handed out as sequences grow (on the host)."""

    def __init__(self, seqs: int, pages: int, kv_heads: int, d: int, page: int, most: int):
        self.keys = torch.zeros((pages, kv_heads, d // 8, page, 8), dtype=torch.bfloat16, device="cuda")
        self.values = torch.zeros((pages, kv_heads, page // 8, d, 8), dtype=torch.bfloat16, device="cuda")
        self.page, self.free = page, list(range(pages))
        self.tables = [[] for _ in range(seqs)]
        self.counts = [0] * seqs
        self.table = torch.full((seqs, -(-most // page)), -1, dtype=torch.int32, device="cuda")
        self.starts = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")

    def grow(self, counts) -> None:
        """Makes room for counts[s] new tokens of each sequence, whose rows a pass takes one sequence after the other.  Where they do not fit, nothing changes."""
        if len(counts) != len(self.counts) or min(counts, default=0) < 0:
            raise ValueError(f"{len(self.counts)} sequences, each with a count of 0 or more, not {counts}")
        lengths = [had + count for had, count in zip(self.counts, counts)]
        missing = [max(0, -(-n // self.page) - len(table)) for n, table in zip(lengths, self.tables)]
        if sum(missing) > len(self.free) or any(len(table) + more > self.table.shape[1] for table, more in zip(self.tables, missing)):
            raise RuntimeError("the cache is full")
        starts = [0]
        for s, (table, more) in enumerate(zip(self.tables, missing)):
            starts.append(starts[-1] + counts[s])
            if more:                                     # (one copy a sequence)
                had = len(table)
                table += [self.free.pop() for _ in range(more)]
                self.table[s, had:had + more] = torch.tensor(table[had:], dtype=torch.int32)
        self.counts = lengths
        self.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        self.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))


def frequencies(pairs: int) -> torch.Tensor:
    return BASE ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)


class QuantizedAttention(NamedTuple):
    norm: torch.Tensor                           # bf16
    qkv: "B.LinearWeights | B.Linear8Weights"    # the queries' rows, the keys', the values'
    o: "Optional[B.LinearWeights | B.Linear8Weights]"      # (None until it is solved: `attend` does not need it)
    heads: int
    kv_heads: int
    d: int
    freqs: torch.Tensor
    window: int = 0
    sinks: int = 0

    def workspace(self, tokens: int, seqs: int) -> torch.Tensor:
        return B.workspace(max(product_workspace_bytes(tokens, self.qkv), product_workspace_bytes(tokens, self.o),
                               B.gptaq_attention_workspace_bytes(tokens, seqs, self.heads, self.kv_heads, self.d)))

    def attend(self, both: torch.Tensor, cache: PagedCache, ws: torch.Tensor) -> torch.Tensor:
        """Attention's output (tokens x heads d) from the rows of the qkv product; their keys and values go to the cache."""
        tokens, heads, kv, d = both.shape[0], self.heads, self.kv_heads, self.d
        q, k, v = (both[:, a * d:b * d].view(tokens, b - a, d) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
        q = B.gptaq_cache_append(q, k, v, cache.keys, cache.values, cache.table, cache.starts, cache.lengths, self.freqs)
        return B.gptaq_attention(q, cache.keys, cache.values, cache.table, cache.starts, cache.lengths, ws, window=self.window, sinks=self.sinks).view(tokens, heads * d)

    def __call__(self, x: torch.Tensor, residual: torch.Tensor, cache: PagedCache, ws: torch.Tensor):
        """(the block's output, x + residual) for the bf16 tokens that the cache has grown by; the caller adds them at its next norm."""
        codes, scales, total = B.gptaq_rms_norm_i8(x, self.norm, EPS, residual=residual)
        y = self.attend(product(codes, scales, self.qkv, ws), cache, ws)
        codes, scales = B.gptaq_quant_activations_i8(y)
        return product(codes, scales, self.o, ws), total


def full_attention(both: torch.Tensor, counts, heads: int, kv: int, d: int, window: int = 0, sinks: int = 0) -> torch.Tensor:
    """The same for whole sequences in fp32, from the rows of the qkv product."""
    freqs = frequencies(d // 2)
    out, first = torch.empty((both.shape[0], heads * d), device="cuda"), 0
    for n in counts:
        rows = both[first:first + n].float()
        at = torch.arange(n, device="cuda")
        angle = at.double()[:, None] * freqs
        cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]

        def heads_of(a, b, turn):
            t = rows[:, a * d:b * d].view(n, b - a, d)
            if turn:
                a, b = t[..., :d // 2], t[..., d // 2:]
                t = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
            return t.transpose(0, 1)
        q, k, v = heads_of(0, heads, True), heads_of(heads, heads + kv, True), heads_of(heads + kv, heads + 2 * kv, False)
        seen = at[None, :] <= at[:, None]
        if window:
            seen &= (at[None, :] > at[:, None] - window) | (at[None, :] < sinks)
        for h in range(heads):
            score = torch.matmul(q[h], k[h // (heads // kv)].t()) / math.sqrt(d)
            w = torch.softmax(torch.where(seen, score, float("-inf")), 1)
            out[first:first + n, h * d:(h + 1) * d] = torch.matmul(w, v[h // (heads // kv)])
        first += n
    return out


def full_precision(x: torch.Tensor, residual: torch.Tensor, norm: torch.Tensor, qkv: torch.Tensor, o: torch.Tensor, counts, heads: int, kv: int, window: int = 0,
                   sinks: int = 0) -> torch.Tensor:
    """The same block with weights in fp32, for whole sequences."""
    h = x.float() + residual.float()
    h = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * norm.float()
    return torch.matmul(full_attention(torch.matmul(h, qkv.t()), counts, heads, kv, o.shape[1] // heads, window, sinks), o.t())


def calibrate(hidden: int, heads: int, kv_heads: int, d: int, seqs: int, tokens: int, bits: int = 8, group: int = 0, act_order: bool = False, window: int = 0,
              sinks: int = 0, seed: int = 0):
    """A random block solved on `seqs` random sequences of `tokens` tokens: (QuantizedAttention, its weights in full precision and as quantised)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    norm = (1.0 + 0.1 * rand(hidden)).to(torch.bfloat16)
    qkv, o = rand((heads + 2 * kv_heads) * d, hidden) / math.sqrt(hidden), rand(hidden, heads * d) / math.sqrt(heads * d)
    x, residual = rand(seqs * tokens, hidden).to(torch.bfloat16), rand(seqs * tokens, hidden).to(torch.bfloat16)
    counts = [tokens] * seqs
    # first input: the model before this block is not quantised here, so both see the same
    h, _ = B.gptaq_rms_norm(x, norm, EPS, residual=residual)
    packed, qkv_q = solve(qkv, h, h, bits, group, act_order)
    # second input: of the full model, and of the one whose qkv is quantised
    full_input = full_attention(torch.matmul(h.float(), qkv.t()).to(torch.bfloat16), counts, heads, kv_heads, d, window, sinks).to(torch.bfloat16)
    block = QuantizedAttention(norm, packed, None, heads, kv_heads, d, frequencies(d // 2), window, sinks)
    cache = PagedCache(seqs, seqs * -(-tokens // 64), kv_heads, d, 64, tokens)
    cache.grow(counts)
    codes, scales = B.gptaq_quant_activations_i8(h)
    both = product(codes, scales, packed, B.workspace(product_workspace_bytes(seqs * tokens, packed)))
    here = block.attend(both, cache, B.workspace(B.gptaq_attention_workspace_bytes(seqs * tokens, seqs, heads, kv_heads, d)))
    packed_o, o_q = solve(o, here, full_input, bits, group, act_order)
    return block._replace(o=packed_o), (norm, qkv, o), (qkv_q, o_q)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=32)
    ap.add_argument("--head-size", type=int, default=128, choices=(64, 96, 128))
    ap.add_argument("--samples", type=int, default=8, help="calibration sequences")
    ap.add_argument("--prompt", type=int, default=2048, help="tokens of a calibration sequence, and of the prompt")
    ap.add_argument("--steps", type=int, default=16, help="tokens behind the prompt, one at a time")
    ap.add_argument("--bits", type=int, default=8, choices=(2, 3, 4, 5, 6, 7, 8))
    ap.add_argument("--group", type=int, default=0, choices=(0, 32, 64, 128))
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--act-order", action="store_true")
    a = ap.parse_args()
    if a.bits > 4:
        a.group = 0                                      # (one scale a row, as layers of more than 4 bits have)
    block, weights, _ = calibrate(a.hidden, a.heads, a.kv_heads, a.head_size, a.samples, a.prompt, a.bits, a.group, a.act_order, a.window, a.sinks)
    n = a.prompt + a.steps
    x, residual = (torch.randn((n, a.hidden), device="cuda").to(torch.bfloat16) for _ in range(2))
    want = full_precision(x, residual, *weights, [n], a.heads, a.kv_heads, a.window, a.sinks)
    cache = PagedCache(1, -(-n // 16), a.kv_heads, a.head_size, 16, n)
    ws = block.workspace(a.prompt, 1)
    first = 0
    for count in [a.prompt] + [1] * a.steps:
        cache.grow([count])
        rows = slice(first, first + count)
        torch.cuda.synchronize()
        began = time.perf_counter()
        y, _ = block(x[rows], residual[rows], cache, ws)
        torch.cuda.synchronize()
        us = (time.perf_counter() - began) * 1e6
        if count > 1 or first + count == n:
            off = (y.float() - want[rows]).norm().item() / want[rows].norm().item()
            print(f"positions {first} to {first + count - 1}: {us:8.1f} us, output {100 * off:.2f} % off the full-precision block's")
        first += count


if __name__ == "__main__":
    main()
