"""From calibration to answers: the MLP of a decoder block, its three layers solved by the library and then run from their codes.

    python -m paper_2504_02692_amd.quantized_mlp [--hidden 4096 --inner 11008 --tokens 32768 --act-order]

Calibration follows Algorithm 2 of the paper: the layers' inputs are taken from the full-precision block and from the block as
it is quantised so far, gate and up share one Hessian.  Afterwards a pass is norm, gate and up, gated activation, down, with 8-bit or
bf16 activations between them.  Weights and inputs are random; the output says how far the quantised MLP is from the full one.
"""
from __future__ import annotations

import argparse
import time
from typing import NamedTuple

import torch

from paper_2504_02692_amd import binding as B

EPS = 1e-5


def solve(W: torch.Tensor, X: torch.Tensor, Xtilde: torch.Tensor, bits: int, group: int, act_order: bool, damp: float = 0.01):
    """(weights as the products read them, dequantised weights in the order of X's columns) of a layer W (fp32) that sees X."""
    m, n = W.shape
    H = torch.zeros((n, n), device="cuda")
    A = torch.zeros_like(H)
    B.gptaq_accumulate(X, Xtilde, H, A, B.workspace(B.gptaq_accumulate_workspace_bytes(X.shape[0], n)))
    perm = None
    if act_order:
        perm = B.gptaq_act_order(H)
        B.gptaq_permute_hessian(H, A, perm, B.workspace(B.gptaq_permute_hessian_workspace_bytes(n)))
    Q = B.gptaq_permute_columns_f32(W, perm) if act_order else W.clone()
    dead, info = B.gptaq_prepare(H, A, damp, B.workspace(B.gptaq_prepare_workspace_bytes(n)))
    codes, scales, zeros = B.gptaq_quantize_layer(Q, H, A, bits, group, False, 128, B.workspace(B.gptaq_quantize_workspace_bytes(m, n)), dead=dead)
    weights = B.gptaq_linear_pack(codes, scales, zeros, group, perm=perm)
    if info[0].item() != 0 or weights.info.item() != 0:
        raise RuntimeError(f"solve failed: info {info.tolist()}, {weights.info.tolist()}")
    return weights, B.gptaq_permute_columns_f32(Q, perm, inverse=True) if act_order else Q


class QuantizedMLP(NamedTuple):
    norm: torch.Tensor                           # bf16
    gate_up: B.LinearWeights                     # gate's rows, then up's
    down: B.LinearWeights

    def workspace(self, tokens: int) -> torch.Tensor:
        return B.workspace(max(B.gptaq_linear_workspace_bytes(tokens, w.m, w.n) for w in (self.gate_up, self.down)))

    def __call__(self, x: torch.Tensor, residual: torch.Tensor, ws: torch.Tensor, eight_bits: bool = True):
        """(the MLP's output, x + residual) for bf16 tokens; the caller adds them at its next norm."""
        inner = self.down.n
        if eight_bits:
            codes, scales, total = B.gptaq_rms_norm_i8(x, self.norm, EPS, residual=residual)
            both = B.gptaq_linear_i8(codes, scales, self.gate_up, ws)
            codes, scales = B.gptaq_silu_mul_i8(both[:, :inner], both[:, inner:])
            return B.gptaq_linear_i8(codes, scales, self.down, ws), total
        h, total = B.gptaq_rms_norm(x, self.norm, EPS, residual=residual)
        both = B.gptaq_linear(h, self.gate_up, ws)
        return B.gptaq_linear(B.gptaq_silu_mul(both[:, :inner], both[:, inner:]), self.down, ws), total


def full_precision(x: torch.Tensor, residual: torch.Tensor, norm: torch.Tensor, gate_up: torch.Tensor, down: torch.Tensor) -> torch.Tensor:
    """The same MLP with weights in fp32."""
    h = x.float() + residual.float()
    h = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * norm.float()
    gate, up = torch.matmul(h, gate_up.t()).chunk(2, 1)
    return torch.matmul(gate / (1.0 + torch.exp(-gate)) * up, down.t())


def calibrate(hidden: int, inner: int, tokens: int, bits: int = 4, group: int = 128, act_order: bool = False, seed: int = 0):
    """A random MLP solved on random tokens: (QuantizedMLP, its weights in full precision and as quantised)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    norm = (1.0 + 0.1 * rand(hidden)).to(torch.bfloat16)
    gate_up, down = 0.02 * rand(2 * inner, hidden), 0.02 * rand(hidden, inner)
    x, residual = rand(tokens, hidden).to(torch.bfloat16), rand(tokens, hidden).to(torch.bfloat16)
    # first input: the block before this MLP is not quantised here, so both models see the same
    h, _ = B.gptaq_rms_norm(x, norm, EPS, residual=residual)
    packed, gate_up_q = solve(gate_up, h, h, bits, group, act_order)
    # second input: of the full model, and of the one whose gate and up are quantised
    gate, up = torch.matmul(h.float(), gate_up.t()).to(torch.bfloat16).chunk(2, 1)
    full_input = B.gptaq_silu_mul(gate, up)
    both = B.gptaq_linear(h, packed, B.workspace(B.gptaq_linear_workspace_bytes(tokens, packed.m, packed.n)))
    here = B.gptaq_silu_mul(both[:, :inner], both[:, inner:])
    packed_down, down_q = solve(down, here, full_input, bits, group, act_order)
    return QuantizedMLP(norm, packed, packed_down), (gate_up, down), (gate_up_q, down_q)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--inner", type=int, default=11008)
    ap.add_argument("--tokens", type=int, default=32768, help="calibration tokens")
    ap.add_argument("--bits", type=int, default=4, choices=(2, 3, 4))
    ap.add_argument("--group", type=int, default=128, choices=(0, 32, 64, 128))
    ap.add_argument("--act-order", action="store_true")
    a = ap.parse_args()
    mlp, (gate_up, down), _ = calibrate(a.hidden, a.inner, a.tokens, a.bits, a.group, a.act_order)
    for tokens in (1, 16, 512, 2048):
        x, residual = (torch.randn((tokens, a.hidden), device="cuda").to(torch.bfloat16) for _ in range(2))
        ws = mlp.workspace(tokens)
        want = full_precision(x, residual, mlp.norm, gate_up, down)
        for eight_bits in (True, False):
            y, _ = mlp(x, residual, ws, eight_bits)
            torch.cuda.synchronize()
            began = time.perf_counter()
            for _ in range(20):
                mlp(x, residual, ws, eight_bits)
            torch.cuda.synchronize()
            us = (time.perf_counter() - began) / 20 * 1e6
            off = (y.float() - want).norm().item() / want.norm().item()
            print(f"{tokens:5d} tokens, {'8-bit' if eight_bits else 'bf16 '} activations: {us:8.1f} us a pass, "
                  f"output {100 * off:.1f} % off the full-precision MLP's")


if __name__ == "__main__":
    main()
