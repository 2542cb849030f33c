"""The operators that run quantised layers where their sums, their memory or their arguments could go wrong.

Where every partial sum, in any order, is a whole number of the smallest unit below 2^24 of these, fp32 holds all of them exactly, and
outputs are equal: in fp32 to the sum, in bfloat16 to the sum rounded to nearest even.
"""
import numpy as np
import pytest
import torch

from paper_2504_02692_amd import binding as B
from tests.test_gpu_serving import bf16, dequantised, f64, pack, quantised, rng

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
