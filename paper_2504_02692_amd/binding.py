"""Thin ctypes binding of libgptaq.so.  Argument marshalling only: every step of the solve
runs in the library's HIP kernels.  torch is used for device memory and the current stream.

The functions carry the names of the C entry points (include/gptaq.h).  There is no CPU or
PyTorch fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgptaq.so")
_lib: Optional[ctypes.CDLL] = None

_c = ctypes
_SIGS = {
    "gptaq_status_string": (_c.c_char_p, [_c.c_int]),
    "gptaq_last_hip_error": (_c.c_int, []),
    "gptaq_accumulate_workspace_bytes": (_c.c_size_t, [_c.c_int64, _c.c_int64]),
    "gptaq_accumulate": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64,
                                    _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "gptaq_accumulate_upper": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64,
                                          _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "gptaq_accumulate_noalloc": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64,
                                            _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gptaq_accumulate_staged": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_void_p,
                                           _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_size_t, _c.POINTER(_c.c_int64),
                                           _c.c_int, _c.c_void_p]),
    "gptaq_accumulate_staged_upper": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64,
                                                 _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_size_t,
                                                 _c.POINTER(_c.c_int64), _c.c_int, _c.c_void_p]),
    "gptaq_symmetrize": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p]),
    "gptaq_prepare_workspace_bytes": (_c.c_size_t, [_c.c_int64]),
    "gptaq_prepare": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_float,
                                 _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "gptaq_quantize_workspace_bytes": (_c.c_size_t, [_c.c_int64, _c.c_int64]),
    "gptaq_quantize_layer": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p,
                                        _c.c_int64, _c.c_void_p, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                        _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_size_t,
                                        _c.c_void_p]),
    "gptaq_quantize_layer_terms": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p,
                                              _c.c_int64, _c.c_void_p, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                              _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_size_t,
                                              _c.c_void_p, _c.c_int]),
    "gptaq_quantize_layer_ex": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p,
                                           _c.c_int64, _c.c_void_p, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                           _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_size_t,
                                           _c.c_void_p, _c.c_int, _c.c_int, _c.c_int]),
    "gptaq_act_order": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p]),
    "gptaq_accumulate_diag": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p]),
    "gptaq_invert_permutation": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p]),
    "gptaq_accumulate_upper_permuted": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_void_p,
                                                   _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_size_t,
                                                   _c.c_void_p]),
    "gptaq_permute_hessian_workspace_bytes": (_c.c_size_t, [_c.c_int64]),
    "gptaq_permute_hessian": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p,
                                         _c.c_size_t, _c.c_void_p]),
    "gptaq_permute_columns_f32": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int64,
                                             _c.c_void_p, _c.c_int, _c.c_void_p]),
    "gptaq_permute_columns_u8": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int64,
                                            _c.c_void_p, _c.c_int, _c.c_void_p]),
    "gptaq_fake_quant_activations": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int64,
                                                _c.c_int, _c.c_float, _c.c_void_p]),
    "gptaq_packed_words_per_row": (_c.c_int64, [_c.c_int64, _c.c_int]),
    "gptaq_pack_codes": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int, _c.c_void_p, _c.c_void_p]),
    "gptaq_linear_weights_bytes": (_c.c_size_t, [_c.c_int64, _c.c_int64, _c.c_int]),
    "gptaq_linear_pack": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int, _c.c_void_p,
                                     _c.c_size_t, _c.c_void_p, _c.c_void_p]),
    "gptaq_linear_workspace_bytes": (_c.c_size_t, [_c.c_int64, _c.c_int64, _c.c_int64]),
    "gptaq_linear": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_size_t, _c.c_int64, _c.c_int64, _c.c_int,
                                _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "gptaq_linear_i8": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_size_t, _c.c_int64,
                                   _c.c_int64, _c.c_int, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "gptaq_rms_norm": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_float,
                                  _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "gptaq_rms_norm_i8": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_float,
                                     _c.c_void_p, _c.c_int64, _c.c_float, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p]),
    "gptaq_silu_mul": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_int64,
                                  _c.c_void_p]),
    "gptaq_silu_mul_i8": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_float, _c.c_void_p,
                                     _c.c_int64, _c.c_void_p, _c.c_void_p]),
    "gptaq_linear8_weights_bytes": (_c.c_size_t, [_c.c_int64, _c.c_int64]),
    "gptaq_linear8_pack": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_void_p,
                                      _c.c_size_t, _c.c_void_p, _c.c_void_p]),
    "gptaq_linear8_workspace_bytes": (_c.c_size_t, [_c.c_int64, _c.c_int64, _c.c_int64]),
    "gptaq_linear8_i8": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_size_t, _c.c_int64, _c.c_int64,
                                    _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int, _c.c_void_p, _c.c_size_t, _c.c_void_p]),
    "gptaq_quant_activations_i8": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_float, _c.c_void_p, _c.c_int64, _c.c_void_p,
                                              _c.c_void_p]),
    "gptaq_cache_append": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64] * 3 + [_c.c_char_p, _c.c_int64, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_int,
                                     _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p]),
    "gptaq_attention_workspace_bytes": (_c.c_size_t, [_c.c_int64] * 5),
    "gptaq_attention": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_char_p] + [_c.c_int64] * 4 + [_c.c_float, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p,
                                   _c.c_size_t, _c.c_void_p]),
    "gptaq_profile_enable": (_c.c_int, [_c.c_int]),
    "gptaq_profile_read": (_c.c_int, [_c.c_int, _c.POINTER(_c.c_int64), _c.POINTER(_c.c_double)]),
    "gptaq_measure_mfma_peak": (_c.c_int, [_c.c_int, _c.c_int, _c.c_void_p, _c.c_size_t, _c.POINTER(_c.c_double),
                                           _c.POINTER(_c.c_double), _c.c_void_p]),
    "gptaq_measure_hbm_copy": (_c.c_int, [_c.c_size_t, _c.c_int, _c.c_void_p, _c.c_size_t, _c.POINTER(_c.c_double),
                                          _c.c_void_p]),
}
EXPORTS = tuple(_SIGS)
PROFILE_TAGS = ("accumulate_gemm", "accumulate_split", "factor_sweep", "p_gemm", "column_loop", "trailing_gemm",
                "trailing_split")


INFO_STALLED = -2 ** 31                          # info[0] of gptaq_prepare: its workgroups lost each other


class GptaqError(RuntimeError):
    pass


def load() -> ctypes.CDLL:
    """Load libgptaq.so (built by paper_2504_02692_amd.build); raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise GptaqError(f"{LIB_PATH} is missing: build it with `python -m paper_2504_02692_amd.build` "
                             "(there is no fallback path)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _check(status: int, what: str) -> None:
    if status != 0:
        lib = load()
        msg = lib.gptaq_status_string(status).decode()
        raise GptaqError(f"{what}: {msg} (status {status}, hip error {lib.gptaq_last_hip_error()})")


# The handle alone: a stream object costs 3 us, as much as the launch of a kernel.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device: Optional[int] = None) -> int:
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device() if device is None else device)
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _ws(ws: torch.Tensor, device: Optional[int] = None) -> int:
    """A workspace's address; on the GPU `device`, where that is given."""
    if not (ws.is_cuda if device is None else ws.get_device() == device) or not ws.is_contiguous():
        raise GptaqError(f"ws: expected contiguous memory of the GPU that runs the call, not of {ws.device}")
    return ws.data_ptr()


def _here(*tensors: Optional[torch.Tensor]) -> int:
    """The current GPU, where all of a call's tensors have to be."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise GptaqError(f"a tensor of {t.device} in a call that runs on GPU {device}")
    return device


def _ld(t: torch.Tensor, rows: int, n: int) -> int:
    """Distance between the rows of a rows x n tensor; of one row alone torch may give any stride."""
    return t.stride(0) if rows > 1 else n


def _need(t: torch.Tensor, dtype, name: str) -> None:
    if not t.is_cuda or t.dtype is not dtype or t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] != 1):
        raise GptaqError(f"{name}: expected a 2-D row-major {dtype} CUDA tensor")


def _need_vec(t: torch.Tensor, dtype, name: str) -> None:
    if not t.is_cuda or t.dtype != dtype or t.dim() != 1 or not t.is_contiguous():
        raise GptaqError(f"{name}: expected a contiguous 1-D {dtype} CUDA tensor")


def workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def gptaq_accumulate_workspace_bytes(tokens: int, n: int) -> int:
    return load().gptaq_accumulate_workspace_bytes(tokens, n)


def gptaq_prepare_workspace_bytes(n: int) -> int:
    return load().gptaq_prepare_workspace_bytes(n)


def gptaq_quantize_workspace_bytes(m: int, n: int) -> int:
    return load().gptaq_quantize_workspace_bytes(m, n)


def _accumulate(name: str, X: torch.Tensor, Xtilde: torch.Tensor, H: torch.Tensor, dXXT: torch.Tensor,
                ws: torch.Tensor) -> None:
    _need(X, torch.bfloat16, "X"); _need(Xtilde, torch.bfloat16, "Xtilde")
    _need(H, torch.float32, "H"); _need(dXXT, torch.float32, "dXXT")
    tokens, n = X.shape
    if Xtilde.shape != X.shape or Xtilde.stride(0) != X.stride(0) or H.shape != (n, n) or dXXT.shape != (n, n) \
            or H.stride(0) != dXXT.stride(0):
        raise GptaqError(f"{name}: shape mismatch")
    _check(getattr(load(), name)(_ptr(X), _ptr(Xtilde), tokens, n, X.stride(0), _ptr(H), _ptr(dXXT),
                                 H.stride(0), _ws(ws), ws.numel(), _stream()), name)


def gptaq_accumulate(X: torch.Tensor, Xtilde: torch.Tensor, H: torch.Tensor, dXXT: torch.Tensor,
                     ws: torch.Tensor) -> None:
    """H += X^T X (upper triangle), dXXT += (Xtilde - X)^T X for token-major bf16 X, Xtilde."""
    _accumulate("gptaq_accumulate", X, Xtilde, H, dXXT, ws)


def gptaq_accumulate_upper(X: torch.Tensor, Xtilde: torch.Tensor, H: torch.Tensor, dXXT: torch.Tensor,
                           ws: torch.Tensor) -> None:
    """gptaq_accumulate that maintains only the entries of dXXT with col >= row (natural column order)."""
    _accumulate("gptaq_accumulate_upper", X, Xtilde, H, dXXT, ws)


def gptaq_accumulate_noalloc(X: torch.Tensor, Xtilde: torch.Tensor, H: torch.Tensor, dXXT: torch.Tensor) -> None:
    """gptaq_accumulate on the library's built-in scratch array (no workspace, no allocation; n <= 16384)."""
    _need(X, torch.bfloat16, "X"); _need(Xtilde, torch.bfloat16, "Xtilde")
    _need(H, torch.float32, "H"); _need(dXXT, torch.float32, "dXXT")
    tokens, n = X.shape
    if Xtilde.shape != X.shape or Xtilde.stride(0) != X.stride(0) or H.shape != (n, n) or dXXT.shape != (n, n) \
            or H.stride(0) != dXXT.stride(0):
        raise GptaqError("gptaq_accumulate_noalloc: shape mismatch")
    _check(load().gptaq_accumulate_noalloc(_ptr(X), _ptr(Xtilde), tokens, n, X.stride(0), _ptr(H), _ptr(dXXT),
                                           H.stride(0), _stream()), "gptaq_accumulate_noalloc")


def gptaq_accumulate_staged(X: Optional[torch.Tensor], Xtilde: Optional[torch.Tensor], H: torch.Tensor, dXXT: torch.Tensor,
                            ws: torch.Tensor, pending: int, flush: bool = False, upper: bool = False) -> int:
    """Appends a chunk to the staged operands in `ws` (products run per 32768 pending tokens or on flush);
    returns the new number of pending tokens.  X, Xtilde may be None with flush=True.
    upper=True calls gptaq_accumulate_staged_upper."""
    fn = "gptaq_accumulate_staged_upper" if upper else "gptaq_accumulate_staged"
    _need(H, torch.float32, "H"); _need(dXXT, torch.float32, "dXXT")
    n = H.shape[0]
    tokens, ldx = 0, n
    if X is not None:
        _need(X, torch.bfloat16, "X"); _need(Xtilde, torch.bfloat16, "Xtilde")
        if X.shape != Xtilde.shape or X.shape[1] != n or X.stride(0) != Xtilde.stride(0) or X.stride(1) != 1:
            raise GptaqError("gptaq_accumulate_staged: shape mismatch")
        tokens, ldx = X.shape[0], X.stride(0)
    if dXXT.shape != (n, n) or H.stride(0) != dXXT.stride(0):
        raise GptaqError("gptaq_accumulate_staged: shape mismatch")
    p = _c.c_int64(int(pending))
    _check(getattr(load(), fn)(_ptr(X), _ptr(Xtilde), tokens, n, ldx, _ptr(H), _ptr(dXXT), H.stride(0),
                               _ws(ws), ws.numel() * ws.element_size(), _c.byref(p), int(bool(flush)),
                               _stream()), fn)
    return p.value


def gptaq_symmetrize(H: torch.Tensor) -> None:
    _need(H, torch.float32, "H")
    _check(load().gptaq_symmetrize(_ptr(H), H.shape[0], H.stride(0), _stream()), "gptaq_symmetrize")


def gptaq_prepare(H: torch.Tensor, dXXT: torch.Tensor, damp: float, ws: torch.Tensor,
                  dead: Optional[torch.Tensor] = None, info: Optional[torch.Tensor] = None):
    """In place: H -> U = L^T (upper), dXXT -> P (strictly upper).  Returns (dead, info) device tensors."""
    _need(H, torch.float32, "H"); _need(dXXT, torch.float32, "dXXT")
    n = H.shape[0]
    if H.shape != (n, n) or dXXT.shape != (n, n) or H.stride(0) != dXXT.stride(0):
        raise GptaqError("gptaq_prepare: shape mismatch")
    if dead is None:
        dead = torch.empty(n, dtype=torch.uint8, device=H.device)
    if info is None:
        info = torch.empty(2, dtype=torch.int32, device=H.device)
    _check(load().gptaq_prepare(_ptr(H), _ptr(dXXT), n, H.stride(0), float(damp), _ptr(dead), _ptr(info),
                                _ws(ws), ws.numel(), _stream()), "gptaq_prepare")
    return dead, info


def gptaq_quantize_layer(W: torch.Tensor, U: torch.Tensor, P: torch.Tensor, bits: int, group: int, sym: bool,
                         blocksize: int, ws: torch.Tensor, dead: Optional[torch.Tensor] = None,
                         codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                         zeros: Optional[torch.Tensor] = None, terms: int = 3, mse_grid: int = 0, mse_steps: int = 0):
    """In place: W -> dequantised quantised weights.  Returns (codes, scales, zeros).
    terms != 3 goes through gptaq_quantize_layer_terms (1: E term only = GPTQ, P may be None)."""
    _need(W, torch.float32, "W"); _need(U, torch.float32, "U")
    m, n = W.shape
    if P is not None:
        _need(P, torch.float32, "P")
        if P.shape != (n, n) or U.stride(0) != P.stride(0):
            raise GptaqError("gptaq_quantize_layer: shape mismatch")
    if U.shape != (n, n):
        raise GptaqError("gptaq_quantize_layer: shape mismatch")
    G = max(1, n // group) if group > 0 else 1
    if codes is None:
        codes = torch.empty((m, n), dtype=torch.uint8, device=W.device)
    if scales is None:
        scales = torch.empty((m, G), dtype=torch.float32, device=W.device)
    if zeros is None:
        zeros = torch.empty((m, G), dtype=torch.float32, device=W.device)
    args = (_ptr(W), m, n, W.stride(0), _ptr(U), _ptr(P), U.stride(0), _ptr(dead), int(bits), int(group),
            int(bool(sym)), int(blocksize), _ptr(codes), _ptr(scales), _ptr(zeros), _ws(ws), ws.numel(), _stream())
    if mse_steps > 0:
        _check(load().gptaq_quantize_layer_ex(*args, int(terms), int(mse_grid), int(mse_steps)), "gptaq_quantize_layer_ex")
    elif terms == 3:
        _check(load().gptaq_quantize_layer(*args), "gptaq_quantize_layer")
    else:
        _check(load().gptaq_quantize_layer_terms(*args, int(terms)), "gptaq_quantize_layer_terms")
    return codes, scales, zeros


gptaq_quantize_layer_terms = gptaq_quantize_layer
gptaq_quantize_layer_ex = gptaq_quantize_layer


def gptaq_profile_enable(mask: int) -> None:
    """Record the kernels whose tag bit (1 << tag) is set in `mask`; 0 switches recording off."""
    _check(load().gptaq_profile_enable(int(mask)), "gptaq_profile_enable")


def gptaq_profile_read(tag: int):
    """(launches, total milliseconds) of the kernels bracketed under `tag` since profiling was enabled."""
    n, ms = _c.c_int64(0), _c.c_double(0.0)
    _check(load().gptaq_profile_read(int(tag), _c.byref(n), _c.byref(ms)), "gptaq_profile_read")
    return n.value, ms.value


def gptaq_measure_mfma_peak(random_data: bool, millis: int = 50):
    """(TFLOP/s, core clock in GHz) of a pure bf16 MFMA loop on every CU, on all-ones or on random operands."""
    ws = workspace(1 << 20)
    tf, ghz = _c.c_double(0.0), _c.c_double(0.0)
    _check(load().gptaq_measure_mfma_peak(int(bool(random_data)), int(millis), _ws(ws), ws.numel() * ws.element_size(),
                                          _c.byref(tf), _c.byref(ghz), _stream()), "gptaq_measure_mfma_peak")
    return tf.value, ghz.value


def gptaq_measure_hbm_copy(nbytes: int = 1 << 30, reps: int = 10) -> float:
    """GB/s (read + written) of a plain streaming copy of `nbytes`."""
    ws = workspace(2 * nbytes)
    g = _c.c_double(0.0)
    _check(load().gptaq_measure_hbm_copy(int(nbytes), int(reps), _ws(ws), ws.numel() * ws.element_size(), _c.byref(g),
                                         _stream()), "gptaq_measure_hbm_copy")
    return g.value


def gptaq_act_order(H: torch.Tensor) -> torch.Tensor:
    """perm (int32, device): inputs in the order of decreasing H[i][i]; a 1-D H is the diagonal itself."""
    if H.dim() == 1:
        _need_vec(H, torch.float32, "H")
    else:
        _need(H, torch.float32, "H")
    n = H.shape[0]
    perm = torch.empty(n, dtype=torch.int32, device=H.device)
    _check(load().gptaq_act_order(_ptr(H), n, H.stride(0) if H.dim() == 2 else 0, _ptr(perm), _stream()), "gptaq_act_order")
    return perm


def gptaq_accumulate_diag(X: torch.Tensor, diag: torch.Tensor) -> None:
    """diag[j] += sum_t X[t][j]^2 (the diagonal of H) for token-major bf16 X."""
    _need(X, torch.bfloat16, "X"); _need_vec(diag, torch.float32, "diag")
    tokens, n = X.shape
    if diag.shape != (n,):
        raise GptaqError("gptaq_accumulate_diag: shape mismatch")
    _check(load().gptaq_accumulate_diag(_ptr(X), tokens, n, X.stride(0), _ptr(diag), _stream()), "gptaq_accumulate_diag")


def gptaq_invert_permutation(perm: torch.Tensor) -> torch.Tensor:
    """inv with inv[perm[r]] = r (int32, device)."""
    if perm.dtype != torch.int32 or perm.dim() != 1 or not perm.is_contiguous():
        raise GptaqError("gptaq_invert_permutation: perm must be a contiguous int32 vector")
    inv = torch.empty_like(perm)
    _check(load().gptaq_invert_permutation(_ptr(perm), perm.numel(), _ptr(inv), _stream()), "gptaq_invert_permutation")
    return inv


def gptaq_accumulate_upper_permuted(X: torch.Tensor, Xtilde: torch.Tensor, inv_perm: torch.Tensor, H: torch.Tensor,
                                    dXXT: torch.Tensor, ws: torch.Tensor) -> None:
    """gptaq_accumulate_upper on the inputs with their channels reordered: input channel j is row / column inv_perm[j]."""
    _need(X, torch.bfloat16, "X"); _need(Xtilde, torch.bfloat16, "Xtilde")
    _need(H, torch.float32, "H"); _need(dXXT, torch.float32, "dXXT")
    tokens, n = X.shape
    if Xtilde.shape != X.shape or Xtilde.stride(0) != X.stride(0) or H.shape != (n, n) or dXXT.shape != (n, n) \
            or H.stride(0) != dXXT.stride(0) or inv_perm.dtype != torch.int32 or inv_perm.shape != (n,) \
            or not inv_perm.is_contiguous():
        raise GptaqError("gptaq_accumulate_upper_permuted: shape mismatch")
    _check(load().gptaq_accumulate_upper_permuted(_ptr(X), _ptr(Xtilde), tokens, n, X.stride(0), _ptr(inv_perm), _ptr(H),
                                                  _ptr(dXXT), H.stride(0), _ws(ws), ws.numel(), _stream()),
           "gptaq_accumulate_upper_permuted")


def gptaq_permute_hessian_workspace_bytes(n: int) -> int:
    return load().gptaq_permute_hessian_workspace_bytes(n)


def gptaq_permute_hessian(H: torch.Tensor, dXXT: torch.Tensor, perm: torch.Tensor, ws: torch.Tensor) -> None:
    _need(H, torch.float32, "H"); _need(dXXT, torch.float32, "dXXT")
    n = H.shape[0]
    if dXXT.shape != (n, n) or H.stride(0) != dXXT.stride(0) or perm.dtype != torch.int32 or perm.numel() != n:
        raise GptaqError("gptaq_permute_hessian: shape mismatch")
    _check(load().gptaq_permute_hessian(_ptr(H), _ptr(dXXT), n, H.stride(0), _ptr(perm), _ws(ws), ws.numel(),
                                        _stream()), "gptaq_permute_hessian")


def _permute_columns(fn, name, src: torch.Tensor, perm: torch.Tensor, inverse: bool) -> torch.Tensor:
    if src.dim() != 2 or src.stride(1) != 1 or perm.dtype != torch.int32 or perm.numel() != src.shape[1]:
        raise GptaqError(f"{name}: shape mismatch")
    out = torch.empty_like(src, memory_format=torch.contiguous_format)
    m, n = src.shape
    _check(fn(_ptr(src), _ptr(out), m, n, src.stride(0), out.stride(0), _ptr(perm), int(bool(inverse)), _stream()), name)
    return out


def gptaq_permute_columns_f32(src: torch.Tensor, perm: torch.Tensor, inverse: bool = False) -> torch.Tensor:
    if src.dtype != torch.float32:
        raise GptaqError("gptaq_permute_columns_f32: expected float32")
    return _permute_columns(load().gptaq_permute_columns_f32, "gptaq_permute_columns_f32", src, perm, inverse)


def gptaq_permute_columns_u8(src: torch.Tensor, perm: torch.Tensor, inverse: bool = False) -> torch.Tensor:
    if src.dtype != torch.uint8:
        raise GptaqError("gptaq_permute_columns_u8: expected uint8")
    return _permute_columns(load().gptaq_permute_columns_u8, "gptaq_permute_columns_u8", src, perm, inverse)


def gptaq_fake_quant_activations(X: torch.Tensor, bits: int, clip: float = 0.9) -> torch.Tensor:
    """Per-token asymmetric fake quantisation of bf16 activations (Section 5.1); returns a new tensor."""
    _need(X, torch.bfloat16, "X")
    Y = torch.empty_like(X, memory_format=torch.contiguous_format)
    tokens, n = X.shape
    _check(load().gptaq_fake_quant_activations(_ptr(X), _ptr(Y), tokens, n, X.stride(0), Y.stride(0), int(bits),
                                               float(clip), _stream()), "gptaq_fake_quant_activations")
    return Y


def gptaq_packed_words_per_row(n: int, bits: int) -> int:
    return load().gptaq_packed_words_per_row(n, bits)


def gptaq_pack_codes(codes: torch.Tensor, bits: int) -> torch.Tensor:
    """(m x n) uint8 codes -> (m x ceil(n*bits/32)) int32 words, code j of a row in bits [j*bits, (j+1)*bits)."""
    if codes.dtype != torch.uint8 or codes.dim() != 2 or codes.stride(1) != 1 or not codes.is_cuda:
        raise GptaqError("gptaq_pack_codes: expected a 2-D row-major uint8 CUDA tensor")
    m, n = codes.shape
    out = torch.empty((m, gptaq_packed_words_per_row(n, bits)), dtype=torch.int32, device=codes.device)
    _check(load().gptaq_pack_codes(_ptr(codes), m, n, codes.stride(0), int(bits), _ptr(out), _stream()),
           "gptaq_pack_codes")
    return out


# ---- running quantised layers

def _address(t: torch.Tensor, device: int, dtype, count: int, name: str, of: str = "LinearWeights") -> int:
    if t.get_device() != device:
        raise GptaqError(f"{of}.{name}: in memory of {t.device}, in a call that runs on GPU {device}")
    if t.dtype is not dtype or t.numel() != count or not t.is_contiguous():
        raise GptaqError(f"{of}.{name}: no longer {count} contiguous {dtype}")
    return t.data_ptr()


class _Weights:
    """Fixed once made; copied, pickled and saved through the constructor (the default sets attributes)."""
    __slots__ = ()

    def __setattr__(self, name, value):
        raise AttributeError(f"{type(self).__name__}.{name}: weights are fixed; lay out new ones with {self._packs}")

    def __reduce__(self):
        return type(self), tuple(getattr(self, name) for name in self.__slots__)


class LinearWeights(_Weights):
    """A layer's weights as gptaq_linear and gptaq_linear_i8 read them: data (uint8), m, n, group (0: one per row), perm, bias, and info,
    an int32 on the GPU that is 0, or 1 + a row whose codes or zeros do not fit in 4 bits.  Fixed once made, as gptaq_linear_pack has checked
    that they fit each other; what a call reads of the tensors is their memory at that time, which has to be of the same kind and size still."""
    __slots__ = ("data", "m", "n", "group", "perm", "bias", "info")
    _packs = "gptaq_linear_pack"

    def __init__(self, data: torch.Tensor, m: int, n: int, group: int, perm: Optional[torch.Tensor], bias: Optional[torch.Tensor],
                 info: torch.Tensor):
        for name, value in zip(self.__slots__, (data, m, n, group, perm, bias, info)):
            object.__setattr__(self, name, value)

    def _args(self, device: int):
        """As the C calls take them, in order; on the GPU `device`."""
        data, perm, bias = self.data, self.perm, self.bias
        size = data.numel()
        return (None if perm is None else _address(perm, device, torch.int32, self.n, "perm"), _address(data, device, torch.uint8, size, "data"), size,
                self.m, self.n, self.group, None if bias is None else _address(bias, device, torch.float32, self.m, "bias"))


def gptaq_linear_weights_bytes(m: int, n: int, group: int) -> int:
    return load().gptaq_linear_weights_bytes(m, n, group)


def gptaq_linear_pack(codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor, group: int,
                      perm: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None) -> LinearWeights:
    """Lays out what gptaq_quantize_layer returned (bits <= 4; group 32, 64, 128, or <= 0 for one per row).  perm: the columns'
    order where the layer was solved with act_order; bias: fp32."""
    _need(codes, torch.uint8, "codes")
    m, n = codes.shape
    G = max(1, n // group) if group > 0 else 1
    for t, name in ((scales, "scales"), (zeros, "zeros")):
        if not t.is_cuda or t.dtype != torch.float32 or t.shape != (m, G) or not t.is_contiguous():
            raise GptaqError(f"gptaq_linear_pack: {name}: expected a contiguous {m} x {G} float32 CUDA tensor")
    if perm is not None:
        _need_vec(perm, torch.int32, "perm")
        if perm.numel() != n:
            raise GptaqError("gptaq_linear_pack: perm: expected one entry per column")
    if bias is not None:
        _need_vec(bias, torch.float32, "bias")
        if bias.numel() != m:
            raise GptaqError("gptaq_linear_pack: bias: expected one entry per row")
    device = _here(codes, scales, zeros, perm, bias)
    data = workspace(gptaq_linear_weights_bytes(m, n, group), codes.device)
    info = torch.empty(1, dtype=torch.int32, device=codes.device)
    _check(load().gptaq_linear_pack(_ptr(codes), _ld(codes, m, n), _ptr(scales), _ptr(zeros), m, n, int(group), _ptr(data), data.numel(),
                                    _ptr(info), _stream(device)), "gptaq_linear_pack")
    return LinearWeights(data, m, n, max(0, int(group)), perm, bias, info)


def gptaq_linear_workspace_bytes(tokens: int, m: int, n: int) -> int:
    return load().gptaq_linear_workspace_bytes(tokens, m, n)


def _linear_out(X: torch.Tensor, tokens: int, n: int, w: _Weights, kind: type, dtype, out: Optional[torch.Tensor], name: str) -> torch.Tensor:
    if not isinstance(w, kind):                          # (the other kind's arguments are others, in another order)
        raise GptaqError(f"{name}: weights: expected the {kind.__name__} that {kind._packs} returns, not {type(w).__name__}")
    if n != w.n:
        raise GptaqError(f"{name}: X has {n} columns, the weights {w.n}")
    if out is None:
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            raise GptaqError(f"{name}: the output is bfloat16 or float32")
        return X.new_empty((tokens, w.m), dtype=dtype)
    _need(out, torch.float32 if out.dtype is torch.float32 else torch.bfloat16, "out")
    if out.shape != (tokens, w.m):
        raise GptaqError(f"{name}: out: shape mismatch")
    return out


def gptaq_linear(X: torch.Tensor, weights: LinearWeights, ws: torch.Tensor, out: Optional[torch.Tensor] = None,
                 dtype=torch.bfloat16) -> torch.Tensor:
    """X W^T + bias for token-major bf16 X; returns (tokens x m), bf16 or fp32 (`dtype`, or the type of `out`)."""
    _need(X, torch.bfloat16, "X")
    device = _here(X, out)
    tokens, n = X.shape
    Y = _linear_out(X, tokens, n, weights, LinearWeights, dtype, out, "gptaq_linear")
    _check(load().gptaq_linear(X.data_ptr(), tokens, _ld(X, tokens, n), *weights._args(device), Y.data_ptr(), _ld(Y, tokens, weights.m),
                               Y.dtype is torch.float32, _ws(ws, device), ws.nbytes, _stream(device)), "gptaq_linear")
    return Y


def gptaq_linear_i8(codes: torch.Tensor, scales: torch.Tensor, weights: LinearWeights, ws: torch.Tensor,
                    out: Optional[torch.Tensor] = None, dtype=torch.bfloat16) -> torch.Tensor:
    """gptaq_linear for 8-bit activations scales[t] * codes[t][:]."""
    _need(codes, torch.int8, "codes"); _need_vec(scales, torch.float32, "scales")
    tokens, n = codes.shape
    if scales.numel() != tokens:
        raise GptaqError("gptaq_linear_i8: scales: expected one per token")
    device = _here(codes, scales, out)
    Y = _linear_out(codes, tokens, n, weights, LinearWeights, dtype, out, "gptaq_linear_i8")
    _check(load().gptaq_linear_i8(codes.data_ptr(), scales.data_ptr(), tokens, _ld(codes, tokens, n), *weights._args(device), Y.data_ptr(),
                                  _ld(Y, tokens, weights.m), Y.dtype is torch.float32, _ws(ws, device), ws.nbytes, _stream(device)), "gptaq_linear_i8")
    return Y


class Linear8Weights(_Weights):
    """A layer's weights as gptaq_linear8_i8 reads them: data (uint8), m, n, bias, and info, an int32 on the GPU that is 0, or 1 + a row whose zero does not
    fit in 8 bits, or -1 - a column that the permutation does not name.  Fixed once made, as LinearWeights are."""
    __slots__ = ("data", "m", "n", "bias", "info")
    _packs = "gptaq_linear8_pack"

    def __init__(self, data: torch.Tensor, m: int, n: int, bias: Optional[torch.Tensor], info: torch.Tensor):
        for name, value in zip(self.__slots__, (data, m, n, bias, info)):
            object.__setattr__(self, name, value)

    def _args(self, device: int):
        """As the C call takes them, in order; on the GPU `device`."""
        data, bias = self.data, self.bias
        size = data.numel()
        return (_address(data, device, torch.uint8, size, "data", "Linear8Weights"), size, self.m, self.n,
                None if bias is None else _address(bias, device, torch.float32, self.m, "bias", "Linear8Weights"))


def gptaq_linear8_weights_bytes(m: int, n: int) -> int:
    return load().gptaq_linear8_weights_bytes(m, n)


def gptaq_linear8_pack(codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor, perm: Optional[torch.Tensor] = None,
                       bias: Optional[torch.Tensor] = None) -> Linear8Weights:
    """Lays out what gptaq_quantize_layer returned (bits <= 8, one scale and zero a row).  perm: the columns' order where the layer was solved with
    act_order; bias: fp32."""
    _need(codes, torch.uint8, "codes")
    m, n = codes.shape
    for t, name in ((scales, "scales"), (zeros, "zeros")):
        if not t.is_cuda or t.dtype != torch.float32 or t.shape != (m, 1) or not t.is_contiguous():
            raise GptaqError(f"gptaq_linear8_pack: {name}: expected a contiguous {m} x 1 float32 CUDA tensor")
    if perm is not None:
        _need_vec(perm, torch.int32, "perm")
        if perm.numel() != n:
            raise GptaqError("gptaq_linear8_pack: perm: expected one entry per column")
    if bias is not None:
        _need_vec(bias, torch.float32, "bias")
        if bias.numel() != m:
            raise GptaqError("gptaq_linear8_pack: bias: expected one entry per row")
    device = _here(codes, scales, zeros, perm, bias)
    data = workspace(gptaq_linear8_weights_bytes(m, n), codes.device)
    info = torch.empty(1, dtype=torch.int32, device=codes.device)
    _check(load().gptaq_linear8_pack(_ptr(codes), _ld(codes, m, n), _ptr(scales), _ptr(zeros), m, n, _ptr(perm), _ptr(data), data.numel(), _ptr(info),
                                     _stream(device)), "gptaq_linear8_pack")
    return Linear8Weights(data, m, n, bias, info)


def gptaq_linear8_workspace_bytes(tokens: int, m: int, n: int) -> int:
    return load().gptaq_linear8_workspace_bytes(tokens, m, n)


def gptaq_linear8_i8(codes: torch.Tensor, scales: torch.Tensor, weights: Linear8Weights, ws: torch.Tensor,
                     out: Optional[torch.Tensor] = None, dtype=torch.bfloat16) -> torch.Tensor:
    """X W^T + bias for 8-bit activations X = scales[t] * codes[t][:] and weights of up to 8 bits; returns (tokens x m), bf16 or fp32."""
    _need(codes, torch.int8, "codes"); _need_vec(scales, torch.float32, "scales")
    tokens, n = codes.shape
    if scales.numel() != tokens:
        raise GptaqError("gptaq_linear8_i8: scales: expected one per token")
    device = _here(codes, scales, out)
    Y = _linear_out(codes, tokens, n, weights, Linear8Weights, dtype, out, "gptaq_linear8_i8")
    _check(load().gptaq_linear8_i8(codes.data_ptr(), scales.data_ptr(), tokens, _ld(codes, tokens, n), *weights._args(device), Y.data_ptr(),
                                   _ld(Y, tokens, weights.m), Y.dtype is torch.float32, _ws(ws, device), ws.nbytes, _stream(device)), "gptaq_linear8_i8")
    return Y


def _like(X: torch.Tensor, out: Optional[torch.Tensor], name: str) -> torch.Tensor:
    if out is None:
        return torch.empty_like(X, memory_format=torch.contiguous_format)
    _need(out, torch.bfloat16, "out")
    if out.shape != X.shape:
        raise GptaqError(f"{name}: out: shape mismatch")
    return out


def _norm_args(X: torch.Tensor, weight: Optional[torch.Tensor], residual: Optional[torch.Tensor], total: Optional[torch.Tensor], name: str):
    _need(X, torch.bfloat16, "X")
    if weight is not None:
        _need_vec(weight, torch.bfloat16, "weight")
        if weight.numel() != X.shape[1]:
            raise GptaqError(f"{name}: weight: expected one entry per column")
    if residual is not None:
        _need(residual, torch.bfloat16, "residual")
        if residual.shape != X.shape:
            raise GptaqError(f"{name}: residual: shape mismatch")
        if total is None:
            return torch.empty_like(X, memory_format=torch.contiguous_format)
    if total is not None:
        _need(total, torch.bfloat16, "total")
        if total.shape != X.shape:
            raise GptaqError(f"{name}: total: shape mismatch")
    return total


def gptaq_rms_norm(X: torch.Tensor, weight: Optional[torch.Tensor], eps: float, residual: Optional[torch.Tensor] = None,
                   total: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None):
    """(Y, total): total = X + residual, Y = its root-mean-square norm times weight (None: ones).  Without a residual and without
    `total`, total is None.  `total` may be the residual itself (in place)."""
    device = _here(X, weight, residual, total, out)
    total = _norm_args(X, weight, residual, total, "gptaq_rms_norm")
    tokens, n = X.shape
    Y = _like(X, out, "gptaq_rms_norm")
    _check(load().gptaq_rms_norm(_ptr(X), _ptr(residual), _ptr(weight), tokens, n, _ld(X, tokens, n), _ld(residual, tokens, n) if residual is not None else 0,
                                 float(eps), _ptr(total), _ld(total, tokens, n) if total is not None else 0, _ptr(Y), _ld(Y, tokens, n), _stream(device)),
           "gptaq_rms_norm")
    return Y, total


def gptaq_rms_norm_i8(X: torch.Tensor, weight: Optional[torch.Tensor], eps: float, residual: Optional[torch.Tensor] = None,
                      total: Optional[torch.Tensor] = None, clip: float = 1.0):
    """(codes, scales, total): gptaq_rms_norm with its output as 8-bit codes and a scale per token."""
    device = _here(X, weight, residual, total)
    total = _norm_args(X, weight, residual, total, "gptaq_rms_norm_i8")
    tokens, n = X.shape
    codes, scales = X.new_empty((tokens, n), dtype=torch.int8), X.new_empty(tokens, dtype=torch.float32)
    _check(load().gptaq_rms_norm_i8(_ptr(X), _ptr(residual), _ptr(weight), tokens, n, _ld(X, tokens, n), _ld(residual, tokens, n) if residual is not None else 0,
                                    float(eps), _ptr(total), _ld(total, tokens, n) if total is not None else 0, float(clip), _ptr(codes), n,
                                    _ptr(scales), _stream(device)), "gptaq_rms_norm_i8")
    return codes, scales, total


def _gated_args(gate: torch.Tensor, up: torch.Tensor, name: str) -> None:
    _need(gate, torch.bfloat16, "gate"); _need(up, torch.bfloat16, "up")
    if gate.shape != up.shape:
        raise GptaqError(f"{name}: shape mismatch")


def gptaq_silu_mul(gate: torch.Tensor, up: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """silu(gate) * up in bf16; gate and up may be the two halves of one product's output."""
    device = _here(gate, up, out)
    _gated_args(gate, up, "gptaq_silu_mul")
    tokens, n = gate.shape
    Y = _like(gate, out, "gptaq_silu_mul")
    _check(load().gptaq_silu_mul(_ptr(gate), _ptr(up), tokens, n, _ld(gate, tokens, n), _ld(up, tokens, n), _ptr(Y), _ld(Y, tokens, n), _stream(device)), "gptaq_silu_mul")
    return Y


def gptaq_silu_mul_i8(gate: torch.Tensor, up: torch.Tensor, clip: float = 1.0):
    """(codes, scales): silu(gate) * up as 8-bit codes and a scale per token."""
    device = _here(gate, up)
    _gated_args(gate, up, "gptaq_silu_mul_i8")
    tokens, n = gate.shape
    codes, scales = gate.new_empty((tokens, n), dtype=torch.int8), gate.new_empty(tokens, dtype=torch.float32)
    _check(load().gptaq_silu_mul_i8(_ptr(gate), _ptr(up), tokens, n, _ld(gate, tokens, n), _ld(up, tokens, n), float(clip), _ptr(codes), n, _ptr(scales),
                                    _stream(device)), "gptaq_silu_mul_i8")
    return codes, scales


def gptaq_quant_activations_i8(X: torch.Tensor, clip: float = 1.0):
    """(codes, scales): bf16 rows as 8-bit codes and a scale per token, scale = clip * max|X| / 127."""
    _need(X, torch.bfloat16, "X")
    device = _here(X)
    tokens, n = X.shape
    codes, scales = X.new_empty((tokens, n), dtype=torch.int8), X.new_empty(tokens, dtype=torch.float32)
    _check(load().gptaq_quant_activations_i8(X.data_ptr(), tokens, n, _ld(X, tokens, n), float(clip), codes.data_ptr(), n, scales.data_ptr(),
                                             _stream(device)), "gptaq_quant_activations_i8")
    return codes, scales


# ---- the cache and attention

_cache = struct.Struct("12q").pack                       # a gptaq_cache


def _need_heads(t: torch.Tensor, shape, name: str):
    """(address, stride of tokens, stride of heads) of a (tokens x heads x d) bf16 tensor of that shape."""
    stride = t.stride()
    if t.dtype is not torch.bfloat16 or len(stride) != 3 or t.shape != shape or (stride[2] != 1 and shape[2] != 1):
        raise GptaqError(f"{name}: expected bfloat16 ({', '.join(map(str, shape))}) with adjacent entries")
    tokens, heads, d = shape                             # (of one token or head alone torch may give any stride)
    head = stride[1] if heads > 1 else d
    return t.data_ptr(), stride[0] if tokens > 1 else heads * head, head


def _cache_args(keys: torch.Tensor, values: torch.Tensor, table: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor, d: int, name: str):
    """The cache as the C calls take it, and kv_heads."""
    bf16, int32, shape, size = torch.bfloat16, torch.int32, keys.shape, table.shape
    if keys.dtype is not bf16 or len(shape) != 5 or shape[2] * 8 != d or shape[4] != 8 or not keys.is_contiguous():
        raise GptaqError(f"{name}: keys: expected contiguous bfloat16 (pages, kv_heads, {d} / 8, page, 8)")
    pages, kv_heads, _, page, _ = shape
    if values.dtype is not bf16 or values.shape != (pages, kv_heads, page // 8, d, 8) or not values.is_contiguous():
        raise GptaqError(f"{name}: values: expected contiguous bfloat16 ({pages}, {kv_heads}, {page} / 8, {d}, 8)")
    if table.dtype is not int32 or len(size) != 2 or (size[1] > 1 and table.stride(1) != 1):
        raise GptaqError(f"{name}: table: expected a row-major int32 tensor with a row for each sequence")
    seqs, width = size
    if lengths.dtype is not int32 or lengths.shape != (seqs,) or not lengths.is_contiguous():
        raise GptaqError(f"{name}: lengths: expected {seqs} contiguous int32, as many as the table has rows")
    if starts.dtype is not int32 or starts.shape != (seqs + 1,) or not starts.is_contiguous():
        raise GptaqError(f"{name}: starts: expected {seqs + 1} contiguous int32")
    return _cache(keys.data_ptr(), values.data_ptr(), pages, kv_heads, page, d, table.data_ptr(), table.stride(0) if seqs > 1 else width, width, starts.data_ptr(),
                  lengths.data_ptr(), seqs), kv_heads


def _heads_of(q: torch.Tensor, name: str):
    shape = q.shape
    if len(shape) != 3:
        raise GptaqError(f"{name}: q: expected (tokens, heads, d)")
    return shape


def gptaq_cache_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, keys: torch.Tensor, values: torch.Tensor, table: torch.Tensor,
                       starts: torch.Tensor, lengths: torch.Tensor, freqs: Optional[torch.Tensor], interleaved: bool = False,
                       out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Writes the keys k, rotated by their positions, and the values v of new tokens into the cache; returns the rotated queries (in `out`, which may be q
    itself).  q, k, v: (tokens, heads, d), for instance parts of one product's rows; sequence s has rows starts[s] .. starts[s + 1] - 1, its
    lengths[s] count them.  freqs: float64, the angle per position of each rotated pair (None: no rotation)."""
    device = _here(q, k, v, keys, values, table, starts, lengths, freqs, out)
    shape = _heads_of(q, "gptaq_cache_append")
    tokens, heads, d = shape
    cache, kv_heads = _cache_args(keys, values, table, starts, lengths, d, "gptaq_cache_append")
    kv_shape = (tokens, kv_heads, d)
    pairs = 0
    if freqs is not None:
        if freqs.dtype is not torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
            raise GptaqError("gptaq_cache_append: freqs: expected a contiguous float64 vector")
        pairs = freqs.numel()
    qp = _need_heads(q, shape, "q")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        op = out.data_ptr(), heads * d, d
    else:
        op = _need_heads(out, shape, "out")
    _check(load().gptaq_cache_append(*qp, *_need_heads(k, kv_shape, "k"), *_need_heads(v, kv_shape, "v"), cache, tokens, heads, _ptr(freqs), pairs, bool(interleaved),
                                     *op, _stream(device)), "gptaq_cache_append")
    return out


def gptaq_attention_workspace_bytes(tokens: int, seqs: int, heads: int, kv_heads: int, d: int) -> int:
    return load().gptaq_attention_workspace_bytes(tokens, seqs, heads, kv_heads, d)


def gptaq_attention(q: torch.Tensor, keys: torch.Tensor, values: torch.Tensor, table: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor,
                    ws: torch.Tensor, window: int = 0, sinks: int = 0, scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Causal attention of new tokens' queries (tokens, heads, d) over the cache, which holds their own keys and values already.  window: positions a
    token sees, itself among them (0: all); sinks: first positions that stay visible.  scale: 1 / sqrt(d) if not given.  `out` may be q itself."""
    device = _here(q, keys, values, table, starts, lengths, out)
    shape = _heads_of(q, "gptaq_attention")
    tokens, heads, d = shape
    cache, _ = _cache_args(keys, values, table, starts, lengths, d, "gptaq_attention")
    qp = _need_heads(q, shape, "q")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        op = out.data_ptr(), heads * d, d
    else:
        op = _need_heads(out, shape, "out")
    _check(load().gptaq_attention(*qp, cache, tokens, heads, int(window), int(sinks), d ** -0.5 if scale is None else float(scale), *op, _ws(ws, device), ws.nbytes,
                                  _stream(device)), "gptaq_attention")
    return out
