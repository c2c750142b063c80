"""Sequence operators on torch tensors: causal convolution, selective scan, gated delta rule, norm, block quantisation, block-scaled product, adapters.

The names and the meaning of every argument mirror include/xl_seq.h; the arithmetic runs in the HIP kernels of libxl_seq.so, and there is no
CPU fallback.  Each call enqueues one kernel (a large product, a long scan of few channels, many tokens of adapters or of the delta rule two and more) on the current stream of its tensors' device and returns without waiting;
what does not fit raises `XlError` before anything is launched.  Inference only: tensors that ask for gradients are refused.
"""
from __future__ import annotations

import ctypes
import importlib
import os
from typing import Optional, Tuple

import torch

from .binding import XlError

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("XL_SEQ_LIBRARY_PATH") or os.path.join(_HERE, "libxl_seq.so")

XL_F32, XL_F16, XL_BF16 = 0, 1, 2
SCALE_BLOCK = 128

# every symbol include/xl_seq.h declares
EXPORTS = ["xl_causal_conv", "xl_selective_scan", "xl_selective_scan_workspace", "xl_quantize_blocks", "xl_block_matmul", "xl_rms_norm", "xl_add_adapters",
           "xl_add_adapters_workspace", "xl_gated_delta_rule", "xl_gated_delta_rule_workspace", "xl_seq_last_error"]

_lib = None
_module = None


def lib() -> ctypes.CDLL:
    """Load libxl_seq.so (raises OSError when it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError(f"{LIB_PATH} is missing: run `python -m paper_2007_06000_amd.build` (there is no fallback)")
        L = ctypes.CDLL(LIB_PATH)
        for name in EXPORTS[:-1]:
            f = getattr(L, name)
            f.argtypes = [ctypes.c_char_p, ctypes.c_void_p]
            f.restype = ctypes.c_int
        for name in EXPORTS:
            if name.endswith("_workspace"):
                f = getattr(L, name)
                f.argtypes = [ctypes.c_char_p]
                f.restype = ctypes.c_longlong
        L.xl_seq_last_error.argtypes = []
        L.xl_seq_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def module():
    """The module that checks tensors and calls libxl_seq.so (csrc/seq_torch.cpp), bound to the loaded library."""
    global _module
    try:
        m = importlib.import_module("._xl_seq", __package__)
    except ModuleNotFoundError as e:
        raise OSError("_xl_seq.so is missing: run `python -m paper_2007_06000_amd.build` (there is no fallback)") from e
    m.bind(*[ctypes.cast(getattr(lib(), name), ctypes.c_void_p).value for name in EXPORTS], XlError)
    _module = m
    return m


def causal_conv(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *, silu: bool = True,
                state: Optional[torch.Tensor] = None, new_state: Optional[torch.Tensor] = None,
                lengths: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Depthwise convolution of x [batch, length, channels] over time with weight [channels, taps] (fp32), bias and SiLU.

    Returns the result and the state [batch, taps - 1, channels] for the next call: the last inputs, oldest first.  `new_state`
    receives it if given (`state` itself may be). With `slots` (int32, one per sequence) the state is a cache of any number of
    rows, updated in place: a sequence reads and writes the row it names, and one outside the cache is absent.  No two sequences of a
    call may name the same row.

    `out` must not share memory with x: a token's inputs are those of the tokens before it too."""
    return (_module or module()).causal_conv(x, weight, bias, silu, state, new_state, lengths, slots, out)


def selective_scan(u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, *,
                   D: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None, delta_bias: Optional[torch.Tensor] = None,
                   softplus: bool = True, state: Optional[torch.Tensor] = None, new_state: Optional[torch.Tensor] = None,
                   lengths: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Selective state-space scan of u and delta [batch, length, channels] with A [channels, states] and B, C [batch, length, states].

    z is the gate; D, delta_bias [channels] and A are fp32, everything else but the states is of u's type.  Returns the result and the
    states [batch, channels, states] (fp32) for the next call; `state`, `new_state`, `slots` as for `causal_conv`.  One token or many: a
    call of length 1 is the step of a generation.  `out` may be u, delta or z itself, and must not share memory with an input otherwise."""
    return (_module or module()).selective_scan(u, delta, A, B, C, D, z, delta_bias, softplus, state, new_state, lengths, slots, out)


def quantize_rows(x: torch.Tensor, *, out: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Activations x [rows, k] as e4m3 numbers and scales [rows, ceil(k / 128)], one for each 128 numbers of a row.

    The rows of `out` begin at multiples of 16 bytes, and the up to 15 bytes from a row's end to the next multiple are set to zero: a slice of a
    wider tensor's columns loses what lies there."""
    return (_module or module()).quantize("quantize_rows", x, 1, out, scales)


def quantize_weight(w: torch.Tensor, *, out: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Weights w [n, k] as e4m3 numbers and scales [ceil(n / 128), ceil(k / 128)], one for each block of 128 x 128; `out` as for `quantize_rows`."""
    return (_module or module()).quantize("quantize_weight", w, SCALE_BLOCK, out, scales)


def block_matmul(a: torch.Tensor, a_scales: torch.Tensor, b: torch.Tensor, b_scales: torch.Tensor, *, bias: Optional[torch.Tensor] = None,
                 dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a [m, k] times the transpose of b [n, k], both e4m3 with the scales of `quantize_rows` and `quantize_weight`; bias [n] is fp32.

    With dtype torch.float32 all sums are fp32.  For 16-bit results the products of a block are added by the 8-bit matrix operation, twice as fast: 1e-5 to
    7e-5 of the result's norm off, less than the rounding to 16 bits."""
    return (_module or module()).block_matmul(a, a_scales, b, b_scales, bias, dtype, out)


def rms_norm(x: torch.Tensor, weight: torch.Tensor, *, residual: Optional[torch.Tensor] = None, new_residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
             out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(x + residual) / sqrt(mean of its squares + eps) * weight for the rows of x [rows, k]; weight [k] is fp32, residual of x's type or fp32.

    Returns the result, of x's type, and the sum, of the residual's type, which is the next layer's residual (without a residual: x itself).  `new_residual` receives
    the sum if given (`residual` itself may be), `out` the result (x itself may be).  The norm is that of the sum before it is rounded to its type."""
    return (_module or module()).rms_norm("rms_norm", x, weight, residual, new_residual, eps, out, None)


def rms_norm_quantized(x: torch.Tensor, weight: torch.Tensor, *, residual: Optional[torch.Tensor] = None, new_residual: Optional[torch.Tensor] = None,
                       eps: float = 1e-6, out: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """`rms_norm` with its fp32 result quantised as by `quantize_rows`, an operand of `block_matmul`: returns the e4m3 numbers, their scales and the sum."""
    return (_module or module()).rms_norm("rms_norm_quantized", x, weight, residual, new_residual, eps, out, scales)


def add_adapters(y: torch.Tensor, x: torch.Tensor, down: torch.Tensor, up: torch.Tensor, index: torch.Tensor, *, scales: Optional[torch.Tensor] = None,
                 lengths: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y[b] + scales[e] * x[b] down[e]^T up[e]^T with the adapter e = index[b] (int32) of each sequence; y[b] itself where there is no such adapter.

    y [batch, length, n] is what the projection that all sequences share makes of x [batch, length, k]; down [adapters, rank, k], up [adapters, n, rank], all of one
    type, rank at most 128; scales [adapters] are fp32.  Tokens past a sequence's own length (`lengths`, int32) come out as zeros.  `out` may be y itself."""
    return (_module or module()).add_adapters(y, x, down, up, index, scales, lengths, out)


def gated_delta_rule(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, g: torch.Tensor, beta: torch.Tensor, *, scale: Optional[float] = None,
                     normalize: bool = False, state: Optional[torch.Tensor] = None, new_state: Optional[torch.Tensor] = None,
                     lengths: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Recurrence of a matrix S [dk, dv] for each head: S <- exp(g) S, S <- S + beta k (v - S^T k)^T, and the result scale * S^T q (scale: dk^-0.5).

    q, k [batch, length, key heads, dk] and v [batch, length, heads, dv] are of one type; neighbouring heads share a key head.  g (at most 0) and beta
    [batch, length, heads] are fp32.  `normalize` divides each token's q and k by sqrt(sum of squares + 1e-6).  Returns the result and the states
    [batch, heads, dk, dv] (fp32) for the next call; `state`, `new_state`, `slots` as for `causal_conv`.  One token or many: a call of length 1 is the step
    of a generation.  `out` must not share memory with an input."""
    return (_module or module()).gated_delta_rule(q, k, v, g, beta, scale, normalize, state, new_state, lengths, slots, out)
