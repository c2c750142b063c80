"""Sequence operators on torch tensors: causal convolution, selective scan, block quantisation, block-scaled product.

The names and the meaning of every argument mirror include/xl_seq.h; the arithmetic runs in the HIP kernels of libxl_seq.so, and there is no
CPU fallback.  Each call enqueues one kernel (a large product two) on the current stream of its tensors' device and returns without waiting;
what does not fit raises `XlError` before anything is launched.  Inference only: tensors that ask for gradients are refused.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Tuple

import torch

from .binding import XL_E_DEVICE, XL_E_SHAPE, XL_E_UNSUPPORTED, XlError

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("XL_SEQ_LIBRARY_PATH") or os.path.join(_HERE, "libxl_seq.so")

XL_F32, XL_F16, XL_BF16 = 0, 1, 2
SCALE_BLOCK = 128
DTYPES = {torch.float32: XL_F32, torch.float16: XL_F16, torch.bfloat16: XL_BF16}

# every symbol include/xl_seq.h declares
EXPORTS = ["xl_causal_conv", "xl_selective_scan", "xl_quantize_blocks", "xl_block_matmul", "xl_seq_last_error"]

# the argument structs: 64-bit numbers, then pointers
_CONV = struct.Struct("=11q8Q")
_SCAN = struct.Struct("=19q13Q")
_QUANTIZE = struct.Struct("=8q3Q")
_MATMUL = struct.Struct("=11q6Q")

_lib = None


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
        L.xl_seq_last_error.argtypes = []
        L.xl_seq_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _fail(status: int, message: str):
    raise XlError(status, message)


def _call(name: str, packed: bytes, device: int):
    f = getattr(_lib or lib(), name)
    if torch._C._cuda_getDevice() == device:
        st = f(packed, torch._C._cuda_getCurrentRawStream(device))
    else:
        with torch.cuda.device(device):
            st = f(packed, torch._C._cuda_getCurrentRawStream(device))
    if st:
        raise XlError(st, lib().xl_seq_last_error().decode())


def _check(what: str, device: torch.device, tensors):
    """(name, tensor or None, type or None, shape or None) each: on the device, of the type and shape, no gradient asked for."""
    if device.type != "cuda":
        _fail(XL_E_DEVICE, f"{what}: tensors must be on a GPU (there is no CPU path)")
    grad = torch.is_grad_enabled()
    for name, t, dtype, shape in tensors:
        if t is None:
            continue
        if t.device != device:
            _fail(XL_E_DEVICE, f"{what}: {name} is on {t.device}, not on {device}")
        if dtype is not None and t.dtype != dtype:
            _fail(XL_E_UNSUPPORTED, f"{what}: {name} is {t.dtype}, not {dtype}")
        if shape is not None and t.shape != shape:
            _fail(XL_E_SHAPE, f"{what}: {name} has shape {tuple(t.shape)}, not {tuple(shape)}")
        if grad and t.requires_grad:
            _fail(XL_E_UNSUPPORTED, f"{what}: {name} asks for a gradient: inference only")


def _rows(what: str, name: str, t: torch.Tensor) -> Tuple[int, int]:
    """Steps between sequences and tokens of [batch, length, width] with a contiguous last dimension."""
    b, n, c = t.stride()
    if c != 1 and t.shape[2] > 1:
        _fail(XL_E_SHAPE, f"{what}: the last dimension of {name} must be contiguous")
    return b, n


def _dense(what: str, name: str, t: Optional[torch.Tensor]) -> int:
    if t is None:
        return 0
    if not t.is_contiguous():
        _fail(XL_E_SHAPE, f"{what}: {name} must be contiguous")
    return t.data_ptr()


def _states(what: str, batch: int, tail: Tuple[int, ...], dtype, device, state, new_state, slots):
    """The state that goes in, the one that comes out and their number of rows."""
    if slots is not None and state is None:
        _fail(XL_E_SHAPE, f"{what}: slots name rows of a state, and none is given")
    rows = state.shape[0] if slots is not None and state.dim() else batch
    if new_state is None:
        new_state = state if slots is not None else torch.empty((batch, *tail), dtype=dtype, device=device)
    return rows, (rows, *tail), new_state


def causal_conv(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *, silu: bool = True,
                state: Optional[torch.Tensor] = None, new_state: Optional[torch.Tensor] = None,
                lengths: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Depthwise convolution of x [batch, length, channels] over time with weight [channels, taps] (fp32), bias and SiLU.

    Returns the result and the state [batch, taps - 1, channels] for the next call: the last inputs, oldest first.  `new_state`
    receives it if given (`state` itself may be). With `slots` (int32, one per sequence) the state is a cache of any number of
    rows, updated in place: a sequence reads and writes the row it names, and one outside the cache is absent."""
    what = "causal_conv"
    if x.dim() != 3 or weight.dim() != 2:
        _fail(XL_E_SHAPE, f"{what}: x is [batch, length, channels] and weight [channels, taps]")
    dtype, device = x.dtype, x.device
    batch, length, channels = x.shape
    taps = weight.shape[1]
    rows, shape, new_state = _states(what, batch, (max(taps - 1, 0), channels), dtype, device, state, new_state, slots)
    if out is None:
        out = torch.empty((batch, length, channels), dtype=dtype, device=device)
    if dtype not in DTYPES:
        _fail(XL_E_UNSUPPORTED, f"{what}: x is {dtype}")
    _check(what, device, (("x", x, None, None), ("weight", weight, torch.float32, (channels, taps)), ("bias", bias, torch.float32, (channels,)),
                          ("state", state, dtype, shape), ("new_state", new_state, dtype, shape), ("lengths", lengths, torch.int32, (batch,)),
                          ("slots", slots, torch.int32, (batch,)), ("out", out, dtype, x.shape)))
    _call("xl_causal_conv", _CONV.pack(
        batch, length, channels, taps, DTYPES[dtype], silu, *_rows(what, "x", x), *_rows(what, "out", out), rows, x.data_ptr(), _dense(what, "weight", weight),
        _dense(what, "bias", bias), _dense(what, "state", state), _dense(what, "new_state", new_state), _dense(what, "lengths", lengths),
        _dense(what, "slots", slots), out.data_ptr()), device.index)
    return out, new_state


def selective_scan(u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, *,
                   D: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None, delta_bias: Optional[torch.Tensor] = None,
                   softplus: bool = True, state: Optional[torch.Tensor] = None, new_state: Optional[torch.Tensor] = None,
                   lengths: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Selective state-space scan of u and delta [batch, length, channels] with A [channels, states] and B, C [batch, length, states].

    z is the gate; D, delta_bias [channels] and A are fp32, everything else but the states is of u's type.  Returns the result and the
    states [batch, channels, states] (fp32) for the next call; `state`, `new_state`, `slots` as for `causal_conv`.  One token or many: a
    call of length 1 is the step of a generation."""
    what = "selective_scan"
    if u.dim() != 3 or A.dim() != 2:
        _fail(XL_E_SHAPE, f"{what}: u is [batch, length, channels] and A [channels, states]")
    dtype, device = u.dtype, u.device
    batch, length, channels = u.shape
    n = A.shape[1]
    rows, shape, new_state = _states(what, batch, (channels, n), torch.float32, device, state, new_state, slots)
    if out is None:
        out = torch.empty((batch, length, channels), dtype=dtype, device=device)
    if dtype not in DTYPES:
        _fail(XL_E_UNSUPPORTED, f"{what}: u is {dtype}")
    wide, f32 = (batch, length, n), torch.float32
    _check(what, device, (("u", u, None, None), ("delta", delta, dtype, u.shape), ("A", A, f32, (channels, n)), ("B", B, dtype, wide), ("C", C, dtype, wide),
                          ("D", D, f32, (channels,)), ("z", z, dtype, u.shape), ("delta_bias", delta_bias, f32, (channels,)), ("state", state, f32, shape),
                          ("new_state", new_state, f32, shape), ("lengths", lengths, torch.int32, (batch,)), ("slots", slots, torch.int32, (batch,)),
                          ("out", out, dtype, u.shape)))
    _call("xl_selective_scan", _SCAN.pack(
        batch, length, channels, n, DTYPES[dtype], softplus, *_rows(what, "u", u), *_rows(what, "delta", delta),
        *(_rows(what, "z", z) if z is not None else (0, 0)), *_rows(what, "out", out), *_rows(what, "B", B), *_rows(what, "C", C), rows, u.data_ptr(), delta.data_ptr(),
        _dense(what, "A", A), B.data_ptr(), C.data_ptr(), _dense(what, "D", D), _dense(what, "delta_bias", delta_bias), z.data_ptr() if z is not None else 0,
        _dense(what, "state", state), _dense(what, "new_state", new_state), _dense(what, "lengths", lengths), _dense(what, "slots", slots),
        out.data_ptr()), device.index)
    return out, new_state


def _quantize(what: str, x: torch.Tensor, block_rows: int, out, scales):
    if x.dim() != 2:
        _fail(XL_E_SHAPE, f"{what}: x is [rows, k]")
    rows, k = x.shape
    device = x.device
    blocks = (k + SCALE_BLOCK - 1) // SCALE_BLOCK
    if out is None:
        wide = (k + 15) // 16 * 16
        out = torch.empty((rows, wide), dtype=torch.float8_e4m3fn, device=device)
        if wide != k:
            out = out[:, :k]
    if scales is None:      # a column for each block: the product reads the scales of neighbouring rows together
        scales = torch.empty((blocks, rows), dtype=torch.float32, device=device).t() if block_rows == 1 else \
            torch.empty(((rows + block_rows - 1) // block_rows, blocks), dtype=torch.float32, device=device)
    if x.dtype not in DTYPES:
        _fail(XL_E_UNSUPPORTED, f"{what}: x is {x.dtype}")
    _check(what, device, (("x", x, None, None), ("out", out, torch.float8_e4m3fn, x.shape),
                          ("scales", scales, torch.float32, ((rows + block_rows - 1) // block_rows, blocks))))
    if k > 1 and (x.stride(1) != 1 or out.stride(1) != 1):
        _fail(XL_E_SHAPE, f"{what}: rows of x and out must be contiguous")
    _readable(what, "out", out)
    _call("xl_quantize_blocks", _QUANTIZE.pack(rows, k, block_rows, DTYPES[x.dtype], x.stride(0), out.stride(0), scales.stride(0), scales.stride(1),
                                               x.data_ptr(), out.data_ptr(), scales.data_ptr()), device.index)
    return out, scales


def _readable(what: str, name: str, t: torch.Tensor):
    """The memory of the last row of 8-bit numbers goes on to the next multiple of 16 bytes."""
    rows, k = t.shape
    if k % 16 and rows and t.storage_offset() + (rows - 1) * t.stride(0) + (k + 15) // 16 * 16 > t.untyped_storage().nbytes():
        _fail(XL_E_SHAPE, f"{what}: the last row of {name} must have memory up to the next multiple of 16 bytes")


def quantize_rows(x: torch.Tensor, *, out: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Activations x [rows, k] as e4m3 numbers and scales [rows, ceil(k / 128)], one for each 128 numbers of a row."""
    return _quantize("quantize_rows", x, 1, out, scales)


def quantize_weight(w: torch.Tensor, *, out: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Weights w [n, k] as e4m3 numbers and scales [ceil(n / 128), ceil(k / 128)], one for each block of 128 x 128."""
    return _quantize("quantize_weight", w, SCALE_BLOCK, out, scales)


def block_matmul(a: torch.Tensor, a_scales: torch.Tensor, b: torch.Tensor, b_scales: torch.Tensor, *, bias: Optional[torch.Tensor] = None,
                 dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a [m, k] times the transpose of b [n, k], both e4m3 with the scales of `quantize_rows` and `quantize_weight`; bias [n] is fp32."""
    what = "block_matmul"
    if a.dim() != 2 or b.dim() != 2:
        _fail(XL_E_SHAPE, f"{what}: a is [m, k] and b [n, k]")
    m, k = a.shape
    n = b.shape[0]
    device = a.device
    if out is None:
        out = torch.empty((m, n), dtype=dtype, device=device)
    else:
        dtype = out.dtype
    if dtype not in DTYPES:
        _fail(XL_E_UNSUPPORTED, f"{what}: the result is {dtype}")
    blocks = (k + SCALE_BLOCK - 1) // SCALE_BLOCK
    f8, f32 = torch.float8_e4m3fn, torch.float32
    _check(what, device, (("a", a, f8, None), ("b", b, f8, (n, k)), ("a_scales", a_scales, f32, (m, blocks)),
                          ("b_scales", b_scales, f32, ((n + SCALE_BLOCK - 1) // SCALE_BLOCK, blocks)), ("bias", bias, f32, (n,)), ("out", out, None, (m, n))))
    if (k > 1 and (a.stride(1) != 1 or b.stride(1) != 1)) or (n > 1 and out.stride(1) != 1):
        _fail(XL_E_SHAPE, f"{what}: rows of a, b and out must be contiguous")
    _readable(what, "a", a)
    _readable(what, "b", b)
    _call("xl_block_matmul", _MATMUL.pack(m, n, k, DTYPES[dtype], a.stride(0), b.stride(0), *a_scales.stride(), *b_scales.stride(),
                                          out.stride(0), a.data_ptr(), b.data_ptr(), a_scales.data_ptr(), b_scales.data_ptr(), _dense(what, "bias", bias),
                                          out.data_ptr()), device.index)
    return out
