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


def _call(f, packed: bytes, device: int):
    if torch._C._cuda_getDevice() == device:
        st = f(packed, torch._C._cuda_getCurrentRawStream(device))
    else:
        with torch.cuda.device(device):
            st = f(packed, torch._C._cuda_getCurrentRawStream(device))
    if st:
        raise XlError(st, lib().xl_seq_last_error().decode())


# A call of one token takes the GPU 2 to 6 us, less than the host needs to check a dozen tensors by their names: what fits is let through by one
# test of a tensor's attributes, and only what does not is looked at again to say why.

def _device(what: str, t: torch.Tensor) -> int:
    if not t.is_cuda:
        _fail(XL_E_DEVICE, f"{what}: tensors must be on a GPU (there is no CPU path)")
    return t.get_device()


def _refuse(what: str, name: str, t: torch.Tensor, dtype, shape, device: int, dense: bool):
    if t.get_device() != device:
        _fail(XL_E_DEVICE, f"{what}: {name} is on {t.device}, not on cuda:{device}")
    if t.dtype != dtype:
        _fail(XL_E_UNSUPPORTED, f"{what}: {name} is {t.dtype}, not {dtype}")
    if t.shape != shape:
        _fail(XL_E_SHAPE, f"{what}: {name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.requires_grad and torch.is_grad_enabled():
        _fail(XL_E_UNSUPPORTED, f"{what}: {name} asks for a gradient: inference only")
    if dense and not t.is_contiguous():
        _fail(XL_E_SHAPE, f"{what}: {name} must be contiguous")


def _check(what: str, name: str, t: torch.Tensor, dtype, shape, device: int):
    """A tensor with strides of its own: on the device, of the type and shape, no gradient asked for."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or t.requires_grad:
        _refuse(what, name, t, dtype, shape, device, False)


def _rows(what: str, name: str, t: torch.Tensor, dtype, shape, device: int) -> Tuple[int, int]:
    """Steps between sequences and tokens of [batch, length, width] with a contiguous last dimension."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or t.requires_grad:
        _refuse(what, name, t, dtype, shape, device, False)
    b, n, c = t.stride()
    if c != 1 and shape[2] > 1:
        _fail(XL_E_SHAPE, f"{what}: the last dimension of {name} must be contiguous")
    return b, n


def _dense(what: str, name: str, t: Optional[torch.Tensor], dtype, shape, device: int) -> int:
    """The address of a contiguous tensor, or 0."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or t.requires_grad or not t.is_contiguous():
        _refuse(what, name, t, dtype, shape, device, True)
    return t.data_ptr()


def _states(what: str, batch: int, tail: Tuple[int, ...], like: torch.Tensor, state, new_state, slots):
    """The state's shape and the one that comes out, which is made like `like` if there is none yet."""
    if slots is None:
        shape = (batch, *tail)
        return shape, like.new_empty(shape) if new_state is None else new_state
    if state is None:
        _fail(XL_E_SHAPE, f"{what}: slots name rows of a state, and none is given")
    return (state.shape[0] if state.dim() else batch, *tail), state if new_state is None else new_state


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
    device, dtype, size = _device(what, x), x.dtype, x.shape
    if dtype not in DTYPES:
        _fail(XL_E_UNSUPPORTED, f"{what}: x is {dtype}")
    batch, length, channels = size
    taps = weight.shape[1]
    shape, new_state = _states(what, batch, (max(taps - 1, 0), channels), x, state, new_state, slots)
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    f32, i32 = torch.float32, torch.int32
    _call((_lib or lib()).xl_causal_conv, _CONV.pack(
        batch, length, channels, taps, DTYPES[dtype], silu, *_rows(what, "x", x, dtype, size, device), *_rows(what, "out", out, dtype, size, device), shape[0],
        x.data_ptr(), _dense(what, "weight", weight, f32, (channels, taps), device), _dense(what, "bias", bias, f32, (channels,), device),
        _dense(what, "state", state, dtype, shape, device), _dense(what, "new_state", new_state, dtype, shape, device),
        _dense(what, "lengths", lengths, i32, (batch,), device), _dense(what, "slots", slots, i32, (batch,), device), out.data_ptr()), device)
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
    device, dtype, size = _device(what, u), u.dtype, u.shape
    if dtype not in DTYPES:
        _fail(XL_E_UNSUPPORTED, f"{what}: u is {dtype}")
    batch, length, channels = size
    n = A.shape[1]
    f32, i32, one, wide = torch.float32, torch.int32, (channels,), (batch, length, n)
    a = _dense(what, "A", A, f32, (channels, n), device)
    shape, new_state = _states(what, batch, (channels, n), A, state, new_state, slots)
    if out is None:
        out = torch.empty_like(u, memory_format=torch.contiguous_format)
    gate, z_batch, z_token = 0, 0, 0
    if z is not None:
        gate = z.data_ptr()
        z_batch, z_token = _rows(what, "z", z, dtype, size, device)
    _call((_lib or lib()).xl_selective_scan, _SCAN.pack(
        batch, length, channels, n, DTYPES[dtype], softplus, *_rows(what, "u", u, dtype, size, device), *_rows(what, "delta", delta, dtype, size, device),
        z_batch, z_token, *_rows(what, "out", out, dtype, size, device), *_rows(what, "B", B, dtype, wide, device), *_rows(what, "C", C, dtype, wide, device),
        shape[0], u.data_ptr(), delta.data_ptr(), a, B.data_ptr(), C.data_ptr(), _dense(what, "D", D, f32, one, device),
        _dense(what, "delta_bias", delta_bias, f32, one, device), gate, _dense(what, "state", state, f32, shape, device),
        _dense(what, "new_state", new_state, f32, shape, device), _dense(what, "lengths", lengths, i32, (batch,), device),
        _dense(what, "slots", slots, i32, (batch,), device), out.data_ptr()), device)
    return out, new_state


def _quantize(what: str, x: torch.Tensor, block_rows: int, out, scales):
    if x.dim() != 2:
        _fail(XL_E_SHAPE, f"{what}: x is [rows, k]")
    device, dtype, size = _device(what, x), x.dtype, x.shape
    if dtype not in DTYPES:
        _fail(XL_E_UNSUPPORTED, f"{what}: x is {dtype}")
    rows, k = size
    shape = ((rows + block_rows - 1) // block_rows, (k + SCALE_BLOCK - 1) // SCALE_BLOCK)
    f8, f32 = torch.float8_e4m3fn, torch.float32
    if out is None:
        wide = (k + 15) // 16 * 16
        out = torch.empty((rows, wide), dtype=f8, device=x.device)
        if wide != k:
            out = out[:, :k]
    if scales is None:      # a column for each block: the product reads the scales of neighbouring rows together
        scales = torch.empty_strided(shape, (1, rows) if block_rows == 1 else (shape[1], 1), dtype=f32, device=x.device)
    _check(what, "x", x, dtype, size, device)
    _check(what, "out", out, f8, size, device)
    _check(what, "scales", scales, f32, shape, device)
    (x_row, x_step), (q_row, q_step) = x.stride(), out.stride()
    if k > 1 and (x_step != 1 or q_step != 1):
        _fail(XL_E_SHAPE, f"{what}: rows of x and out must be contiguous")
    if k % 16:
        _readable(what, "out", out)
    _call((_lib or lib()).xl_quantize_blocks, _QUANTIZE.pack(rows, k, block_rows, DTYPES[dtype], x_row, q_row, *scales.stride(), x.data_ptr(), out.data_ptr(),
                                                             scales.data_ptr()), device)
    return out, scales


def _readable(what: str, name: str, t: torch.Tensor):
    """The memory of the last row of 8-bit numbers goes on to the next multiple of 16 bytes."""
    rows, k = t.shape
    if rows and t.storage_offset() + (rows - 1) * t.stride(0) + (k + 15) // 16 * 16 > t.untyped_storage().nbytes():
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
    device, (m, k) = _device(what, a), a.shape
    n = b.shape[0]
    shape, blocks, f8, f32 = (m, n), (k + SCALE_BLOCK - 1) // SCALE_BLOCK, torch.float8_e4m3fn, torch.float32
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=a.device)
    else:
        dtype = out.dtype
        _check(what, "out", out, dtype, shape, device)
    if dtype not in DTYPES:
        _fail(XL_E_UNSUPPORTED, f"{what}: the result is {dtype}")
    _check(what, "a", a, f8, (m, k), device)
    _check(what, "b", b, f8, (n, k), device)
    _check(what, "a_scales", a_scales, f32, (m, blocks), device)
    _check(what, "b_scales", b_scales, f32, ((n + SCALE_BLOCK - 1) // SCALE_BLOCK, blocks), device)
    (a_row, a_step), (b_row, b_step), (y_row, y_step) = a.stride(), b.stride(), out.stride()
    if (k > 1 and (a_step != 1 or b_step != 1)) or (n > 1 and y_step != 1):
        _fail(XL_E_SHAPE, f"{what}: rows of a, b and out must be contiguous")
    if k % 16:
        _readable(what, "a", a)
        _readable(what, "b", b)
    _call((_lib or lib()).xl_block_matmul, _MATMUL.pack(
        m, n, k, DTYPES[dtype], a_row, b_row, *a_scales.stride(), *b_scales.stride(), y_row, a.data_ptr(), b.data_ptr(), a_scales.data_ptr(), b_scales.data_ptr(),
        _dense(what, "bias", bias, f32, (n,), device), out.data_ptr()), device)
    return out
