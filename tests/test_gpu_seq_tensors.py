"""The sequence operators as calls among others: errors, versions and gradients of tensors, memory that results share."""
import ctypes

import pytest
import torch

from paper_2007_06000_amd import seq

pytestmark = pytest.mark.gpu


def operators():
    """(name, call) of every operator; a call takes the result's place or None."""
    g = torch.Generator("cuda").manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, w, B = r(2, 9, 16), r(16, 4), r(2, 9, 4)
    A = -torch.rand(16, 4, generator=g, device="cuda")
    q, s = seq.quantize_rows(x[0])
    return [("causal_conv", lambda out=None: seq.causal_conv(x, w, out=out)), ("selective_scan", lambda out=None: seq.selective_scan(x, x, A, B, B, out=out)),
            ("quantize_rows", lambda out=None: seq.quantize_rows(x[0], out=out)), ("quantize_weight", lambda out=None: seq.quantize_weight(x[0], out=out)),
            ("block_matmul", lambda out=None: (seq.block_matmul(q, s, q, s[:1], out=out),))]


def test_an_error_that_another_call_left_is_not_this_calls():
    hip = ctypes.CDLL(seq.LIB_PATH)         # the runtime that the library is linked with
    for name, call in operators():
        want = call()
        torch.cuda.synchronize()
        assert hip.hipSetDevice(1 << 20) != 0, "the device exists"
        try:
            got = call()
        finally:
            hip.hipGetLastError()
        assert all(torch.equal(a.float(), b.float()) for a, b in zip(got, want)), name
