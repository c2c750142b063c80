"""The sequence operators as calls among others: errors, versions and gradients of tensors, memory that results share."""
import ctypes
import os
import subprocess
import sysconfig

import pytest
import torch
from torch.utils.cpp_extension import include_paths, library_paths

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


def versions(*tensors):
    return [t._version for t in tensors]


def test_tensors_that_a_call_writes_get_a_new_version():
    x, w, B = torch.randn(2, 9, 16, device="cuda"), torch.randn(16, 4, device="cuda"), torch.randn(2, 9, 4, device="cuda")
    A, slots = -torch.rand(16, 4, device="cuda"), torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    for make, call in ((lambda: torch.zeros(3, 3, 16, device="cuda"), lambda **k: seq.causal_conv(x, w, **k)),
                       (lambda: torch.zeros(3, 16, 4, device="cuda"), lambda **k: seq.selective_scan(x, x, A, B, B, **k))):
        out, cache = torch.empty_like(x), make()
        before, inputs = versions(out, cache), versions(x, w, B, A, slots)
        call(state=cache, slots=slots, out=out)
        assert [a > b for a, b in zip(versions(out, cache), before)] == [True, True]
        state, new = make()[:2].clone(), make()[:2].clone()
        before = versions(state, new)
        call(state=state, new_state=new)
        assert versions(state) == before[:1] and versions(new)[0] > before[1]
        before = versions(out)
        with pytest.raises(seq.XlError):
            call(state=state[:1], out=out)
        assert versions(out) == before and versions(x, w, B, A, slots) == inputs
    q, s = seq.quantize_rows(x[0])
    for call, given in ((lambda: seq.quantize_rows(x[0], out=q, scales=s), (q, s)), (lambda: seq.quantize_weight(x[0], out=q), (q,)),
                        (lambda: seq.block_matmul(q, s, q, s[:1], out=room), (room := torch.empty(9, 9, device="cuda"),))):
        before = versions(*given)
        call()
        assert all(a > b for a, b in zip(versions(*given), before))


def test_somebody_elses_backward_pass_notices_that_its_tensor_was_overwritten():
    x, w = torch.randn(2, 9, 16, device="cuda"), torch.randn(16, 4, device="cuda")
    out, leaf = torch.randn(2, 9, 16, device="cuda"), torch.ones(2, 9, 16, device="cuda", requires_grad=True)
    loss = (leaf * out).sum()           # keeps out for the gradient of leaf
    seq.causal_conv(x, w, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_results_made_in_inference_mode_may_be_written_again():
    x, w = torch.randn(2, 9, 16, device="cuda"), torch.randn(16, 4, device="cuda")
    with torch.inference_mode():
        out, state = seq.causal_conv(x, w)
    assert out.is_inference()
    want = out.clone()
    seq.causal_conv(x, w, out=out, new_state=state)
    assert torch.equal(out, want)


def test_a_recorded_steps_tensors_get_a_new_version_with_every_step():
    from paper_2007_06000_amd.scan_block import ScanBlock, TokenStep, random_weights
    step = TokenStep(ScanBlock(random_weights(64, 128)), 2)
    x = torch.randn(2, 1, 64, device="cuda").bfloat16()
    leaf = torch.ones(2, 1, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    loss = (leaf * step(x)).sum()
    before = versions(step.y, *step.cache)
    step(x)
    assert all(a > b for a, b in zip(versions(step.y, *step.cache), before))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_tensors_that_carry_a_tangent_are_refused():
    from torch.autograd import forward_ad
    x, w, B = torch.randn(2, 9, 16, device="cuda"), torch.randn(16, 4, device="cuda"), torch.randn(2, 9, 4, device="cuda")
    A = -torch.rand(16, 4, device="cuda")
    q, s = seq.quantize_rows(x[0])
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: seq.causal_conv(dual(x), w), lambda: seq.causal_conv(x, dual(w)), lambda: seq.causal_conv(x, w, dual(w[:, 0].contiguous())),
                     lambda: seq.selective_scan(dual(x), x, A, B, B), lambda: seq.selective_scan(x, x, dual(A), B, B), lambda: seq.selective_scan(x, x, A, B, dual(B)),
                     lambda: seq.selective_scan(x, x, A, B, B, z=dual(x)), lambda: seq.quantize_rows(dual(x[0])), lambda: seq.quantize_weight(dual(x[0])),
                     lambda: seq.block_matmul(q, dual(s), q, s[:1]), lambda: seq.block_matmul(q, s, q, s[:1], bias=dual(x[0, :, 0].contiguous()))):
            with torch.no_grad(), pytest.raises(seq.XlError, match="tangent"):      # no_grad is about backward passes only
                call()
        with torch.inference_mode():
            seq.causal_conv(dual(x), w)         # no gradients of any kind are asked for here
        seq.causal_conv(x, w)


def test_views_whose_numbers_are_to_be_negated_are_refused():
    pairs = torch.randn(2, 9, 1, 2, device="cuda")
    x, w = torch.view_as_complex(pairs).conj().imag, torch.randn(1, 4, device="cuda")       # -pairs[..., 1], read through a mark on the tensor
    assert x.is_neg()
    with pytest.raises(seq.XlError, match="negated"):
        seq.causal_conv(x, w)
    y, _ = seq.causal_conv(x.resolve_neg(), w)
    want, _ = seq.causal_conv(-pairs[..., 1].contiguous(), w)
    assert torch.equal(y, want)
    with pytest.raises(seq.XlError, match="negated"):
        seq.quantize_rows(x[..., 0][:, :1])


F8 = torch.float8_e4m3fn


def refused(call, what):
    with pytest.raises(seq.XlError, match=f"shares memory with {what}"):
        call()


def test_results_that_share_memory_with_what_is_still_to_be_read_are_refused():
    wide = torch.randn(2, 40, 96, device="cuda")
    x, w = wide[:, :, :32], torch.randn(32, 4, device="cuda")
    before = wide.clone()
    refused(lambda: seq.causal_conv(x, w, out=x), "x")
    refused(lambda: seq.causal_conv(x, w, out=wide[:, :, 31:63]), "x")
    refused(lambda: seq.causal_conv(x[:, 1:], w, out=x[:, :-1]), "x")
    refused(lambda: seq.causal_conv(x[:1], w, out=wide.view(-1)[:40 * 32].view(1, 40, 32)), "x")
    states = torch.randn(1000, device="cuda")
    refused(lambda: seq.causal_conv(x, w, state=states[:192].view(2, 3, 32), new_state=states[96:288].view(2, 3, 32)), "state")
    refused(lambda: seq.causal_conv(x, w, new_state=wide.view(-1)[:192].view(2, 3, 32)), "x")
    refused(lambda: seq.causal_conv(x, w, out=wide[:, :, 32:64], new_state=wide.view(-1)[96 * 10 + 32:96 * 10 + 32 + 192].view(2, 3, 32)), "new_state")
    refused(lambda: seq.causal_conv(x[:1, :30], states[:128].view(32, 4), out=states[:960].view(1, 30, 32)), "weight")

    A, state = -torch.rand(32, 32, device="cuda"), torch.randn(3, 32, 32, device="cuda")
    u, B, C = (torch.randn(2, 40, 32, device="cuda") for _ in range(3))
    refused(lambda: seq.selective_scan(u, u, A, B, C, out=B), "B")
    refused(lambda: seq.selective_scan(u, u, A, B, C, out=C), "C")
    refused(lambda: seq.selective_scan(x, u, A, B, C, out=wide[:, :, 16:48]), "u")
    refused(lambda: seq.selective_scan(u, x, A, B, C, out=wide[:, :, 16:48]), "delta")
    refused(lambda: seq.selective_scan(u, u, A, B, C, z=x, out=wide[:, :, 16:48]), "z")
    refused(lambda: seq.selective_scan(u, u, A, B, C, new_state=B.view(-1)[:2048].view(2, 32, 32)), "B")
    refused(lambda: seq.selective_scan(u, u, A, B, C, state=state[:2], new_state=state[1:]), "state")

    memory = torch.randn(40, 48, device="cuda")
    refused(lambda: seq.quantize_rows(memory, out=memory.view(torch.uint8).view(-1)[:40 * 48].view(40, 48).view(F8)), "x")
    refused(lambda: seq.quantize_rows(memory, scales=memory[:, 5:6]), "x")
    room = torch.zeros(40, 48, dtype=torch.uint8, device="cuda")
    refused(lambda: seq.quantize_rows(memory[:, :40], out=room.view(F8)[:, :40], scales=room.view(torch.float32)[:, 10:11]), "scales")       # in the bytes behind a row
    q, s = seq.quantize_rows(memory)
    numbers = q.view(torch.uint8).view(torch.float32)
    refused(lambda: seq.block_matmul(q, s, q[:12], s[:1], out=numbers), "a")
    refused(lambda: seq.block_matmul(q[:20], s[:20], q[28:], s[:1], out=numbers[20:]), "b")
    torch.cuda.synchronize()
    assert torch.equal(wide, before)


@pytest.mark.parametrize("length", [1, 2, 90, 2304])
def test_results_may_lie_beside_the_inputs_and_in_their_place_as_a_whole(length):
    g = torch.Generator("cuda").manual_seed(length)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    wide, w, A = r(2, length, 64), r(32, 4), -torch.rand(32, 8, generator=g, device="cuda")
    B, C = r(2, length, 8), r(2, length, 8)
    left, right = wide[:, :, :32], wide[:, :, 32:]
    y, state = seq.causal_conv(left, w)
    got, other = seq.causal_conv(left, w, out=right)
    assert torch.equal(got, y) and torch.equal(other, state)
    delta = right.clone() - 3
    y, state = seq.selective_scan(left, delta, A, B, C)
    got, other = seq.selective_scan(left, delta, A, B, C, out=delta)
    assert got is delta and torch.equal(got, y) and torch.equal(other, state)
    rows = left.reshape(-1, 32)
    q, s = seq.quantize_rows(rows)
    both = torch.zeros(2 * length, 96, dtype=torch.uint8, device="cuda").view(F8)
    got, _ = seq.quantize_rows(rows, out=both[:, 32:64])
    assert torch.equal(got.float(), q.float()) and not both.float()[:, :32].any() and not both.float()[:, 64:].any()


def test_results_come_from_the_devices_allocator_wherever_the_inputs_came_from(tmp_path):
    lib = os.path.join(tmp_path, "foreign.so")
    system = [*include_paths(), sysconfig.get_path("include"), "/opt/rocm/include"]
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-fPIC", "-D__HIP_PLATFORM_AMD__", *[f for p in system for f in ("-isystem", p)], "-shared", "-o", lib,
                    os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "foreign_allocator.cpp"), *["-L" + p for p in library_paths()],
                    "-ltorch_python", "-ltorch_cpu", "-lc10"], check=True, capture_output=True, text=True)
    foreign = ctypes.PyDLL(lib)
    foreign.foreign_float_tensor.restype, foreign.foreign_float_tensor.argtypes = ctypes.py_object, [ctypes.c_longlong, ctypes.c_longlong]
    foreign.foreign_calls.restype = ctypes.c_longlong
    x = foreign.foreign_float_tensor(40, 100)
    made = foreign.foreign_calls()
    assert made == 1
    x.copy_(torch.randn(40, 100))
    w, B, A = torch.randn(100, 4, device="cuda"), torch.randn(1, 40, 4, device="cuda"), -torch.rand(100, 4, device="cuda")
    y, state = seq.causal_conv(x[None], w)
    _, scan_state = seq.selective_scan(x[None], x[None], A, B, B)
    q, s = seq.quantize_rows(x)
    assert foreign.foreign_calls() == made and y.device == state.device == q.device == s.device == x.device
    want = x.clone()
    assert torch.equal(y, seq.causal_conv(want[None], w)[0]) and torch.equal(q.float(), seq.quantize_rows(want)[0].float()) and scan_state.shape == (1, 100, 4)


def test_results_whose_rows_share_memory_are_refused():
    x, w, memory = torch.randn(3, 5, 16, device="cuda"), torch.randn(16, 4, device="cuda"), torch.zeros(4000, device="cuda")
    B, A = torch.randn(3, 5, 4, device="cuda"), -torch.rand(16, 4, device="cuda")
    for steps in ((16, 16, 1), (64, 16, 1), (40, 20, 1), (16, 40, 1)):
        out = memory.as_strided((3, 5, 16), steps)
        for call in (lambda: seq.causal_conv(x, w, out=out), lambda: seq.selective_scan(x, x, A, B, B, out=out)):
            with pytest.raises(seq.XlError, match="share memory with each other"):
                call()
    y, _ = seq.causal_conv(x, w)
    for steps in ((80, 16, 1), (100, 20, 1), (16, 48, 1), (20, 90, 1)):         # sequences outermost or tokens, with gaps or without
        assert torch.equal(seq.causal_conv(x, w, out=memory.as_strided((3, 5, 16), steps))[0], y)
    with pytest.raises(seq.XlError, match="share memory with each other"):
        seq.quantize_rows(x[0], scales=memory[:1].expand(5, 1))
