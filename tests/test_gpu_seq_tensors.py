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
