"""The selective scan against its definition in 64 bits."""
import struct

import numpy as np
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import seq
from paper_2007_06000_amd.binding import XlError
from test_gpu_seq_conv import HALF, f64, near

pytestmark = pytest.mark.gpu


def inputs(batch, length, channels, states, dtype, seed=0, step=(-2.0, 1.0)):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return {"u": r(batch, length, channels).to(dtype).cuda(), "delta": (step[0] + step[1] * r(batch, length, channels)).to(dtype).cuda(),
            "A": -(1 + torch.arange(states) * (1 + 0.1 * torch.rand(channels, states, generator=g))).cuda(),
            "B": r(batch, length, states).to(dtype).cuda(), "C": r(batch, length, states).to(dtype).cuda(), "D": r(channels).cuda(),
            "z": r(batch, length, channels).to(dtype).cuda(), "delta_bias": (0.1 * r(channels)).cuda(), "state": r(batch, channels, states).cuda()}


def check(p, y, new, what, lengths=None, softplus=True, rows=slice(None)):
    batch, length, channels = p["u"].shape
    n = [length] * batch if lengths is None else [min(max(int(v), 0), length) for v in lengths]
    bias = p.get("delta_bias")
    want, bound, last, last_bound = ref.selective_scan(f64(p["u"]), f64(p["delta"]), f64(p["A"]), f64(p["B"]), f64(p["C"]), f64(p.get("D")), f64(p.get("z")),
                                                       np.zeros(channels) if bias is None else f64(bias), f64(p.get("state")), n, softplus)
    near(y, want, bound, f"{what}: y")
    near(new, last, last_bound, f"{what}: state")


def run(p, **more):
    return seq.selective_scan(**p, **more)


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("batch,length,channels,states", [
    (1, 1, 1, 1), (2, 1, 64, 16), (3, 3, 40, 16), (1, 16, 16, 16), (2, 17, 33, 13), (1, 64, 64, 16), (2, 65, 20, 4), (1, 130, 100, 16), (2, 300, 18, 7),
    (1, 50, 24, 32), (2, 77, 9, 50), (1, 140, 12, 64), (1, 40, 7, 128), (2, 9, 5, 100), (1, 515, 40, 2)])
def test_against_the_definition(batch, length, channels, states, dtype):
    p = inputs(batch, length, channels, states, dtype)
    check(p, *run(p), "all")
    bare = {k: p[k] for k in ("u", "delta", "A", "B", "C")}
    check(bare, *run(bare), "bare")


@pytest.mark.parametrize("length", [1, 90])
def test_steps_without_softplus(length):
    p = inputs(2, length, 48, 16, torch.float32)
    p["delta"], p["delta_bias"] = p["delta"].abs() * 0.1, p["delta_bias"].abs()
    check(p, *run(p, softplus=False), "plain steps", softplus=False)


@pytest.mark.parametrize("step", [(-9.0, 0.5), (3.0, 2.0), (30.0, 10.0)])
def test_small_and_large_steps(step):
    """From states that keep everything to ones that forget it within a token (exponentials that underflow)."""
    p = inputs(1, 100, 32, 16, torch.float32, step=step)
    check(p, *run(p), f"steps {step}")


@pytest.mark.parametrize("states", [16, 64, 5])
@pytest.mark.parametrize("lengths", [[0, 1, 63, 64, 200], [200, -3, 65, 9999, 2]])
def test_sequences_of_their_own_lengths(lengths, states):
    p = inputs(5, 200, 36, states, torch.bfloat16)
    clean = {k: v.clone() for k, v in p.items()}
    for b, n in enumerate(lengths):
        for k in ("u", "delta", "B", "C", "z"):
            p[k][b, max(n, 0):] = float("nan")          # never read
    y, new = run(p, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    check(clean, y, new, "lengths", lengths)
    for b, n in enumerate(lengths):
        assert not y[b, max(n, 0):].any()
        if n <= 0:
            assert torch.equal(new[b], p["state"][b])


def asks_for_a_workspace(p):
    batch, length, channels = p["u"].shape
    sizes = struct.pack("=20q14Q", batch, length, channels, p["A"].shape[1], *[0] * 30)
    return seq.lib().xl_selective_scan_workspace(sizes) > 0


@pytest.mark.parametrize("dtype,batch,length,channels,states", [
    (torch.bfloat16, 1, 2304, 64, 16), (torch.float32, 2, 2100, 33, 13), (torch.float16, 3, 2049, 20, 3), (torch.bfloat16, 1, 2500, 28, 8),
    (torch.float32, 1, 2050, 12, 30), (torch.float16, 1, 2090, 11, 64)])
def test_long_sequences_of_few_channels_are_worked_on_in_parts(dtype, batch, length, channels, states):
    p = inputs(batch, length, channels, states, dtype, step=(-5.0, 1.0))
    assert asks_for_a_workspace(p)
    check(p, *run(p), "all")
    bare = {k: p[k] for k in ("u", "delta", "A", "B", "C")}
    check(bare, *run(bare), "bare")


# 2100 tokens of six sequences of 33 channels: parts of 384
@pytest.mark.parametrize("lengths", [[0, 1, 383, 384, 385, 2100], [768, 2099, 1537, 1536, -1, 5000]])
def test_parts_of_sequences_of_their_own_lengths(lengths):
    p = inputs(6, 2100, 33, 16, torch.bfloat16, step=(-5.0, 1.0))
    assert asks_for_a_workspace(p)
    clean = {k: v.clone() for k, v in p.items()}
    for b, n in enumerate(lengths):
        for k in ("u", "delta", "B", "C", "z"):
            p[k][b, max(n, 0):] = float("nan")          # never used
    state = p["state"]
    y, new = run(p, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), new_state=state, out=p["u"])      # everything in place
    assert new is state and y is p["u"]
    check(clean, y, new, "lengths", lengths)
    for b, n in enumerate(lengths):
        assert not y[b, max(n, 0):].any()
        if n <= 0:
            assert torch.equal(new[b], clean["state"][b])


def test_parts_of_sequences_in_a_cache():
    p = inputs(3, 2200, 40, 16, torch.float32, step=(-5.0, 1.0))
    assert asks_for_a_workspace(p)
    cache = torch.full((5, 40, 16), 7.0, device="cuda")
    slots = [4, -1, 0]
    cache[[4, 0]] = p["state"][[0, 2]]
    y, new = seq.selective_scan(**{**p, "state": cache}, slots=torch.tensor(slots, dtype=torch.int32, device="cuda"))
    assert new is cache and not y[1].any() and (cache[1:4] == 7).all()
    part = {k: v if k in ("A", "D", "delta_bias") else v[[0, 2]] for k, v in p.items()}
    check(part, y[[0, 2]], cache[[4, 0]], "cache")


def test_pieces_and_single_tokens_continue_a_sequence():
    p = inputs(2, 150, 40, 16, torch.float32)
    state, got = p["state"].clone(), []
    for a, b in ((0, 1), (1, 2), (2, 90), (90, 90), (90, 93), (93, 149), (149, 150)):
        piece = {k: v[:, a:b] if k in ("u", "delta", "B", "C", "z") else v for k, v in p.items()}
        piece["state"] = state
        y, new = run(piece, new_state=state)
        assert new is state
        got.append(y)
    check(p, torch.cat(got, 1), state, "pieces")


@pytest.mark.parametrize("length", [1, 70])
def test_slots_name_rows_of_a_cache(length):
    p = inputs(4, length, 24, 16, torch.bfloat16)
    cache = torch.randn(6, 24, 16, device="cuda")
    before = cache.clone()
    y, new = run({**p, "state": cache}, slots=torch.tensor([4, -1, 0, 6], dtype=torch.int32, device="cuda"))
    assert new is cache and not y[1].any() and not y[3].any()
    some = {k: v if k in ("A", "D", "delta_bias") else v[[0, 2]] for k, v in p.items()}
    check({**some, "state": before[[4, 0]]}, y[[0, 2]], cache[[4, 0]], "slots")
    assert torch.equal(cache[[1, 2, 3, 5]], before[[1, 2, 3, 5]])


@pytest.mark.parametrize("length", [1, 100])
@pytest.mark.parametrize("offset,width", [(0, 128), (64, 128), (5, 133), (2, 70)])
def test_strides_and_alignment(offset, width, length):
    p = inputs(2, length, 64, 16, torch.float16)
    for k in ("u", "z", "delta"):
        wide = torch.full((2, length, width), float("nan"), dtype=torch.float16, device="cuda")
        wide[:, :, offset:offset + 64] = p[k]
        p[k] = wide[:, :, offset:offset + 64]
    both = torch.cat([p["B"], p["C"], p["B"][:, :, :offset]], 2)
    p["B"], p["C"] = both[:, :, :16], both[:, :, 16:32]
    out = torch.full((2, length, width), 7.0, dtype=torch.float16, device="cuda")
    y, new = run(p, out=out[:, :, offset:offset + 64])
    check(p, y, new, "strided")
    out[:, :, offset:offset + 64] = 7
    assert (out == 7).all()
    for k in ("u", "z", "delta", "B", "C"):             # tokens outermost
        p[k] = p[k].transpose(0, 1).contiguous().transpose(0, 1)
    check(p, *run(p), "transposed")


@pytest.mark.parametrize("length", [1, 200])
@pytest.mark.parametrize("over", ["u", "z"])
def test_the_result_may_take_an_inputs_place(over, length):
    p = inputs(2, length, 48, 16, torch.bfloat16)
    y, new = run(p)
    got, same = run(p, out=p[over])
    assert got is p[over] and torch.equal(got, y) and torch.equal(same, new)


def test_a_result_does_not_depend_on_the_rest_of_the_batch():
    p = inputs(5, 333, 80, 16, torch.bfloat16)
    y, new = run(p)
    for b in (0, 4):
        one = {k: v if k in ("A", "D", "delta_bias") else v[b:b + 1] for k, v in p.items()}
        check(one, *run(one), "alone")
        check(one, y[b:b + 1], new[b:b + 1], "in a batch")


@pytest.mark.parametrize("length", [1, 80])
def test_infinities_stay_with_their_channel_and_come_after_their_token(length):
    p = inputs(1, length, 32, 16, torch.float32)
    at = length // 2
    p["u"][0, at, 7] = float("inf")
    p["u"][0, at, 9] = float("nan")
    y, new = run(p)
    clean = torch.ones(32, dtype=torch.bool, device="cuda")
    clean[[7, 9]] = False
    assert torch.isfinite(y[0, :, clean]).all() and torch.isfinite(new[0, clean]).all() and torch.isfinite(y[0, :at]).all()
    assert not torch.isfinite(y[0, at:, ~clean]).any() and not torch.isfinite(new[0, ~clean]).any()


def test_offsets_beyond_32_bits():
    big = torch.empty(5 << 31, dtype=torch.int8, device="cuda").view(torch.float16)
    p = inputs(2, 3, 64, 16, torch.float16)
    u = big.as_strided((2, 3, 64), ((1 << 30) + 640, 1 << 30, 1))
    u.copy_(p["u"])
    p["u"] = u
    check(p, *run(p), "far apart, 3 tokens")
    p = inputs(2, 64, 64, 16, torch.float16)
    u = big.as_strided((2, 64, 64), ((1 << 31) + 6400, 1 << 25, 1))
    u.copy_(p["u"])
    p["u"] = u
    check(p, *run(p), "far apart, 64 tokens")


def test_refusals():
    p = inputs(2, 5, 16, 16, torch.bfloat16)
    for change in (dict(delta=p["delta"].float()), dict(A=p["A"].bfloat16()), dict(A=p["A"][:8]), dict(B=p["B"][:, :, :8]), dict(D=p["D"][:1]), dict(z=p["z"][:1]),
                   dict(state=p["state"].bfloat16()), dict(state=p["state"][:1]), dict(A=torch.zeros(16, 129, device="cuda")), dict(A=p["A"].t()), dict(u=p["u"][0]),
                   dict(A=p["A"].clone().requires_grad_()), dict(C=p["C"].cpu()), dict(u=p["u"].double()), dict(state=None, slots=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(XlError):
            run({**p, **change})
