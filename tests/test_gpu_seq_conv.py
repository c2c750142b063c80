"""The causal convolution against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import seq
from paper_2007_06000_amd.binding import XlError

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # of a unit in the last place


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def near(got, want, bound, what):
    """Within the bound of the fp32 arithmetic and the rounding to the result's type."""
    half = HALF[got.dtype]
    got = f64(got)
    off = np.abs(got - want) - (bound + half * (np.abs(want) + bound) + 2.0 ** -24)
    assert np.isfinite(got).all() and (off <= 0).all(), f"{what}: {off.max():.3g} beyond the bound at {np.unravel_index(off.argmax(), off.shape)}"


def inputs(batch, length, channels, taps, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return r(batch, length, channels).to(dtype).cuda(), r(channels, taps).cuda(), r(channels).cuda(), r(batch, taps - 1, channels).to(dtype).cuda()


def check(x, w, bias, state, lengths, silu, y, new, what):
    n = [x.shape[1]] * x.shape[0] if lengths is None else [min(max(int(v), 0), x.shape[1]) for v in lengths]
    want, bound, last = ref.causal_conv(f64(x), f64(w), np.zeros(x.shape[2]) if bias is None else f64(bias), f64(state), n, silu)
    near(y, want, bound, what)
    assert np.array_equal(f64(new), last), what


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("batch,length,channels,taps", [(1, 1, 1, 2), (2, 1, 64, 4), (3, 2, 40, 4), (2, 5, 24, 3), (1, 131, 8, 2), (2, 70, 1000, 4), (5, 33, 17, 3), (1, 4, 512, 4)])
def test_against_the_definition(batch, length, channels, taps, dtype):
    x, w, bias, state = inputs(batch, length, channels, taps, dtype)
    for st in (state, None):
        for silu in (True, False):
            y, new = seq.causal_conv(x, w, bias if silu else None, state=st, silu=silu)
            check(x, w, bias if silu else None, st, None, silu, y, new, f"state={st is not None} silu={silu}")


@pytest.mark.parametrize("lengths", [[0, 1, 2, 3, 37], [37, 0, -5, 1000, 36]])
def test_sequences_of_their_own_lengths(lengths):
    x, w, bias, state = inputs(5, 37, 48, 4, torch.bfloat16)
    for b, n in enumerate(lengths):
        x[b, max(n, 0):] = float("nan")         # never read
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    y, new = seq.causal_conv(x, w, bias, state=state, lengths=n)
    check(torch.nan_to_num(x), w, bias, state, lengths, True, y, new, "lengths")
    for b, k in enumerate(lengths):
        assert not y[b, max(k, 0):].any()


def test_pieces_and_single_tokens_continue_a_sequence():
    x, w, bias, _ = inputs(3, 40, 72, 4, torch.float16)
    whole, last = seq.causal_conv(x, w, bias)
    state, got = None, []
    for a, b in ((0, 2), (2, 3), (3, 20), (20, 20), (20, 39), (39, 40)):
        y, state = seq.causal_conv(x[:, a:b], w, bias, state=state, new_state=state)      # in place from the second piece on
        got.append(y)
    assert torch.equal(torch.cat(got, 1), whole) and torch.equal(state, last)


def test_a_long_sequence_may_overwrite_the_state_it_began_with():
    x, w, bias, state = inputs(2, 500, 64, 4, torch.bfloat16)
    y, new = seq.causal_conv(x, w, bias, state=state)
    again, same = seq.causal_conv(x, w, bias, state=state, new_state=state)
    assert same is state and torch.equal(y, again) and torch.equal(new, state)


def test_slots_name_rows_of_a_cache():
    x, w, bias, _ = inputs(4, 6, 32, 3, torch.float32)
    cache = torch.randn(7, 2, 32, device="cuda")
    before = cache.clone()
    slots = torch.tensor([5, -1, 0, 7], dtype=torch.int32, device="cuda")       # two of them absent
    y, new = seq.causal_conv(x, w, bias, state=cache, slots=slots)
    assert new is cache and not y[1].any() and not y[3].any()
    check(x[[0, 2]], w, bias, before[[5, 0]], None, True, y[[0, 2]], cache[[5, 0]], "slots")
    assert torch.equal(cache[[1, 2, 3, 4, 6]], before[[1, 2, 3, 4, 6]])


@pytest.mark.parametrize("offset,width", [(0, 96), (48, 96), (3, 97), (1, 50)])
def test_strides_and_alignment(offset, width):
    x = torch.randn(2, 45, width, device="cuda").bfloat16()[:, :, offset:offset + 48]
    _, w, bias, state = inputs(2, 1, 48, 4, torch.bfloat16)
    out = torch.full((2, 46, width), 7.0, dtype=torch.bfloat16, device="cuda")
    y, new = seq.causal_conv(x, w, bias, state=state, out=out[:, :45, offset:offset + 48])
    check(x, w, bias, state, None, True, y, new, "strided")
    out[:, :45, offset:offset + 48] = 7
    assert (out == 7).all()                     # nothing beside it was written
    t = torch.randn(45, 2, 48, device="cuda").bfloat16().transpose(0, 1)        # tokens outermost
    y, new = seq.causal_conv(t, w, bias, state=state)
    check(t, w, bias, state, None, True, y, new, "transposed")


def test_offsets_beyond_32_bits():
    big = torch.empty(3 * (1 << 31) + 4096, dtype=torch.int8, device="cuda").view(torch.float16)
    x = big.as_strided((2, 3, 64), ((1 << 30) + 640, 1 << 30, 1))
    x.copy_(torch.randn(2, 3, 64))
    _, w, bias, _ = inputs(1, 1, 64, 4, torch.float16)
    y, new = seq.causal_conv(x, w, bias)
    check(x, w, bias, None, None, True, y, new, "far apart")


def test_refusals():
    x, w, bias, state = inputs(2, 5, 16, 4, torch.bfloat16)
    for f in (lambda: seq.causal_conv(x, w.half()), lambda: seq.causal_conv(x, w, bias[:8]), lambda: seq.causal_conv(x, w, state=state.float()),
              lambda: seq.causal_conv(x, w, state=state[:, :2]), lambda: seq.causal_conv(x.transpose(1, 2), w[:5]), lambda: seq.causal_conv(x, w[:, :1]),
              lambda: seq.causal_conv(x.double(), w), lambda: seq.causal_conv(x, w, lengths=torch.tensor([1, 2], device="cuda")),
              lambda: seq.causal_conv(x, w, slots=torch.tensor([1, 0], dtype=torch.int32, device="cuda")), lambda: seq.causal_conv(x, w.cpu()),
              lambda: seq.causal_conv(x, w.requires_grad_()), lambda: seq.causal_conv(x[0], w)):
        with pytest.raises(XlError):
            f()
    with torch.no_grad():
        seq.causal_conv(x, w)
