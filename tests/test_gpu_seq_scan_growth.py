"""Scans whose states grow: positive A, or negative steps.  What a run of tokens multiplies a state by may lie outside fp32 while the state itself stays inside."""
import pytest
import torch

from test_gpu_seq_scan import check, inputs, run

pytestmark = pytest.mark.gpu
# (length, channels): one token after the other; tiles of few and of many workgroups; parts
SHAPES = [(8, 16), (70, 16), (300, 40), (2304, 64)]


def growing(length, channels, states, per_token, first, last, softplus, negative):
    """Steps that multiply a state by e^per_token between the tokens `first` and `last`, and by one elsewhere."""
    p = inputs(2, length, channels, states, torch.float32, seed=length)
    del p["delta_bias"]
    sign = -1.0 if negative else 1.0
    p["A"] = torch.full((channels, states), sign * per_token, device="cuda")
    live = torch.zeros(1, length, 1, device="cuda")
    live[:, first:last] = 1
    # softplus(0.541325) = 1, softplus(-200) = 0
    p["delta"] = (live * 200.541325 - 200 if softplus else sign * live).expand(2, length, channels).contiguous()
    return p


@pytest.mark.parametrize("states", [16, 5, 30])
@pytest.mark.parametrize("softplus,negative", [(True, False), (False, False), (False, True)])
@pytest.mark.parametrize("length,channels", SHAPES)
def test_states_that_are_still_zero_stay_zero_however_much_they_would_grow(length, channels, softplus, negative, states):
    half = length // 2
    p = growing(length, channels, states, 20.0 if length < 1000 else 0.8, 0, half + 1, softplus, negative)
    del p["state"]
    p["u"][:, :half] = 0            # the first input meets a zero state; what comes behind does not grow
    check(p, *run(p, softplus=softplus), "zero at first", softplus=softplus)


@pytest.mark.parametrize("states", [16, 5, 30])
@pytest.mark.parametrize("length,channels", SHAPES)
def test_small_states_may_grow_by_more_than_the_largest_number(length, channels, states):
    first, tokens = (0, min(length, 16)) if length < 1000 else (256, 256)               # within one part
    p = growing(length, channels, states, 120.0 / tokens, first, first + tokens, False, False)      # e^120 is 1e52
    p["u"][:, :first + tokens] = 0
    p["state"] = p["state"] * 1e-30
    check(p, *run(p, softplus=False), "small at first", softplus=False)


@pytest.mark.parametrize("length,channels", SHAPES)
def test_growth_and_decay_cancel(length, channels):
    """A state goes up by e^60 and down again by as much, several times: no token's state is out of range."""
    p = inputs(1, length, channels, 16, torch.float32, seed=1)
    del p["delta_bias"]
    p["A"] = torch.ones(channels, 16, device="cuda")
    turns = torch.arange(length, device="cuda") // 4 % 2
    p["delta"] = ((1 - 2 * turns) * 15.0)[None, :, None].expand(1, length, channels).contiguous()
    p["u"] = p["u"] * 1e-12
    check(p, *run(p, softplus=False), "up and down", softplus=False)


@pytest.mark.parametrize("length,channels", SHAPES)
def test_an_infinite_state_stays_infinite(length, channels):
    p = inputs(1, length, channels, 16, torch.float32, step=(3.0, 0.1))
    p["B"], p["u"] = p["B"].abs() + 0.1, p["u"].abs() + 0.1
    p["A"] = p["A"].clamp(-16, -8)
    p["u"][:, 3] = float("inf")
    _, state = run(p)
    assert (state == float("inf")).all()
