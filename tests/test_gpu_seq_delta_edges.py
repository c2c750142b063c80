"""The gated delta rule where numbers, places and sizes come to an end."""
import numpy as np
import pytest
import torch

from paper_2007_06000_amd import seq
from test_gpu_seq_conv import HALF, f64
from test_gpu_seq_delta import compare, inputs, reference, spread

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length", [5, 64, 100])        # token by token, in chunks
@pytest.mark.parametrize("dk", [5, 64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("where", ["state", "correction", "product"])
def test_a_result_of_16_bits_is_rounded_once(where, dtype, dk, length):
    """Half a step and 2^-20 above one: every sum of these calls is a number of 24 bits, and rounds to the step above.  What is rounded to 16 bits on the way there lands on the tie, and then on one."""
    half = HALF[dtype]
    value = 1 + half + 2.0 ** -20
    zeros = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    q, k, v = zeros(1, length, 1, dk), zeros(1, length, 1, dk), zeros(1, length, 1, 20)
    beta, state = zeros(1, length, 1), zeros(1, 1, dk, 20)
    q[..., 0], k[0, 0, 0, 0], v[0, 0] = 1, 1, 1
    if where == "state":
        state[0, 0, 0] = value
    elif where == "correction":
        beta[0, 0] = value
    else:
        q[..., :3], k[0, 0, 0, 1], k[0, 0, 0, 2], beta[0, 0] = 1, half, 2.0 ** -20, 1
    y, _ = seq.gated_delta_rule(q.to(dtype), k.to(dtype), v.to(dtype), zeros(1, length, 1), beta, scale=1.0, state=state)
    assert (f64(y) == 1 + 2 * half).all()
