"""Low-rank adapters where numbers, places and sizes come to an end."""
import pytest
import torch

from paper_2007_06000_amd import seq
from test_gpu_seq_conv import HALF, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length", [3, 4200])           # in one kernel, in two
@pytest.mark.parametrize("rank", [3, 16, 20, 64, 100])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
def test_a_result_of_16_bits_is_rounded_once(dtype, rank, length):
    """down x is half a step and 2^-20 above one, a number of 24 bits, and rounds to the step above.  Rounded to 16 bits on its way into the second product it lands on the tie, and then on one."""
    half = HALF[dtype]
    x, down, up = torch.ones(1, length, 3), torch.zeros(1, rank, 3), torch.zeros(1, 70, rank)
    down[0, rank - 1], up[:, :, rank - 1] = torch.tensor([1, half, 2.0 ** -20]), 1
    y = torch.zeros(1, length, 70, dtype=dtype, device="cuda")
    out = seq.add_adapters(y, *[t.to(dtype).cuda() for t in (x, down, up)], torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert (f64(out) == 1 + 2 * half).all()
