"""The root-mean-square norm where numbers and rows come to an end."""
import numpy as np
import pytest
import torch

from paper_2007_06000_amd import seq
from test_gpu_seq_conv import f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [32769, 1 << 20, (1 << 24) + 77])
@pytest.mark.parametrize("value", [0.95, 1.05])
def test_long_rows_of_one_number(value, k):
    """In fp32 every square is rounded the same way when it joins a sum, the more the larger the sum.  Sums in 64 bits leave the mean's rounding (half of it: a root), the root and three products."""
    x, w = torch.full((1, k), value, device="cuda"), torch.ones(k, device="cuda")
    y, _ = seq.rms_norm(x, w)
    v = float(x[0, 0])
    want = v / np.sqrt(v * v + 1e-6)
    assert (np.abs(f64(y) - want) <= 8 * 2.0 ** -24 * want).all()
