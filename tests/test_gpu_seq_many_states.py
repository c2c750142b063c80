"""Scans of more than 64 states whose rows of B and C are read one number at a time: more numbers in a row than a wave has lanes."""
import pytest
import torch

from paper_2007_06000_amd import seq
from test_gpu_seq_conv import HALF
from test_gpu_seq_scan import check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("batch,length,channels,states", [(1, 16, 4, 65), (2, 33, 9, 66), (1, 90, 30, 101), (1, 40, 301, 127), (3, 130, 5, 97)])
def test_odd_numbers_of_states(batch, length, channels, states, dtype):
    p = inputs(batch, length, channels, states, dtype, seed=states)
    check(p, *seq.selective_scan(**p), "all")
    bare = {k: p[k] for k in ("u", "delta", "A", "B", "C")}
    check(bare, *seq.selective_scan(**bare), "bare")


@pytest.mark.parametrize("states", [72, 100, 128])
def test_rows_that_are_not_aligned(states):
    p = inputs(2, 50, 12, states, torch.bfloat16, seed=states)
    both = torch.full((2, 50, 2 * states + 3), float("nan"), device="cuda").bfloat16()
    both[:, :, 1:states + 1], both[:, :, states + 2:2 * states + 2] = p["B"], p["C"]
    p["B"], p["C"] = both[:, :, 1:states + 1], both[:, :, states + 2:2 * states + 2]
    check(p, *seq.selective_scan(**p), "unaligned")


@pytest.mark.parametrize("states", [72, 101, 128])
def test_rows_that_lie_across_each_other(states):
    p = inputs(1, 50, 12, states, torch.float32, seed=states)
    p["u"] = p["u"][:, :1].expand(1, 50, 12)
    p["B"] = p["B"].reshape(-1).as_strided((1, 50, states), (0, 1, 1))
    check(p, *seq.selective_scan(**p), "across")
