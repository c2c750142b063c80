"""From a fused convolution block's feature maps into a scan block: all positions at once, and position by position from a recorded step."""
import pytest
import torch

import xl_workloads as W
from paper_2007_06000_amd.scan_block import ScanBlock, TokenStep, random_weights
from paper_2007_06000_amd.session import Session
from test_gpu_seq_block import TOLERANCE, apart, definition
from test_gpu_seq_conv import f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(TOLERANCE), ids=str)
def test_positions_of_a_stems_maps_as_sequences(dtype):
    wl = W.config(2, n=2, hw=20)
    stem = Session(wl, *W.make_tensors(wl))
    maps = stem.run().clone()
    batch, width = maps.shape[:2]
    block = ScanBlock(random_weights(width, 2 * width), dtype=dtype)
    x = maps.flatten(2).transpose(1, 2)
    x = (x / x.square().mean().sqrt()).to(dtype)            # tokens outermost: the block lays them out
    y, (conv, scan) = block(x)
    want = definition(block, f64(x), [x.shape[1]] * batch)
    assert apart(y, want[0]) < TOLERANCE[dtype] and apart(conv, want[1]) < TOLERANCE[dtype] and apart(scan, want[2]) < TOLERANCE[dtype]
    step = TokenStep(block, batch)
    by_token = torch.cat([step(x[:, t:t + 1]).clone() for t in range(x.shape[1])], 1)
    assert apart(by_token, want[0]) < TOLERANCE[dtype] and apart(step.cache[1], want[2]) < TOLERANCE[dtype]
    again = stem.run()                                      # the stem is what it was
    assert torch.equal(again, maps)
