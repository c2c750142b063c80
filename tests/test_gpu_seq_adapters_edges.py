"""Low-rank adapters where numbers, places and sizes come to an end."""
import pytest
import torch

from paper_2007_06000_amd import seq
from test_gpu_seq_adapters import check, inputs
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


# batch, length, k, n, rank, adapters: two kernels, k and out's columns in several parts, every width of rank
CUT = [(2, 2100, 1100, 2100, 12, 3), (2, 2100, 1100, 2100, 20, 2), (1, 4200, 1030, 2056, 50, 1), (1, 4200, 1030, 2056, 100, 2), (3, 1450, 2100, 2049, 128, 4), (5, 1000, 1537, 4161, 7, 2)]


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("size", CUT, ids=lambda s: "x".join(map(str, s)))
def test_k_and_the_columns_of_the_result_in_several_parts(size, dtype):
    p = inputs(*size, dtype, seed=sum(size))
    batch, length = size[:2]
    n = [length * (b + 1) // batch - b % 2 * 17 for b in range(batch)]      # up to all, and inside of a tile
    lengths = torch.tensor(n, dtype=torch.int32, device="cuda")
    for b in range(batch):
        p["x"][b, n[b]:] = float("nan")
    want = seq.add_adapters(**p, lengths=lengths)
    check(p, want, "parts", n)
    y = p["y"].clone()
    assert seq.add_adapters(**{**p, "y": y}, lengths=lengths, out=y) is y and torch.equal(y, want)
    wide = torch.full((batch, length, size[3] + 9), 3.0, dtype=dtype, device="cuda")        # rows that begin anywhere
    out = seq.add_adapters(**p, lengths=lengths, out=wide[..., 5:-4])
    assert torch.equal(out, want) and (wide[..., :5] == 3).all() and (wide[..., -4:] == 3).all()


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("rank", [8, 128])
@pytest.mark.parametrize("batch,length,k,n", [(32, 1, 2048, 4096), (1, 1, 4096, 4096), (3, 5, 520, 1001), (2, 300, 130, 64)])
def test_usual_ranks(batch, length, k, n, rank, dtype):
    p = inputs(batch, length, k, n, rank, 3, dtype, seed=rank)
    if batch >= 3:
        p["index"][1] = -1
    check(p, seq.add_adapters(**p), "ranks")
