"""The root-mean-square norm where numbers and rows come to an end."""
import numpy as np
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import seq
from test_gpu_seq_conv import f64, near
from test_gpu_seq_norm import inputs

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


@pytest.mark.parametrize("quantized", [False, True])
def test_the_longest_row(quantized):
    """As many numbers as a size may have, 4096 fewer than 32 bits count: a turn of a workgroup goes past them."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough memory is free")
    k, step = (1 << 31) - 1 - 4096, 1 << 26
    x = torch.empty(1, k, dtype=torch.bfloat16, device="cuda")
    w = torch.empty(k, device="cuda")
    g = torch.Generator("cuda").manual_seed(0)
    squares = 0.0
    for at in range(0, k, step):
        n = min(step, k - at)
        x[0, at:at + n].copy_(torch.randn(n, generator=g, device="cuda"))
        w[at:at + n].copy_(torch.rand(n, generator=g, device="cuda") + 0.5)
        squares += float(x[0, at:at + n].double().square().sum())
    inverse = (squares / k + 1e-6) ** -0.5
    if quantized:
        q, scales, _ = seq.rms_norm_quantized(x, w)
        assert not q.as_strided((1, q.stride(0)), (q.stride(0), 1)).view(torch.uint8)[:, k:].any()
    else:
        y, _ = seq.rms_norm(x, w)
    for at in range(0, k, step):
        n = min(step, k - at)
        want = x[0, at:at + n].double() * w[at:at + n].double() * inverse
        off = 16 * 2.0 ** -24 * want.abs()
        if quantized:       # half a step of e4m3
            s = scales[0, at // 128:(at + n + 127) // 128].double().repeat_interleave(128)[:n]
            got = q[0, at:at + n].float().double() * s
            off += 2.0 ** -4 * 1.0001 * want.abs() + 2.0 ** -10 * s
        else:               # of bf16
            got = y[0, at:at + n].double()
            off += 2.0 ** -8 * 1.0001 * want.abs() + 2.0 ** -134
        assert ((got - want).abs() <= off).all(), at
    del x, w
    torch.cuda.empty_cache()


@pytest.mark.parametrize("k", [1, 96, 1500, 9000, 40000])
def test_an_eps_that_counts_beside_the_largest_squares(k):
    x, _, w = inputs(3, k, torch.float32, None)
    for size, eps in ((1e18, 1e38), (1e19, 3e38), (1.5e19, 3.4e38), (1e19, 1e37), (3e38, 3.4e38), (1.0, 3.4e38)):
        at = x.sign() * size
        want, bound, _ = ref.rms_norm(f64(at), None, f64(w), eps)
        near(seq.rms_norm(at, w, eps=eps)[0], want, bound, (size, eps))


@pytest.mark.parametrize("k", [96, 1500, 9000, 40000])
def test_small_numbers_beside_the_largest(k):
    """A result is a number of 24 bits wherever it is one of the normal ones, whatever size the row's largest number has."""
    x = torch.full((1, k), 2.0 ** -59, device="cuda")
    x[0, k // 2] = 1.5 * 2.0 ** 66
    x[0, 1::2] *= 1 + torch.arange(k // 2, device="cuda") * 2.0 ** -23
    w = torch.ones(k, device="cuda")
    want, bound, _ = ref.rms_norm(f64(x), None, f64(w), 1e-6)
    y = f64(seq.rms_norm(x, w)[0])
    assert (np.abs(want) > 2.0 ** -126).all() and (np.abs(y - want) <= bound + 2.0 ** -149).all()


@pytest.mark.parametrize("k", [7, 200, 1001, 3001, 40009])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")], ids=str)
def test_what_lies_behind_a_row_of_eight_bits_is_zero(bad, k):
    for at in (0, k - 1):
        x, r, w = inputs(3, k, torch.bfloat16, torch.bfloat16)
        x[1, at] = bad
        q, _, _ = seq.rms_norm_quantized(x, w, residual=r)
        assert not q.as_strided((3, q.stride(0)), (q.stride(0), 1)).view(torch.uint8)[:, k:].any()


@pytest.mark.parametrize("k", [7, 200, 1001, 40009])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")], ids=str)
@pytest.mark.parametrize("quantize", [seq.quantize_rows, seq.quantize_weight], ids=["rows", "weight"])
def test_what_lies_behind_a_row_of_the_quantiser_is_zero(quantize, bad, k):
    for at in (0, k - 1):
        x, _, _ = inputs(3, k, torch.bfloat16, None)
        x[1, at] = bad
        q, _ = quantize(x)
        assert not q.as_strided((3, q.stride(0)), (q.stride(0), 1)).view(torch.uint8)[:, k:].any()
