"""Block quantisation and the block-scaled product against their definitions."""
import numpy as np
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import seq
from paper_2007_06000_amd.binding import XlError
from test_gpu_seq_conv import HALF, f64

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def e4m3(q):
    """fp32 numbers rounded to e4m3 (on the CPU)."""
    return torch.from_numpy(np.ascontiguousarray(q)).to(F8)


def same(got, want):
    got, want = got.cpu().float().numpy(), want.float().numpy()
    return np.array_equal(got, want, equal_nan=True) and np.array_equal(np.signbit(got), np.signbit(want)) or np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 128), (3, 129), (17, 64), (16, 520), (130, 1000), (257, 17), (5, 4096)])
def test_quantised_numbers_are_the_definitions(rows, k, dtype):
    g = torch.Generator().manual_seed(rows + k)
    x = (torch.randn(rows, k, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))).to(dtype)
    for f, block in ((seq.quantize_rows, 1), (seq.quantize_weight, 128)):
        q, s = f(x.cuda())
        want, scales = ref.quantize(x.float().numpy(), block)
        assert q.dtype == F8 and q.shape == x.shape and q.stride(0) % 16 == 0
        assert np.array_equal(s.cpu().numpy(), scales), f.__name__
        assert same(q, e4m3(want)), f.__name__


def test_scales_at_the_ends_of_the_range():
    x = torch.zeros(7, 256)
    x[1, 3] = 1e-45
    x[2] = 2.0 ** -126
    x[3, :] = torch.finfo(torch.float32).max
    x[4, 0], x[4, 200] = float("inf"), 3.0
    x[5, 7] = float("nan")
    x[6] = torch.linspace(-500, 500, 256)
    q, s = seq.quantize_rows(x.cuda())
    want, scales = ref.quantize(x.numpy(), 1)
    assert np.array_equal(s.cpu().numpy(), scales, equal_nan=True)
    assert same(q, e4m3(want))
    got = q.float().cpu()
    assert torch.isnan(got[4, 0]) and not got[4, 1:128].any() and got[4, 200] == 448 and torch.isnan(got[5, :128]).all() and not got[5, 128:].any()


def test_quantiser_takes_strided_rows_and_writes_nothing_beside_its_own():
    wide = torch.randn(20, 333, device="cuda").half()
    for off in (0, 8, 3):
        x = wide[:, off:off + 200]
        room = torch.full((20, 288), 1.0, device="cuda").to(F8)
        scales = torch.full((20, 5), -1.0, device="cuda")
        q, s = seq.quantize_rows(x, out=room[:, :200], scales=scales[:, 1:3])
        want, ws = ref.quantize(x.cpu().float().numpy(), 1)
        assert same(q, e4m3(want)) and np.array_equal(s.cpu().numpy(), ws)
        assert (room[:, 208:].float() == 1).all() and not room[:, 200:208].float().any() and (scales[:, [0, 3, 4]] == -1).all()


def operands(m, n, k, seed=0):
    g = torch.Generator().manual_seed(seed)
    a = torch.randn(m, k, generator=g) * torch.exp(torch.randn(m, 1, generator=g))
    return *seq.quantize_rows(a.cuda()), *seq.quantize_weight(torch.randn(n, k, generator=g).cuda()), torch.randn(n, generator=g).cuda()


def check(a, sa, b, sb, bias, y, what):
    want, mag = ref.block_matmul(f64(a.float()), f64(sa), f64(b.float()), f64(sb), np.zeros(b.shape[0]) if bias is None else f64(bias))
    k = a.shape[1]
    # 16-bit results: the 8-bit operation adds with 14 bits or more, and the result is rounded; 32-bit results: 128 products, then the blocks, in fp32
    half = HALF[y.dtype]
    tol = (2.0 ** -14 * mag if y.dtype != torch.float32 else (128 + k // 128 + 8) * 2.0 ** -24 * mag) + half * np.abs(want) * 1.01 + 2.0 ** -24
    got = f64(y)
    off = np.abs(got - want) - tol
    assert np.isfinite(got).all() and (off <= 0).all(), f"{what}: {off.max():.3g} beyond the bound at {np.unravel_index(off.argmax(), off.shape)}"


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 16, 128), (1, 1000, 512), (2, 130, 96), (16, 64, 256), (17, 33, 129), (33, 128, 384), (64, 512, 1000), (65, 96, 640),
                                   (100, 257, 2048), (128, 128, 128), (129, 300, 520), (255, 256, 1024), (300, 500, 333), (513, 129, 64), (1000, 1000, 200)])
def test_product_against_the_definition(m, n, k, dtype):
    a, sa, b, sb, bias = operands(m, n, k)
    check(a, sa, b, sb, bias, seq.block_matmul(a, sa, b, sb, bias=bias, dtype=dtype), "with bias")
    check(a, sa, b, sb, None, seq.block_matmul(a, sa, b, sb, dtype=dtype), "without")


@pytest.mark.parametrize("m", [1, 40, 200])
def test_what_lies_behind_a_row_does_not_matter(m):
    k, n = 200, 70
    a, sa, b, sb, bias = operands(m, n, k)
    wa, wb = (torch.full((t.shape[0], 256), float("nan"), device="cuda").to(F8) for t in (a, b))
    wa[:, :k], wb[:, :k] = a, b
    got = seq.block_matmul(wa[:, :k], sa, wb[:, :k], sb, bias=bias)
    assert torch.equal(got, seq.block_matmul(a, sa, b, sb, bias=bias))


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("m", [3, 150])
def test_strided_results_and_scales(m, dtype):
    a, sa, b, sb, bias = operands(m, 90, 300)
    want = seq.block_matmul(a, sa, b, sb, bias=bias, dtype=dtype)
    for off, width in ((0, 96), (3, 101), (4, 128)):
        out = torch.full((m, width), 7.0, dtype=dtype, device="cuda")
        got = seq.block_matmul(a, sa.contiguous(), b, sb.t().contiguous().t(), bias=bias, out=out[:, off:off + 90])
        assert torch.equal(got, want)
        out[:, off:off + 90] = 7
        assert (out == 7).all()


@pytest.mark.parametrize("m", [2, 200])
def test_no_columns_to_add_leave_the_bias(m):
    f8 = lambda r: torch.empty(r, 0, dtype=F8, device="cuda")  # noqa: E731
    bias = torch.randn(40, device="cuda")
    y = seq.block_matmul(f8(m), torch.empty(m, 0, device="cuda"), f8(40), torch.empty(1, 0, device="cuda"), bias=bias, dtype=torch.float32)
    assert torch.equal(y, bias.expand(m, 40))


@pytest.mark.parametrize("m", [4, 140])
def test_not_a_number_stays_in_its_row_and_column(m):
    a, sa, b, sb, bias = operands(m, 150, 260)
    clean = seq.block_matmul(a, sa, b, sb, bias=bias)
    a.view(torch.uint8)[1, 5] = 0x7f
    y = seq.block_matmul(a, sa, b, sb, bias=bias)
    assert torch.isnan(y[1]).all()
    y[1] = clean[1]
    assert torch.equal(y, clean)
    sb[1, 0] = float("inf")
    y = seq.block_matmul(a, sa, b, sb, bias=bias)
    rows = [i for i in range(m) if i != 1]
    assert not torch.isfinite(y[:, 128:]).any() and torch.equal(y[rows][:, :128], clean[rows][:, :128])


@pytest.mark.parametrize("m", [5, 300])
def test_offsets_beyond_32_bits(m):
    a, sa, b, sb, bias = operands(m, 20, 64)
    big = torch.empty((1 << 32) + (1 << 20), dtype=torch.uint8, device="cuda").view(F8)
    far = big.as_strided((m, 64), ((1 << 32) // (m - 1) // 16 * 16, 1))
    far.copy_(a)
    assert torch.equal(seq.block_matmul(far, sa, b, sb, bias=bias), seq.block_matmul(a, sa, b, sb, bias=bias))
    x = big.view(torch.uint8).view(torch.float16).as_strided((3, 64), (1 << 30, 1))
    x.copy_(torch.randn(3, 64))
    q, s = seq.quantize_rows(x)
    q2, s2 = seq.quantize_rows(x.contiguous())
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s, s2)


def test_refusals():
    a, sa, b, sb, bias = operands(20, 30, 40)
    f = seq.block_matmul
    for call in (lambda: f(a.float(), sa, b, sb), lambda: f(a, sa[:5], b, sb), lambda: f(a, sa, b[:, :16], sb), lambda: f(a, sa, b, sb, bias=bias[:3]),
                 lambda: f(a, sa, b, sb, dtype=torch.float64), lambda: f(a, sa, b, sb, bias=bias.half()), lambda: f(a.contiguous(), sa, b, sb),
                 lambda: f(a, sa, b, sb, out=torch.empty(20, 31, device="cuda")), lambda: f(a, sa.cpu(), b, sb), lambda: f(a.t(), sa, b, sb),
                 lambda: seq.quantize_rows(bias), lambda: seq.quantize_rows(torch.zeros(4, 8, device="cuda").double()),
                 lambda: seq.quantize_rows(torch.zeros(8, 4, device="cuda").t()), lambda: seq.quantize_rows(torch.zeros(4, 40, device="cuda"), out=torch.empty(4, 40, device="cuda").to(F8)),
                 lambda: seq.quantize_weight(torch.zeros(4, 40, device="cuda", requires_grad=True))):
        with pytest.raises(XlError):
            call()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("m,n,k", [(4096, 2048, 128), (2100, 4000, 130), (3000, 3000, 1040), (5000, 1800, 384), (1030, 9000, 256), (16000, 600, 520)])
def test_large_products_against_a_smaller_part_of_them(m, n, k, dtype):
    """Every row and column of the large tiles' kernel, rows and columns in samples against the definition."""
    a, sa, b, sb, bias = operands(m, n, k)
    y = seq.block_matmul(a, sa, b, sb, bias=bias, dtype=dtype)
    rows = torch.cat([torch.arange(0, m, 97), torch.arange(m - 40, m)]).cuda()
    check(a.view(torch.uint8)[rows].view(F8), sa[rows], b, sb, bias, y[rows], "rows")
    cols = (n + 127) // 128
    for j in (0, cols // 2, cols - 1):          # whole columns of 128
        at = slice(128 * j, min(n, 128 * (j + 1)))
        check(a, sa, b[at], sb[j:j + 1], bias[at], y[:, at], f"columns of block {j}")


def test_large_product_with_numbers_behind_the_rows_and_a_wider_result():
    m, n, k = 2300, 3900, 200
    a, sa, b, sb, bias = operands(m, n, k)
    wa, wb = (torch.full((t.shape[0], 256), float("nan"), device="cuda").to(F8) for t in (a, b))
    wa[:, :k], wb[:, :k] = a, b
    want = seq.block_matmul(a, sa, b, sb, bias=bias)
    assert torch.equal(seq.block_matmul(wa[:, :k], sa, wb[:, :k], sb, bias=bias), want)
    for off in (0, 8, 3):
        out = torch.full((m, n + 20), 7.0, dtype=torch.bfloat16, device="cuda")
        assert torch.equal(seq.block_matmul(a, sa.contiguous(), b, sb, bias=bias, out=out[:, off:off + n]), want)
        out[:, off:off + n] = 7
        assert (out == 7).all()
