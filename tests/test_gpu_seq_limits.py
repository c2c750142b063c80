"""Calls that need more threads than one launch can have: sizes that still fit a device's memory."""
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import seq
from test_gpu_seq_conv import f64, near

pytestmark = pytest.mark.gpu
GB = 1 << 30


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 * GB:
        pytest.skip("not enough memory is free")
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("with_slots", [False, True])
def test_convolution_of_more_numbers_than_a_launch_has_threads(with_slots):
    batch, channels, step = 1 << 20, 4099, 1 << 16
    base = (torch.arange(batch + channels, device="cuda") % 61).float()
    x = base.as_strided((batch, 1, channels), (1, 1, 1))
    weight, bias = torch.tensor([[0.5, 2.0]], device="cuda").repeat(channels, 1), torch.arange(channels, device="cuda", dtype=torch.float32)
    numbers = torch.arange(batch, device="cuda", dtype=torch.float32)
    state = numbers[:, None, None].expand(batch, 1, channels).contiguous()      # every row its own number
    lengths = (torch.arange(batch, device="cuda") % 3 != 0).int()
    rows, slots, here = torch.arange(batch, device="cuda"), None, torch.ones(batch, dtype=torch.bool, device="cuda")
    if with_slots:
        rows = (rows * 5 + 3) % batch           # every row once, but for sequences that are absent
        slots = rows.int()
        slots[7::1000] = -1
        here = slots >= 0
    y, new = seq.causal_conv(x, weight, bias, silu=False, state=state, new_state=state, lengths=lengths, slots=slots)
    assert new is state
    for b in range(0, batch, step):             # small numbers and halves: exact in fp32
        at = slice(b, b + step)
        inputs, live = x[at, 0], (here[at] & (lengths[at] > 0))[:, None]
        row = numbers[rows[at]][:, None]
        assert torch.equal(y[at, 0], torch.where(live, 0.5 * row + 2 * inputs + bias, torch.zeros_like(bias))), b
        assert torch.equal(state[rows[at], 0], torch.where(live, inputs, row.expand_as(inputs))), b


@pytest.mark.parametrize("length,states,batch,channels,dtype", [(1, 65, 1 << 14, 8200, torch.float32), (25, 33, 1 << 14, 8200, torch.float16)])
def test_scan_of_more_channels_than_a_launch_has_threads(length, states, batch, channels, dtype):
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    # two sequences that take turns, of every tenth channel's numbers: 64 and 10 different ones
    two = {"u": r(2, length, 10).to(dtype), "delta": (r(2, length, 10) - 2).to(dtype), "B": r(2, length, states).to(dtype), "C": r(2, length, states).to(dtype)}
    A, D = -torch.rand(10, states, generator=g) - 0.1, r(10)
    wide = lambda t: t.cuda().repeat(1, 1, channels // 10).repeat(batch // 2, 1, 1) if t.shape[2] == 10 else t.cuda().repeat(batch // 2, 1, 1)  # noqa: E731
    p = {k: wide(v) for k, v in two.items()}
    y, new = seq.selective_scan(**p, A=A.cuda().repeat(channels // 10, 1), D=D.cuda().repeat(channels // 10))
    want, bound, last, last_bound = ref.selective_scan(*[f64(two[k]) for k in ("u", "delta")], f64(A), f64(two["B"]), f64(two["C"]), f64(D), None, torch.zeros(10).numpy(), None, [length] * 2, True)
    y, new = y.view(batch // 2, 2, length, channels // 10, 10), new.view(batch // 2, 2, channels // 10, 10, states)
    near(y[0, :, :, 0], want, bound, "y")
    near(new[0, :, 0], last, last_bound, "state")
    for b in range(0, batch // 2, 256):         # and all the others the same
        assert torch.equal(y[b:b + 256], y[:1, :, :, :1].expand(min(256, batch // 2 - b), -1, -1, channels // 10, -1)), b
        assert torch.equal(new[b:b + 256], new[:1, :, :1].expand(min(256, batch // 2 - b), -1, channels // 10, -1, -1)), b


def bytes_of(rows, k, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randint(0, 256, (rows, k), generator=g, device="cuda", dtype=torch.uint8) & 0xbf).view(torch.float8_e4m3fn)      # magnitudes below 2


def check(a, sa, b, sb, bias, y):
    """y [m, n] of 32 bits in parts against sums in 64 bits: 16 products, a scale, a bias, in fp32."""
    step = max(1, (1 << 27) // y.shape[1])
    for i in range(0, y.shape[0], step):
        at = slice(i, i + step)
        for j in range(0, y.shape[1], 1 << 24):
            cols = slice(j, j + (1 << 24))
            scales = sb.repeat_interleave(128, 0)[cols][:y.shape[1] - j]
            left, right = a[at].double() * sa[at].double(), b[cols].double() * scales.double()
            want, mag = left @ right.t().contiguous(), left.abs() @ right.abs().t().contiguous()
            if bias is not None:
                want, mag = want + bias[cols].double(), mag + bias[cols].abs().double()
            off = (y[at, cols].double() - want).abs() - 24 * 2.0 ** -24 * mag
            assert (off <= 0).all(), (i, j, off.max())
            del want, mag, off


def test_product_of_more_columns_than_a_launch_has_threads():
    n, k = (1 << 27) + 137, 16
    a, b = bytes_of(2, k, 1), bytes_of(n, k, 2)
    sa, sb = torch.rand(2, 1, device="cuda") + 0.5, torch.rand(-(-n // 128), 1, device="cuda") + 0.5
    bias = torch.randn(n, device="cuda")
    check(a, sa, b, sb, bias, seq.block_matmul(a, sa, b, sb, bias=bias, dtype=torch.float32))


def test_product_of_more_rows_than_a_launch_has_threads():
    m, n, k = (1 << 27) + 45, 40, 16
    a, b = bytes_of(m, k, 3), bytes_of(n, k, 4)
    sa = torch.empty_strided((m, 1), (1, m), device="cuda")         # a column for each block, too long for the tiles' 31 bits
    sa.uniform_(0.5, 1.5)
    sb = torch.rand(1, 1, device="cuda") + 0.5
    check(a, sa, b, sb, None, seq.block_matmul(a, sa, b, sb, dtype=torch.float32))
