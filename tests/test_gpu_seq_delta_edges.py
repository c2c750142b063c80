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


@pytest.mark.parametrize("with_slots", [False, True])
@pytest.mark.parametrize("length", [60, 140])           # one chunk of each sequence, three and the states between them
def test_more_sequences_than_the_workspace_has_room_for(length, with_slots):
    """4200 heads that take 133 KB a chunk, of 1400 sequences: they go in two pieces, the second from about sequence 1311 on."""
    p = inputs(1400, length, 3, 3, 129, 8, torch.bfloat16)
    rows = torch.arange(1400)
    if with_slots:
        rows = (rows * 3 + 5) % 1400
        p["state"] = torch.randn(1400, 3, 129, 8, device="cuda") * 0.1
    slots = rows.int().cuda() if with_slots else None
    lengths = (torch.arange(1400) * 7 % (length + 1)).int().cuda()
    cache = p["state"].clone()
    got, new = seq.gated_delta_rule(**{**p, "state": cache}, normalize=True, slots=slots, lengths=lengths)
    at = [0, 1, 655, 1300, *range(1308, 1316), 1399]
    some = {**{f: t[at].contiguous() for f, t in p.items() if f != "state"}, "state": p["state"][rows[at].cuda()]}
    n = [int(lengths[b]) for b in at]
    compare(got[at], new[rows[at].cuda()], reference(some, n), "some", spread(some, n, True))
    # the others as in calls of their own, which are small enough for one piece
    for first in range(0, 1400, 200):
        part = slice(first, first + 200)
        y, s = seq.gated_delta_rule(**{**{f: t[part] for f, t in p.items() if f != "state"}, "state": p["state"][rows[part].cuda()]}, normalize=True, lengths=lengths[part])
        assert torch.equal(y, got[part]) and torch.equal(s, new[rows[part].cuda()]), first


def test_a_sequence_of_more_heads_than_the_workspace_has_room_for():
    """A chunk of 4200 heads with keys of their own does not fit: token by token."""
    p = inputs(2, 70, 4200, 4200, 129, 4, torch.bfloat16)
    got, new = seq.gated_delta_rule(**p, normalize=True)
    some = {f: (t[:, ::1400] if f == "state" else t[:, :, ::1400]).contiguous() for f, t in p.items()}
    compare(got[:, :, ::1400], new[:, ::1400], reference(some), "some")


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("step", [1, 4])                # numbers one by one, four at a time
@pytest.mark.parametrize("length", [5, 64, 100, 130])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")], ids=str)
def test_values_that_overlap_are_those_of_tokens_that_exist(bad, length, step, dtype):
    """Windows of one run of memory: behind the last token's row there are numbers of that row, not of a token."""
    p = inputs(1, length, 1, 2, 64, 36, dtype)
    room = torch.randn((length - 1) * step + 72, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    p["v"] = room.as_strided((1, length, 2, 36), (room.numel(), step, 36, 1))
    y0, s0 = seq.gated_delta_rule(**p, normalize=True)
    compare(y0, s0, reference(p), "windows", spread(p, [length], True))
    room[-1] = bad                                      # the last number of the last token and head
    y, s = seq.gated_delta_rule(**p, normalize=True)
    assert not torch.isfinite(y[0, -1, 1, 35]) and not torch.isfinite(s[0, 1, :, 35]).any()
    y[0, -1, 1, 35], s[0, 1, :, 35] = y0[0, -1, 1, 35], s0[0, 1, :, 35]
    assert torch.equal(y, y0) and torch.equal(s, s0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("length,t", [(5, 4), (5, 1), (64, 63), (100, 99), (100, 30), (130, 64), (130, 63)])
def test_a_key_whose_square_leaves_fp32(length, t, dtype):
    """A key of 3e19 writes states of that size; nothing that the formula asks for is larger."""
    p = inputs(1, length, 1, 2, 64, 24, dtype, normalized=True)
    p["k"][..., 7] = 0                                  # no other key has this number
    p["q"][..., 7] = 2.0 ** -64
    p["state"][:, :, 7] = 0
    p["k"][0, t] = 0
    y0, s0 = seq.gated_delta_rule(**p, scale=1.0)       # without the token's key: nothing is written there
    p["k"][0, t, 0, 7] = 3e19
    y, s = seq.gated_delta_rule(**p, scale=1.0)
    size = f64(p["k"])[0, t, 0, 7]
    after = np.cumsum(f64(p["g"])[0, t:], 0) - f64(p["g"])[0, t]          # [tokens, heads]
    row = size * f64(p["beta"])[0, t][:, None] * f64(p["v"])[0, t] * np.exp(after)[..., None]      # [tokens, heads, dv]
    # a factor e^G is off by 2^-24 of G's size and some units, a product by 2^-24, and states before it are what they were
    off = (32 + np.abs(after).max()) * 2.0 ** -24
    assert (np.abs(f64(s)[0, :, 7] - row[-1]) <= off * np.abs(row[-1])).all()
    others = torch.arange(64, device="cuda") != 7
    assert torch.allclose(s[:, :, others], s0[:, :, others], rtol=1e-5, atol=1e-6)
    want = f64(y0)[0, t:] + 2.0 ** -64 * row
    # each of the two results is rounded to its type, and their fp32 sums of 64 products
    assert (np.abs(f64(y)[0, t:] - want) <= 2 * HALF[dtype] * (np.abs(f64(y0)[0, t:]) + np.abs(want)) + (off + 256 * 2.0 ** -24) * (1 + np.abs(row) * 2.0 ** -64)).all()
    assert torch.equal(y[:, :t], y0[:, :t])


def test_pieces_recorded_and_replayed():
    """Several launches that share a workspace, three chunks and two pieces: the same from a graph, again and again, with calls of its own kind in between."""
    p = inputs(1400, 140, 3, 3, 129, 8, torch.bfloat16)
    static = {f: t.clone() for f, t in p.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        seq.gated_delta_rule(**static, normalize=True)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        results = seq.gated_delta_rule(**static, normalize=True)
    for i in range(3):
        static["v"].copy_(p["v"] * (1 + i))
        graph.replay()
        want = seq.gated_delta_rule(**{**p, "v": p["v"] * (1 + i)}, normalize=True)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want)), i
