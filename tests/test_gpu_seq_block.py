"""The sequence operators together: a scan block over prompts and over single tokens, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import seq
from paper_2007_06000_amd.binding import XlError
from paper_2007_06000_amd.scan_block import ScanBlock, TokenStep, random_weights
from test_gpu_seq_conv import f64

pytestmark = pytest.mark.gpu

# A rounding of relative size e before a quantiser lands on another 8-bit number for about 2 e / 2^-3 of the numbers, and each of those is off by
# 2^-3 of itself: an error of 2^-3 sqrt(16 e) of the norm.  fp32 results with sums of a few hundred terms have e = 1e-5: 1.6e-3 for a
# quantiser; bf16 ones e = 2^-9: 2.2e-2.  Four quantisers and what the layers behind them make of it: twelve times the one and five times the other.
TOLERANCE = {torch.float32: 2e-2, torch.bfloat16: 1e-1}


def product(x, matrix):
    """The definition's quantisation of x, times the block's own 8-bit weights."""
    q, s = ref.quantize(x.astype(np.float32), 1)
    q = f64(torch.from_numpy(q).to(torch.float8_e4m3fn))
    w, ws = (f64(t) for t in matrix)
    return ref.block_matmul(q, s.astype(np.float64), w, ws, np.zeros(len(w)))[0]


def definition(block, x, lengths):
    """y, the convolution's state and the scan's."""
    v = {name: f64(t) for name, t in block.vectors.items()}
    b, n, _ = x.shape

    def project(name, t):
        return product(t.reshape(b * n, -1), block.matrices[name]).reshape(b, n, -1)

    hz = project("in_proj", x)
    h, z = hz[..., :block.inner], hz[..., block.inner:]
    h, _, conv = ref.causal_conv(h, v["conv"], v["conv_bias"], None, lengths, True)
    rBC = project("x_proj", h)
    r, B, C = np.split(rBC, [block.rank, block.rank + block.states], 2)
    y, _, scan, _ = ref.selective_scan(h, project("dt_proj", r), v["A"], B, C, v["D"], z, v["dt_bias"], None, lengths, True)
    return project("out_proj", y), conv, scan


def apart(got, want):
    got, want = f64(got) if torch.is_tensor(got) else got, f64(want) if torch.is_tensor(want) else want
    assert got.shape == want.shape and np.isfinite(got).all()
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("dtype", list(TOLERANCE), ids=str)
@pytest.mark.parametrize("width,inner,states,lengths", [(64, 128, 16, [9, 9]), (40, 72, 7, [23, 0, 1]), (136, 272, 16, [70])])
def test_a_prompt_is_the_definitions(width, inner, states, lengths, dtype):
    block = ScanBlock(random_weights(width, inner, states), dtype=dtype)
    g = torch.Generator().manual_seed(width)
    x = torch.randn(len(lengths), max(lengths), width, generator=g).to(dtype)
    y, (conv, scan) = block(x.cuda(), lengths=torch.tensor(lengths, dtype=torch.int32).cuda())
    want = definition(block, f64(x), lengths)
    assert apart(conv, want[1]) < TOLERANCE[dtype] and apart(scan, want[2]) < TOLERANCE[dtype]
    live = np.arange(max(lengths))[None] < np.array(lengths)[:, None]
    assert apart(f64(y)[live], want[0][live]) < TOLERANCE[dtype]


@pytest.mark.parametrize("dtype", list(TOLERANCE), ids=str)
def test_parts_and_single_tokens_go_on_where_the_prompt_ended(dtype):
    block = ScanBlock(random_weights(64, 128), dtype=dtype)
    x = torch.randn(3, 30, 64, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    whole, last = block(x)
    parts, state = [], None
    for t in (slice(0, 17), slice(17, 18), slice(18, 26), *(slice(i, i + 1) for i in range(26, 30))):
        y, state = block(x[:, t], state)
        parts.append(y)
    assert apart(torch.cat(parts, 1), whole) < TOLERANCE[dtype]
    assert apart(state[0], last[0]) < TOLERANCE[dtype] and apart(state[1], last[1]) < TOLERANCE[dtype]


def test_no_tokens_leave_the_states_as_they_are():
    block = ScanBlock(random_weights(64, 128))
    _, state = block(torch.randn(2, 5, 64, generator=torch.Generator().manual_seed(5)).bfloat16().cuda())
    y, after = block(torch.zeros(2, 0, 64, dtype=torch.bfloat16, device="cuda"), state)
    assert y.shape == (2, 0, 64) and torch.equal(after[0], state[0]) and torch.equal(after[1], state[1])


def test_slots_of_a_cache_belong_to_their_sequences():
    block = ScanBlock(random_weights(64, 128), dtype=torch.float32)
    x = torch.randn(3, 12, 64, generator=torch.Generator().manual_seed(2)).cuda()
    cache = block.cache(6)
    for t in cache:
        t[2:4] = 7.0
    slots = torch.tensor([4, 0, 5], dtype=torch.int32).cuda()
    block(x[:, :11], cache, slots=slots)
    order = torch.tensor([2, 0]).cuda()                     # two of the three go on, in another order
    y, same = block(x[order, 11:], cache, slots=slots[order].contiguous())
    assert same[0] is cache[0] and same[1] is cache[1]
    whole, last = block(x)
    assert apart(y, whole[order, 11:]) < TOLERANCE[torch.float32]
    for got, want in zip(cache, last):
        assert apart(got[slots[order].long()], want[order]) < TOLERANCE[torch.float32]
        assert (got[2:4] == 7).all() and not got[1].any()


def test_a_recorded_step_gives_what_the_eager_one_gives():
    block = ScanBlock(random_weights(64, 128))
    x = torch.randn(4, 12, 64, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    step = TokenStep(block, 4)
    for _ in range(2):
        step.reset()
        state = block.cache(4)
        for t in range(12):
            y, state = block(x[:, t:t + 1], state)          # eager work between the replays
            got = step(x[:, t:t + 1])
            torch.cuda.synchronize()
            assert torch.equal(got, y) and torch.equal(step.cache[0], state[0]) and torch.equal(step.cache[1], state[1]), t


def test_every_operator_can_be_recorded():
    """Also where a call has two kernels: a large product, and a scan in parts with its workspace."""
    g = torch.Generator().manual_seed(6)
    r = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    x, w, filters = r(4200, 1024), r(4096, 1024), r(64, 4).float()
    u, B, C = r(1, 4100, 64), r(1, 4100, 16), r(1, 4100, 16)
    A = -torch.arange(1.0, 17).repeat(64, 1).cuda()
    wq, ws = seq.quantize_weight(w)

    def run():
        h, _ = seq.causal_conv(u, filters)
        y, state = seq.selective_scan(h, u - 4, A, B, C, z=u)
        return seq.block_matmul(*seq.quantize_rows(x), wq, ws), y, state

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(4):
        x.copy_(r(4200, 1024))
        u.copy_(r(1, 4100, 64))
        want = run()                                        # eager work between the replays
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), i


def test_work_follows_the_current_stream():
    block = ScanBlock(random_weights(64, 128))
    x = torch.randn(2, 300, 64, generator=torch.Generator().manual_seed(4)).bfloat16()
    want, state = block(x.cuda())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got, other = block(x.pin_memory().cuda(non_blocking=True))
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(other[0], state[0]) and torch.equal(other[1], state[1])


def test_results_are_ordinary_tensors():
    x = torch.randn(5, 200, generator=torch.Generator().manual_seed(7)).cuda()
    filters = torch.ones(200, 4, device="cuda")
    before = torch.cuda.memory_allocated()
    q, s = seq.quantize_rows(x)
    y, state = seq.causal_conv(x[None], filters)
    assert torch.cuda.memory_allocated() > before
    assert q.device == x.device and q.untyped_storage().nbytes() >= 5 * 208 and s.stride() == (1, 5)
    assert not y.is_inference() and not y.requires_grad and y.is_contiguous()
    w = y.clone().requires_grad_()
    (w * y).sum().backward()                                # a constant in somebody's graph
    assert torch.equal(w.grad, y) and y.resize_(1, 2, 200).shape == (1, 2, 200)
    with torch.inference_mode():
        z = seq.causal_conv(x[None], filters)[0]
        assert z.is_inference()
    other = torch.from_dlpack(x)                            # memory that torch did not allocate, as far as the tensor knows
    q2, s2 = seq.quantize_rows(other)
    assert torch.equal(q2.float(), q.float()) and torch.equal(s2, s)
    del q, s, y, state, w, z, q2, s2, other
    assert torch.cuda.memory_allocated() == before


def test_what_does_not_fit_a_block_is_refused():
    block = ScanBlock(random_weights(64, 128))
    x = torch.zeros(2, 3, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (lambda: block(x[0]), lambda: block(x[..., :40]), lambda: block(x, slots=slots), lambda: block(x, block.cache(3)),
                lambda: block(x, lengths=slots[:1]), lambda: block(x, lengths=slots.long()), lambda: block(x.cpu())):
        with pytest.raises(XlError):
            bad()
    assert seq.module() is seq.module()
