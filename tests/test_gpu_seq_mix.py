"""Norm, projection with adapters, convolution and delta rule together, as a mixer layer runs them; and as calls among others: graphs, streams, versions, places far apart."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2007_06000_amd import seq
from test_gpu_seq_adapters import check as check_adapters
from test_gpu_seq_adapters import inputs as adapter_inputs
from test_gpu_seq_conv import f64
from test_gpu_seq_delta import compare, reference
from test_gpu_seq_delta import inputs as delta_inputs
from test_gpu_seq_norm import inputs as norm_inputs
from test_gpu_seq_norm import run as run_norm

pytestmark = pytest.mark.gpu


class Layer:
    """h, z = in_proj(norm(x + residual)) + adapters; q, k, v = conv(h); residual + out_proj(delta rule(q, k, v))"""

    def __init__(self, width, key_heads, heads, dk, dv, dtype, adapters=3, rank=8, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
        self.sizes, self.dtype, self.inner = (key_heads, heads, dk, dv), dtype, 2 * key_heads * dk + heads * dv
        n = self.inner + 2 * heads          # behind the rest what makes decays and steps
        self.norm = 1 + 0.1 * r(width)
        self.in_proj, self.out_proj = seq.quantize_weight(r(n, width) * width ** -0.5), seq.quantize_weight(r(width, heads * dv) * (heads * dv) ** -0.5)
        self.down, self.up = (r(adapters, rank, width) * width ** -0.5).to(dtype), (0.2 * r(adapters, n, rank)).to(dtype)
        self.filters, self.bias = r(self.inner, 4) * 0.5, 0.1 * r(self.inner)

    def cache(self, rows):
        key_heads, heads, dk, dv = self.sizes
        return torch.zeros(rows, 3, self.inner, dtype=self.dtype, device="cuda"), torch.zeros(rows, heads, dk, dv, device="cuda")

    def __call__(self, x, residual, index, cache, slots, lengths=None):
        batch, length, width = x.shape
        key_heads, heads, dk, dv = self.sizes
        q8, s8, residual = seq.rms_norm_quantized(x.view(-1, width), self.norm, residual=residual)
        normed = (q8.float() * s8.repeat_interleave(128, 1)[:, :width]).to(self.dtype).view(batch, length, width)
        h = seq.block_matmul(q8, s8, *self.in_proj, dtype=self.dtype).view(batch, length, -1)
        h = seq.add_adapters(h, normed, self.down, self.up, index, lengths=lengths, out=h)
        gates = h[..., self.inner:].float()
        mixed, _ = seq.causal_conv(h[..., :self.inner], self.filters, self.bias, state=cache[0], slots=slots, lengths=lengths)
        q, k, v = mixed.split((key_heads * dk, key_heads * dk, heads * dv), 2)
        y, _ = seq.gated_delta_rule(q.view(batch, length, key_heads, dk), k.view(batch, length, key_heads, dk), v.view(batch, length, heads, dv),
                                    -torch.nn.functional.softplus(gates[..., :heads] - 3), torch.sigmoid(gates[..., heads:]), normalize=True, state=cache[1], slots=slots, lengths=lengths)
        out = seq.block_matmul(*seq.quantize_rows(y.view(batch * length, heads * dv)), *self.out_proj, dtype=self.dtype).view(batch, length, width)
        return out, residual.view(batch, length, width)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_a_layer_at_once_and_in_pieces(dtype):
    """The same tokens as a prompt, in pieces and token by token; what differs is how sums are ordered, and now and then the rounding of an 8-bit operand."""
    batch, length, width = 3, 90, 160
    layer = Layer(width, 2, 4, 32, 24, dtype)
    g = torch.Generator().manual_seed(5)
    x, residual = (torch.randn(batch, length, width, generator=g).to(dtype).cuda() for _ in range(2))
    index, slots = torch.tensor([2, -1, 0], dtype=torch.int32, device="cuda"), torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    cache = layer.cache(5)
    want, kept = layer(x, residual.view(-1, width), index, cache, slots)
    assert torch.isfinite(want.float()).all() and (want.float().norm(dim=-1) > 0).all()
    pieces = layer.cache(5)
    at, got = 0, []
    for n in (64, 20, 1, 1, 4):
        y, r = layer(x[:, at:at + n].contiguous(), residual[:, at:at + n].reshape(-1, width), index, pieces, slots)
        assert torch.equal(r, kept[:, at:at + n])
        got.append(y)
        at += n
    got = torch.cat(got, 1)
    # roundings of 16 bits make some numbers land on the other side of an 8-bit step (2^-4) behind them
    off = (got.float() - want.float()).norm() / want.float().norm()
    assert off < (2e-2 if dtype == torch.float32 else 6e-2), off
    assert (pieces[1] - cache[1]).norm() < (2e-2 if dtype == torch.float32 else 6e-2) * cache[1].norm()
    for row in (1, 3):
        assert not pieces[0][row].any() and not pieces[1][row].any()


def test_a_layer_of_sequences_of_their_own_lengths():
    width, layer = 96, Layer(96, 1, 2, 16, 16, torch.float32)
    g = torch.Generator().manual_seed(6)
    x, residual = torch.randn(3, 70, width, generator=g).cuda(), torch.randn(3, 70, width, generator=g).cuda()
    index, slots, lengths = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 1, 2], [0, 1, 2], [70, 0, 33]))
    cache = layer.cache(3)
    y, _ = layer(x, residual.view(-1, width), index, cache, slots, lengths)
    for b, n in enumerate(lengths.tolist()):
        one = layer.cache(1)
        if n:
            want, _ = layer(x[b:b + 1, :n].contiguous(), residual[b, :n], index[b:b + 1], one, torch.zeros(1, dtype=torch.int32, device="cuda"))
            assert (y[b, :n] - want[0]).norm() < 2e-2 * want.norm()
        assert torch.allclose(cache[1][b], one[1][0], atol=2e-2) and torch.allclose(cache[0][b], one[0][0], atol=1e-4)


def calls():
    """(name, tensors that are read, call(tensors) -> results) of the operators, small and large."""
    out = []
    for rows, k in ((3, 100), (40, 5000)):
        x, r, w = norm_inputs(rows, k, torch.bfloat16, torch.bfloat16)
        out.append((f"norm {k}", (x, r), lambda x, r, w=w: seq.rms_norm(x, w, residual=r)))
        out.append((f"quantized norm {k}", (x, r), lambda x, r, w=w: seq.rms_norm_quantized(x, w, residual=r)))
    for size in ((4, 1, 64, 128, 8, 2), (2, 3000, 96, 160, 16, 2)):
        p = adapter_inputs(*size, torch.bfloat16)
        out.append((f"adapters {size}", (p["y"], p["x"]), lambda y, x, p=p: (seq.add_adapters(**{**p, "y": y, "x": x}),)))
    for size in ((2, 1, 1, 2, 64, 64), (2, 200, 1, 2, 64, 48)):
        p = delta_inputs(*size, torch.bfloat16)
        out.append((f"delta {size}", (p["q"], p["v"], p["state"]), lambda q, v, state, p=p: seq.gated_delta_rule(**{**p, "q": q, "v": v, "state": state}, normalize=True)))
    return out


def same(a, b):
    return all(torch.equal(s.float().nan_to_num(7.0), t.float().nan_to_num(7.0)) for s, t in zip(a, b))


def test_recorded_and_replayed():
    """Two graphs of every call, replayed in turn with other inputs and eager calls in between."""
    for name, tensors, call in calls():
        side, graphs = torch.cuda.Stream(), []
        for _ in range(2):
            static = [t.clone() for t in tensors]
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                call(*static)
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                results = call(*static)
            graphs.append((static, graph, results))
        for i in range(3):
            for static, graph, results in graphs:
                for s, t in zip(static, tensors):
                    s.copy_(t * (1 + i))
                graph.replay()
                want = call(*[t * (1 + i) for t in tensors])
                torch.cuda.synchronize()
                assert same(results, want), (name, i)


def test_on_two_streams_at_once():
    for name, tensors, call in calls():
        want = call(*tensors)
        torch.cuda.synchronize()
        streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
        for i in range(6):
            with torch.cuda.stream(streams[i % 2]):
                got.append(call(*tensors))
        torch.cuda.synchronize()
        assert all(same(g, want) for g in got), name


def test_an_error_that_another_call_left_is_not_this_calls():
    hip = ctypes.CDLL(seq.LIB_PATH)
    for name, tensors, call in calls():
        want = call(*tensors)
        torch.cuda.synchronize()
        assert hip.hipSetDevice(1 << 20) != 0
        try:
            got = call(*tensors)
        finally:
            hip.hipGetLastError()
        assert same(got, want), name


def test_tensors_that_a_call_writes_get_a_new_version_and_others_do_not():
    x, r, w = norm_inputs(4, 64, torch.float32, torch.float32)
    a, d = adapter_inputs(2, 3, 16, 24, 4, 2, torch.float32), delta_inputs(2, 3, 1, 2, 16, 24, torch.float32)
    out, y, o, cache = torch.empty_like(x), a["y"].clone(), torch.empty_like(d["v"]), d["state"].clone()
    q, s = seq.quantize_rows(x)
    slots = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    written = (out, r, q, s, y, o, cache)
    before, inputs = [t._version for t in written], [x, w, *a.values(), *d.values(), slots]
    versions = [t._version for t in inputs]
    seq.rms_norm(x, w, residual=r, new_residual=r, out=out)
    seq.rms_norm_quantized(x, w, out=q, scales=s)
    seq.add_adapters(**{**a, "y": y}, out=y)
    seq.gated_delta_rule(**{**d, "state": cache}, slots=slots, out=o)
    assert all(t._version > v for t, v in zip(written, before)) and [t._version for t in inputs] == versions


def test_tangents_and_negated_views_are_refused():
    from torch.autograd import forward_ad
    x, r, w = norm_inputs(4, 64, torch.float32, torch.float32)
    a, d = adapter_inputs(2, 3, 16, 24, 4, 2, torch.float32), delta_inputs(2, 3, 1, 2, 16, 24, torch.float32)
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: seq.rms_norm(dual(x), w), lambda: seq.rms_norm_quantized(x, w, residual=dual(r)), lambda: seq.add_adapters(**{**a, "up": dual(a["up"])}),
                     lambda: seq.gated_delta_rule(**{**d, "g": dual(d["g"])}), lambda: seq.gated_delta_rule(**{**d, "k": dual(d["k"])})):
            with torch.no_grad(), pytest.raises(seq.XlError, match="tangent"):
                call()
    minus = torch.view_as_complex(torch.randn(4, 1, 2, device="cuda")).conj().imag
    with pytest.raises(seq.XlError, match="negated"):
        seq.rms_norm(minus, w[:1])


def test_rows_further_apart_than_32_bits_count():
    far = (1 << 31) + 64
    room = torch.zeros(far + 40000, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(0)
    x = room.as_strided((2, 300), (far, 1))
    x.copy_(torch.randn(2, 300, generator=g).cuda())
    w = torch.ones(300, device="cuda")
    run_norm(x, None, w)
    out = room.as_strided((2, 300), (far, 1), 400)
    y, _ = seq.rms_norm(x.contiguous(), w, out=out)
    assert torch.equal(out, seq.rms_norm(x.contiguous(), w)[0])
    for length in (3, 200):             # sequences far apart
        p = adapter_inputs(2, length, 40, 24, 8, 2, torch.bfloat16)
        wide = room.as_strided((2, length, 64), (far, 64, 1), 1000)
        wide[..., :40].copy_(p["x"])
        wide[..., 40:].copy_(p["y"])
        check_adapters(p, seq.add_adapters(**{**p, "x": wide[..., :40], "y": wide[..., 40:]}, out=wide[..., 40:]), "far")
        d = delta_inputs(2, length, 1, 1, 64, 24, torch.bfloat16)
        view = room.as_strided((2, length, 152), (far, 152, 1), 1000)
        for t, at in (("q", 0), ("k", 64), ("v", 128)):
            view[..., at:at + d[t].shape[3]].copy_(d[t][:, :, 0])
        got, new = seq.gated_delta_rule(**{**d, "q": view[..., None, :64], "k": view[..., None, 64:128], "v": view[..., None, 128:]}, normalize=True)
        compare(got, new, reference(d), "far")
    d = delta_inputs(1, 20, 1, 1, 64, 16, torch.bfloat16)       # tokens far apart: 20 x 100 M numbers
    step = 100_000_000
    view = room.as_strided((1, 20, 1, 16), (0, step, 16, 1), 0)
    view.copy_(d["v"])
    got, new = seq.gated_delta_rule(**{**d, "v": view}, normalize=True)
    compare(got, new, reference(d), "tokens far apart")


def test_more_chunks_than_are_prepared_at_once():
    """1024 heads: a workspace of half a gigabyte holds some eleven of the seventeen chunks, and the states wait between them."""
    p = delta_inputs(64, 1050, 16, 16, 64, 16, torch.bfloat16)
    lengths = torch.tensor([1050, 0, 63, 700, 705] * 13, dtype=torch.int32, device="cuda")[:64]
    got, new = seq.gated_delta_rule(**p, normalize=True, lengths=lengths)
    for b in (0, 1, 2, 3, 4, 63):
        h = slice(b % 16, b % 16 + 1)
        one = {f: (t[b:b + 1, h] if f == "state" else t[b:b + 1, :, h]).contiguous() for f, t in p.items()}
        compare(got[b:b + 1, :, h], new[b:b + 1, h], reference(one, [int(lengths[b])]), f"sequence {b}")
    again, _ = seq.gated_delta_rule(**p, normalize=True, lengths=lengths)
    assert torch.equal(again, got) and np.isfinite(f64(got[0])).all()


def test_more_work_than_a_launch_has_workgroups():
    """A launch has a million workgroups at most; what is more goes round in them."""
    x, w = torch.randn(5_000_003, 8, device="cuda"), torch.rand(8, device="cuda") + 0.5
    y, _ = seq.rms_norm(x, w)
    want = x.double() / (x.double().square().mean(1, keepdim=True) + 1e-6).sqrt() * w.double()
    assert ((y.double() - want).abs() <= 70 * 2.0 ** -24 * want.abs() + 1e-40).all()        # as the definition's bound
    q, s, _ = seq.rms_norm_quantized(x, w)
    assert ((q.float() * s - y).abs() <= 2.0 ** -4 * 1.001 * y.abs() + 2.0 ** -10 * s).all()
    p = adapter_inputs(1 << 20, 1, 8, 24, 2, 5, torch.float32)
    got = seq.add_adapters(**p)
    at = torch.arange(0, 1 << 20, 10007, device="cuda")
    some = {f: t[at] if f in ("x", "y", "index") else t for f, t in p.items()}
    check_adapters(some, got[at], "many sequences")
    d = delta_inputs(4096, 20, 16, 16, 4, 4, torch.float32)         # 65536 heads: token by token
    y, new = seq.gated_delta_rule(**d, normalize=True)
    some = {f: t[::1365].contiguous() for f, t in d.items()}
    compare(y[::1365].contiguous(), new[::1365].contiguous(), reference(some), "many heads")
