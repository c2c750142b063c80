"""A scan block: the four sequence operators together, as a mixer behind a convolutional stem uses them.

    h, z     = in_proj(x)                        product of 8-bit numbers, [tokens, width] -> [tokens, 2 inner]
    h        = causal_conv(h)                    short convolution over time and SiLU
    r, B, C  = x_proj(h)                         [tokens, inner] -> [tokens, rank + 2 states]
    delta    = dt_proj(r)                        [tokens, rank] -> [tokens, inner]
    y        = out_proj(selective_scan(h, delta, A, B, C, D, z))

Every product quantises its rows on the way in (one scale for 128 numbers); weights are quantised once, when the block is made.  Between the
operators a tensor is never copied: the halves of in_proj and the three parts of x_proj are read where they lie.

`python -m paper_2007_06000_amd.scan_block` reads the feature maps of a fused convolution block as sequences, takes them through a scan block at
once and position by position (launched one by one, and as a recorded graph), and prints the times and how far the results are apart.
"""
from __future__ import annotations

import math
from typing import Dict, Optional, Tuple

import torch
from torch.autograd import forward_ad

from . import seq
from .binding import XL_E_SHAPE, XL_E_UNSUPPORTED, XlError

State = Tuple[torch.Tensor, torch.Tensor]


def random_weights(width: int, inner: int, states: int = 16, rank: Optional[int] = None, taps: int = 4, seed: int = 0) -> Dict[str, torch.Tensor]:
    """fp32 weights on the CPU: steps between 1e-3 and 1e-1, A = -1 .. -states."""
    g = torch.Generator().manual_seed(seed)
    rank = rank or max(1, width // 16)

    def matrix(n, k):
        return torch.randn(n, k, generator=g) / math.sqrt(k)

    steps = torch.exp(torch.empty(inner).uniform_(math.log(1e-3), math.log(1e-1), generator=g))
    return {"in_proj": matrix(2 * inner, width), "conv": torch.randn(inner, taps, generator=g) / math.sqrt(taps), "conv_bias": torch.zeros(inner),
            "x_proj": matrix(rank + 2 * states, inner), "dt_proj": matrix(inner, rank), "dt_bias": torch.log(torch.expm1(steps)),
            "A": -torch.arange(1.0, states + 1).repeat(inner, 1), "D": torch.ones(inner), "out_proj": matrix(width, inner)}


class ScanBlock:
    """Weights as `random_weights` names them; activations in `dtype`.

    The four products have 8-bit operands in every `dtype`, those that make the steps and state vectors too: what a step depends on is
    rounded to four significant bits for each product.  float32 takes the sums and the activations between the operators to 32 bits."""

    def __init__(self, weights: Dict[str, torch.Tensor], device: int = 0, dtype: torch.dtype = torch.bfloat16):
        self.dev, self.dtype = torch.device("cuda", device), dtype
        w = {name: t.to(self.dev, torch.float32).contiguous() for name, t in weights.items()}
        self.inner, self.taps = w["conv"].shape
        self.states, self.rank, self.width = w["A"].shape[1], w["dt_proj"].shape[1], w["in_proj"].shape[1]
        self.matrices = {name: seq.quantize_weight(w.pop(name)) for name in ("in_proj", "x_proj", "dt_proj", "out_proj")}
        self.vectors = w

    def cache(self, rows: int) -> State:
        """States of `rows` sequences that have not begun."""
        return (torch.zeros(rows, self.taps - 1, self.inner, dtype=self.dtype, device=self.dev),
                torch.zeros(rows, self.inner, self.states, dtype=torch.float32, device=self.dev))

    def _product(self, name: str, x: torch.Tensor) -> torch.Tensor:
        """x [batch, length, k], whose tokens lie at even steps, times a matrix."""
        batch, length, k = x.shape
        rows = x.as_strided((batch * length, k), (x.stride(1) if length > 1 else x.stride(0), 1))
        weight, scales = self.matrices[name]
        return seq.block_matmul(*seq.quantize_rows(rows), weight, scales, dtype=self.dtype).view(batch, length, weight.shape[0])

    def __call__(self, x: torch.Tensor, state: Optional[State] = None, *, lengths: Optional[torch.Tensor] = None,
                 slots: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, State]:
        """x [batch, length, width], one token or many, and the states that the last call returned (`state`, None at the start of a sequence).

        `lengths` (int32) gives each sequence's own length; what is computed for the tokens behind it means nothing.  With `slots` (int32)
        `state` is a cache of many sequences' states, updated in place: sequence i has its states in row slots[i]."""
        if x.dim() != 3 or x.shape[2] != self.width:
            raise XlError(XL_E_SHAPE, f"scan block: x has shape {tuple(x.shape)}, not [batch, length, {self.width}]")
        x = x.contiguous()
        conv_state, scan_state = state if state is not None else (None, None)
        v, inner, rank, n = self.vectors, self.inner, self.rank, self.states
        h, z = self._product("in_proj", x).split(inner, 2)
        h, conv_state = seq.causal_conv(h, v["conv"], v["conv_bias"], state=conv_state, lengths=lengths, slots=slots)
        r, B, C = self._product("x_proj", h).split((rank, n, n), 2)
        delta = self._product("dt_proj", r)
        y, scan_state = seq.selective_scan(h, delta, v["A"], B, C, D=v["D"], z=z, delta_bias=v["dt_bias"], state=scan_state, lengths=lengths, slots=slots)
        return self._product("out_proj", y), (conv_state, scan_state)


class TokenStep:
    """One token for each row of a cache, recorded once as a graph: a step is then a copy of its input and one launch for the whole block."""

    def __init__(self, block: ScanBlock, batch: int):
        self.block, self.cache = block, block.cache(batch)
        self.slots = torch.arange(batch, dtype=torch.int32, device=block.dev)
        self.x = torch.zeros(batch, 1, block.width, dtype=block.dtype, device=block.dev)
        side = torch.cuda.Stream(block.dev)
        side.wait_stream(torch.cuda.current_stream(block.dev))
        with torch.cuda.stream(side):
            block(self.x, self.cache, slots=self.slots)
        torch.cuda.current_stream(block.dev).wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph, stream=side):         # by itself it would take a stream of the device that is current
            self.y, _ = block(self.x, self.cache, slots=self.slots)
        self.written = [t for t in (self.y, *self.cache) if not t.is_inference()]
        self.reset()

    def reset(self):
        for t in self.cache:
            t.zero_()

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        """x [batch, 1, width]; the result is overwritten by the next step."""
        if x.shape != self.x.shape:
            raise XlError(XL_E_SHAPE, f"token step: x has shape {tuple(x.shape)}, not {tuple(self.x.shape)}")
        if (x.requires_grad and torch.is_grad_enabled()) or forward_ad.unpack_dual(x).tangent is not None:
            raise XlError(XL_E_UNSUPPORTED, "token step: x asks for a gradient: inference only")
        self.x.copy_(x)
        self.graph.replay()
        torch.autograd.graph.increment_version(self.written)    # for whoever has saved one of them for a backward pass
        return self.y


def _main():
    import xl_workloads as W

    from .session import Session

    wl = W.config(2)                                            # convolution and pooling of 8 x 64 x 56 x 56, fused
    stem = Session(wl, *W.make_tensors(wl))
    maps = stem.run()
    block = ScanBlock(random_weights(maps.shape[1], 2 * maps.shape[1]))
    x = maps.flatten(2).transpose(1, 2).to(block.dtype).contiguous()      # positions as tokens
    x = x / x.float().square().mean().sqrt().to(x.dtype)
    batch, length, width = x.shape

    def timed(f, reps):
        f()
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(reps):
            f()
        b.record()
        b.synchronize()
        return a.elapsed_time(b) / reps * 1e3

    whole, _ = block(x)
    step = TokenStep(block, batch)
    by_token = torch.cat([step(x[:, t:t + 1]).clone() for t in range(length)], 1)
    apart = ((by_token.float() - whole.float()).norm() / whole.float().norm()).item()
    state = block(x)[1]
    print(f"{batch} maps of {length} positions, {width} channels, {block.inner} inside, {block.states} states")
    print(f"all positions at once          {timed(lambda: block(x), 50):9.1f} us")
    print(f"one position, launched singly  {timed(lambda: block(x[:, -1:], state), 200):9.1f} us")
    print(f"one position, as a graph       {timed(lambda: step(x[:, -1:]), 200):9.1f} us")
    print(f"position by position against at once: {apart:.2e} of the result's norm")


if __name__ == "__main__":
    _main()
