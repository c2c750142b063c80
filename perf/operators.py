"""Performance cases of the sequence operators: causal convolution, selective scan, block quantisation, block-scaled product.

They are the layers of a scan block, the mixer that follows a convolutional stem when the positions of its feature map are
read as a sequence: a projection (block-scaled product of 8-bit numbers), a short causal depthwise convolution, the selective
state-space scan, and the projection back.  Every case is one call of one operator on one batch.  A case holds

    kind       conv | scan | quantize | matmul
    dtype      of the activations (matmul: of the result)
    conv       batch, length, channels, taps; state: whether a state of earlier tokens goes in
    scan       batch, length, channels, states; state; ragged: the sequences have lengths of their own, from none to all
    quantize   rows, k (the length of a row)
    matmul     m, n, k; bias

The path is inference only: there is no backward direction and no optimiser.
"""
import torch

own = False

BLOCK = 128                                     # numbers that share a scale
E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -126
DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
MAX_STATE_STEPS = 2 * 12321 * 2048 * 16         # of a drawn scan: the largest listed one's
MAX_ELEMENTS = 2 * 12321 * 2048                 # of a drawn scan's or convolution's input


def listed():
    return [
        # One token of 16 sequences through the convolution: the smallest call, bound by its launch.
        {"name": "conv_token_b16", "kind": "conv", "dtype": "bfloat16", "batch": 16, "length": 1, "channels": 1024, "taps": 4,
         "state": True},
        # Eight 55x55 feature maps read as sequences, the input half of a wider tensor.
        {"name": "conv_55x55_b8", "kind": "conv", "dtype": "bfloat16", "batch": 8, "length": 3025, "channels": 2048, "taps": 4,
         "state": False},
        # One token of 64 sequences through the scan: reads and writes the states, little else.
        {"name": "scan_token_b64", "kind": "scan", "dtype": "bfloat16", "batch": 64, "length": 1, "channels": 2048, "states": 16,
         "state": True, "ragged": False},
        # One 56x56 feature map: a single long sequence, few channels to fill the chip with.
        {"name": "scan_56x56_b1", "kind": "scan", "dtype": "bfloat16", "batch": 1, "length": 3136, "channels": 1024, "states": 16,
         "state": False, "ragged": False},
        # Sequences of their own lengths (none, a part, all of 27x27), odd numbers of channels and states, fp32.
        {"name": "scan_27x27_b5_ragged", "kind": "scan", "dtype": "float32", "batch": 5, "length": 729, "channels": 333, "states": 13,
         "state": True, "ragged": True},
        # Two 111x111 feature maps (the stem's output): the largest scan.
        {"name": "scan_111x111_b2", "kind": "scan", "dtype": "bfloat16", "batch": 2, "length": 12321, "channels": 2048, "states": 16,
         "state": False, "ragged": False},
        # The tokens of a serving step on their way into a projection.
        {"name": "quantize_64", "kind": "quantize", "dtype": "bfloat16", "rows": 64, "k": 1024},
        # All positions of two 111x111 maps: bound by memory.
        {"name": "quantize_24642", "kind": "quantize", "dtype": "bfloat16", "rows": 24642, "k": 4096},
        # A projection of 16 tokens: bound by reading the weights.
        {"name": "matmul_token_b16", "kind": "matmul", "dtype": "bfloat16", "m": 16, "n": 4096, "k": 2048, "bias": False},
        # The narrow projection that makes step sizes and both state vectors of a 56x56 map.
        {"name": "matmul_56x56_n96", "kind": "matmul", "dtype": "bfloat16", "m": 3136, "n": 96, "k": 1024, "bias": False},
        # A classifier over 27x27 positions: nothing divides by a block or a tile; fp32 logits.
        {"name": "matmul_27x27_n1000", "kind": "matmul", "dtype": "float32", "m": 729, "n": 1000, "k": 520, "bias": True},
        # A projection of two 111x111 maps: bound by the matrix cores.
        {"name": "matmul_24642", "kind": "matmul", "dtype": "bfloat16", "m": 24642, "n": 4096, "k": 4096, "bias": False},
    ]


def _size(rng, lo, hi):
    """A size of [lo, hi], spread over its logarithm: a power of two or an odd number."""
    v = lo * (hi / lo) ** rng.random()
    if rng.random() < 0.4:
        p = 1 << max(0, round(v).bit_length() - 1)
        if lo <= p <= hi:
            return p
    return min(hi, max(lo, int(v) | 1))


def _too_long(c):
    x = c["batch"] * c["length"] * c["channels"]
    return x > MAX_ELEMENTS or x * c["states"] > MAX_STATE_STEPS


def draw(rng):
    kind = rng.choice(["conv", "scan", "scan", "quantize", "matmul", "matmul"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if kind == "conv":
        c = {"kind": kind, "dtype": dtype, "batch": _size(rng, 1, 64), "length": rng.choice([1, _size(rng, 1, 12321)]),
             "channels": _size(rng, 8, 4096), "taps": rng.choice([2, 3, 4]), "state": rng.random() < 0.5}
        while c["batch"] > 1 and c["batch"] * c["length"] * c["channels"] > MAX_ELEMENTS:
            c["batch"] //= 2
    elif kind == "scan":
        c = {"kind": kind, "dtype": dtype, "batch": _size(rng, 1, 64), "length": rng.choice([1, _size(rng, 1, 12321), _size(rng, 1, 12321)]),
             "channels": _size(rng, 8, 4096), "states": rng.choice([16, 16, _size(rng, 1, 64)]), "state": rng.random() < 0.5,
             "ragged": rng.random() < 0.3}
        while _too_long(c):
            if c["batch"] > 1:
                c["batch"] //= 2
            else:
                c["channels"] = c["channels"] // 2 | 1
    elif kind == "quantize":
        c = {"kind": kind, "dtype": dtype, "rows": _size(rng, 1, 24642), "k": _size(rng, 8, 4096)}
    else:
        c = {"kind": kind, "dtype": dtype, "m": _size(rng, 1, 24642), "n": _size(rng, 8, 4096), "k": _size(rng, 16, 4096),
             "bias": rng.random() < 0.5}
    return c


def _lengths(c, gen):
    """From none to all of the tokens, evenly spread, in an order of the seed's."""
    b, n = c["batch"], c["length"]
    even = torch.arange(b, dtype=torch.float64) * n / max(1, b - 1) if b > 1 else torch.full((1,), float(n), dtype=torch.float64)
    return even.round().to(torch.int32)[torch.randperm(b, generator=gen)].cuda()


def _quantized(x, rows):
    """x [R, K] as 8-bit numbers and their scales, one for each `rows` x 128 block; the scales lie as the operators give them."""
    r, k = x.shape
    rb, kb = -(-r // rows), -(-k // BLOCK)
    wide = torch.zeros(rb * rows, kb * BLOCK, dtype=torch.float32, device=x.device)
    wide[:r, :k] = x.float()
    blocks = wide.view(rb, rows, kb, BLOCK)
    scale = (blocks.abs().amax((1, 3)) / E4M3_MAX).clamp_min(MIN_SCALE)
    q = (blocks / scale[:, None, :, None]).reshape(wide.shape)[:r, :k].to(torch.float8_e4m3fn)
    return q, scale


def _rows_of_16_bytes(q):
    """The same numbers in rows that begin at multiples of 16 bytes, as the quantiser leaves them."""
    r, k = q.shape
    wide = torch.zeros(r, -(-k // 16) * 16, dtype=torch.uint8, device=q.device).view(torch.float8_e4m3fn)
    wide[:, :k].copy_(q)
    return wide[:, :k]


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    s = {"case": dict(case)}
    if case["kind"] == "conv":
        b, n, c, k = case["batch"], case["length"], case["channels"], case["taps"]
        s["x"] = normal(b, n, 2 * c).to(dt)[:, :, :c]           # the projection makes the gate's half beside it
        s["weight"] = normal(c, k, std=k ** -0.5)
        s["bias"] = normal(c, std=0.1)
        s["state"] = normal(b, k - 1, c).to(dt) if case["state"] else None
    elif case["kind"] == "scan":
        b, n, d, m = case["batch"], case["length"], case["channels"], case["states"]
        s["u"] = torch.nn.functional.silu(normal(b, n, d)).to(dt)
        s["delta"] = normal(b, n, d, std=0.5).to(dt)
        s["z"] = normal(b, n, 2 * d).to(dt)[:, :, d:]
        both = normal(b, n, 2 * m).to(dt)                       # B and C come out of one projection
        s["B"], s["C"] = both[:, :, :m], both[:, :, m:]
        s["A"] = -torch.arange(1, m + 1, device="cuda", dtype=torch.float32) * (1 + 0.1 * torch.rand(d, m, generator=gen, device="cuda"))
        step = torch.exp(torch.rand(d, generator=gen, device="cuda") * 4.6 - 6.9)      # 0.001 to 0.1
        s["delta_bias"] = step + torch.log(-torch.expm1(-step))
        s["D"] = 1 + normal(d, std=0.1)
        s["state"] = normal(b, d, m) if case["state"] else None
        s["lengths"] = _lengths(case, host) if case["ragged"] else None
    elif case["kind"] == "quantize":
        x = normal(case["rows"], case["k"])
        x *= torch.exp(normal(case["rows"], 1))                 # tokens differ in scale
        s["x"] = x.to(dt)
    else:
        m, n, k = case["m"], case["n"], case["k"]
        a, sa = _quantized(normal(m, k) * torch.exp(normal(m, 1, std=0.5)), 1)
        b, sb = _quantized(normal(n, k, std=k ** -0.5), BLOCK)
        s["a"], s["a_scales"] = _rows_of_16_bytes(a), sa.t().contiguous().t()
        s["b"], s["b_scales"] = _rows_of_16_bytes(b), sb.contiguous()
        s["bias"] = normal(n) if case["bias"] else None
    return s


def _conv(s):
    x, w = s["x"].float(), s["weight"]
    n, k = x.shape[1], w.shape[1]
    before = torch.zeros_like(x[:, :1]).expand(-1, k - 1, -1) if s["state"] is None else s["state"].float()
    wide = torch.cat([before, x], 1)
    y = (wide.unfold(1, k, 1) * w).sum(-1) + s["bias"]
    y = y / (1 + torch.exp(-y))
    return {"y": y.to(s["x"].dtype), "state": wide[:, n:].to(s["x"].dtype)}


def _scan(s):
    u, dtype = s["u"].float(), s["u"].dtype
    raw = s["delta"].float() + s["delta_bias"]
    delta = torch.clamp_min(raw, 0) + torch.log1p(torch.exp(-raw.abs()))
    n = u.shape[1]
    if s["lengths"] is not None:
        inside = torch.arange(n, device=u.device)[None, :, None] < s["lengths"][:, None, None]
        delta = delta * inside
    a = torch.exp(delta[..., None] * s["A"])                                            # [batch, token, channel, state]
    h = (delta * u)[..., None] * s["B"].float()[:, :, None, :]
    if s["state"] is not None:
        h[:, 0] += a[:, 0] * s["state"]
    step = 1
    while step < n:             # after each round every token has the sum over twice as many tokens before it
        h[:, step:] += a[:, step:] * h[:, :-step]
        a[:, step:] = a[:, step:] * a[:, :-step]
        step *= 2
    y = (h * s["C"].float()[:, :, None, :]).sum(-1) + s["D"] * u
    z = s["z"].float()
    y = y * (z / (1 + torch.exp(-z)))
    if s["lengths"] is not None:
        y = torch.where(inside, y, torch.zeros_like(y))
    return {"y": y.to(dtype), "state": h[:, -1].clone()}


def _matmul(s):
    def wide(q, scales, rows):
        r, k = q.shape
        return q.float() * scales.repeat_interleave(rows, 0)[:r].repeat_interleave(BLOCK, 1)[:, :k]

    y = wide(s["a"], s["a_scales"], 1) @ wide(s["b"], s["b_scales"], BLOCK).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": y.to(DTYPES[s["case"]["dtype"]])}


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        from paper_2007_06000_amd import seq
        if kind == "conv":
            y, new = seq.causal_conv(s["x"], s["weight"], s["bias"], state=s["state"])
            return {"y": y, "state": new}
        if kind == "scan":
            y, new = seq.selective_scan(s["u"], s["delta"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"], delta_bias=s["delta_bias"],
                                        state=s["state"], lengths=s["lengths"])
            return {"y": y, "state": new}
        if kind == "quantize":
            q, scales = seq.quantize_rows(s["x"])
            return {"q": q, "scales": scales}
        return {"y": seq.block_matmul(s["a"], s["a_scales"], s["b"], s["b_scales"], bias=s["bias"], dtype=DTYPES[s["case"]["dtype"]])}
    if kind == "conv":
        return _conv(s)
    if kind == "scan":
        return _scan(s)
    if kind == "quantize":
        q, scales = _quantized(s["x"], 1)
        return {"q": q, "scales": scales}
    return _matmul(s)


def work(case):
    c = case
    size = DTYPES[c["dtype"]].itemsize
    if c["kind"] == "conv":
        x = c["batch"] * c["length"] * c["channels"]
        state = c["batch"] * (c["taps"] - 1) * c["channels"] * size
        return {"bytes": 2 * x * size + (1 + c["state"]) * state + c["channels"] * (c["taps"] + 1) * 4, "flops": x * (2 * c["taps"] + 4)}
    if c["kind"] == "scan":
        b, n, d, m = c["batch"], c["length"], c["channels"], c["states"]
        tokens = b * n
        if c["ragged"] and b > 1:       # the lengths are evenly spread from none to all
            tokens = sum(int(round(i * n / (b - 1))) for i in range(b))
        inputs = tokens * (3 * d + 2 * m) * size
        return {"bytes": inputs + b * n * d * size + (1 + c["state"]) * b * d * m * 4 + d * (m + 2) * 4,
                "flops": tokens * d * (7 * m + 12)}      # a state: product, exponential, two products and two sums
    if c["kind"] == "quantize":
        x = c["rows"] * c["k"]
        return {"bytes": x * (size + 1) + c["rows"] * -(-c["k"] // BLOCK) * 4, "flops": 2 * x}
    m, n, k = c["m"], c["n"], c["k"]
    scales = (m + -(-n // BLOCK)) * -(-k // BLOCK) * 4
    return {"bytes": (m + n) * k + scales + m * n * size + c["bias"] * n * 4, "flops": 2 * m * n * k}


def exact(case, seed):
    """From the definitions, in 64 bits: the convolution tap by tap, the scan token by token, the product block by block."""
    s = prepare(case, seed)
    if case["kind"] == "conv":
        x, w = s["x"].double(), s["weight"].double()
        n, k = x.shape[1], w.shape[1]
        y = torch.zeros_like(x) + s["bias"].double()
        last = []
        for j in range(k):              # tap j sees the input k - 1 - j tokens earlier
            back = k - 1 - j
            y[:, back:] += w[:, j] * x[:, :max(0, n - back)]
            if s["state"] is not None:
                for t in range(min(back, n)):
                    y[:, t] += w[:, j] * s["state"][:, t + j].double()
        for t in range(n - (k - 1), n):
            at = k - 1 + t
            last.append(x[:, t] if t >= 0 else s["state"][:, at].double() if s["state"] is not None else torch.zeros_like(x[:, 0]))
        return {"y": y * torch.sigmoid(y), "state": torch.stack(last, 1)}
    if case["kind"] == "scan":
        u, A = s["u"].double(), s["A"].double()
        b, n, d = u.shape
        delta = torch.nn.functional.softplus(s["delta"].double() + s["delta_bias"].double(), threshold=40.0)
        B, C = s["B"].double(), s["C"].double()
        h = torch.zeros(b, d, A.shape[1], dtype=torch.float64, device=u.device) if s["state"] is None else s["state"].double()
        y = torch.zeros_like(u)
        for t in range(n):
            new = torch.exp(delta[:, t, :, None] * A) * h + (delta[:, t] * u[:, t])[..., None] * B[:, t, None, :]
            h = new if s["lengths"] is None else torch.where((t < s["lengths"])[:, None, None], new, h)
            y[:, t] = (h * C[:, t, None, :]).sum(-1)
        z = s["z"].double()
        y = (y + s["D"].double() * u) * z * torch.sigmoid(z)
        if s["lengths"] is not None:
            y[torch.arange(n, device=u.device)[None] >= s["lengths"][:, None]] = 0
        return {"y": y, "state": h}
    if case["kind"] == "quantize":
        x = s["x"].double()
        r, k = x.shape
        q, scales = torch.empty_like(x), []
        for at in range(0, k, BLOCK):
            part = x[:, at:at + BLOCK]
            scales.append((part.abs().max(1)[0] / E4M3_MAX).clamp_min(MIN_SCALE))
            q[:, at:at + BLOCK] = part / scales[-1][:, None]
        return {"q": q, "scales": torch.stack(scales, 1)}
    m, n, k = case["m"], case["n"], case["k"]
    y = torch.zeros(m, n, dtype=torch.float64, device="cuda")
    if s["bias"] is not None:
        y += s["bias"].double()
    for i, at in enumerate(range(0, k, BLOCK)):
        part = s["a"][:, at:at + BLOCK].double() @ s["b"][:, at:at + BLOCK].double().t()
        part *= s["a_scales"][:, i].double()[:, None]
        part *= s["b_scales"][:, i].double().repeat_interleave(BLOCK)[:n]
        y += part
    return {"y": y}
