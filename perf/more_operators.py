"""Performance cases of the operators around a block-scaled projection: norm, low-rank adapters, gated delta rule.

A mixer layer adds its input to the residual and norms the sum on the way into its 8-bit projection, low-rank adapters of many
requests go beside that projection, and the gated delta rule is the recurrence between the projections: a matrix of states for each head
that every token decays, corrects and reads.  Every case is one call of one operator on one batch.  A case holds

    kind       norm | delta | adapters
    dtype      of the activations
    norm       rows, k (the length of a row); residual: whether one is added, in place ("" | "same" type | "float32"); quantized: e4m3 and scales
    delta      batch, length, key_heads, heads, dk, dv; state; ragged: the sequences have lengths of their own, from none to all;
               normalize: whether the operator brings queries and keys to length one
    adapters   batch, length, k, n, rank, adapters: how many there are; ragged

The path is inference only: there is no backward direction and no optimiser.
"""
import torch

own = False

BLOCK = 128                                     # numbers that share a scale
E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -126
EPS = 1e-6
CHUNK = 64                                      # tokens that the plain delta rule takes at once
DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
MAX_NUMBERS = 24642 * 4096                      # of a drawn norm's input, of an adapter call's input and result
MAX_HEAD_NUMBERS = 2 * 12321 * 16 * 128         # of a drawn delta rule's values
MAX_STATE_STEPS = 2 * 12321 * 16 * 128 * 128    # of a drawn delta rule: the largest listed one's


def listed():
    return [
        # The tokens of a serving step on their way into a projection: the smallest norm, bound by its launch.
        {"name": "norm_token_b16", "kind": "norm", "dtype": "bfloat16", "rows": 16, "k": 2048, "residual": "same", "quantized": True},
        # Five 27x27 feature maps read as sequences, fp32 throughout; nothing divides by a block or a vector.
        {"name": "norm_27x27_b5", "kind": "norm", "dtype": "float32", "rows": 3645, "k": 1001, "residual": "same", "quantized": False},
        # All positions of two 111x111 maps: bound by memory.
        {"name": "norm_24642", "kind": "norm", "dtype": "bfloat16", "rows": 24642, "k": 4096, "residual": "same", "quantized": True},
        # One token of 16 sequences, small heads: the smallest call of the recurrence.
        {"name": "delta_token_b16", "kind": "delta", "dtype": "bfloat16", "batch": 16, "length": 1, "key_heads": 4, "heads": 8, "dk": 64, "dv": 64,
         "state": True, "ragged": False, "normalize": True},
        # One token of 64 sequences: reads and writes 67 MB of states, little else.
        {"name": "delta_token_b64", "kind": "delta", "dtype": "bfloat16", "batch": 64, "length": 1, "key_heads": 8, "heads": 16, "dk": 128, "dv": 128,
         "state": True, "ragged": False, "normalize": True},
        # One 56x56 feature map: a single long sequence, few heads to fill the chip with.
        {"name": "delta_56x56_b1", "kind": "delta", "dtype": "bfloat16", "batch": 1, "length": 3136, "key_heads": 8, "heads": 8, "dk": 128, "dv": 128,
         "state": False, "ragged": False, "normalize": True},
        # Sequences of their own lengths (none, a part, all of 27x27), odd sizes of heads, fp32, keys of length one already.
        {"name": "delta_27x27_b5_ragged", "kind": "delta", "dtype": "float32", "batch": 5, "length": 729, "key_heads": 3, "heads": 6, "dk": 45, "dv": 77,
         "state": True, "ragged": True, "normalize": False},
        # Two 111x111 feature maps (the stem's output): the largest recurrence.
        {"name": "delta_111x111_b2", "kind": "delta", "dtype": "bfloat16", "batch": 2, "length": 12321, "key_heads": 8, "heads": 16, "dk": 128, "dv": 128,
         "state": False, "ragged": False, "normalize": True},
        # One token of 32 requests, each with an adapter of its own: bound by reading them.
        {"name": "adapters_token_b32", "kind": "adapters", "dtype": "bfloat16", "batch": 32, "length": 1, "k": 2048, "n": 4096, "rank": 16, "adapters": 40,
         "ragged": False},
        # Prompts of their own lengths and few adapters, one of them without any: odd sizes, fp32.
        {"name": "adapters_27x27_b5_ragged", "kind": "adapters", "dtype": "float32", "batch": 5, "length": 729, "k": 520, "n": 1000, "rank": 13, "adapters": 3,
         "ragged": True},
        # One 56x56 map as the prompt of one request.
        {"name": "adapters_56x56_b1", "kind": "adapters", "dtype": "float16", "batch": 1, "length": 3136, "k": 1024, "n": 4096, "rank": 64, "adapters": 4,
         "ragged": False},
        # Two 111x111 maps: bound by memory.
        {"name": "adapters_111x111_b2", "kind": "adapters", "dtype": "bfloat16", "batch": 2, "length": 12321, "k": 4096, "n": 4096, "rank": 32, "adapters": 8,
         "ragged": False},
    ]


def _size(rng, lo, hi):
    """A size of [lo, hi], spread over its logarithm: a power of two or an odd number."""
    v = lo * (hi / lo) ** rng.random()
    if rng.random() < 0.4:
        p = 1 << max(0, round(v).bit_length() - 1)
        if lo <= p <= hi:
            return p
    return min(hi, max(lo, int(v) | 1))


def draw(rng):
    kind = rng.choice(["norm", "delta", "delta", "adapters"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if kind == "norm":
        c = {"kind": kind, "dtype": dtype, "rows": _size(rng, 1, 24642), "k": _size(rng, 8, 16384), "residual": rng.choice(["", "same", "same", "float32"]),
             "quantized": rng.random() < 0.5}
        while c["rows"] * c["k"] > MAX_NUMBERS:
            c["rows"] //= 2
    elif kind == "delta":
        groups, key_heads = rng.choice([1, 1, 2, 3, 4]), _size(rng, 1, 16)
        c = {"kind": kind, "dtype": dtype, "batch": _size(rng, 1, 64), "length": rng.choice([1, _size(rng, 1, 12321), _size(rng, 1, 12321)]),
             "key_heads": key_heads, "heads": key_heads * groups, "dk": rng.choice([64, 128, _size(rng, 8, 256)]), "dv": rng.choice([64, 128, _size(rng, 8, 256)]),
             "state": rng.random() < 0.5, "ragged": rng.random() < 0.3, "normalize": rng.random() < 0.5}

        def too_long():
            rows = c["batch"] * c["length"] * c["heads"]
            return rows * max(c["dk"], c["dv"]) > MAX_HEAD_NUMBERS or rows * c["dk"] * c["dv"] > MAX_STATE_STEPS
        while too_long():
            if c["batch"] > 1:
                c["batch"] //= 2
            elif c["key_heads"] > 1:
                c["key_heads"] //= 2
                c["heads"] = c["key_heads"] * groups
            else:
                c["length"] = c["length"] // 2 | 1
    else:
        c = {"kind": kind, "dtype": dtype, "batch": _size(rng, 1, 64), "length": rng.choice([1, _size(rng, 1, 12321), _size(rng, 1, 12321)]),
             "k": _size(rng, 16, 4096), "n": _size(rng, 16, 4096), "rank": rng.choice([8, 16, 32, 64, _size(rng, 1, 128)]), "adapters": _size(rng, 1, 64),
             "ragged": rng.random() < 0.3}
        while c["batch"] > 1 and c["batch"] * c["length"] * max(c["k"], c["n"]) > MAX_NUMBERS:
            c["batch"] //= 2
        if c["dtype"] == "float32":
            c["rank"] = min(c["rank"], 32)
    return c


def _lengths(c, gen):
    """From none to all of the tokens, evenly spread, in an order of the seed's."""
    b, n = c["batch"], c["length"]
    even = torch.arange(b, dtype=torch.float64) * n / max(1, b - 1) if b > 1 else torch.full((1,), float(n), dtype=torch.float64)
    return even.round().to(torch.int32)[torch.randperm(b, generator=gen)].cuda()


def _index(c):
    """The adapter of each sequence: all of them in turn, and where there are three sequences or more the second has none."""
    which = torch.arange(c["batch"], dtype=torch.int32) % c["adapters"]
    if c["batch"] >= 3:
        which[1] = -1
    return which


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    s = {"case": dict(case)}
    if case["kind"] == "norm":
        rows, k = case["rows"], case["k"]
        s["x"] = normal(rows, k, std=0.5).to(dt)
        s["residual"] = None
        if case["residual"]:                                    # grows from layer to layer, tokens differ in scale
            r = normal(rows, k) * torch.exp(normal(rows, 1))
            s["residual"] = r.to(dt if case["residual"] == "same" else torch.float32)
        s["weight"] = 1 + normal(k, std=0.2)
    elif case["kind"] == "delta":
        b, n, hk, h, dk, dv = (case[f] for f in ("batch", "length", "key_heads", "heads", "dk", "dv"))
        # q, k and v are parts of one projection, behind a short convolution and SiLU
        both = torch.nn.functional.silu(normal(b, n, 2 * hk * dk + h * dv)).to(dt)
        if not case["normalize"]:
            qk = both[..., :2 * hk * dk].float().view(b, n, 2 * hk, dk)
            both[..., :2 * hk * dk] = (qk / (qk.square().sum(-1, keepdim=True) + EPS).sqrt()).view(b, n, -1).to(dt)
        s["q"] = both[..., :hk * dk].view(b, n, hk, dk)
        s["k"] = both[..., hk * dk:2 * hk * dk].view(b, n, hk, dk)
        s["v"] = both[..., 2 * hk * dk:].view(b, n, h, dv)
        rate = torch.exp(torch.rand(h, generator=gen, device="cuda") * 2.77)            # 1 to 16
        step = torch.exp(torch.rand(b, n, h, generator=gen, device="cuda") * 4.6 - 6.9)    # 0.001 to 0.1
        s["g"] = -rate * step
        s["beta"] = torch.sigmoid(normal(b, n, h))
        s["state"] = normal(b, h, dk, dv, std=dk ** -0.5) if case["state"] else None
        s["lengths"] = _lengths(case, host) if case["ragged"] else None
    else:
        b, n, k, m, rank, many = (case[f] for f in ("batch", "length", "k", "n", "rank", "adapters"))
        s["x"], s["y"] = normal(b, n, k).to(dt), normal(b, n, m).to(dt)
        s["down"] = normal(many, rank, k, std=k ** -0.5).to(dt)
        s["up"] = normal(many, m, rank, std=rank ** -0.5).to(dt)
        s["scales"] = 0.25 + torch.rand(many, generator=gen, device="cuda")
        s["index"] = _index(case).cuda()
        s["lengths"] = _lengths(case, host) if case["ragged"] else None
    return s


def _norm(s):
    x, k = s["x"].float(), s["x"].shape[1]
    r = x if s["residual"] is None else x + s["residual"].float()
    y = r * torch.rsqrt((r * r).sum(1, keepdim=True) / k + EPS) * s["weight"]
    out = {} if s["residual"] is None else {"residual": r.to(s["residual"].dtype)}
    if not s["case"]["quantized"]:
        return {"y": y.to(s["x"].dtype), **out}
    blocks = torch.nn.functional.pad(y, (0, -k % BLOCK)).view(y.shape[0], -1, BLOCK)
    scales = (blocks.abs().amax(2) / E4M3_MAX).clamp_min(MIN_SCALE)
    q = (blocks / scales[..., None]).view(y.shape[0], -1)[:, :k].to(torch.float8_e4m3fn)
    return {"q": q, "scales": scales, **out}


def _delta(s):
    """Chunks of tokens: inside one the corrections solve a triangular system, from one to the next the states go through an affine map."""
    dtype, h = s["v"].dtype, s["v"].shape[2]
    b, n, hk, dk = s["q"].shape
    dv, c = s["v"].shape[3], min(CHUNK, s["q"].shape[1])
    many = -(-n // c)
    g, beta = s["g"], s["beta"]
    inside = None
    if s["lengths"] is not None:
        inside = torch.arange(n, device=g.device)[None, :, None] < s["lengths"][:, None, None]
        g, beta = g * inside, beta * inside

    def chunks(t):              # [b, n, heads, d] -> [b, heads, chunk, token, d], fp32, zeros behind the end
        t = torch.nn.functional.pad(t.float(), (0, 0, 0, 0, 0, many * c - n))
        return t.view(b, many, c, t.shape[2], t.shape[3]).permute(0, 3, 1, 2, 4)

    q, k, v = chunks(s["q"]), chunks(s["k"]), chunks(s["v"]).contiguous()
    if s["case"]["normalize"]:
        q, k = (t / ((t * t).sum(-1, keepdim=True) + EPS).sqrt() for t in (q, k))
    q, k = (t.repeat_interleave(h // hk, 1).contiguous() for t in (q * dk ** -0.5, k))
    g, beta = chunks(g[..., None])[..., 0], chunks(beta[..., None])
    G = g.double().cumsum(-1)
    between = torch.exp((G[..., :, None] - G[..., None, :]).clamp_max(0)).float()
    kt = k.transpose(-1, -2).contiguous()
    # (I + A)^-1 of a strictly lower triangular A, whose powers end: (I - A)(I + A^2)(I + A^4) ..., in 64 bits, for keys that point the same way
    power = -(beta * (k @ kt) * between).tril(-1).double()
    solve, step = torch.eye(c, dtype=torch.float64, device=g.device) + power, 2
    while step < c:
        power = power @ power
        solve = solve + solve @ power
        step *= 2
    solve = solve.float()
    since = torch.exp(G).float()[..., None]                     # decay from the chunk's begin, and to its end
    until = torch.exp(G[..., -1:] - G).float()[..., None]
    w, u = solve @ (beta * since * k), solve @ (beta * v)
    ends = (k * until).transpose(-1, -2).contiguous()
    # states behind a chunk: move @ states before it + add; after each round over twice as many chunks
    move = since[..., -1:, :] * torch.eye(dk, device=g.device) - ends @ w
    add = ends @ u
    if s["state"] is not None:
        add[:, :, 0] += move[:, :, 0] @ s["state"]
    step = 1
    while step < many:
        add[:, :, step:] += move[:, :, step:] @ add[:, :, :-step]
        move[:, :, step:] = move[:, :, step:] @ move[:, :, :-step]
        step *= 2
    first = torch.zeros_like(add[:, :, :1]) if s["state"] is None else s["state"][:, :, None]
    before = torch.cat([first, add[:, :, :-1]], 2)
    y = (since * q) @ before + ((q @ kt) * between).tril() @ (u - w @ before)
    y = y.permute(0, 2, 3, 1, 4).reshape(b, many * c, h, dv)[:, :n]
    if inside is not None:
        y = torch.where(inside[..., None], y, torch.zeros_like(y))
    return {"y": y.to(dtype), "state": add[:, :, -1].clone()}


def _adapters(s):
    x, y = s["x"].float(), s["y"].float()
    there = s["index"] >= 0
    at = s["index"].clamp_min(0).long()
    t = x @ s["down"][at].float().transpose(1, 2).contiguous()
    t = t * (s["scales"][at] * there)[:, None, None]
    out = y + t @ s["up"][at].float().transpose(1, 2).contiguous()
    if s["lengths"] is not None:
        inside = torch.arange(x.shape[1], device=x.device)[None, :, None] < s["lengths"][:, None, None]
        out = torch.where(inside, out, torch.zeros_like(out))
    return {"out": out.to(s["y"].dtype)}


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        from paper_2007_06000_amd import seq
        if kind == "norm":
            if s["case"]["quantized"]:
                q, scales, r = seq.rms_norm_quantized(s["x"], s["weight"], residual=s["residual"], eps=EPS)
                out = {"q": q, "scales": scales}
            else:
                y, r = seq.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS)
                out = {"y": y}
            return out if s["residual"] is None else {**out, "residual": r}
        if kind == "delta":
            y, new = seq.gated_delta_rule(s["q"], s["k"], s["v"], s["g"], s["beta"], normalize=s["case"]["normalize"], state=s["state"], lengths=s["lengths"])
            return {"y": y, "state": new}
        return {"out": seq.add_adapters(s["y"], s["x"], s["down"], s["up"], s["index"], scales=s["scales"], lengths=s["lengths"])}
    return _norm(s) if kind == "norm" else _delta(s) if kind == "delta" else _adapters(s)


def work(case):
    c = case
    size = DTYPES[c["dtype"]].itemsize
    if c["kind"] == "norm":
        x, residual = c["rows"] * c["k"], {"": 0, "same": size, "float32": 4}[c["residual"]]
        result = x + c["rows"] * -(-c["k"] // BLOCK) * 4 if c["quantized"] else x * size
        return {"bytes": x * (size + 2 * residual) + result + c["k"] * 4, "flops": x * (6 + 2 * c["quantized"])}
    b, n = c["batch"], c["length"]
    lengths = [n] * b
    if c["ragged"] and b > 1:           # evenly spread from none to all
        lengths = [int(round(i * n / (b - 1))) for i in range(b)]
    tokens = sum(lengths)
    if c["kind"] == "delta":
        hk, h, dk, dv = c["key_heads"], c["heads"], c["dk"], c["dv"]
        return {"bytes": tokens * ((2 * hk * dk + h * dv) * size + 2 * h * 4) + b * n * h * dv * size + (1 + c["state"]) * b * h * dk * dv * 4,
                "flops": tokens * h * 7 * dk * dv}      # of a state: the decay, and a product and a sum for the correction, the update and the result
    which = [int(i) for i in _index(c)]
    used = len({i for i in which if i >= 0})
    # lengths come in an order of the seed's: the sequence without an adapter is taken to be an average one
    adapted = tokens * sum(i >= 0 for i in which) / b
    return {"bytes": int(adapted * c["k"] * size) + (tokens + b * n) * c["n"] * size + used * c["rank"] * (c["k"] + c["n"]) * size,
            "flops": int(adapted * 2 * c["rank"] * (c["k"] + c["n"]))}


def exact(case, seed):
    """From the definitions, in 64 bits: the norm row by row, the delta rule token by token, the adapters sequence by sequence."""
    s = prepare(case, seed)
    if case["kind"] == "norm":
        r = s["x"].double()
        if s["residual"] is not None:
            r = r + s["residual"].double()
        y = r / torch.sqrt(r.pow(2).mean(1) + EPS)[:, None] * s["weight"].double()
        out = {} if s["residual"] is None else {"residual": r}
        if not case["quantized"]:
            return {"y": y, **out}
        q, scales = torch.empty_like(y), []
        for at in range(0, y.shape[1], BLOCK):
            part = y[:, at:at + BLOCK]
            scales.append((part.abs().max(1)[0] / E4M3_MAX).clamp_min(MIN_SCALE))
            q[:, at:at + BLOCK] = part / scales[-1][:, None]
        return {"q": q, "scales": torch.stack(scales, 1), **out}
    if case["kind"] == "delta":
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        b, n, h, dv = v.shape
        dk = q.shape[3]
        if case["normalize"]:
            q, k = (t / torch.sqrt(t.pow(2).sum(-1) + EPS)[..., None] for t in (q, k))
        head = torch.arange(h, device=v.device) // (h // q.shape[2])
        decay, beta = torch.exp(s["g"].double()), s["beta"].double()
        S = torch.zeros(b, h, dk, dv, dtype=torch.float64, device=v.device) if s["state"] is None else s["state"].double()
        y = torch.zeros_like(v)
        for t in range(n):
            kt, qt = k[:, t, head, :, None], q[:, t, head, :, None]
            new = S * decay[:, t, :, None, None]
            error = v[:, t] - (new * kt).sum(2)
            new += kt * (beta[:, t, :, None] * error)[:, :, None, :]
            S = new if s["lengths"] is None else torch.where((t < s["lengths"])[:, None, None, None], new, S)
            y[:, t] = (new * qt).sum(2) * dk ** -0.5
        if s["lengths"] is not None:
            y[torch.arange(n, device=v.device)[None] >= s["lengths"][:, None]] = 0
        return {"y": y, "state": S}
    out = s["y"].double()
    lengths = [case["length"]] * case["batch"] if s["lengths"] is None else s["lengths"].tolist()
    for i, a in enumerate(s["index"].tolist()):
        m = lengths[i]
        if a >= 0 and m:
            inner = s["x"][i, :m].double() @ s["down"][a].double().t()
            out[i, :m] += s["scales"][a].double() * (inner @ s["up"][a].double().t())
        out[i, m:] = 0
    return {"out": out}
