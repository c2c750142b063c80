"""The gated delta rule against its definition in 64 bits: prompts, single tokens, states in a cache."""
import numpy as np
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import seq
from paper_2007_06000_amd.binding import XlError
from test_gpu_seq_conv import HALF, f64

pytestmark = pytest.mark.gpu


def inputs(batch, length, key_heads, heads, dk, dv, dtype, seed=0, normalized=False, alike=0.5):
    """Keys lean the same way, as behind a SiLU; decays between almost none and a sixth a token."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q, k = r(batch, length, key_heads, dk) + alike, r(batch, length, key_heads, dk) + alike
    if normalized:
        q, k = (t / t.norm(dim=-1, keepdim=True) for t in (q, k))
    decay = -torch.exp(torch.rand(heads, generator=g) * 2.77) * torch.exp(torch.rand(batch, length, heads, generator=g) * 4.6 - 6.9)
    return {"q": q.to(dtype).cuda(), "k": k.to(dtype).cuda(), "v": r(batch, length, heads, dv).to(dtype).cuda(), "g": decay.cuda(),
            "beta": torch.sigmoid(r(batch, length, heads)).cuda(), "state": (r(batch, heads, dk, dv) * dk ** -0.5).cuda()}


def reference(p, lengths=None, normalize=True, scale=None):
    length = p["q"].shape[1]
    n = [length] * p["q"].shape[0] if lengths is None else [min(max(int(v), 0), length) for v in lengths]
    clean = {f: np.nan_to_num(f64(p[f])) for f in ("q", "k", "v", "g", "beta")}
    s = p["q"].shape[3] ** -0.5 if scale is None else scale
    return ref.gated_delta_rule(*clean.values(), s, normalize, f64(p.get("state")), n, p["v"].dtype != torch.float32)


def spread(p, lengths, normalize):
    """The largest sum of magnitudes in a row of (I + A)^-1 over all chunks of 64 tokens: how much the corrections of a chunk may outgrow what they are made of."""
    k, g, beta = (np.nan_to_num(f64(p[f]), neginf=-128) for f in ("k", "g", "beta"))
    if normalize:
        k = k / np.sqrt((k ** 2).sum(-1, keepdims=True) + 1e-6)
    most, group = 1.0, g.shape[2] // k.shape[2]
    for b, n in enumerate(lengths):
        for t in range(0, n, 64):
            at = slice(t, min(t + 64, n))
            for h in range(g.shape[2]):
                G = np.clip(g[b, at, h], -128, 0).cumsum()
                keys = k[b, at, h // group]
                A = np.tril(beta[b, at, h][:, None] * (keys @ keys.T) * np.exp(np.minimum(G[:, None] - G[None], 0)), -1)
                most = max(most, np.abs(np.linalg.inv(np.eye(len(G)) + A)).sum(1).max())
    return most


def compare(got, new, want, what, outgrown=1.0):
    """A chunk's corrections are sums over T = (I + A)^-1 whose terms' magnitudes are up to `outgrown` (the largest row of |T|) times the result's size; what T, its product with the right side, the
    product of keys and corrections and the right side itself are rounded by is at most 2^-24 of that each, with either sign: 4 outgrown 2^-24 of the states' norm, 8 standing for a row of T
    where there is little growth and for the token by token form's dk sums."""
    y, bound, S, S_bound = want
    half = HALF[got.dtype]
    got, new = f64(got), f64(new)
    assert np.isfinite(got).all() and np.isfinite(new).all(), what
    off = np.abs(got - y) - (bound + half * (np.abs(y) + bound) + 2.0 ** -24)
    assert (off <= 0).all(), f"{what}: y is {off.max():.3g} beyond the bound at {np.unravel_index(off.argmax(), off.shape)}"
    apart = np.sqrt(((new - S) ** 2).sum(2)) - S_bound - 2.0 ** -24 * np.sqrt((S ** 2).sum(2)) - 1e-37
    assert (apart <= 0).all(), f"{what}: a column is {apart.max():.3g} beyond the bound"
    # roundings have either sign: of some thousand numbers' 2-norm little is left of the sum of the bounds
    if S.size > 1000 and np.linalg.norm(S) > 0:
        assert np.linalg.norm(new - S) < 4 * max(8, outgrown) * 2.0 ** -24 * np.linalg.norm(S), f"{what}: states are {np.linalg.norm(new - S) / np.linalg.norm(S):.3g} off"


def check(p, what="", lengths=None, normalize=True, scale=None, **more):
    got, new = seq.gated_delta_rule(**p, normalize=normalize, scale=scale, lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"), **more)
    length = p["q"].shape[1]
    n = [length] * p["q"].shape[0] if lengths is None else [min(max(int(v), 0), length) for v in lengths]
    compare(got, new, reference(p, lengths, normalize, scale), what, spread(p, n, normalize))
    return got, new


SIZES = [  # batch, length, key heads, heads, dk, dv
    (1, 1, 1, 1, 1, 1), (2, 1, 1, 2, 64, 64), (3, 1, 2, 2, 128, 128), (2, 1, 2, 6, 45, 77), (1, 1, 1, 1, 256, 32), (2, 2, 1, 1, 17, 33), (1, 7, 2, 4, 64, 32), (1, 16, 1, 1, 128, 40),
    (1, 63, 1, 2, 64, 16), (2, 64, 1, 1, 128, 32), (1, 65, 2, 2, 64, 64), (1, 128, 1, 3, 100, 50), (2, 129, 1, 2, 8, 8), (1, 200, 1, 1, 256, 24), (1, 150, 2, 4, 129, 17), (3, 77, 1, 1, 3, 5),
    (1, 330, 1, 2, 128, 128), (1, 100, 1, 1, 250, 3), (1, 40, 3, 6, 32, 20), (1, 70, 1, 1, 65, 130)]


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(size, dtype):
    p = inputs(*size, dtype, seed=sum(size))
    check(p, "state")
    p.pop("state")
    check(p, "no state")


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("size", [(2, 1, 1, 2, 64, 64), (1, 90, 1, 2, 64, 32), (1, 140, 1, 1, 128, 16), (1, 70, 1, 1, 200, 16)], ids=lambda s: "x".join(map(str, s)))
def test_keys_that_come_normalised(size, dtype):
    check(inputs(*size, dtype, normalized=True), normalize=False)
    check(inputs(*size, dtype, normalized=True, seed=1), normalize=False, scale=-1.5)


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("lengths", [[0, 1, 63, 64, 65], [150, 0, -5, 1000, 149], [0, 0, 0, 0, 0], [2, 3, 127, 128, 129]])
def test_sequences_of_their_own_lengths(lengths, dtype):
    p = inputs(5, 150, 1, 2, 64, 48, dtype)
    for b, n in enumerate(lengths):
        for f in ("q", "k", "v", "g", "beta"):
            p[f][b, max(n, 0):] = float("nan")         # never read
    got, new = check(p, lengths=lengths)
    for b, n in enumerate(lengths):
        assert not got[b, max(n, 0):].any()
        if n <= 0:
            assert torch.equal(new[b], p["state"][b])


@pytest.mark.parametrize("length", [1, 5, 100])
def test_a_cache_of_slots(length):
    p = inputs(5, length, 1, 2, 64, 40, torch.bfloat16)
    cache = torch.randn(7, 2, 64, 40, device="cuda") * 0.1
    before = cache.clone()
    slots = torch.tensor([4, -1, 0, 7, 6], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([length, length, 0, length, max(1, length // 2)], dtype=torch.int32, device="cuda")
    p.pop("state")
    got, back = seq.gated_delta_rule(**p, normalize=True, state=cache, slots=slots, lengths=lengths)
    assert back is cache
    for b, slot in enumerate(slots.tolist()):
        if not 0 <= slot < 7:
            assert not got[b].any()
            continue
        one = {f: t[b:b + 1] for f, t in p.items()}
        compare(got[b:b + 1], cache[slot:slot + 1], reference({**one, "state": before[slot:slot + 1]}, [int(lengths[b])]), f"sequence {b}")
    for slot in (1, 2, 3, 5):
        assert torch.equal(cache[slot], before[slot])
    assert torch.equal(cache[0], before[0])         # a length of zero


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
def test_a_prompt_in_pieces_and_token_by_token(dtype):
    p = inputs(2, 139, 2, 4, 64, 64, dtype)
    want = reference(p)
    outs, state = [], p.pop("state")
    for a, b in ((0, 64), (64, 70), (70, 71), (71, 135), (135, 136), (136, 139)):
        y, state = seq.gated_delta_rule(**{f: t[:, a:b] for f, t in p.items()}, normalize=True, state=state, new_state=state)
        outs.append(y)
    compare(torch.cat(outs, 1), state, want, "pieces")


@pytest.mark.parametrize("length", [1, 3, 80])
def test_layouts(length):
    """Parts of one projection, heads in front of the tokens, odd addresses; a result inside of a wider tensor."""
    b, hk, h, dk, dv = 2, 2, 4, 40, 24
    p = inputs(b, length, hk, h, dk, dv, torch.bfloat16)
    want, state = check(p)
    wide = torch.cat([torch.zeros(b, length, 3, device="cuda", dtype=torch.bfloat16), p["q"].flatten(2), p["k"].flatten(2), p["v"].flatten(2)], 2)
    views = {**p, "q": wide[..., 3:3 + hk * dk].view(b, length, hk, dk), "k": wide[..., 3 + hk * dk:3 + 2 * hk * dk].view(b, length, hk, dk), "v": wide[..., 3 + 2 * hk * dk:].view(b, length, h, dv),
             "g": torch.stack([p["g"], p["beta"]], 2)[:, :, 0], "beta": torch.cat([p["g"], p["beta"]], 2)[:, :, h:]}
    room = torch.full((b, length, h * dv + 7), 5.0, dtype=torch.bfloat16, device="cuda")
    out = room[..., 5:5 + h * dv].view(b, length, h, dv)
    got, new = seq.gated_delta_rule(**views, normalize=True, out=out)
    assert got is out and torch.equal(got, want) and torch.equal(new, state) and (room[..., :5] == 5).all() and (room[..., -2:] == 5).all()
    turned = {**p, **{f: p[f].transpose(1, 2).contiguous().transpose(1, 2) for f in ("q", "k", "v")}}
    got, new = seq.gated_delta_rule(**turned, normalize=True)
    assert torch.equal(got, want) and torch.equal(new, state)
    shared = {**p, "q": p["q"][:, :, :1].expand(b, length, hk, dk), "k": p["k"][:, :, :1].expand(b, length, hk, dk)}
    check(shared, "one head for all")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("length", [1, 4, 64, 150])
def test_decays_at_their_ends(length, dtype):
    p = inputs(1, length, 1, 2, 64, 32, dtype)
    p["g"][:, :, 0] = 0
    p["g"][:, ::3, 1] = -float("inf")           # forgets everything now and then
    p["g"][:, 1::3, 1] = -500.0
    check(p, "ends")
    p["g"][:, :, 0] = 3.0                       # counts as 0
    check(p, "above")
    p["g"][:] = -100.0
    check(p, "all forgotten")
    p["g"][:] = -1e-8
    p["beta"][:] = 0                            # nothing is ever corrected
    got, new = check(p, "no correction")
    assert torch.allclose(new, p["state"], rtol=1e-5)


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("length", [64, 200])
def test_keys_that_are_all_the_same(length, dtype):
    """The corrections of a chunk then depend on each other as much as they can."""
    p = inputs(1, length, 1, 2, 64, 32, dtype)
    p["k"][:] = p["k"][:, :1]
    p["beta"][..., 0] = 1
    p["g"][..., 0] = 0
    check(p, "same")
    p["beta"][:] = 1.9                          # reflects
    check(p, "reflections")
    p["k"][:] = 0
    check(p, "zero keys")


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")], ids=str)
@pytest.mark.parametrize("length,t", [(1, 0), (3, 1), (64, 63), (64, 0), (130, 70), (130, 64), (130, 5)])
def test_infinities_and_nan_do_not_reach_earlier_tokens_or_other_columns(length, t, bad, dtype):
    p = inputs(2, length, 2, 4, 64, 40, dtype)
    y0, s0 = seq.gated_delta_rule(**p, normalize=True)
    v = p["v"].clone()
    v[1, t, 2, 7] = bad
    y, s = seq.gated_delta_rule(**{**p, "v": v}, normalize=True)
    assert not torch.isfinite(y[1, t:, 2, 7]).any() and not torch.isfinite(s[1, 2, :, 7]).any()
    y[1, t:, 2, 7], s[1, 2, :, 7] = y0[1, t:, 2, 7], s0[1, 2, :, 7]
    assert torch.equal(y, y0) and torch.equal(s, s0)
    for f, at in (("k", (1, t, 1, 3)), ("beta", (1, t, 3)), ("g", (1, t, 3))):
        if f == "g" and bad > 0:
            continue                    # a decay above 0 counts as 0
        w = p[f].clone()
        w[at] = bad
        y, s = seq.gated_delta_rule(**{**p, f: w}, normalize=True)
        heads = [2, 3] if f == "k" else [3]
        for h in heads:
            assert not torch.isfinite(s[1, h]).any() and not torch.isfinite(y[1, t:, h]).any(), f
            y[1, t:, h], s[1, h] = y0[1, t:, h], s0[1, h]
        assert torch.equal(y, y0) and torch.equal(s, s0), f
    q = p["q"].clone()
    q[1, t, 1, 3] = bad
    y, s = seq.gated_delta_rule(**{**p, "q": q}, normalize=True)
    assert not torch.isfinite(y[1, t, 2:]).any() and torch.equal(s, s0)
    y[1, t, 2:] = y0[1, t, 2:]
    assert torch.equal(y, y0)
    state = p["state"].clone()
    state[0, 1, 5, 9] = bad
    y, s = seq.gated_delta_rule(**{**p, "state": state}, normalize=True)
    assert not torch.isfinite(y[0, :, 1, 9]).any() and not torch.isfinite(s[0, 1, :, 9]).all()
    y[0, :, 1, 9], s[0, 1, :, 9] = y0[0, :, 1, 9], s0[0, 1, :, 9]
    assert torch.equal(y, y0) and torch.equal(s, s0)


@pytest.mark.parametrize("length", [1, 100])
def test_many_sequences_and_heads(length):
    p = inputs(9, length, 4, 12, 64, 64, torch.bfloat16)
    check(p)


def test_large_and_small_numbers():
    for size in (1e-12, 1e12):
        p = inputs(1, 100, 1, 1, 64, 32, torch.float32)
        p["v"] *= size
        p["state"] *= size
        got, new = seq.gated_delta_rule(**p, normalize=True)
        y, bound, S, S_bound = reference(p)
        assert (np.abs(f64(got) - y) <= bound + 2.0 ** -24 * np.abs(y)).all() and np.linalg.norm(f64(new) - S) < 2e-6 * np.linalg.norm(S)


def test_nothing_to_do():
    p = inputs(2, 3, 1, 2, 16, 24, torch.bfloat16)
    none = {f: t[:0] for f, t in p.items()}
    assert seq.gated_delta_rule(**none)[0].shape == (0, 3, 2, 24)
    y, new = seq.gated_delta_rule(**{f: t if f == "state" else t[:, :0] for f, t in p.items()})
    assert y.shape == (2, 0, 2, 24) and torch.equal(new, p["state"])
    y, new = seq.gated_delta_rule(**{f: t[:, :0] for f, t in p.items() if f != "state"})
    assert not new.any()
    y, new = seq.gated_delta_rule(**{**p, "v": p["v"][..., :0], "state": p["state"][..., :0]})
    assert y.shape == (2, 3, 2, 0) and new.shape == (2, 2, 16, 0)


def test_what_does_not_fit_is_refused():
    p = inputs(2, 3, 2, 4, 32, 24, torch.bfloat16)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    wide = torch.zeros(2, 3, 2, 257, device="cuda", dtype=torch.bfloat16)
    for change in (dict(q=p["q"][:, :2]), dict(k=p["k"][:1]), dict(k=p["k"][..., :31]), dict(k=p["k"].half()), dict(q=p["q"].transpose(2, 3)), dict(v=p["v"][:, :, :3]), dict(v=p["v"].float()),
                   dict(g=p["g"].half()), dict(g=p["g"][..., :3]), dict(g=p["g"].transpose(1, 2)), dict(beta=p["beta"].double()), dict(beta=p["beta"][:1]), dict(state=p["state"].half()),
                   dict(state=p["state"][:1]), dict(state=p["state"].transpose(2, 3).contiguous()), dict(state=p["state"].transpose(2, 3).contiguous().transpose(2, 3)), dict(lengths=i32(1)),
                   dict(lengths=torch.tensor([1, 2], device="cuda")), dict(slots=i32(0)), dict(slots=i32(0, 1), state=None), dict(new_state=p["state"][:, :2]), dict(out=p["v"]), dict(out=p["v"].float()),
                   dict(new_state=p["state"].view(-1)[1:].new_zeros(2, 4, 32, 24).half()), dict(q=wide, k=wide, state=None), dict(q=p["q"][:, :, :0], k=p["k"][:, :, :0]), dict(scale=float("inf")),
                   dict(scale=float("nan")), dict(q=p["q"].cpu()), dict(v=p["v"].cpu()), dict(q=p["q"].clone().requires_grad_()), dict(state=p["state"].clone().requires_grad_()),
                   dict(out=torch.zeros(2, 4, 3, 24, device="cuda", dtype=torch.bfloat16).transpose(1, 2)), dict(out=torch.zeros(1, 1, 4, 24, device="cuda", dtype=torch.bfloat16).expand(2, 3, 4, 24))):
        with pytest.raises(XlError):
            seq.gated_delta_rule(**{**p, **change})
    half = torch.zeros(3, 4, 32, 24, device="cuda")
    with pytest.raises(XlError, match="shares memory"):
        seq.gated_delta_rule(**{**p, "state": half[:2]}, new_state=half[1:])
    with pytest.raises(XlError, match="heads of out"):
        seq.gated_delta_rule(**p, out=torch.zeros(2, 3, 4, 48, device="cuda", dtype=torch.bfloat16)[..., :24])
