"""Low-rank adapters beside a shared projection against their definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import seq
from paper_2007_06000_amd.binding import XlError
from test_gpu_seq_conv import HALF, f64, near

pytestmark = pytest.mark.gpu


def inputs(batch, length, k, n, rank, adapters, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    index = torch.randint(0, adapters, (batch,), generator=g, dtype=torch.int32)
    return {"y": r(batch, length, n).to(dtype).cuda(), "x": r(batch, length, k).to(dtype).cuda(), "down": (r(adapters, rank, k) * k ** -0.5).to(dtype).cuda(),
            "up": r(adapters, n, rank).to(dtype).cuda(), "index": index.cuda(), "scales": (0.5 + torch.rand(adapters, generator=g)).cuda()}


def check(p, got, what, lengths=None):
    length = p["x"].shape[1]
    n = [length] * p["x"].shape[0] if lengths is None else [min(max(int(v), 0), length) for v in lengths]
    # what lies past a sequence's end is never read
    live = torch.arange(length)[None, :, None] < torch.tensor(n)[:, None, None]
    clean = {f: torch.where(live, p[f].cpu(), torch.zeros((), dtype=p[f].dtype)) for f in ("x", "y")}
    want, bound = ref.add_adapters(f64(clean["y"]), f64(clean["x"]), f64(p["down"]), f64(p["up"]), f64(p.get("scales")), p["index"].tolist(), n, p["y"].dtype != torch.float32)
    near(got, want, bound, what)


SIZES = [  # batch, length, k, n, rank, adapters
    (1, 1, 1, 1, 1, 1), (3, 1, 64, 64, 8, 2), (32, 1, 256, 512, 16, 40), (5, 1, 100, 77, 3, 4), (2, 2, 520, 1000, 13, 3), (7, 5, 33, 130, 5, 2), (2, 17, 128, 96, 32, 3), (1, 64, 512, 256, 64, 1),
    (3, 65, 200, 300, 128, 2), (1, 200, 1024, 160, 16, 1), (4, 130, 72, 520, 127, 2), (2, 300, 48, 16, 1, 2), (16, 3, 1000, 640, 20, 5), (1, 1, 4096, 4096, 16, 1), (2, 33, 31, 17, 96, 2),
    (260, 17, 40, 72, 4, 7), (1, 4200, 600, 100, 16, 1), (2, 2100, 72, 264, 40, 2), (5, 900, 1100, 40, 7, 3), (3, 1500, 33, 65, 100, 2), (300, 18, 8, 30, 20, 2)]


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(size, dtype):
    p = inputs(*size, dtype, seed=sum(size))
    check(p, seq.add_adapters(**p), "scales")
    p.pop("scales")
    check(p, seq.add_adapters(**p), "no scales")


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("length", [1, 9, 150, 800])
def test_sequences_without_an_adapter_keep_their_projection(length, dtype):
    p = inputs(6, length, 96, 200, 24, 3, dtype)
    p["index"] = torch.tensor([0, -1, 2, 3, 1 << 30, -(1 << 31)], dtype=torch.int32, device="cuda")
    p["x"][1] = float("nan")            # nobody asks for it
    got = seq.add_adapters(**p)
    for b in (1, 3, 4, 5):
        assert torch.equal(got[b], p["y"][b])
    p["x"][1] = 0
    check(p, got, "absent")


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("lengths", [[0, 1, 2, 63, 150], [150, 0, -5, 1000, 149], [0, 0, 0, 0, 0], [64, 65, 128, 16, 17]])
@pytest.mark.parametrize("length", [150, 1000])        # in one kernel, in two
def test_sequences_of_their_own_lengths(length, lengths, dtype):
    p = inputs(5, length, 80, 144, 16, 2, dtype)
    for b, n in enumerate(lengths):
        p["x"][b, max(n, 0):] = float("nan")
        p["y"][b, max(n, 0):] = float("nan")
    got = seq.add_adapters(**p, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    check(p, got, "lengths", lengths)
    for b, n in enumerate(lengths):
        assert not got[b, max(n, 0):].any()


@pytest.mark.parametrize("length", [1, 12, 140, 1500])
def test_views_odd_addresses_and_in_place(length):
    g = torch.Generator().manual_seed(1)
    wide = torch.randn(3, length, 300, generator=g).bfloat16().cuda()
    base = inputs(3, length, 101, 99, 12, 2, torch.bfloat16)
    p = {**base, "x": wide[:, :, 1:102], "y": wide[:, :, 150:249]}
    whole = {**p, "x": p["x"].contiguous(), "y": p["y"].contiguous()}
    want = seq.add_adapters(**whole)
    check(whole, want, "contiguous")
    near(seq.add_adapters(**p), f64(want), 2.0 ** -7 * np.abs(f64(want)), "views")      # a step: the order of the sums may differ
    kept = wide.clone()
    out = seq.add_adapters(**p, out=p["y"])
    assert out is p["y"] and torch.equal(wide[:, :, :150], kept[:, :, :150]) and torch.equal(wide[:, :, 249:], kept[:, :, 249:])
    check(whole, out, "in place")
    turned = inputs(length, 3, 101, 99, 12, 2, torch.bfloat16)
    q = {**turned, "x": turned["x"].transpose(0, 1).contiguous().transpose(0, 1), "y": turned["y"].transpose(0, 1).contiguous().transpose(0, 1)}
    check(turned, seq.add_adapters(**q), "tokens in front")


@pytest.mark.parametrize("dtype", list(HALF), ids=str)
@pytest.mark.parametrize("length", [1, 100, 2100])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")], ids=str)
def test_infinities_and_nan_stay_in_their_row(length, bad, dtype):
    p = inputs(2, length, 70, 90, 9, 2, dtype)
    want = seq.add_adapters(**p)
    t = length // 2
    p["x"][1, t, 33] = bad
    got = seq.add_adapters(**p)
    assert not torch.isfinite(got[1, t]).any()
    got[1, t] = want[1, t]
    assert torch.equal(got, want)
    p["x"][1, t, 33] = 0
    p["y"][0, t, 5] = bad
    got = seq.add_adapters(**p)
    assert not torch.isfinite(got[0, t, 5]) and torch.isfinite(got[0, t, :5]).all() and torch.isfinite(got[0, t, 6:]).all()


def test_a_state_of_large_numbers_in_16_bits():
    """down x beyond the range of fp16 between two fp16 factors."""
    p = inputs(2, 40, 64, 64, 8, 2, torch.float16)
    p["x"] *= 1000
    p["down"] *= 1000
    p["up"] *= 1e-4
    check(p, seq.add_adapters(**p), "large")


def test_nothing_to_do():
    p = inputs(2, 3, 16, 24, 4, 2, torch.bfloat16)
    none = {**p, "y": p["y"][:0], "x": p["x"][:0], "index": p["index"][:0]}
    assert seq.add_adapters(**none).shape == (0, 3, 24)
    assert seq.add_adapters(**{**p, "y": p["y"][:, :0], "x": p["x"][:, :0]}).shape == (2, 0, 24)
    assert seq.add_adapters(**{**p, "y": p["y"][:, :, :0], "up": p["up"][:, :0]}).shape == (2, 3, 0)
    assert torch.equal(seq.add_adapters(**{**p, "x": p["x"][:, :, :0], "down": p["down"][:, :, :0]}), p["y"])
    assert torch.equal(seq.add_adapters(**{**p, "down": p["down"][:0], "up": p["up"][:0], "scales": p["scales"][:0]}), p["y"])


def test_what_does_not_fit_is_refused():
    p = inputs(3, 4, 32, 48, 8, 2, torch.bfloat16)
    for change in (dict(x=p["x"][:2]), dict(x=p["x"][:, :3]), dict(x=p["x"].half()), dict(x=p["x"][..., ::2]), dict(down=p["down"][:, :, :31]), dict(down=p["down"][0]), dict(up=p["up"][:, :, :7]),
                   dict(up=p["up"][:1]), dict(up=p["up"].float()), dict(index=p["index"].long()), dict(index=p["index"][:2]), dict(scales=p["scales"].half()), dict(scales=p["scales"][:1]),
                   dict(lengths=p["index"][:2]), dict(out=p["y"].float()), dict(out=p["y"][:2]), dict(out=p["x"].repeat(1, 1, 2)[:, :, :48].transpose(0, 1)),
                   dict(down=torch.zeros(2, 129, 32, device="cuda", dtype=torch.bfloat16), up=torch.zeros(2, 48, 129, device="cuda", dtype=torch.bfloat16)),
                   dict(down=torch.zeros(2, 0, 32, device="cuda", dtype=torch.bfloat16), up=torch.zeros(2, 48, 0, device="cuda", dtype=torch.bfloat16)),
                   dict(y=p["y"].cpu()), dict(x=p["x"].cpu()), dict(x=p["x"].clone().requires_grad_()), dict(out=p["y"].view(-1)[:48].expand(3, 4, 48))):
        with pytest.raises(XlError):
            seq.add_adapters(**{**p, **change})
    square = inputs(3, 4, 32, 32, 8, 2, torch.bfloat16)
    for out in (square["x"], square["down"].view(-1)[:384].view(3, 4, 32)):
        with pytest.raises(XlError, match="shares memory"):
            seq.add_adapters(**square, out=out)
