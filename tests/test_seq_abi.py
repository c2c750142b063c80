"""CPU checks of the sequence operators: the library's exports, the argument structs, what is refused, and the definitions they are tested against."""
import ctypes
import os
import re
import struct

import numpy as np
import pytest
import torch

from oracle import seq as ref
from paper_2007_06000_amd import binding as B
from paper_2007_06000_amd import seq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "xl_seq.h")).read()


def fields(name):
    """[(field, 'q' for a number, 'Q' for a pointer)] of a struct of the header."""
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), HEADER, re.S)[1], flags=re.S)
    out = []
    for decl in filter(str.strip, body.split(";")):
        pointer = "*" in decl
        names = re.sub(r"\b(const|void|float|int|long)\b|\*", " ", decl)
        out += [(n.strip(), "Q" if pointer else "q") for n in names.split(",")]
    return out


# the argument structs: 64-bit numbers, then pointers
STRUCTS = {"xl_causal_conv": ("xl_causal_conv_args", struct.Struct("=11q8Q")), "xl_selective_scan": ("xl_scan_args", struct.Struct("=20q14Q")),
           "xl_quantize_blocks": ("xl_quantize_args", struct.Struct("=8q3Q")), "xl_block_matmul": ("xl_block_matmul_args", struct.Struct("=11q6Q"))}


def call(name, **values):
    """The status of one call with the given fields, everything else 0."""
    args, layout = STRUCTS[name]
    names = [f for f, _ in fields(args)]
    assert set(values) <= set(names)
    return getattr(seq.lib(), name)(layout.pack(*[values.get(f, 0) for f in names]), None), seq.lib().xl_seq_last_error().decode()


def test_library_exports_every_declared_symbol():
    assert set(re.findall(r"\b(xl_[a-z_]+)\s*\(", HEADER)) == set(seq.EXPORTS)
    lib = ctypes.CDLL(seq.LIB_PATH)
    for name in seq.EXPORTS:
        assert hasattr(lib, name), name


@pytest.mark.parametrize("name", STRUCTS)
def test_packed_arguments_have_the_layout_of_the_structs(name):
    args, layout = STRUCTS[name]
    kinds = [k for _, k in fields(args)]
    assert kinds == sorted(kinds, key="qQ".index)
    assert layout.format == "=%dq%dQ" % (kinds.count("q"), kinds.count("Q")) and layout.size == 8 * len(kinds)


P = 1 << 20         # stands for a pointer: nothing here gets as far as reading through it
CONV = dict(batch=2, length=3, channels=8, taps=4, dtype=seq.XL_BF16, x_batch=24, x_token=8, y_batch=24, y_token=8, nslots=2, x=P, weight=P, y=P)
SCAN = dict(batch=2, length=3, channels=8, states=16, dtype=seq.XL_BF16, u_batch=24, u_token=8, delta_batch=24, delta_token=8, y_batch=24, y_token=8,
            b_batch=48, b_token=16, c_batch=48, c_token=16, nslots=2, u=P, delta=P, A=P, B=P, C=P, y=P)
QUANT = dict(rows=3, k=40, block_rows=1, dtype=seq.XL_BF16, x_row=40, q_row=48, scale_row=1, scale_block=3, x=P, q=P, scales=P)
MATMUL = dict(m=3, n=5, k=40, dtype=seq.XL_BF16, a_row=48, b_row=48, a_scale_row=1, a_scale_block=1, b_scale_row=1, b_scale_block=1, y_row=5, a=P, b=P,
              a_scales=P, b_scales=P, y=P)
BASE = {"xl_causal_conv": CONV, "xl_selective_scan": SCAN, "xl_quantize_blocks": QUANT, "xl_block_matmul": MATMUL}
REFUSED = [
    ("xl_causal_conv", B.XL_E_NULL, dict(x=0)), ("xl_causal_conv", B.XL_E_NULL, dict(y=0)), ("xl_causal_conv", B.XL_E_NULL, dict(weight=0)),
    ("xl_causal_conv", B.XL_E_UNSUPPORTED, dict(taps=1)), ("xl_causal_conv", B.XL_E_UNSUPPORTED, dict(taps=5)), ("xl_causal_conv", B.XL_E_UNSUPPORTED, dict(dtype=3)),
    ("xl_causal_conv", B.XL_E_SHAPE, dict(batch=-1)), ("xl_causal_conv", B.XL_E_SHAPE, dict(length=1 << 31)), ("xl_causal_conv", B.XL_E_SHAPE, dict(channels=-8)),
    ("xl_causal_conv", B.XL_E_SHAPE, dict(batch=1 << 20, length=1 << 20, channels=1 << 20)), ("xl_causal_conv", B.XL_E_SHAPE, dict(x_token=-8)),
    ("xl_causal_conv", B.XL_E_SHAPE, dict(y_token=7)), ("xl_causal_conv", B.XL_E_SHAPE, dict(y_batch=0)), ("xl_causal_conv", B.XL_E_SHAPE, dict(nslots=1, state=P)),
    ("xl_causal_conv", B.XL_E_SHAPE, dict(nslots=-1, new_state=P, slots=P)), ("xl_causal_conv", B.XL_E_ALIGN, dict(x=P + 1)), ("xl_causal_conv", B.XL_E_ALIGN, dict(bias=P + 2)),
    ("xl_causal_conv", B.XL_E_ALIGN, dict(state=P + 1)), ("xl_causal_conv", B.XL_E_ALIGN, dict(lengths=P + 2)),
    ("xl_selective_scan", B.XL_E_NULL, dict(u=0)), ("xl_selective_scan", B.XL_E_NULL, dict(delta=0)), ("xl_selective_scan", B.XL_E_NULL, dict(A=0)),
    ("xl_selective_scan", B.XL_E_NULL, dict(B=0)), ("xl_selective_scan", B.XL_E_NULL, dict(C=0)), ("xl_selective_scan", B.XL_E_NULL, dict(y=0)),
    ("xl_selective_scan", B.XL_E_UNSUPPORTED, dict(states=0)), ("xl_selective_scan", B.XL_E_UNSUPPORTED, dict(states=129)), ("xl_selective_scan", B.XL_E_UNSUPPORTED, dict(dtype=-1)),
    ("xl_selective_scan", B.XL_E_SHAPE, dict(delta_token=-1)), ("xl_selective_scan", B.XL_E_SHAPE, dict(y_token=4)), ("xl_selective_scan", B.XL_E_SHAPE, dict(z=P, z_batch=-1)),
    ("xl_selective_scan", B.XL_E_SHAPE, dict(nslots=1, new_state=P)), ("xl_selective_scan", B.XL_E_ALIGN, dict(state=P + 2)), ("xl_selective_scan", B.XL_E_ALIGN, dict(C=P + 1)),
    ("xl_selective_scan", B.XL_E_ALIGN, dict(z=P + 1)), ("xl_selective_scan", B.XL_E_ALIGN, dict(workspace=P + 8)), ("xl_selective_scan", B.XL_E_ALIGN, dict(D=P + 2)),
    ("xl_quantize_blocks", B.XL_E_NULL, dict(x=0)), ("xl_quantize_blocks", B.XL_E_NULL, dict(q=0)), ("xl_quantize_blocks", B.XL_E_NULL, dict(scales=0)),
    ("xl_quantize_blocks", B.XL_E_UNSUPPORTED, dict(block_rows=2)), ("xl_quantize_blocks", B.XL_E_UNSUPPORTED, dict(dtype=7)), ("xl_quantize_blocks", B.XL_E_SHAPE, dict(rows=-1)),
    ("xl_quantize_blocks", B.XL_E_SHAPE, dict(q_row=32)), ("xl_quantize_blocks", B.XL_E_SHAPE, dict(scale_block=-1)), ("xl_quantize_blocks", B.XL_E_SHAPE, dict(x_row=-40)),
    ("xl_quantize_blocks", B.XL_E_ALIGN, dict(q=P + 8)), ("xl_quantize_blocks", B.XL_E_ALIGN, dict(q_row=40)), ("xl_quantize_blocks", B.XL_E_ALIGN, dict(x=P + 1)),
    ("xl_block_matmul", B.XL_E_NULL, dict(a=0)), ("xl_block_matmul", B.XL_E_NULL, dict(b=0)), ("xl_block_matmul", B.XL_E_NULL, dict(a_scales=0)),
    ("xl_block_matmul", B.XL_E_NULL, dict(b_scales=0)), ("xl_block_matmul", B.XL_E_NULL, dict(y=0)), ("xl_block_matmul", B.XL_E_UNSUPPORTED, dict(dtype=9)),
    ("xl_block_matmul", B.XL_E_SHAPE, dict(m=-1)), ("xl_block_matmul", B.XL_E_SHAPE, dict(n=1 << 32)), ("xl_block_matmul", B.XL_E_SHAPE, dict(a_row=32)),
    ("xl_block_matmul", B.XL_E_SHAPE, dict(b_row=16)), ("xl_block_matmul", B.XL_E_SHAPE, dict(y_row=4)), ("xl_block_matmul", B.XL_E_SHAPE, dict(a_scale_row=-1)),
    ("xl_block_matmul", B.XL_E_ALIGN, dict(a=P + 8)), ("xl_block_matmul", B.XL_E_ALIGN, dict(b_row=40)), ("xl_block_matmul", B.XL_E_ALIGN, dict(y=P + 1)),
    ("xl_block_matmul", B.XL_E_ALIGN, dict(a_scales=P + 2)),
]


@pytest.mark.parametrize("name,status,change", REFUSED, ids=lambda v: str(v))
def test_what_does_not_fit_is_refused(name, status, change):
    st, message = call(name, **{**BASE[name], **change})
    assert st == status and message.startswith(name[3:])


@pytest.mark.parametrize("name,empty", [("xl_causal_conv", dict(batch=0)), ("xl_causal_conv", dict(channels=0)), ("xl_causal_conv", dict(length=0, x=0, y=0)),
                                        ("xl_selective_scan", dict(batch=0)), ("xl_selective_scan", dict(length=0, u=0, delta=0, y=0)), ("xl_quantize_blocks", dict(rows=0, x=0)),
                                        ("xl_quantize_blocks", dict(k=0)), ("xl_block_matmul", dict(m=0, a=0)), ("xl_block_matmul", dict(n=0))], ids=str)
def test_nothing_to_do_is_no_error(name, empty):
    assert call(name, **{**BASE[name], **empty})[0] == B.XL_OK


def test_a_scan_asks_for_a_workspace_where_it_can_use_one():
    names = [f for f, _ in fields("xl_scan_args")]

    def ask(**sizes):
        return seq.lib().xl_selective_scan_workspace(STRUCTS["xl_selective_scan"][1].pack(*[{**SCAN, **sizes}.get(f, 0) for f in names]))

    few = ask(batch=1, length=12321, channels=256, states=16)
    assert few > 0 and few % 16 == 0 and few % (2 * 4 * 256 * 16) == 0
    assert ask(batch=1, length=12321, channels=250, states=13) > 0
    assert not ask(batch=1, length=1, channels=256, states=16) and not ask(batch=64, length=12321, channels=4096, states=16)
    for bad in (dict(batch=-1), dict(length=1 << 40), dict(channels=1 << 62), dict(states=0), dict(states=129), dict(batch=0), dict(batch=1 << 30, channels=1 << 30)):
        assert ask(**{**dict(batch=1, length=12321, channels=256, states=16), **bad}) == 0
    assert seq.lib().xl_selective_scan_workspace(None) == 0


@pytest.mark.parametrize("name", STRUCTS)
def test_no_arguments_at_all(name):
    assert getattr(seq.lib(), name)(None, None) == B.XL_E_NULL


def test_tensors_on_the_cpu_are_refused():
    x = torch.zeros(1, 2, 8)
    for f in (lambda: seq.causal_conv(x, torch.zeros(8, 4)), lambda: seq.selective_scan(x, x, torch.zeros(8, 16), torch.zeros(1, 2, 16), torch.zeros(1, 2, 16)),
              lambda: seq.quantize_rows(x[0]), lambda: seq.quantize_weight(x[0])):
        with pytest.raises(B.XlError) as e:
            f()
        assert e.value.status == B.XL_E_DEVICE


def test_the_definitions_agree_with_torch_in_64_bits():
    g = np.random.default_rng(0)
    x, w, bias = g.standard_normal((2, 9, 5)), g.standard_normal((5, 3)), g.standard_normal(5)
    y, _, new = ref.causal_conv(x, w, bias, None, [9, 9], True)
    t = torch.nn.functional.conv1d(torch.from_numpy(x).transpose(1, 2), torch.from_numpy(w)[:, None], torch.from_numpy(bias), padding=2, groups=5)[:, :, :9]
    assert np.allclose(y, torch.nn.functional.silu(t).transpose(1, 2).numpy(), atol=1e-12) and np.array_equal(new, x[:, 7:])
    # a scan with a constant step and A = 0 is a running sum
    u, B1 = g.standard_normal((1, 7, 3)), np.ones((1, 7, 1))
    y, bound, h, _ = ref.selective_scan(u, np.full_like(u, 0.5), np.zeros((3, 1)), B1, B1, None, None, np.zeros(3), None, [7], False)
    assert np.allclose(y, 0.5 * u.cumsum(1)) and np.allclose(h[0, :, 0], y[0, -1]) and (bound < 1e-5).all()
    q, s = ref.quantize(np.array([[448.0, 1.0, -2.0], [0.0, 0.0, 0.0]]), 1)
    assert np.array_equal(q, [[448, 1, -2], [0, 0, 0]]) and s[0, 0] == 1 and s[1, 0] == np.float32(2.0 ** -126)
    a, b = g.standard_normal((3, 200)), g.standard_normal((130, 200))
    ones = np.ones
    y, mag = ref.block_matmul(a, ones((3, 2)), b, ones((2, 2)), np.zeros(130))
    assert np.allclose(y, a @ b.T) and (mag >= np.abs(y)).all()
