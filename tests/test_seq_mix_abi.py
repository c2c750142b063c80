"""CPU checks of the operators around a projection: argument structs, what is refused, host code under sanitizers, and the definitions they are tested against."""
import os
import re
import struct
import subprocess

import numpy as np
import pytest
import torch
from test_sanitizers import CLANG, ENV, HERE, OUT, ROOT, SAN

from oracle import seq as ref
from paper_2007_06000_amd import binding as B
from paper_2007_06000_amd import seq

HEADER = open(os.path.join(ROOT, "include", "xl_seq.h")).read()
# 64-bit numbers, a double where there is one, then pointers
STRUCTS = {"xl_rms_norm": ("xl_rms_norm_args", struct.Struct("=11q1d6Q")), "xl_add_adapters": ("xl_adapters_args", struct.Struct("=14q9Q")),
           "xl_gated_delta_rule": ("xl_delta_args", struct.Struct("=26q1d11Q"))}


def fields(name):
    """[(field, 'q' for a number, 'd' for a double, 'Q' for a pointer)] of a struct of the header."""
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), HEADER, re.S)[1], flags=re.S)
    out = []
    for decl in filter(str.strip, body.split(";")):
        kind = "Q" if "*" in decl else "d" if "double" in decl else "q"
        out += [(n.strip(), kind) for n in re.sub(r"\b(const|void|float|double|int|long)\b|\*", " ", decl).split(",")]
    return out


def pack(name, values):
    args, layout = STRUCTS[name]
    names = [f for f, _ in fields(args)]
    assert set(values) <= set(names), set(values) - set(names)
    return layout.pack(*[values.get(f, 0) for f in names])


def call(name, **values):
    return getattr(seq.lib(), name)(pack(name, values), None), seq.lib().xl_seq_last_error().decode()


@pytest.mark.parametrize("name", STRUCTS)
def test_packed_arguments_have_the_layout_of_the_structs(name):
    args, layout = STRUCTS[name]
    kinds = "".join(k for _, k in fields(args))
    assert kinds == "q" * kinds.count("q") + "d" * kinds.count("d") + "Q" * kinds.count("Q")
    assert layout.format == "=" + "".join("%d%s" % (kinds.count(k), k) for k in "qdQ" if k in kinds) and layout.size == 8 * len(kinds)


P = 1 << 20         # stands for a pointer: nothing here gets as far as reading through it
NORM = dict(rows=3, k=40, dtype=seq.XL_BF16, residual_dtype=seq.XL_F32, x_row=40, residual_row=40, new_residual_row=40, y_row=40, eps=1e-6, x=P, residual=P, new_residual=P, weight=P, y=P)
QNORM = dict(NORM, quantized=1, y_row=48, scale_row=1, scale_block=3, scales=P)
ADAPT = dict(batch=2, length=3, k=8, n=16, rank=4, adapters=2, dtype=seq.XL_BF16, x_batch=24, x_token=8, y_batch=48, y_token=16, out_batch=48, out_token=16, workspace_bytes=1 << 40, x=P, y=P,
             down=P, up=P, index=P, out=P, workspace=P)
DELTA = dict(batch=2, length=3, key_heads=1, heads=2, dk=8, dv=4, dtype=seq.XL_BF16, q_batch=24, q_token=8, q_head=8, k_batch=24, k_token=8, k_head=8, v_batch=24, v_token=8, v_head=4, y_batch=24,
             y_token=8, y_head=4, g_batch=6, g_token=2, beta_batch=6, beta_token=2, nslots=2, workspace_bytes=1 << 40, scale=1.0, q=P, k=P, v=P, g=P, beta=P, y=P, workspace=P)
BASE = {"xl_rms_norm": NORM, "xl_add_adapters": ADAPT, "xl_gated_delta_rule": DELTA}
NULL, SHAPE, ALIGN, UNSUPPORTED = B.XL_E_NULL, B.XL_E_SHAPE, B.XL_E_ALIGN, B.XL_E_UNSUPPORTED
REFUSED = [
    *[("xl_rms_norm", NULL, {f: 0}) for f in ("x", "weight", "y")], ("xl_rms_norm", NULL, {**QNORM, "scales": 0}), ("xl_rms_norm", UNSUPPORTED, dict(dtype=3)),
    ("xl_rms_norm", UNSUPPORTED, dict(residual_dtype=seq.XL_F16)), ("xl_rms_norm", UNSUPPORTED, dict(residual_dtype=9)), ("xl_rms_norm", SHAPE, dict(rows=-1)), ("xl_rms_norm", SHAPE, dict(k=1 << 31)),
    ("xl_rms_norm", SHAPE, dict(rows=1 << 30, k=1 << 20)), *[("xl_rms_norm", SHAPE, dict(eps=e)) for e in (0.0, -1.0, 1e-39, 1e39, float("nan"), float("inf"))],
    ("xl_rms_norm", SHAPE, dict(x_row=-1)), ("xl_rms_norm", SHAPE, dict(residual_row=-40)), ("xl_rms_norm", SHAPE, dict(new_residual_row=39)), ("xl_rms_norm", SHAPE, dict(y_row=39)),
    ("xl_rms_norm", SHAPE, {**QNORM, "scale_block": -1}), ("xl_rms_norm", SHAPE, {**QNORM, "scale_row": -1}), ("xl_rms_norm", SHAPE, {**QNORM, "y_row": 32}), ("xl_rms_norm", ALIGN, {**QNORM, "y_row": 40}),
    ("xl_rms_norm", ALIGN, {**QNORM, "y": P + 8}), ("xl_rms_norm", ALIGN, {**QNORM, "scales": P + 2}), ("xl_rms_norm", ALIGN, dict(x=P + 1)), ("xl_rms_norm", ALIGN, dict(weight=P + 2)),
    ("xl_rms_norm", ALIGN, dict(residual=P + 2)), ("xl_rms_norm", ALIGN, dict(new_residual=P + 2)), ("xl_rms_norm", ALIGN, dict(y=P + 1)),
    *[("xl_add_adapters", NULL, {f: 0}) for f in ("x", "y", "down", "up", "index", "out")], *[("xl_add_adapters", UNSUPPORTED, c) for c in (dict(dtype=3), dict(rank=0), dict(rank=129), dict(rank=-1))],
    *[("xl_add_adapters", SHAPE, c) for c in (dict(batch=-1), dict(length=1 << 31), dict(k=-1), dict(n=1 << 40), dict(adapters=-1), dict(batch=1 << 20, length=1 << 20), dict(adapters=1 << 30, k=1 << 20),
                                              dict(x_token=-1), dict(y_batch=-1), dict(out_token=15), dict(out_batch=8))],
    *[("xl_add_adapters", ALIGN, {f: P + 1}) for f in ("x", "y", "down", "up", "index", "scales", "lengths", "out", "workspace")],
    *[("xl_gated_delta_rule", NULL, {f: 0}) for f in ("q", "k", "v", "g", "beta", "y")], *[("xl_gated_delta_rule", UNSUPPORTED, c) for c in (dict(dtype=3), dict(dk=0), dict(dk=257), dict(dk=-1))],
    *[("xl_gated_delta_rule", SHAPE, c) for c in (dict(batch=-1), dict(length=1 << 31), dict(heads=-2), dict(heads=3, key_heads=2), dict(key_heads=0), dict(key_heads=-1), dict(dv=-1), dict(dv=1 << 40),
                                                  dict(batch=1 << 20, length=1 << 20), dict(q_token=-1), dict(k_batch=-1), dict(k_head=-1, key_heads=2), dict(v_head=-4), dict(y_head=3), dict(y_token=3),
                                                  dict(g_token=-1), dict(beta_batch=-1), dict(nslots=1, state=P), dict(nslots=-1, state=P, slots=P), dict(scale=float("nan")), dict(scale=float("inf")),
                                                  dict(scale=1e39))],
    *[("xl_gated_delta_rule", ALIGN, {f: P + 1}) for f in ("q", "k", "v", "g", "beta", "state", "new_state", "lengths", "slots", "y", "workspace")]]


@pytest.mark.parametrize("name,status,change", REFUSED, ids=lambda v: str(v))
def test_what_does_not_fit_is_refused(name, status, change):
    st, message = call(name, **{**BASE[name], **change})
    assert st == status and message.startswith(name[3:])


@pytest.mark.parametrize("name,empty", [("xl_rms_norm", dict(rows=0, x=0)), ("xl_rms_norm", dict(k=0, weight=0)), ("xl_add_adapters", dict(batch=0, index=0)), ("xl_add_adapters", dict(length=0, x=0)),
                                        ("xl_add_adapters", dict(n=0, up=0)), ("xl_gated_delta_rule", dict(batch=0)), ("xl_gated_delta_rule", dict(heads=0)), ("xl_gated_delta_rule", dict(dv=0, v=0)),
                                        ("xl_gated_delta_rule", dict(length=0, q=0, k=0, v=0, y=0))], ids=str)
def test_nothing_to_do_is_no_error(name, empty):
    assert call(name, **{**BASE[name], **empty})[0] == B.XL_OK


@pytest.mark.parametrize("name", STRUCTS)
def test_no_arguments_at_all(name):
    assert getattr(seq.lib(), name)(None, None) == B.XL_E_NULL


@pytest.mark.parametrize("name", ["xl_add_adapters", "xl_gated_delta_rule"])
def test_a_workspace_is_asked_for_within_bounds(name):
    def ask(**sizes):
        return getattr(seq.lib(), name + "_workspace")(pack(name, {**BASE[name], **sizes}))

    assert getattr(seq.lib(), name + "_workspace")(None) == 0
    assert ask(batch=0) == 0 and ask(length=0) == 0
    for sizes in (dict(length=1), dict(length=100), dict(length=12321), dict(batch=300, length=700)):
        need = ask(**sizes)
        assert 0 <= need < 1 << 40 and need % 16 == 0
        if need:
            assert call(name, **{**BASE[name], **sizes, "workspace": 0})[0] == B.XL_E_NULL
            assert call(name, **{**BASE[name], **sizes, "workspace_bytes": need - 1})[0] == B.XL_E_NULL
    for bad in (dict(batch=-1), dict(length=1 << 40), dict(batch=1 << 30, length=1 << 30), dict(dtype=7)):
        assert ask(**bad) == 0


def test_tensors_on_the_cpu_are_refused():
    x = torch.zeros(2, 3, 8)
    for f in (lambda: seq.rms_norm(x[0], x[0, 0]), lambda: seq.rms_norm_quantized(x[0], x[0, 0]), lambda: seq.add_adapters(x, x, x, x, torch.zeros(2, dtype=torch.int32)),
              lambda: seq.gated_delta_rule(x[:, :, None], x[:, :, None], x[:, :, None], x[..., :1], x[..., :1])):
        with pytest.raises(B.XlError) as e:
            f()
        assert e.value.status == B.XL_E_DEVICE


def test_c_abi_under_address_and_undefined_behaviour_sanitizers():
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ with sanitizer runtimes in this image")
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "seq_mix_asan")
    csrc = os.path.join(ROOT, "paper_2007_06000_amd", "csrc")
    cmd = [CLANG, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + csrc, *SAN,
           os.path.join(csrc, "seq_api.cpp"), os.path.join(csrc, "seq_mix_api.cpp"), os.path.join(HERE, "seq_mix_asan.cpp"), "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, env=ENV, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "ERROR: AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-4000:]


def test_the_definitions_say_what_the_formulas_say():
    g = np.random.default_rng(0)
    x, r, w = g.standard_normal((3, 10)), g.standard_normal((3, 10)), g.standard_normal(10)
    y, _, s = ref.rms_norm(x, r, w, 0.25)
    assert np.array_equal(s, x + r) and np.allclose((y / w) ** 2 * (np.mean(s ** 2, 1, keepdims=True) + 0.25), s ** 2)
    # an adapter is a matrix of low rank
    y, x, down, up = g.standard_normal((2, 4, 6)), g.standard_normal((2, 4, 5)), g.standard_normal((3, 2, 5)), g.standard_normal((3, 6, 2))
    out, _ = ref.add_adapters(y, x, down, up, np.array([1.0, 2.0, 3.0]), [2, -1], [4, 3], False)
    assert np.allclose(out[0], y[0] + 3 * np.einsum("tk,nk->tn", x[0], up[2] @ down[2])) and np.array_equal(out[1, :3], y[1, :3]) and not out[1, 3].any()
    # without forgetting and with orthogonal keys of length one, a step of one stores a value that its key reads back
    n, d = 6, 5
    k = np.linalg.qr(g.standard_normal((n, n)))[0][None, :, None]
    v = g.standard_normal((1, n, 1, d))
    zeros, ones = np.zeros((1, n, 1)), np.ones((1, n, 1))
    y, bound, S, _ = ref.gated_delta_rule(k, k, v, zeros, ones, 1.0, False, None, [n], False)
    assert np.allclose(y, v) and np.allclose(np.einsum("ij,ti->tj", S[0, 0], k[0, :, 0]), v[0, :, 0]) and (bound < 1e-3).all()
    # the same as a product of matrices: S_t = e^g (I - beta k k^T) S + beta k v^T
    q, k, v = g.standard_normal((1, n, 1, 4)), g.standard_normal((1, n, 1, 4)), g.standard_normal((1, n, 2, d))
    gate, beta, S0 = -g.random((1, n, 2)), g.random((1, n, 2)), g.standard_normal((1, 2, 4, d))
    y, _, new, _ = ref.gated_delta_rule(q, k, v, gate, beta, 0.5, True, S0, [n], False)
    for h in range(2):
        S = S0[0, h]
        for t in range(n):
            kt, qt = (a[0, t, 0] / np.sqrt(a[0, t, 0] @ a[0, t, 0] + 1e-6) for a in (k, q))
            S = np.exp(gate[0, t, h]) * (np.eye(4) - beta[0, t, h] * np.outer(kt, kt)) @ S + beta[0, t, h] * np.outer(kt, v[0, t, h])
            assert np.allclose(y[0, t, h], 0.5 * S.T @ qt)
        assert np.allclose(new[0, h], S)
