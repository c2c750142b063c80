"""Build libxl.so (HIP kernels + host planner + C ABI) and libxl_seq.so (sequence operators) for gfx950 with hipcc, and with the host compiler
_xl_seq.so, the Python module that hands torch tensors to libxl_seq.so.

Run as `python -m paper_2007_06000_amd.build`; the libraries land next to this
file so that they travel with the source tree.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libxl.so")
# (source, object name, extra defines): kernels.hip is compiled once for the fp32 variants and once for each part of the
# split-bf16 ones
SOURCES = [("kernels.hip", "kernels", []),
           *[("kernels.hip", f"kernels_split_{part}{pr}", [f"-DXL_TU_SPLIT={part}", f"-DXL_TU_PR={pr}"] + extra)
             for part, extra in (("A", []), ("B", []), ("C", []), ("D", ["-DXL_TU_CHAIN"]), ("E", ["-DXL_TU_KSPLIT"]), ("F", []), ("G", ["-DXL_TU_HEAD"])) for pr in (1, 2)],
           ("plan.cpp", "plan", []), ("api.cpp", "api", []), ("static_run.hip", "static_run", [])]
HEADERS = [os.path.join(CSRC, "xl_internal.h"), os.path.join(CSRC, "plan.h"), os.path.join(CSRC, "thin_conv.h"),
           os.path.join(CSRC, "split_conv.h"), os.path.join(CSRC, "dw_conv.h"), os.path.join(CSRC, "chain_conv.h"),
           os.path.join(CSRC, "ksplit_conv.h"), os.path.join(CSRC, "direct_conv.h"), os.path.join(CSRC, "head_conv.h"), os.path.join(CSRC, "stem_conv.h"),
           os.path.join(ROOT, "include", "xl.h")]
SEQ_LIB = os.path.join(HERE, "libxl_seq.so")
SEQ_SOURCES = [("seq_api.cpp", "seq_api", []), ("seq_conv.hip", "seq_conv", []), ("seq_scan.hip", "seq_scan", []),
               ("seq_quant.hip", "seq_quant", []), ("seq_matmul.hip", "seq_matmul", []), ("seq_mix_api.cpp", "seq_mix_api", []),
               ("seq_norm.hip", "seq_norm", []), ("seq_adapters.hip", "seq_adapters", []), ("seq_delta.hip", "seq_delta", [])]
SEQ_HEADERS = [os.path.join(CSRC, "seq_internal.h"), os.path.join(CSRC, "seq_launch.h"), os.path.join(CSRC, "seq_checks.h"), os.path.join(CSRC, "seq_e4m3.h"), os.path.join(CSRC, "seq_parts.h"),
               os.path.join(ROOT, "include", "xl_seq.h"), os.path.join(ROOT, "include", "xl.h")]
MODULE = os.path.join(HERE, "_xl_seq.so")

# packed-fp32 instructions are switched off for all device code
HIPCC_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
               "-Wno-cuda-compat", "-Wno-pass-failed",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def _filter(stderr: str) -> str:
    keep = [ln for ln in stderr.splitlines() if "packed-fp32-ops" not in ln]
    return "\n".join(keep)


def _compile(item, headers, force: bool) -> str:
    src, name, defines = item
    obj = os.path.join(OBJ, name + ".o")
    path = os.path.join(CSRC, src)
    newest = max(os.path.getmtime(p) for p in [path] + headers)
    if not force and os.path.exists(obj) and os.path.getmtime(obj) >= newest:
        return obj
    cmd = [_hipcc()] + HIPCC_FLAGS + defines + ["-x", "hip", "-c", path, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    msg = _filter(r.stderr)
    if msg.strip():
        sys.stderr.write(msg + "\n")
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}")
    return obj


def _build_module(force: bool) -> str:
    src = os.path.join(CSRC, "seq_torch.cpp")
    newest = max(os.path.getmtime(p) for p in [src, os.path.join(CSRC, "seq_overlap.h")] + SEQ_HEADERS[-2:])
    if not force and os.path.exists(MODULE) and os.path.getmtime(MODULE) >= newest:
        return MODULE
    from torch.utils.cpp_extension import include_paths, library_paths     # both name only files of the installed torch
    system = [*include_paths(), sysconfig.get_path("include"), "/opt/rocm/include"]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__", *[f for p in system for f in ("-isystem", p)],
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-shared", "-o", MODULE, src, *["-L" + p for p in library_paths()],
           "-ltorch_python", "-ltorch_cpu", "-lc10_hip", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.stderr.strip():
        sys.stderr.write(r.stderr + "\n")
    if r.returncode != 0:
        raise RuntimeError("the host compiler failed on seq_torch.cpp")
    return MODULE


def _link(lib: str, objs, force: bool) -> None:
    if force or not os.path.exists(lib) or any(os.path.getmtime(o) > os.path.getmtime(lib) for o in objs):
        cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", lib] + objs
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(_filter(r.stderr) + "\n")
            raise RuntimeError("link failed")


def build(force: bool = False, verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    items = [(s, HEADERS) for s in SOURCES] + [(s, SEQ_HEADERS) for s in SEQ_SOURCES]
    with ThreadPoolExecutor(max_workers=len(items) + 1) as ex:
        module = ex.submit(_build_module, force)
        objs = list(ex.map(lambda item: _compile(*item, force), items))
        module.result()
    for lib, part in ((LIB, objs[:len(SOURCES)]), (SEQ_LIB, objs[len(SOURCES):])):
        _link(lib, part, force)
        if verbose:
            print("built", lib)
    if verbose:
        print("built", MODULE)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv)
