"""Host code of the sequence operators under sanitizers, and the wait states in their compiled kernels (CPU only)."""
import os
import shutil
import subprocess

import pytest
import test_matrix_operation_waits as waits
from test_sanitizers import CLANG, ENV, HERE, OUT, ROOT, SAN

from paper_2007_06000_amd import seq

# wait states before any other instruction may touch the result: eight 4-cycle passes, plus 4
NEED_F8 = {"v_mfma_f32_16x16x128_f8f6f4": 12}


def test_c_abi_under_address_and_undefined_behaviour_sanitizers():
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ with sanitizer runtimes in this image")
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "seq_asan")
    csrc = os.path.join(ROOT, "paper_2007_06000_amd", "csrc")
    cmd = [CLANG, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + csrc, *SAN,
           os.path.join(csrc, "seq_api.cpp"), os.path.join(HERE, "seq_asan.cpp"), "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, env=ENV, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "ERROR: AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-4000:]


@pytest.mark.skipif(not os.path.exists(waits.OBJDUMP), reason="no disassembler")
def test_results_of_matrix_operations_are_not_touched_early(tmp_path, monkeypatch):
    for op, need in NEED_F8.items():
        monkeypatch.setitem(waits.NEED, op, need)
    lib = shutil.copy(seq.LIB_PATH, tmp_path)
    subprocess.run([waits.OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, capture_output=True)
    seen = {}
    for part in sorted(tmp_path.glob("*gfx950")):
        listing = subprocess.run([waits.OBJDUMP, "-d", str(part)], check=True, capture_output=True, text=True).stdout
        for name, ins in waits.functions(listing):
            bad, _ = waits.early_uses(ins)
            assert not bad, (name, bad[:4])
            for op, *_ in ins:
                seen[op] = seen.get(op, 0) + 1
    assert seen["v_mfma_f32_16x16x128_f8f6f4"] > 200 and seen["v_mfma_f32_16x16x32_bf16"] > 100
    # no packed arithmetic in 32 bits, hardly a spill
    assert not [op for op in seen if op.startswith(("v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32"))]
    assert sum(n for op, n in seen.items() if op.startswith("scratch_")) < 32
