"""CPU checks of the operators around a projection at the ends of their sizes: how much workspace is asked for."""
import itertools

import pytest

from paper_2007_06000_amd import seq
from test_seq_mix_abi import BASE, pack

NAME = "xl_gated_delta_rule"


@pytest.mark.parametrize("dtype", [seq.XL_F32, seq.XL_F16, seq.XL_BF16])
def test_the_workspace_of_a_delta_rule_has_a_bound(dtype):
    """Half a gigabyte of chunks, and where they do not all fit the states of the sequences whose chunks do."""
    for batch, (key_heads, heads), length, dk, dv in itertools.product((1, 3, 64, 700, 4095, 100000), ((1, 1), (16, 16), (4, 16), (1, 4095), (2100, 2100), (65535, 65535)), (13, 41, 64, 1000, 100000),
                                                                      (8, 64, 128, 256), (8, 128)):
        need = getattr(seq.lib(), NAME + "_workspace")(pack(NAME, dict(BASE[NAME], batch=batch, key_heads=key_heads, heads=heads, length=length, dk=dk, dv=dv, dtype=dtype)))
        assert 0 <= need <= (1 << 29) + batch * heads * dk * dv * 4 + 16, (batch, key_heads, heads, length, dk, dv, need)
        if length <= 64:        # one chunk a sequence
            assert need <= 1 << 29
