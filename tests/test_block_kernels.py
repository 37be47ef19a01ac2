"""What the compiler made of the kernels around the feed-forward block (no GPU): the symbols the header declares, matrix ops without hazards, registers that are not spilled."""
import ctypes
import os
import re

import pytest

from test_kernel_hazards import _hazards

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2503_16672_amd", "libffn24.so")


@pytest.mark.skipif(not os.path.exists(LIB), reason="libffn24.so not built (python -m paper_2503_16672_amd.build)")
def test_header_symbols_are_exported_and_bound():
    from paper_2503_16672_amd import block
    names = re.findall(r"FFN24_API\s+\w+\s+(\w+)\s*\(", open(os.path.join(ROOT, "include", "ffn24_block.h")).read())
    assert sorted(names) == sorted(block.EXPORTS) and len(names) == 17
    lib = ctypes.CDLL(LIB)
    for n in names:
        assert hasattr(lib, n), n
    block.lib()


@pytest.mark.parametrize("unit,least", [("k_gated", 500), ("k_i8", 500), ("k_few", 100)])
def test_no_operand_or_result_is_touched_too_close_to_a_matrix_op(assembly, unit, least):
    ops, early, late = _hazards(assembly[unit])
    assert ops > least and not early and not late, (unit, ops, early[:5], late[:5])


# A norm's workgroup of 16 waves (more than 8192 columns) has 128 registers a lane.
SPILLS = {"k_norm": lambda name: "Li2ELi16ELi1E" in name}


@pytest.mark.parametrize("unit", ["k_gated", "k_i8", "k_few", "k_norm"])
def test_kernels_do_not_spill(assembly, unit):
    found = re.findall(r"\.name:\s+(_Z\S+)\n.*?\.vgpr_spill_count:\s+(\d+)", assembly[unit], re.S)
    assert found
    bad = [(n, s) for n, s in found if int(s) and not SPILLS.get(unit, lambda name: False)(n)]
    assert not bad, bad


def test_int8_ops_are_the_wide_ones(assembly):
    """The 16 x 16 x 64 and 32 x 32 x 32 integer ops, not their halves."""
    assert assembly["k_i8"].count("v_mfma_i32_16x16x64_i8") >= 64 and assembly["k_i8"].count("v_mfma_i32_32x32x32_i8") >= 32
    assert not re.search(r"v_mfma_i32_(16x16x32|32x32x16)_i8", assembly["k_i8"])
