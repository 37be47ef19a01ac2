"""What the compiler made of the kernels on mx4 weights and of the experts (no GPU): the symbols the header declares, matrix ops without hazards, registers that are not
spilled; and what the library refuses before it touches the GPU."""
import ctypes
import os
import re

import pytest

from test_kernel_hazards import _hazards

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2503_16672_amd", "libffn24.so")
built = pytest.mark.skipif(not os.path.exists(LIB), reason="libffn24.so not built (python -m paper_2503_16672_amd.build)")


@built
def test_header_symbols_are_exported_and_bound():
    from paper_2503_16672_amd import serve
    names = re.findall(r"FFN24_API\s+\w+\s+(\w+)\s*\(", open(os.path.join(ROOT, "include", "ffn24_serve.h")).read())
    assert sorted(names) == sorted(serve.EXPORTS) and len(names) == 15
    lib = ctypes.CDLL(LIB)
    for n in names:
        assert hasattr(lib, n), n
    serve.lib()


@pytest.mark.parametrize("unit,least", [("k_mx4", 500), ("k_experts", 100)])
def test_no_operand_or_result_is_touched_too_close_to_a_matrix_op(assembly, unit, least):
    ops, early, late = _hazards(assembly[unit])
    assert ops > least and not early and not late, (unit, ops, early[:5], late[:5])


@pytest.mark.parametrize("unit", ["k_mx4", "k_experts"])
def test_kernels_do_not_spill(assembly, unit):
    found = re.findall(r"\.name:\s+(_Z\S+)\n.*?\.vgpr_spill_count:\s+(\d+)", assembly[unit], re.S)
    assert found and not [(n, s) for n, s in found if int(s)]


def test_accumulators_stay_where_they_are(assembly):
    """Between the ops of the GEMM's loops no accumulator is moved: the scaled op's builtin would copy them."""
    ops = re.findall(r"v_mfma_scale_f32_16x16x128_f8f6f4 a\[(\d+):\d+\], \S+ \S+ a\[(\d+):\d+\],", assembly["k_mx4"])
    assert len(ops) >= 500 and all(a == b for a, b in ops)


@built
def test_arguments_are_checked_before_the_gpu_is_touched():
    from paper_2503_16672_amd import serve
    L, a = serve.lib(), 0x1000
    NULL, SHAPE, ALIGN, DTYPE = -1, -2, -3, -4
    assert L.quantise_mx4(a, 4, 48, 0, a, a, None) == SHAPE and L.quantise_mx4(a, -1, 64, 0, a, a, None) == SHAPE and L.quantise_mx4(a, 4, (1 << 17) + 32, 0, a, a, None) == SHAPE
    assert L.quantise_mx4(a, 4, 64, 2, a, a, None) == DTYPE and L.quantise_mx4(a, 4, 64, 1, a, None, None) == NULL and L.quantise_mx4(a + 4, 4, 64, 0, a, a, None) == ALIGN
    assert L.dequantise_mx4(a, a, 4, 16, 0, a, None) == SHAPE and L.dequantise_mx4(a, a, 4, 64, 5, a, None) == DTYPE
    assert L.dequantise_mx4(a, None, 4, 64, 0, a, None) == NULL and L.dequantise_mx4(a, a, 4, 64, 0, a + 8, None) == ALIGN
    assert L.quantise_mx4(None, 0, 64, 0, None, None, None) == 0 and L.dequantise_mx4(None, None, 0, 64, 0, None, None) == 0
    assert L.mx4_weight_bytes(100, 64) == -1 and L.mx4_weight_bytes(64, 12) == -1 and L.mx4_weight_bytes(64, (1 << 20) + 8) == -1
    assert L.mx4_weight_bytes(128, 64) == 4096 + 1024 and L.mx4_weight_bytes(544, 72) == 2 * (5 * 4096 + 2 * 1024)
    assert L.mx4_weight(a, 64, 72, 1, a, None) == SHAPE and L.mx4_weight(None, 64, 64, 0, a, None) == NULL and L.mx4_weight(a, 64, 64, 0, a + 1, None) == ALIGN
    assert L.mx4_weight_codes(a, None, 64, 64, 0, a, None) == NULL and L.mx4_weight_codes(a, a, 33, 64, 0, a, None) == SHAPE
    assert L.linear_mx4_scratch(-1, 64, 64) == -1 and L.linear_mx4_scratch(1 << 21, 64, 64) == -1 and L.linear_mx4_scratch(0, 64, 64) == 0
    assert L.linear_mx4(a, 100, a, 64, 64, a, None, None) == NULL and L.linear_mx4(a, 100, a, 64, 60, a, a, None) == SHAPE and L.linear_mx4(a, 100, a, 64, 64, a + 2, a, None) == ALIGN
    assert L.linear_mx4(None, 0, None, 64, 64, None, None, None) == 0
    h = ctypes.c_void_p()
    new = lambda *args: L.gated_mx4_ctx_create(ctypes.byref(h), *args)
    assert new(0, 64, 64, 0) == SHAPE and new(4, 96, 64, 0) == SHAPE and new(4, 64, 1 << 18, 0) == SHAPE and new(4, 64, 64, 2) == DTYPE and new((1 << 20) + 1, 64, 64, 0) == SHAPE
    assert L.gated_mx4_ctx_create(None, 4, 64, 64, 0) == NULL and L.gated_mx4_fwd(None, a, 4, a, None) == NULL and L.gated_mx4_set_weights(None, a, a, None) == NULL
    new = lambda *args: L.moe_ctx_create(ctypes.byref(h), *args)
    assert new(65, 64, 64, 4, 2, 0, 1, 0) == SHAPE and new(4, 64, 96, 4, 2, 0, 1, 0) == SHAPE and new(4, 1 << 15, 64, 4, 2, 0, 1, 0) == SHAPE
    assert new(4, 64, 64, 257, 2, 0, 1, 0) == SHAPE and new(4, 64, 64, 4, 5, 0, 1, 0) == SHAPE and new(4, 64, 64, 32, 17, 0, 1, 0) == SHAPE and new(4, 64, 64, 4, 0, 0, 1, 0) == SHAPE
    assert new(4, 64, 64, 4, 2, 3, 1, 0) == DTYPE and new(4, 64, 64, 4, 2, 0, 1, 2) == DTYPE and L.moe_ctx_create(None, 4, 64, 64, 4, 2, 0, 1, 0) == NULL
    assert L.moe_fwd(None, a, 4, a, None, None, None) == NULL and L.moe_set_weights(None, a, a, a, None) == NULL
    assert L.gated_mx4_ctx_destroy(None) == 0 and L.moe_ctx_destroy(None) == 0 and h.value is None
