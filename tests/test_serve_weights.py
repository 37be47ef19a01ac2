"""Weights laid out for the products: no entry point takes a gated block's interleaved halves, so none makes them (no GPU: refused before anything is launched)."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHAPE = -2
built = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2503_16672_amd", "libffn24.so")), reason="libffn24.so not built (python -m paper_2503_16672_amd.build)")


@built
@pytest.mark.parametrize("K,N", [(64, 64), (32, 128), (1088, 1408), (4096, 32768)])
@pytest.mark.parametrize("reserved", [1, -1, 2])
def test_the_reserved_argument_is_refused(K, N, reserved):
    from paper_2503_16672_amd import serve
    L, a = serve.lib(), 0x1000
    assert L.mx4_weight(a, K, N, reserved, a, None) == SHAPE
    assert L.mx4_weight_codes(a, a, K, N, reserved, a, None) == SHAPE


def test_no_layout_of_halves_is_offered():
    text = open(os.path.join(ROOT, "include", "ffn24_serve.h")).read()
    assert "halves" not in text
