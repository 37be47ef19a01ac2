"""Weights laid out for the products: no entry point takes a gated block's interleaved halves, so none makes them (no GPU: refused before anything is launched); their size is the header's."""
import os
import re

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


@built
def test_the_size_is_the_one_that_the_header_states():
    from paper_2503_16672_amd import serve
    text = " ".join(open(os.path.join(ROOT, "include", "ffn24_serve.h")).read().split())
    assert "ceil(N / 64) (4096 s + 1024 ceil(s / 4)) with s = ceil(K / 128)" in text
    assert not re.search(r"17/32 bytes for each value|in mx4 17/64 of it", text)      # (a block of 64 rows, four steps of 128 k: smaller ones are filled up)
    up = lambda a, b: -(-a // b)
    for K in (32, 64, 96, 128, 544, 1088, 2048, 4096, 1 << 17):
        for N in (8, 64, 72, 704, 2944, 1 << 20):
            s = up(K, 128)
            size = serve.lib().mx4_weight_bytes(K, N)
            assert size == up(N, 64) * (4096 * s + 1024 * up(s, 4))
            assert size >= 17 * K * N / 32 and (size == 17 * K * N / 32) == (K % 512 == 0 and N % 64 == 0)
