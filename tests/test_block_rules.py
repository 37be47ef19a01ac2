"""Which kernels the sizes of the int8 tests reach, by the rules of csrc/tile_rule.hpp compiled for the host: a rule that changes must not leave a path without a test."""
import shutil
import subprocess

import pytest

import test_gpu_i8
from test_gpu_i8_split import ROWS, SIZES
from test_tile_rule import RULE

MAIN = """
#include "%s"
#include <cstdio>
int main() {
  char kind; int T, K, N;
  while (std::scanf(" %%c %%d %%d %%d", &kind, &T, &K, &N) == 4) {       // p: product of T x K and K x N; g: gated block of T tokens, D = K, F = N
    const bool few = kind == 'p' ? ffn24::few_i8_tokens(T, K) : ffn24::few_gated_i8_tokens(T, K, N);
    const int k = kind == 'p' ? K : N, n = kind == 'p' ? N : K;
    const ffn24::EdgeSplit s = ffn24::pick_edge_split(n, T, (k + 127) / 128 * 64);
    std::printf("%%d %%d %%d\\n", few, s.tile, s.splits);
  }
}
"""


@pytest.fixture(scope="module")
def path(tmp_path_factory):
    """(kind, size) -> "few", or the GEMM core's tile and parts."""
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.cpp").write_text(MAIN % RULE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(d / "rule"), str(d / "rule.cpp")], check=True)

    def one(kind, size):
        out = subprocess.run([str(d / "rule")], input=f"{kind} {size[0]} {size[1]} {size[2]}", capture_output=True, text=True, check=True).stdout
        few, tile, splits = map(int, out.split())
        return "few" if few else (tile, splits)
    return one


def _sizes(test):
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and "," in m.args[0])


def test_split_sizes_split_the_down_product_on_the_core(path):
    """With codes in panel form: all three tiles that a split may take, from 2 to 16 parts."""
    paths = [path("g", s) for s in SIZES]
    assert all(p != "few" and p[1] > 1 for p in paths), paths
    assert {p[0] for p in paths} == {2, 3, 4} and min(p[1] for p in paths) == 2 and max(p[1] for p in paths) == 16
    assert any(s[2] % 128 for s in SIZES) and any(s[0] > 256 for s in SIZES)


def test_company_sizes_take_every_kind_of_path(path):
    D, F, counts = ROWS
    paths = [path("g", (t, D, F)) for t in counts]
    assert "few" in paths and any(p != "few" and p[1] > 1 for p in paths) and any(p != "few" and p[1] == 1 for p in paths), paths


def test_sizes_of_the_int8_tests_take_every_kind_of_path(path):
    products = [path("p", s) for s in _sizes(test_gpu_i8.test_product)]
    assert "few" in products and any(p != "few" and p[1] == 1 for p in products) and any(p != "few" and p[1] > 1 for p in products), products
    gated = [path("g", s) for s in _sizes(test_gpu_i8.test_gated_block)]
    assert "few" in gated and any(p != "few" and p[1] == 1 for p in gated), gated
