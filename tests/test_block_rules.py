"""Which kernels the sizes of the int8 and the gated block's tests reach, by the rules of csrc/tile_rule.hpp compiled for the host: a rule that changes must not leave a path without a test."""
import shutil
import subprocess

import pytest

import test_gpu_gated
import test_gpu_gated_paths
import test_gpu_i8
import test_gpu_i8_tiles
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
    std::printf("%%d %%d %%d %%d\\n", few, s.tile, s.splits, ffn24::pick_edge_tile(2 * N, T, (K + 127) / 128 * 64));
  }
}
"""


@pytest.fixture(scope="module")
def path(tmp_path_factory):
    """(kind, size) -> "few", or the GEMM core's tile and parts of the product (the down product of a block); up: the tile of a block's gate and up product."""
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.cpp").write_text(MAIN % RULE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(d / "rule"), str(d / "rule.cpp")], check=True)

    def one(kind, size, up=False):
        out = subprocess.run([str(d / "rule")], input=f"{kind} {size[0]} {size[1]} {size[2]}", capture_output=True, text=True, check=True).stdout
        few, tile, splits, first = map(int, out.split())
        return "few" if few else first if up else (tile, splits)
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


def test_large_tile_sizes_take_the_large_tiles(path):
    products = [path("p", s) for s in _sizes(test_gpu_i8.test_product) + test_gpu_i8_tiles.PRODUCTS]
    assert {p[0] for p in products if p != "few" and p[1] == 1} == {0, 1, 2, 3, 4}, products
    gated = _sizes(test_gpu_i8.test_gated_block) + test_gpu_i8_tiles.GATED
    assert {path("g", s)[0] for s in gated if path("g", s) != "few" and path("g", s)[1] == 1} == {0, 1, 2, 3, 4}
    assert {path("g", s, up=True) for s in gated + SIZES} - {"few"} == {0, 1, 2, 3, 4}


BF16 = """
#include "%s"
#include <cstdio>
using namespace ffn24;
int main() {
  int T, D, F;
  while (std::scanf("%%d %%d %%d", &T, &D, &F) == 3) {
    const int K = (T + 63) / 64 * 64;
    const EdgeSplit y = pick_edge_split(D, T, F), x = pick_edge_split(D, T, 2 * F);
    const bool panels = gated_dx_panels(T, D, F);
    const int dh = pick_edge_tile(F, T, D), shared = panels ? 0 : pick_grads_tile(T, D, F, K);
    std::printf("up%%d dh%%d ", pick_edge_tile(2 * F, T, D), dh == 3 ? 4 : dh);                                                  // (dH has no 128 x 64)
    if (few_tokens(T, D, F)) std::printf("few "); else std::printf("down%%d%%s ", y.tile, y.splits > 1 ? "split" : "");
    if (shared) std::printf("shared%%d\\n", shared);
    else std::printf("dx%%d%%s wgrad%%d\\n", x.tile, panels ? "panels" : x.splits > 1 ? "split" : "", pick_edge_tile(D, 2 * F, K, F, D));
  }
}
"""


def test_sizes_of_the_gated_tests_take_every_launch(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    (tmp_path / "rule.cpp").write_text(BF16 % RULE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(tmp_path / "rule"), str(tmp_path / "rule.cpp")], check=True)
    sizes = test_gpu_gated.SIZES + test_gpu_gated_paths.SIZES
    out = subprocess.run([str(tmp_path / "rule")], input="\n".join("%d %d %d" % s for s in sizes), capture_output=True, text=True, check=True).stdout.split()
    want = {f"{k}{i}" for k in ("up", "down", "dx", "wgrad") for i in range(5)} | {f"dh{i}" for i in (0, 1, 2, 4)} | {f"shared{i}" for i in (1, 2, 3, 4)}
    want |= {f"{k}{i}split" for k in ("down", "dx") for i in (2, 3, 4)} | {"dx0panels", "few"}
    assert not want - set(out), sorted(want - set(out))
