"""Which kernels the sizes of the mx4 and expert tests reach, by the rules of csrc/mx4_rule.hpp compiled for the host: a rule that changes must not leave a path without a test."""
import os
import shutil
import subprocess

import pytest

import test_gpu_moe
import test_gpu_mx4

RULE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_16672_amd", "csrc", "mx4_rule.hpp")
MAIN = """
#include "%s"
#include <cstdio>
using namespace ffn24;
void product(const char* name, int T, int K, int N, bool fused) {
  const int steps = (K + 127) / 128;
  if (!fused) std::printf("%%s-tokens-%%d ", name, mx4_tokens_rows(T, steps));
  if (mx4_few(T, K, N)) std::printf("%%s-few-%%s-%%d-%%d ", name, fused ? "fused" : "operand", T > 16 ? 2 : 1, T > 16 ? 1 : mx4_few_groups(N, steps));
  else { const Mx4Plan p = mx4_plan(N, T, steps, true); std::printf("%%s-tile%%d%%s ", name, p.tile, p.splits > 1 ? "split" : ""); }
}
int main() {
  char kind; int T, K, N, E, k;
  while (std::scanf(" %%c %%d %%d %%d %%d %%d", &kind, &T, &K, &N, &E, &k) == 6) {
    if (kind == 'p') product("p", T, K, N, mx4_few_fused(T, K));
    if (kind == 'g') {                                       // T tokens, D = K, F = N
      if (mx4_few_gated(T)) std::printf("up-few-%%s ", mx4_few_fused(T, K) ? "fused" : "operand");
      else std::printf("up-tile%%d ", mx4_plan(2 * N, T, (K + 127) / 128, false).tile);
      product("down", T, N, K, false);
    }
    if (kind == 'm') for (int mx4 = 0; mx4 < 2; mx4++) {
      const int slots = T * k < E ? T * k : E, strips = N / 32 * slots, waves = mx4 ? few_up_waves(strips, (K + 127) / 128) : 8;
      const bool halves = !mx4 && few_up_halves(strips);
      std::printf("%%s-", mx4 ? "mx4" : "bf16");
      if (T == 1) std::printf("one-%%s ", halves ? "half" : "whole");
      else if (T <= 16) std::printf("few-%%s ", waves == 4 ? "4" : halves ? "half" : "8");
      else if (moe_crowded(T, k, E)) std::printf("crowded ");
      else std::printf("passes-%%d ", waves);
      const int steps = mx4 ? (N + 127) / 128 : N / 32;
      std::printf("%%s-down%%d-%%s ", mx4 ? "mx4" : "bf16", T <= 16 ? 1 : 4, moe_down_splits(K / 16, slots * ((steps + 7) / 8)) > 1 ? "shared" : "alone");
    }
  }
}
"""


@pytest.fixture(scope="module")
def paths(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.cpp").write_text(MAIN % RULE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(d / "rule"), str(d / "rule.cpp")], check=True)

    def of(kind, sizes):
        lines = "\n".join(" ".join(map(str, (kind, *s, *([0] * (5 - len(s)))))) for s in sizes)
        return set(subprocess.run([str(d / "rule")], input=lines, capture_output=True, text=True, check=True).stdout.split())
    return of


def _sizes(test):
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == "T,D,F")


def test_products_take_every_kernel(paths):
    want = {f"p-tile{i}" for i in range(4)} | {"p-tile3split", "p-few-operand-2-1", "p-tokens-1", "p-tokens-4"} | {f"p-few-{s}-1-{g}" for s in ("fused", "operand") for g in (1, 2, 4)}
    assert not want - (paths("p", test_gpu_mx4.PRODUCTS) | {p.replace("down", "p") for p in paths("g", _sizes(test_gpu_mx4.test_gated_block))})


def test_gated_blocks_take_every_kernel(paths):
    got = paths("g", _sizes(test_gpu_mx4.test_gated_block))
    want = {f"up-tile{i}" for i in range(4)} | {"up-few-fused", "up-few-operand", "down-few-operand-1-1", "down-few-operand-2-1", "down-tile3split", "down-tile3"}
    assert not want - got, want - got


def test_experts_take_every_kernel(paths):
    got = paths("m", [(T, D, F, E, k) for T, D, F, E, k in test_gpu_moe.CASES])
    want = {f"{t}-{p}" for t in ("bf16", "mx4") for p in ("one-whole", "few-8", "crowded", "passes-8", "down1-alone", "down1-shared", "down4-alone", "down4-shared")}
    want |= {"bf16-one-half", "bf16-few-half", "mx4-few-4", "mx4-passes-4"}
    assert not want - got, want - got
