// Which tile, split and kernel an mx4 product takes: rules on its sizes alone.
#pragma once

namespace ffn24 {

// Block tiles (channels x tokens) of mx4_core.hpp, ns a step of 128 k and of what a tile costs besides
struct Mx4Tile { int m, n, per_step, fixed; };
constexpr Mx4Tile MX4_TILES[] = {{256, 256, 640, 4500}, {256, 128, 360, 3500}, {128, 128, 250, 3000}, {128, 64, 170, 2500}};
constexpr int MX4_NUM_TILES = 4, MX4_CUS = 256, MX4_SPLITS = 16;

inline long long mx4_tiles(const Mx4Tile& t, int M, int N) { return ((M + t.m - 1LL) / t.m) * ((N + t.n - 1LL) / t.n); }
// rounds of the chip (two of the small tiles share a CU at nearly their own rate) x a tile
inline long long mx4_time(const Mx4Tile& t, long long tiles, int steps) { return (tiles + MX4_CUS - 1) / MX4_CUS * ((long long)t.per_step * steps + t.fixed); }

struct Mx4Plan { int tile, splits, part; };
// M channels, N tokens, `steps` of k; split: whether the reduction may be split (its sums then cost a launch and their way through memory)
inline Mx4Plan mx4_plan(int M, int N, int steps, bool split) {
  N = (N + 63) / 64 * 64;      // (the scratch of a context is made for whole 64s)
  Mx4Plan best{0, 1, steps};
  long long best_time = -1;
  for (int i = 0; i < MX4_NUM_TILES; i++) {
    const Mx4Tile& t = MX4_TILES[i];
    const long long tiles = mx4_tiles(t, M, N);
    for (int s = 1; s <= (split ? MX4_SPLITS : 1); s++) {
      const int part = ((steps + s - 1) / s + 3) / 4 * 4;
      if (s > 1 && (part < 8 || (s - 1) * part >= steps || tiles * s > 2 * MX4_CUS)) continue;
      const long long time = mx4_time(t, tiles * s, s > 1 ? part : steps) + (s > 1 ? 5000 + 8LL * s * M * N / 5000 : 0);
      if (best_time < 0 || time < best_time) { best = Mx4Plan{i, s, s > 1 ? part : steps}; best_time = time; }
    }
  }
  return best;
}

constexpr long long MX4_SPLIT_MOST = 1LL << 25;   // results of a product that could be split: two rounds of the largest tile

// Few tokens: the kernels of k_experts.hip or the GEMM.  A product's tokens to mx4 in its own kernel, or by a launch before it.
constexpr int FEW_MX4_TOKENS = 32;
inline bool mx4_few_fused(int T) { return T <= 16; }
inline bool mx4_few(int T, int, int) { return T <= FEW_MX4_TOKENS; }
inline bool mx4_few_gated(int T, int, int) { return T <= FEW_MX4_TOKENS; }

// Experts: waves a workgroup of the up projection of `strips` strips, half strips, and over how many workgroups a strip's experts of the down projection are dealt out
// (`units`: of eight steps, at most, that a strip has)
inline int few_up_waves(int strips, int nt) { return strips >= 1024 && nt == 1 ? 4 : 8; }
inline bool few_up_halves(int strips) { return strips < 256; }
constexpr int MOE_SPLITS = 8;
inline int moe_down_splits(int strips, int units) {
  const int fill = 256 / strips, most = units / 16;              // (two units a wave at least)
  int s = fill < most ? fill : most;
  s = s < MOE_SPLITS ? s : MOE_SPLITS;
  return s > 2 ? s : 1;
}

}  // namespace ffn24
