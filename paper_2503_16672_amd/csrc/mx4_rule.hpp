// Which tile, split and kernel an mx4 product takes: rules on its sizes alone.
#pragma once

namespace ffn24 {

// Block tiles (channels x tokens) of mx4_core.hpp, in ns: a step of 128 k where the chip is nearly empty and where every CU has its tiles, what a launch takes besides, and
// what the results of a tile take where all go out together.  (M N K, 256 x 256 / 256 x 128 / 128 x 128 / 128 x 64, us: 4096 64 16384 73, 42, 26, 21.5; 5888 1000 1088 15.8, 10.2, 8.5, 8.0; 4096 4096
// 4096 34.3, 35.4, 37.9, 44.9; 2048 4096 8192 54, 33.7, 35.4, 43.3; 16384 8192 4096 264, 255, 279, -; 4096 8192 16384 210, 221, 247, -)
struct Mx4Tile { int m, n, lone, busy, launch, out; };
constexpr Mx4Tile MX4_TILES[] = {{256, 256, 530, 770, 5100, 7500}, {256, 128, 293, 410, 4900, 2000}, {128, 128, 181, 240, 3200, 1000}, {128, 64, 152, 149, 2000, 600}};
constexpr int MX4_NUM_TILES = 4, MX4_CUS = 256, MX4_SPLITS = 16;

inline long long mx4_tiles(const Mx4Tile& t, int M, int N) { return ((M + t.m - 1LL) / t.m) * ((N + t.n - 1LL) / t.n); }
inline long long mx4_time(const Mx4Tile& t, long long tiles, int steps) {
  const long long full = tiles < MX4_CUS ? tiles : MX4_CUS, a_cu = (tiles + MX4_CUS - 1) / MX4_CUS;
  return t.launch + a_cu * (steps * (t.lone * (MX4_CUS - full) + t.busy * full) + t.out * full) / MX4_CUS;
}

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
      const long long time = mx4_time(t, tiles * s, s > 1 ? part : steps) + (s > 1 ? 3500 + 8LL * s * M * N / 5000 : 0);
      if (best_time < 0 || time < best_time) { best = Mx4Plan{i, s, s > 1 ? part : steps}; best_time = time; }
    }
  }
  return best;
}

constexpr long long MX4_SPLIT_MOST = 1LL << 25;   // results of a product that could be split: two rounds of the largest tile

// Few tokens: the kernels of k_experts.hip or the GEMM.  A product's tokens come to mx4 in its own kernel where a workgroup can hold them, or by a launch before it.
constexpr int FEW_MX4_TOKENS = 32, MX4_FUSED_VALUES = 1 << 16;
inline bool mx4_few_fused(int T, int K) { return T <= 16 && (long long)T * K <= MX4_FUSED_VALUES; }
inline bool mx4_few(int T, int, int) { return T <= FEW_MX4_TOKENS; }
inline bool mx4_few_gated(int T, int, int) { return T <= FEW_MX4_TOKENS; }

// Experts: waves a workgroup of the up projection of `strips` strips, half strips, and over how many workgroups a strip's experts of the down projection are dealt out
// (`units`: of eight steps, at most, that a strip has)
inline int few_up_waves(int strips) { return strips >= 1024 ? 4 : 8; }
inline bool few_up_halves(int strips) { return strips < 256; }
constexpr int MOE_SPLITS = 8;
inline int moe_down_splits(int strips, int units) {
  const int fill = 256 / strips, most = units / 16;              // (two units a wave at least)
  int s = fill < most ? fill : most;
  s = s < MOE_SPLITS ? s : MOE_SPLITS;
  return s > 2 ? s : 1;
}

}  // namespace ffn24
