// Which tile, split and kernel an mx4 product takes: rules on its sizes alone.
// Figures here are of passes over the same weights one after the other, unless "cold" is said: up to 256 MB of them are then in the last-level cache.  Cold, from HBM (copies in turn), few
// tokens take 1 to 2 us more: 1 2048 8192 3.0, 4.3; 16 4096 4096 6.4, 7.1; 16 8192 8192 9.3, 11.4; gated 16 4096 16384 25.2, 26.6; experts 1 2048 1024 32 4 20.1, 21.5.
#pragma once

namespace ffn24 {

// Block tiles (channels x tokens) of mx4_core.hpp, in ns: a step of 128 k where the chip is nearly empty and where every CU has its tiles, what a launch takes besides, and
// what the results of a tile take where all go out together.  (M N K, 256 x 256 / 256 x 128 / 128 x 128 / 128 x 64, us: 4096 64 16384 73, 42, 26, 21.5; 5888 1000 1088 15.8, 10.2,
// 8.5, 8.0; 4096 4096 4096 34.3, 35.4, 37.9, 44.9; 2048 4096 8192 54, 33.7, 35.4, 43.3; 16384 8192 4096 264, 255, 279, -; 4096 8192 16384 210, 221, 247, -)
struct Mx4Tile { int m, n, lone, busy, launch, out; };
constexpr Mx4Tile MX4_TILES[] = {{256, 256, 530, 770, 5100, 7500}, {256, 128, 293, 410, 4900, 2000}, {128, 128, 181, 240, 3200, 1000}, {128, 64, 152, 149, 2000, 600}};
constexpr int MX4_NUM_TILES = 4, MX4_CUS = 256, MX4_SPLITS = 16;

inline long long mx4_tiles(const Mx4Tile& t, int M, int N) { return ((M + t.m - 1LL) / t.m) * ((N + t.n - 1LL) / t.n); }
inline long long mx4_time(const Mx4Tile& t, long long tiles, int steps) {
  const long long full = tiles < MX4_CUS ? tiles : MX4_CUS, a_cu = (tiles + MX4_CUS - 1) / MX4_CUS;
  return t.launch + a_cu * (steps * (t.lone * (MX4_CUS - full) + t.busy * full) + t.out * full) / MX4_CUS;
}

struct Mx4Plan { int tile, splits, part; };
// M channels, N tokens, `steps` of k.  split: whether the reduction may be split over several workgroups a tile, on the smallest tile (its sums then cost a launch and their way
// through memory; us, 128 x 64 / 128 x 128 tiles at their best split: 4096 64 16384 12.2, 13.4; 4096 128 16384 14.0, 15.4; 1024 64 16384 10.1, 11.3; unsplit 21.5, 21.6, 18.1)
inline Mx4Plan mx4_plan(int M, int N, int steps, bool split) {
  N = (N + 63) / 64 * 64;      // (the scratch of a context is made for whole 64s)
  Mx4Plan best{0, 1, steps};
  long long best_time = -1;
  for (int i = 0; i < MX4_NUM_TILES; i++) {
    const Mx4Tile& t = MX4_TILES[i];
    const long long tiles = mx4_tiles(t, M, N);
    for (int s = 1; s <= (split && i == MX4_NUM_TILES - 1 ? MX4_SPLITS : 1); s++) {
      const int part = ((steps + s - 1) / s + 3) / 4 * 4;
      if (s > 1 && (part < 8 || (s - 1) * part >= steps || tiles * s > 2 * MX4_CUS)) continue;
      const long long time = mx4_time(t, tiles * s, s > 1 ? part : steps) + (s > 1 ? 3500 + 8LL * s * M * N / 5000 : 0);
      if (best_time < 0 || time < best_time) { best = Mx4Plan{i, s, s > 1 ? part : steps}; best_time = time; }
    }
  }
  return best;
}

constexpr long long MX4_SPLIT_MOST = 1LL << 21;   // results of a product that could be split: 256 tiles of 128 x 64

// Few tokens: the kernels of k_experts.hip or the GEMM.  us, few tokens' kernel / GEMM.  Products (T K N): 16 4096 32768 11.2, 12.9; 16 16384 4096 8.7, 12.3; 24 16384 4096 9.6, 12.3;
// 24 5440 2048 4.2, 7.6; 24 1408 512 3.4, 4.7; the other way round 24 4096 32768 14.3, 13.0; 24 2048 10880 8.6, 5.1; 24 28672 8192 26.9, 23.2: from 17 tokens on where the GEMM would
// have to split the reduction.  Gate and up (T D F): 16 4096 16384 12.4, 13.2; 16 2048 5440 4.9, 5.4; 24 4096 16384 16.2, 13.4; 24 2048 5440 5.8, 5.5.  Up to 16 tokens of wide layers the
// GEMM is ahead on weights in the last-level cache and behind on cold ones, which a model's are.  Whole calls, cold: 16 8192 57344 45.0, 51.0 (warm 43.4, 39.5); 16 16384 32768 51.9, 55.1
// (51.3, 46.9); 16 8192 28672 25.3, 29.0 (23.5, 23.4); 16 4096 65536 27.8, 31.5 (25.9, 25.4); 16 16384 16384 27.5, 33.4; 16 8192 131072 91, 112; gated 16 8192 28672 67, 75 (68, 81); 16 4096
// 16384 26.0, 31.8; 16 8192 65536 132, 164.
constexpr int FEW_MX4_TOKENS = 16, FEW_MX4_MORE = 32;
inline bool mx4_few(int T, int K, int N) { return T <= FEW_MX4_TOKENS || (T <= FEW_MX4_MORE && K >= N && N <= 4096); }
inline bool mx4_few_gated(int T) { return T <= FEW_MX4_TOKENS; }
// Their tokens come to mx4 in the kernel itself, by every workgroup, or by a launch before it.  us, both: products (T K N) 8 4096 32768 11.8, 12.7; 16 2048 8192 5.0, 5.4; 1 28672
// 8192 19.7, 24.3; 3 16384 4096 9.3, 9.9; 4 16384 4096 10.2, 9.9; 8 8192 8192 11.4, 9.8; 16 4096 4096 7.0, 5.7; gated (T D F) 1 4096 16384 20.7, 22.4; 12 4096 16384 23.0, 23.6;
// 16 4096 16384 24.2, 23.7.
constexpr int MX4_FUSED_VALUES = 3 << 14;
inline bool mx4_few_fused(int T, int K) { return T <= FEW_MX4_TOKENS && (long long)T * K <= MX4_FUSED_VALUES; }
// That launch: rows in fours, of 16, that a wave takes of its four steps; one until there are eight waves a CU.  us with one / four (product and launch): 333 1088 4168 7.8, 9.1;
// 8192 512 1024 13.5, 15.7; 2048 4096 1024 16.4, 17.3; 4096 4096 1024 21.5, 21.6; 8192 4096 1024 35.7, 35.4.
inline int mx4_tokens_rows(int T, int steps) { return (long long)((T + 15) / 16) * ((steps + 3) / 4) < 2048 ? 1 : 4; }
// Groups of 16 channels a strip.  A wave takes 8 KiB at a time, so a short reduction needs wide strips for eight waves to have work, and a long one many strips where channels are
// few.  us with 1, 2, 4 groups, 16 tokens (K N): 16384 4096 10.6, 12.2, 16.9; 28672 4096 15.1, 18.5, 27.0; 8192 2048 5.9, 6.4, 8.1; 8192 4096 6.9, 6.5, 8.0; 4096 4096 5.7, 5.4,
// 6.4; 8192 8192 10.5, 8.7, 11.1; 2048 8192 6.5, 4.6, 4.9; 4096 24576 15.8, 11.6, 12.6; 8192 28672 26.3, 22.9, 21.9; 4096 32768 19.5, 14.2, 13.6; 2048 16384 10.6, 6.6, 5.8; 1536
// 8960 7.6, 5.2, 4.5; 1024 32768 13.2, 7.1, 4.9.
inline int mx4_few_groups(int N, int steps) {
  if (N >= 28672 || (N > 8192 && steps <= 16)) return 4;
  return N <= 4096 && steps >= 40 && 50 * steps >= N ? 1 : 2;
}

// Experts (T D F E k, us).
// Waves a workgroup of the up projection: eight, for what they have on their way; four where a reduction has no two loads of four KiB for each of eight (mx4, fewer than 24 steps
// of 128) and the strips are so many that more workgroups of fewer waves fill the CUs as well.  Mx4, 4 / 8 waves: 16 1024 1024 64 2 26.6, 28.3; 8 1024 512 128 8 31.7, 33.3; 37
// 2048 1024 64 4 53.8, 55.6; 64 2048 768 128 8 89.5, 92.3; 16 2880 1472 128 4 84.8, 85.2; the other way round 64 3584 1024 64 4 78.4, 76.8; 8 4096 2048 64 4 75.3, 73.2; 4 2048
// 1024 32 4 (512 strips) 24.8, 24.1.
inline int few_up_waves(int strips, int steps) { return steps < 24 && strips >= 768 ? 4 : 8; }
// Strips of half the width where there are fewer whole ones than CUs.  Bf16, whole / half: 1 2048 1024 32 4 (128 strips) 21.2, 19.9; 2 2048 1024 32 2 25.0, 23.2; 2 1024 512 32 4
// 21.2, 20.2; the other way round 1 2048 1024 32 8 (256) 27.5, 28.4.
inline bool few_up_halves(int strips) { return strips < 256; }
// From 17 tokens on an expert may have more than 16: one pass over its weights with 64 tokens beside them (half the workgroups a CU, for the registers) where it has many,
// otherwise a pass for each 16. Bf16, passes / one: 64 2048 1024 16 4 75.7, 65.6; 64 4096 2048 16 4 199, 157; 32 1088 704 8 4 30.1, 27.0; the other way round 37 1088 704 24 4
// 38.2, 40.5; 64 2048 1024 16 2 53.5, 54.6.  At T k = 10 E (64 1088 704 24 4) 44.8, 43.3; mx4 29.9, 30.4.  The choices here are spread evenly and only their mean is known to the host: where
// all 64 tokens choose the same eight experts, passes read their gate and up weights four times (bf16 4096 2048 64 8: 241 us, where one pass over those weights is 40; spread 490).
inline bool moe_crowded(int T, int k, int E) { return T * k > 12 * E; }
// Groups of 16 channels a strip of the down projection has, of bf16 experts (pairs: T k): every strip reads the tokens' activations (4 bytes a value), so wide ones read fewer bytes and
// narrow ones are more workgroups, without or with fewer sums of a launch of their own.  1, 2, 4 groups, each with its splits: 64 4096 2048 64 8 541, 504, 488; 64 4096 2048 16 4 169,
// 158, 153; 48 3584 1024 64 4 239, 227, 224; 12 2880 1472 16 2 81.5, 78.6, 70; 64 2304 1024 16 4 79, 67.5, 66.6; 64 2560 1024 16 2 66, 61.3, 62.5; 64 2048 768 128 8 205, 195, 197; 64 2048
// 1024 16 4 61.6, 59.9, 61.1; 20 1536 1024 32 4 66.5, 60.9, 62.8; 64 1536 512 16 16 56.6, 51.7, 51.8; short reductions 64 8192 512 8 2 73, 66.0, 67.7; 64 4096 768 32 4 116, 112, 111; 64 4096
// 512 16 2 50.3, 51.2, 53.1; few channels 64 1024 2048 32 4 89.0, 86.1, 95; 64 1024 4096 16 4 110, 105, 117; 64 1024 1024 32 4 53.8, 54.1, 60; 64 1088 704 24 4 43.4, 43.7, 46.9; 64 512 1024
// 64 8 58.7, 64.1, 73.6; few pairs 1 2048 1024 32 4 19.5, 20.0, 20.2; 2 1024 512 32 4 20.7, 21.2, 22.0; 2 4096 2048 16 2 37.9, 38.3, 38.1; 1 4096 2048 64 8 76.8, 75.7, 75.3; 3 2048 1024 32 4
// 42.3, 41.8, 41.6; 2 4096 2048 64 8 138, 133, 131.
inline int moe_down_groups(int pairs, int D, int F) { return pairs < 12 || D < 1024 || (D < 1280 && F < 2048) ? 1 : D < 2560 || F < 1024 ? 2 : 4; }
// Over how many workgroups the experts of a strip of the down projection are dealt out (`units`: of eight steps, at most, that a strip has): as many as fill the CUs, where the
// sums' own launch does not cost more.  1 / chosen: bf16 64 2048 768 128 8 235, 202 (2); 16 2048 1024 32 4 75.2, 69.1 (2); 37 1088 704 24 4 47.1, 38.5 (3); 64 1024 2048 32 4 121,
// 81 (4); mx4 64 2048 768 128 8 89.5, 76.5; 8 1088 704 24 4 (24 units) 24.1, 23.7; with less work than that: 1 2048 1024 32 4 bf16 (16 units) 18.9, 19.8, mx4 15.2, 17.0; and at
// 180 strips of 2880 channels two lose 2 to 8 %.
constexpr int MOE_SPLITS = 8;
inline int moe_down_splits(int strips, int units) {
  const int fill = 256 / strips, most = units / 8;               // (a unit a wave at least)
  int s = fill < most ? fill : most;
  s = s < MOE_SPLITS ? s : MOE_SPLITS;
  return s > 1 && units >= 24 ? s : 1;
}

}  // namespace ffn24
