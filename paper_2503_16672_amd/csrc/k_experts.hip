// Few tokens: products with weights in the operand form of mx4_core.hpp (mx4, or bf16 in the same order), and the mixture of experts made of them.  Bound by the weights' bytes.
//
// A wave streams weights from memory straight into operands of the 16 x 16 matrix ops (rows: output channels, columns: tokens, 16 at a time); the eight waves of a
// workgroup share the reduction of a strip of channels and add up through LDS in a fixed order.  A wave has 8 KiB of weights on their way while it works on 8 KiB.
//
// Mixture of experts, four launches:
//   router   logits X Wr in 64 bits, a part of D a workgroup (a product of two bf16 is exact in fp32; in 64 bits the choice between near experts is the definition's)
//   pick     a token's k largest by their rank, ties to the lowest index; shares
//   up       a workgroup a strip of 32 features of a chosen expert: h = a(G) U for the tokens that chose it; a row of H for each (token, choice)
//   down     a workgroup a strip of 16 channels and all chosen experts one after the other: the shares' sum stays in LDS, in the order of the experts
#include "mx4_core.hpp"
#include "stream_core.hpp"

namespace ffn24 {
namespace {

constexpr int WAVES = 8, THREADS = 64 * WAVES, RED = 17;   // RED: pitch of the sums' image [channel][16 tokens]

// Workgroup ids go round the 8 XCDs; an XCD gets a run of neighbouring strips instead (a strip of 16 channels is a KiB of every 4: a quarter of an L2's channels)
__device__ __forceinline__ unsigned run_of(unsigned id, unsigned n) {
  const unsigned per = n >> 3, more = n & 7u, xcd = id & 7u;
  return xcd * per + min(xcd, more) + (id >> 3);
}

// Where a wave's weights are: the strip's codes and scales, bytes from a step (four steps' scales) to the next
struct Strip { const char* codes; const char* scales; int steps; };

// U steps of RG groups of 16 channels
template <bool MX4, int RG, int U>
struct Weights {
  static constexpr int SU = (U + 3) / 4;
  u32x4 w[U][RG];
  uint32_t s[MX4 ? SU : 1][MX4 ? RG : 1];
  // from step s0 (a multiple of U) on; steps beyond the last read the last one and are not used
  __device__ __forceinline__ void load(const Strip& p, int s0, int lane) {
#pragma unroll
    for (int j = 0; j < U; j++) {
      const char* at = p.codes + (size_t)min(s0 + j, p.steps - 1) * MX4_PANEL + lane * 16;
#pragma unroll
      for (int g = 0; g < RG; g++) w[j][g] = ld_stream(reinterpret_cast<const u32x4*>(at + g * 1024));
    }
    if constexpr (MX4) {
#pragma unroll
      for (int j = 0; j < SU; j++) {
        const char* at = p.scales + (size_t)(min(s0 + 4 * j, p.steps - 1) >> 2) * 1024 + lane * 4;
#pragma unroll
        for (int g = 0; g < RG; g++) s[j][g] = *reinterpret_cast<const uint32_t*>(at + g * 256);
      }
    }
  }
};

// Tokens of one step: an operand (and its scale) of 16 of them
struct TokenOp { u32x4 x; uint32_t s; };
// SRC 0: rows of bf16 as they are; 1: rows of bf16 to mx4; 2: the mx4 operand form
enum { ROWS_BF16 = 0, ROWS_TO_MX4 = 1, OPERAND_MX4 = 2 };
struct Tokens { const char* p; const char* scales; int K, steps; };   // rows [..][K], or codes and scales
template <int SRC>
__device__ __forceinline__ TokenOp token_op(const Tokens& t, int row, bool on, int step, int q) {
  TokenOp o{{0u, 0u, 0u, 0u}, 0u};
  if constexpr (SRC == ROWS_BF16) {
    const int k = 32 * step + 8 * q;
    if (on && k < t.K) o.x = *reinterpret_cast<const u32x4*>(t.p + ((size_t)row * t.K + k) * 2);
  } else if constexpr (SRC == ROWS_TO_MX4) {
    const int k = MX4_STEP * step + 32 * q;
    if (on && k < t.K) {
      const u32x4* p = reinterpret_cast<const u32x4*>(t.p + ((size_t)row * t.K + k) * 2);
      u32x4 v[4];
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] = p[i];
      uint32_t top = 0u;
#pragma unroll
      for (int i = 0; i < 4; i++) top = i8_top8(v[i], top);
      o.s = mx4_scale_code(top);
      const float s = mx4_scale(o.s);
#pragma unroll
      for (int i = 0; i < 4; i++) o.x[i] = mx4_codes8(v[i], s);
    }
  } else {
    if (on) {
      o.x = *reinterpret_cast<const u32x4*>(t.p + mx4_code_at(row, 4 * step + q, t.steps));
      o.s = static_cast<uint8_t>(t.scales[mx4_scale_at(row, 4 * step + q, t.steps)]);
    }
  }
  return o;
}

template <bool MX4>
__device__ __forceinline__ void few_op(const u32x4& w, uint32_t sw, const TokenOp& x, f32x4& acc) {
  if constexpr (MX4) {
    const i32x4 a = __builtin_bit_cast(i32x4, w), b = __builtin_bit_cast(i32x4, x.x);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1), __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1), acc, 4, 4,
                                                           0, (int)sw, 0, (int)x.s);
  } else {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x.x), acc, 0, 0, 0);
  }
}
// the ops of U steps for up to NT groups of 16 tokens; row[i]: the lane's row of group i, on[i]: whether there is one; groups: how many there are
template <bool MX4, int SRC, int RG, int U, int NT>
__device__ __forceinline__ void few_steps(const Weights<MX4, RG, U>& w, const Tokens& t, const int (&row)[NT], const bool (&on)[NT], int groups, int s0, int steps, int q,
                                          f32x4 (&acc)[RG][NT]) {
#pragma unroll
  for (int j = 0; j < U; j++) {
    if (s0 + j >= steps) break;
#pragma unroll
    for (int i = 0; i < NT; i++) {
      if (NT > 1 && i >= groups) break;
      const TokenOp x = token_op<SRC>(t, row[i], on[i], s0 + j, q);
#pragma unroll
      for (int g = 0; g < RG; g++) few_op<MX4>(w.w[j][g], MX4 ? w.s[MX4 ? j / 4 : 0][MX4 ? g : 0] >> (8 * ((s0 + j) & 3)) : 0u, x, acc[g][i]);
    }
  }
}

// The channel of a strip's row r (0 .. 16 RG - 1) from the strip's block of 64 on; g0: the strip's first group in its block
__device__ __forceinline__ int channel_of(int g, int r) { return 32 * (g >> 1) + 8 * (r >> 2) + 4 * (g & 1) + (r & 3); }

// ------------------------------------------------------------------------------------------------ experts' lists
constexpr int MOE_E = 256, MOE_PAIRS = 1024;   // most experts; most (token, choice) pairs
struct MoeLists {
  int count[MOE_E], at[MOE_E + 1], cursor[MOE_E], active[MOE_E], list[MOE_PAIRS], n_active;
};
// From the picks of all pairs: the chosen experts in ascending order, and each one's pairs.  (The order of an expert's pairs is as it comes: it says which column of
// an op a token is, which no result depends on.)
__device__ __forceinline__ void moe_lists(const int* __restrict__ picks, int pairs, MoeLists& l) {
  const int tid = threadIdx.x;
  if (tid < MOE_E) l.count[tid] = 0;
  __syncthreads();
  for (int p = tid; p < pairs; p += THREADS) atomicAdd(&l.count[picks[p]], 1);
  __syncthreads();
  if (tid < 64) {                                              // four experts a lane
    int n[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      n[i] = l.count[4 * tid + i];
      sum += n[i] | (n[i] > 0 ? 1 << 16 : 0);                  // pairs below, chosen experts above
    }
    int upto = sum;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int x = __shfl_up(upto, s, 64);
      if (tid >= s) upto += x;
    }
    int run = upto - sum;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int e = 4 * tid + i;
      l.at[e] = l.cursor[e] = run & 0xFFFF;
      if (n[i] > 0) l.active[run >> 16] = e;
      run += n[i] | (n[i] > 0 ? 1 << 16 : 0);
    }
    if (tid == 63) {
      l.at[MOE_E] = run & 0xFFFF;
      l.n_active = run >> 16;
    }
  }
  __syncthreads();
  for (int p = tid; p < pairs; p += THREADS) l.list[atomicAdd(&l.cursor[picks[p]], 1)] = p;
  __syncthreads();
}

// ------------------------------------------------------------------------------------------------ up
struct UpArgs {
  const char* w; size_t w_stride;      // weights of an expert (operand form, codes then scales) and bytes to the next expert's
  size_t scales_at;                    // where an expert's scales start
  int steps, K, F, T;                  // steps of K; features
  Gate gate;
  const char* x;                       // bf16 [T][K]
  char* h; char* h_scales; int h_steps;   // bf16 rows [..][F], or the mx4 operand form
  const int* picks; int k;             // MOE: [T][k]
};

// grid (F / 32, slots).  A slot is a chosen expert; without MOE there is one, and it has all tokens.
template <bool MX4, int NT, bool MOE>
__global__ void __launch_bounds__(THREADS) few_up_kernel(UpArgs e) {
  constexpr int RG = 4, U = 2, SRC = MX4 ? ROWS_TO_MX4 : ROWS_BF16;
  __shared__ __attribute__((aligned(16))) float red[WAVES * 64 * RED];
  __shared__ MoeLists lists[MOE ? 1 : 1];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned id = run_of(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y), slot = id / gridDim.x;
  const int strip = (int)(id - slot * gridDim.x);
  int expert = 0, n = e.T, first = 0;
  if constexpr (MOE) {
    moe_lists(e.picks, e.T * e.k, lists[0]);
    if ((int)slot >= lists[0].n_active) return;
    expert = lists[0].active[slot];
    first = lists[0].at[expert];
    n = lists[0].count[expert];
  }
  const char* codes = e.w + (size_t)expert * e.w_stride;
  const Strip w{codes + (size_t)strip * e.steps * MX4_PANEL, codes + e.scales_at + (size_t)strip * ((e.steps + 3) >> 2) * 1024, e.steps};
  const Tokens x{e.x, nullptr, e.K, 0};

  for (int t0 = 0; t0 < n; t0 += 16 * NT) {
    int row[NT];
    bool on[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) {
      const int at = t0 + 16 * i + c;
      on[i] = at < n;
      const int p = on[i] ? (MOE ? lists[0].list[first + at] : at) : 0;
      row[i] = MOE ? p / e.k : p;
    }
    const int groups = min((n - t0 + 15) >> 4, NT);
    f32x4 acc[RG][NT];
#pragma unroll
    for (int g = 0; g < RG; g++)
#pragma unroll
      for (int i = 0; i < NT; i++) acc[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    Weights<MX4, RG, U> now, next;
    int s = wave * U;
    if (s < e.steps) now.load(w, s, lane);
    for (; s < e.steps; s += WAVES * U) {
      const bool more = s + WAVES * U < e.steps;
      if (more) next.load(w, s + WAVES * U, lane);
      few_steps<MX4, SRC, RG, U, NT>(now, x, row, on, groups, s, e.steps, q, acc);
      if (more) now = next;
    }
    for (int i = 0; i < groups; i++) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NT; j++)
        if (j == i) {
#pragma unroll
          for (int g = 0; g < RG; g++)
#pragma unroll
            for (int v = 0; v < 4; v++) red[(wave * 64 + 16 * g + 4 * q + v) * RED + c] = acc[g][j][v];
        }
      __syncthreads();
      // 32 neighbouring lanes have the features of a token
      const int f = tid & 31, tok = tid >> 5, r = ((f >> 2) & 1) * 16 + 4 * (f >> 3) + (f & 3), at = t0 + 16 * i + tok;
      float gate = 0.f, up = 0.f;
#pragma unroll
      for (int k = 0; k < WAVES; k++) {
        gate += red[(k * 64 + r) * RED + tok];
        up += red[(k * 64 + 32 + r) * RED + tok];
      }
      const float h = gate_act(e.gate, gate) * up;
      const int dest = at < n ? (MOE ? lists[0].list[first + at] : at) : 0;
      if constexpr (MX4) {
        uint32_t top = magnitude(h);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
        const uint32_t code = mx4_scale_code(top);
        uint32_t word = (__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, h, 0.f, mx4_scale(code), 0) & 15u) << (4 * (f & 7));
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) word |= (uint32_t)__shfl_xor((int)word, d, 64);
        if (at < n && (f & 7) == 0) *reinterpret_cast<uint32_t*>(e.h + mx4_code_at(dest, strip, e.h_steps) + (f >> 1)) = word;
        if (at < n && f == 0) e.h_scales[mx4_scale_at(dest, strip, e.h_steps)] = (char)code;
      } else {
        if (at < n) reinterpret_cast<uint16_t*>(e.h)[(size_t)dest * e.F + 32 * strip + f] = (uint16_t)pack_bf16x2(h, 0.f);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ a product by itself
struct RowsArgs {
  const char* w; const char* w_scales; int steps, K, N, T;
  const char* x; const char* x_scales; int x_steps;
  uint16_t* out;
};
template <bool MX4, int RG, int NT, int SRC>
__global__ void __launch_bounds__(THREADS) few_rows_kernel(RowsArgs e) {
  constexpr int U = SRC == ROWS_TO_MX4 && RG == 1 ? 4 : 8 / RG;
  __shared__ __attribute__((aligned(16))) float red[WAVES * 16 * RG * RED];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int strip = (int)run_of(blockIdx.x, gridDim.x), block = strip / (4 / RG), g0 = strip % (4 / RG) * RG;
  const Strip w{e.w + (size_t)block * e.steps * MX4_PANEL + g0 * 1024, e.w_scales + (size_t)block * ((e.steps + 3) >> 2) * 1024 + g0 * 256, e.steps};
  const Tokens x{e.x, e.x_scales, e.K, e.x_steps};
  int row[NT];
  bool on[NT];
#pragma unroll
  for (int i = 0; i < NT; i++) {
    row[i] = 16 * i + c;
    on[i] = row[i] < e.T;
  }
  f32x4 acc[RG][NT];
#pragma unroll
  for (int g = 0; g < RG; g++)
#pragma unroll
    for (int i = 0; i < NT; i++) acc[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  Weights<MX4, RG, U> now, next;
  int s = wave * U;
  if (s < e.steps) now.load(w, s, lane);
  for (; s < e.steps; s += WAVES * U) {
    const bool more = s + WAVES * U < e.steps;
    if (more) next.load(w, s + WAVES * U, lane);
    few_steps<MX4, SRC, RG, U, NT>(now, x, row, on, NT, s, e.steps, q, acc);
    if (more) now = next;
  }
#pragma unroll
  for (int i = 0; i < NT; i++) {
    if (i > 0) __syncthreads();
#pragma unroll
    for (int g = 0; g < RG; g++)
#pragma unroll
      for (int v = 0; v < 4; v++) red[(wave * 16 * RG + 16 * g + 4 * q + v) * RED + c] = acc[g][i][v];
    __syncthreads();
    for (int o = tid; o < 16 * RG * 16; o += THREADS) {
      const int r = o % (16 * RG), tok = o / (16 * RG), t = 16 * i + tok, ch = 64 * block + channel_of(g0 + r / 16, r % 16);
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < WAVES; k++) sum += red[(k * 16 * RG + r) * RED + tok];
      if (t < e.T && ch < e.N) e.out[(size_t)t * e.N + ch] = (uint16_t)pack_bf16x2(sum, 0.f);
    }
  }
}

// ------------------------------------------------------------------------------------------------ down, with the shares
struct DownArgs {
  const char* w; size_t w_stride, scales_at;
  int steps, F, D, T, k;
  const char* h; const char* h_scales; int h_steps;   // rows by pair
  const int* picks; const float* shares;
  uint16_t* out;
};
constexpr int SUM = 20;                                    // pitch of a token's 16 channels
constexpr int down_lds(int T) { return WAVES * T * SUM * 4; }

// grid (D / 16)
template <bool MX4, int NT>
__global__ void __launch_bounds__(THREADS) moe_down_kernel(DownArgs e) {
  constexpr int U = 8, SRC = MX4 ? OPERAND_MX4 : ROWS_BF16;
  extern __shared__ __attribute__((aligned(16))) float sums[];   // [wave][token][SUM]
  __shared__ MoeLists lists;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int strip = (int)run_of(blockIdx.x, gridDim.x), block = strip >> 2, g0 = strip & 3;
  for (int i = tid; i < WAVES * e.T * SUM; i += THREADS) sums[i] = 0.f;
  moe_lists(e.picks, e.T * e.k, lists);
  float* mine = sums + wave * e.T * SUM;
  const Tokens x{e.h, e.h_scales, e.F, e.h_steps};
  const int units = (e.steps + U - 1) / U, total = lists.n_active * units;   // units of U steps, the experts' one after the other, dealt out to the waves
  auto strip_of = [&](int i, int& expert) {
    expert = lists.active[i / units];
    const char* codes = e.w + (size_t)expert * e.w_stride;
    return Strip{codes + (size_t)block * e.steps * MX4_PANEL + g0 * 1024, codes + e.scales_at + (size_t)block * ((e.steps + 3) >> 2) * 1024 + g0 * 256, e.steps};
  };
  Weights<MX4, 1, U> now, next;
  int i = wave, expert = 0;
  if (i < total) now.load(strip_of(i, expert), i % units * U, lane);
  for (; i < total; i += WAVES) {
    const bool more = i + WAVES < total;
    int then = 0;
    if (more) next.load(strip_of(i + WAVES, then), (i + WAVES) % units * U, lane);
    const int n = lists.count[expert], first = lists.at[expert];
    for (int t0 = 0; t0 < n; t0 += 16 * NT) {
      int row[NT];
      bool on[NT];
#pragma unroll
      for (int g = 0; g < NT; g++) {
        const int at = t0 + 16 * g + c;
        on[g] = at < n;
        row[g] = on[g] ? lists.list[first + at] : 0;
      }
      f32x4 acc[1][NT];
#pragma unroll
      for (int g = 0; g < NT; g++) acc[0][g] = f32x4{0.f, 0.f, 0.f, 0.f};
      few_steps<MX4, SRC, 1, U, NT>(now, x, row, on, min((n - t0 + 15) >> 4, NT), i % units * U, e.steps, q, acc);
#pragma unroll
      for (int g = 0; g < NT; g++)
        if (on[g]) {                                       // (a token chooses an expert once: no two lanes of a quarter have the same one)
          const float p = e.shares[row[g]];
          f32x4* to = reinterpret_cast<f32x4*>(mine + row[g] / e.k * SUM + 4 * q);
          f32x4 y = *to;
#pragma unroll
          for (int v = 0; v < 4; v++) y[v] += p * acc[0][g][v];
          *to = y;
        }
    }
    if (more) now = next;
    expert = then;
  }
  __syncthreads();
  for (int o = tid; o < 16 * e.T; o += THREADS) {
    const int r = o & 15, t = o >> 4, ch = 64 * block + channel_of(g0, r);
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < WAVES; k++) y += sums[(k * e.T + t) * SUM + r];
    if (ch < e.D) e.out[(size_t)t * e.D + ch] = (uint16_t)pack_bf16x2(y, 0.f);
  }
}

// ------------------------------------------------------------------------------------------------ router
constexpr int ROUTE_D = 64, ROUTE_T = 8;   // of D and of the tokens a workgroup
// grid (D / 64, T / 8); parts [D / 64][T][E]
__global__ void __launch_bounds__(256) moe_router_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ Wr, int T, int D, int E, double* __restrict__ parts) {
  __shared__ float x[ROUTE_T][ROUTE_D];
  __shared__ double sums[256 * ROUTE_T];
  const int tid = threadIdx.x, d0 = blockIdx.x * ROUTE_D, t0 = blockIdx.y * ROUTE_T, tokens = min(T - t0, ROUTE_T);
  for (int i = tid; i < tokens * ROUTE_D; i += 256) x[i / ROUTE_D][i % ROUTE_D] = bf16_lo_to_f32(X[(size_t)(t0 + i / ROUTE_D) * D + d0 + i % ROUTE_D]);
  __syncthreads();
  const int ways = 256 / E, way = tid / E, ex = tid - way * E;   // the rows of Wr are dealt out to `ways` groups of E work items
  double acc[ROUTE_T] = {};
  if (way < ways) {
    for (int d = way; d < ROUTE_D; d += ways) {
      const float w = bf16_lo_to_f32(Wr[(size_t)(d0 + d) * E + ex]);
#pragma unroll
      for (int t = 0; t < ROUTE_T; t++)
        if (t < tokens) acc[t] += (double)(x[t][d] * w);
    }
#pragma unroll
    for (int t = 0; t < ROUTE_T; t++)
      if (t < tokens) sums[(t * ways + way) * E + ex] = acc[t];
  }
  __syncthreads();
  for (int i = tid; i < tokens * E; i += 256) {
    const int t = i / E, n = i - t * E;
    double s = 0.0;
    for (int k = 0; k < ways; k++) s += sums[(t * ways + k) * E + n];
    parts[((size_t)blockIdx.x * T + t0 + t) * E + n] = s;
  }
}

// A value as an integer of the same order; NaN below all
__device__ __forceinline__ unsigned long long order_of(double x) {
  const unsigned long long b = __builtin_bit_cast(unsigned long long, x + 0.0);   // (-0 is 0)
  return x != x ? 0ull : b >> 63 ? ~b : b | 1ull << 63;
}
// a workgroup a token
__global__ void __launch_bounds__(256) moe_pick_kernel(const double* __restrict__ parts, int n_parts, int T, int E, int k, int renormalise, int* __restrict__ picks,
                                                       float* __restrict__ shares) {
  __shared__ unsigned long long order[MOE_E];
  __shared__ double logit[MOE_E], chosen[16];
  __shared__ float part[4];
  const int t = blockIdx.x, e = threadIdx.x;
  double s = 0.0;
  if (e < E) {
    const double* p = parts + (size_t)t * E + e;
#pragma unroll 8
    for (int i = 0; i < n_parts; i++) s += p[(size_t)i * T * E];
    order[e] = order_of(s);
    logit[e] = s;
  }
  __syncthreads();
  int rank = MOE_E;
  if (e < E) {
    const unsigned long long mine = order[e];
    rank = 0;
    for (int i = 0; i < E; i++) rank += order[i] > mine || (order[i] == mine && i < e);
    if (rank < k) {
      picks[t * k + rank] = e;
      chosen[rank] = s;
    }
  }
  __syncthreads();
  // shares: exp(l - largest) over its sum, of the chosen or of all
  const float x = e < E && (rank < k || !renormalise) ? expf((float)(s - chosen[0])) : 0.f;
  float sum = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
  if ((e & 63) == 0) part[e >> 6] = sum;
  __syncthreads();
  if (rank < k) shares[t * k + rank] = x / (part[0] + part[1] + part[2] + part[3]);
}

template <int NT, bool MOE>
int launch_up(const UpArgs& a, bool mx4, int slots, hipStream_t s) {
  const dim3 grid((unsigned)(a.F / 32), (unsigned)slots);
  if (mx4) hipLaunchKernelGGL((few_up_kernel<true, NT, MOE>), grid, dim3(THREADS), 0, s, a);
  else hipLaunchKernelGGL((few_up_kernel<false, NT, MOE>), grid, dim3(THREADS), 0, s, a);
  return (int)hipGetLastError();
}
template <bool MX4, int NT>
int launch_down(const DownArgs& a, hipStream_t s) {
  auto kern = moe_down_kernel<MX4, NT>;
  static std::atomic<bool> configured[MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), down_lds(MOE_TOKENS), configured)) return rc;
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.D / 16)), dim3(THREADS), down_lds(a.T), s, a);
  return (int)hipGetLastError();
}
template <int RG, int SRC>
int launch_rows(const RowsArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(RG == 1 ? (a.N + 31) / 32 * 2 : (a.N + 16 * RG - 1) / (16 * RG)));   // (two groups of 16 share 32 channels)
  if (a.T <= 16) hipLaunchKernelGGL((few_rows_kernel<true, RG, 1, SRC>), grid, dim3(THREADS), 0, s, a);
  else hipLaunchKernelGGL((few_rows_kernel<true, RG, 2, SRC>), grid, dim3(THREADS), 0, s, a);
  return (int)hipGetLastError();
}
}  // namespace

size_t moe_parts_size(int T, int D, int E) { return (size_t)(D / ROUTE_D) * T * E * sizeof(double); }

int launch_moe_route(const void* X, const void* Wr, int T, int D, int E, int k, bool renormalise, void* parts, int* picks, float* shares, hipStream_t s) {
  const int n = D / ROUTE_D;
  hipLaunchKernelGGL(moe_router_kernel, dim3((unsigned)n, (unsigned)((T + ROUTE_T - 1) / ROUTE_T)), dim3(256), 0, s, static_cast<const uint16_t*>(X),
                     static_cast<const uint16_t*>(Wr), T, D, E, static_cast<double*>(parts));
  hipLaunchKernelGGL(moe_pick_kernel, dim3((unsigned)T), dim3(256), 0, s, static_cast<const double*>(parts), n, T, E, k, (int)renormalise, picks, shares);
  return (int)hipGetLastError();
}

int launch_moe_experts(const MoeWeights& w, const void* X, int T, int D, int F, int E, int k, float c1, float c3, const int* picks, const float* shares, void* H, int h_rows,
                       void* Y, hipStream_t s) {
  UpArgs up{};
  up.w = static_cast<const char*>(w.up); up.w_stride = w.up_stride; up.scales_at = w.up_scales;
  up.K = D; up.F = F; up.T = T; up.steps = w.mx4 ? mx4_steps(D) : D / 32; up.gate = Gate{c1, c3};
  up.x = static_cast<const char*>(X);
  const Mx4Operand h = mx4_operand(H, h_rows, F);
  up.h = const_cast<char*>(w.mx4 ? h.codes : static_cast<const char*>(H));
  up.h_scales = const_cast<char*>(h.scales);
  up.h_steps = h.steps;
  up.picks = picks; up.k = k;
  const int slots = T * k < E ? T * k : E;
  const int rc = T <= 16 ? launch_up<1, true>(up, w.mx4, slots, s) : T <= 32 ? launch_up<2, true>(up, w.mx4, slots, s) : launch_up<4, true>(up, w.mx4, slots, s);
  if (rc) return rc;
  DownArgs d{};
  d.w = static_cast<const char*>(w.down); d.w_stride = w.down_stride; d.scales_at = w.down_scales;
  d.steps = w.mx4 ? mx4_steps(F) : F / 32; d.F = F; d.D = D; d.T = T; d.k = k;
  d.h = up.h; d.h_scales = h.scales; d.h_steps = h.steps;
  d.picks = picks; d.shares = shares; d.out = static_cast<uint16_t*>(Y);
  if (T <= 16) return w.mx4 ? launch_down<true, 1>(d, s) : launch_down<false, 1>(d, s);
  return w.mx4 ? launch_down<true, 4>(d, s) : launch_down<false, 4>(d, s);
}

int launch_few_mx4_up(const Mx4Operand& w, const void* X, int T, int D, int F, float c1, float c3, const Mx4Operand& h, hipStream_t s) {
  UpArgs up{};
  up.w = w.codes; up.scales_at = (size_t)(w.scales - w.codes);
  up.K = D; up.F = F; up.T = T; up.steps = w.steps; up.gate = Gate{c1, c3};
  up.x = static_cast<const char*>(X);
  up.h = const_cast<char*>(h.codes); up.h_scales = const_cast<char*>(h.scales); up.h_steps = h.steps;
  return T <= 16 ? launch_up<1, false>(up, true, 1, s) : launch_up<2, false>(up, true, 1, s);
}
// Strips of 64, 32 or 16 channels: at least 512 workgroups if there are that many
int launch_few_mx4_rows(const Mx4Operand& w, int K, int N, const void* X, const Mx4Operand* x, int T, void* Y, hipStream_t s) {
  RowsArgs a{w.codes, w.scales, w.steps, K, N, T, static_cast<const char*>(X), nullptr, 0, static_cast<uint16_t*>(Y)};
  if (x) { a.x = x->codes; a.x_scales = x->scales; a.x_steps = x->steps; }
  if (N >= 512 * 64) return x ? launch_rows<4, OPERAND_MX4>(a, s) : launch_rows<4, ROWS_TO_MX4>(a, s);
  if (N >= 512 * 32) return x ? launch_rows<2, OPERAND_MX4>(a, s) : launch_rows<2, ROWS_TO_MX4>(a, s);
  return x ? launch_rows<1, OPERAND_MX4>(a, s) : launch_rows<1, ROWS_TO_MX4>(a, s);
}

}  // namespace ffn24
