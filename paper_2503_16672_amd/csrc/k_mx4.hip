// mx4 numbers (mx4_core.hpp): quantisation and back, the weights' layout, the products of many tokens.
//
//   scale = 2^(floor(log2 max |block|) - 2) over 32 neighbours of a row (no less than 2^-127);  code = x / scale to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even
// code).  Both rounding kernels and the tokens' are bound by memory and move every byte once, 16 bytes a lane, non-temporal: 16384 x 4096 bf16 26 us to codes and scales and 28 back
// (170 MB, 6.4 and 6.0 TB/s: the largest copy here reaches 6.4, reads alone 7.1), 1031 x 1056 fp32 2.9 and 3.5 us (a launch); 8192 x 4096 tokens to the operand form 17 us (5.0 TB/s).  The
// weights' layout, once: 4096 x 16384 42 us.
#include "mx4_core.hpp"
#include "launch_edge.hpp"
#include "mx4_rule.hpp"

namespace ffn24 {
namespace {

// Eight values of a row: as bf16 or fp32 in memory
template <bool F32> struct Eight;
template <> struct Eight<false> {
  u32x4 w;
  __device__ __forceinline__ void load(const void* p, size_t i) { w = ld_stream(static_cast<const u32x4*>(p) + i); }
  __device__ __forceinline__ uint32_t top() const { return mx4_top8(w); }
  __device__ __forceinline__ uint32_t codes(float s) const { return mx4_codes8(w, s); }
};
template <> struct Eight<true> {
  f32x4 x[2];
  __device__ __forceinline__ void load(const void* p, size_t i) {
    x[0] = ld_stream(static_cast<const f32x4*>(p) + 2 * i);
    x[1] = ld_stream(static_cast<const f32x4*>(p) + 2 * i + 1);
  }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t t = 0u;
#pragma unroll
    for (int i = 0; i < 8; i++) t = max(t, magnitude(x[i / 4][i % 4]));
    return t;
  }
  __device__ __forceinline__ uint32_t codes(float s) const {
    const float v[8] = {x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]};
    return mx4_codes8(v, s);
  }
};

constexpr int ROUND_U = 4;      // pieces of 8 values a work item
// Row-major codes and scales: a stream of blocks.  Four lanes have a block, each 8 values.
template <bool F32>
__global__ void __launch_bounds__(256) quantise_mx4_kernel(const void* __restrict__ X, size_t pieces, uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const size_t at = (size_t)blockIdx.x * (256 * ROUND_U) + threadIdx.x;
  Eight<F32> x[ROUND_U];
#pragma unroll
  for (int u = 0; u < ROUND_U; u++)
    if (at + 256 * u < pieces) x[u].load(X, at + 256 * u);
#pragma unroll
  for (int u = 0; u < ROUND_U; u++) {
    const size_t i = at + 256 * u;
    if (i >= pieces) break;                                    // (pieces is a multiple of 4: a block's lanes leave together)
    const uint32_t code = mx4_scale_code(quad_max(x[u].top()));
    st_stream(codes + i, x[u].codes(mx4_scale(code)));
    if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)code;
  }
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
template <bool F32>
__global__ void __launch_bounds__(256) dequantise_mx4_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, size_t pieces, void* __restrict__ Y) {
  const size_t at = (size_t)blockIdx.x * (256 * ROUND_U) + threadIdx.x;
  uint32_t w[ROUND_U], c[ROUND_U];
#pragma unroll
  for (int u = 0; u < ROUND_U; u++) {
    const size_t i = at + 256 * u;
    if (i < pieces) {
      w[u] = ld_stream(codes + i);
      c[u] = scales[i >> 2];
    }
  }
#pragma unroll
  for (int u = 0; u < ROUND_U; u++) {
    const size_t i = at + 256 * u;
    if (i >= pieces) break;
    const float s = mx4_scale(c[u]);
    const bool nan = c[u] == 255u;
    if constexpr (F32) {
      f32x4 o[2];
#define FFN24_PAIR(j) { const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], s, j); o[j / 2][2 * (j % 2)] = v[0]; o[j / 2][2 * (j % 2) + 1] = v[1]; }
      FFN24_PAIR(0) FFN24_PAIR(1) FFN24_PAIR(2) FFN24_PAIR(3)
#undef FFN24_PAIR
      if (nan) o[0] = o[1] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
      st_stream(static_cast<f32x4*>(Y) + 2 * i, o[0]);
      st_stream(static_cast<f32x4*>(Y) + 2 * i + 1, o[1]);
    } else {
      u32x4 o;
#define FFN24_PAIR(j) o[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], s, j));
      FFN24_PAIR(0) FFN24_PAIR(1) FFN24_PAIR(2) FFN24_PAIR(3)
#undef FFN24_PAIR
      if (nan) o = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
      st_stream(static_cast<u32x4*>(Y) + i, o);
    }
  }
}

// Tokens to the operand form: a wave takes 4 R of 16 rows and four steps, 4 rows and a step (256 bytes of each, whole lines) a load.  Four lanes have a block of 32.
template <int R>
__global__ void __launch_bounds__(256) mx4_tokens_kernel(const uint16_t* __restrict__ X, int T, int K, int steps, char* __restrict__ codes, char* __restrict__ scales) {
  const int quads = (steps + 3) >> 2;
  const int id = blockIdx.x * 4 + (threadIdx.x >> 6), part = id / quads, S = id - part * quads, lane = threadIdx.x & 63, c = lane >> 4, q = (lane >> 2) & 3, p = lane & 3;
  const int group = part / (4 / R), i0 = part % (4 / R) * R;
  if (16 * group >= T) return;
  u32x4 w[4][R];                                               // [step][4 rows]
#pragma unroll
  for (int j = 0; j < 4; j++)
#pragma unroll
    for (int i = 0; i < R; i++) {
      const int k = 128 * (4 * S + j) + 8 * (lane & 15), r = 16 * group + 4 * (i0 + i) + c;
      w[j][i] = k < K && r < T ? ld_stream(reinterpret_cast<const u32x4*>(X + (size_t)r * K + k)) : u32x4{0u, 0u, 0u, 0u};
    }
  char* out = codes + mx4_code_at(16 * group, 16 * S, steps) + q * 256 + 4 * p;
#pragma unroll
  for (int i = 0; i < R; i++) {
    const int r = 4 * (i0 + i) + c;
    uint32_t mine = 0u;                                        // the scales of the quarter's four steps
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const uint32_t code = mx4_scale_code(quad_max(mx4_top8(w[j][i])));
      mine |= code << (8 * j);
      if (4 * S + j < steps) *reinterpret_cast<uint32_t*>(out + (size_t)j * MX4_PANEL + r * 16) = mx4_codes8(w[j][i], mx4_scale(code));
    }
    if (p == 0) *reinterpret_cast<uint32_t*>(scales + mx4_scale_at(16 * group + r, 16 * S + q, steps)) = mine;
  }
}

// Weights to the operand form, a workgroup 64 rows and a step: lane = channel of the block, wave = quarter of the step.  FORM 0: bf16 W [K][N] to mx4; 1: codes [N][K / 2] and
// scales [N][K / 32]; 2: bf16 W as bf16, 32 k a step.  F > 0: bf16 W is [gate | up] of F channels each.  grid (blocks, steps, matrices)
enum { FROM_BF16 = 0, FROM_CODES = 1, KEEP_BF16 = 2 };
template <int FORM>
__global__ void __launch_bounds__(256) operand_weight_kernel(const void* __restrict__ W, const uint8_t* __restrict__ Ws, int K, int N, int F, int steps, char* __restrict__ codes,
                                                             char* __restrict__ scales, size_t w_stride, size_t code_stride, size_t scale_stride) {
  constexpr int KS = FORM == KEEP_BF16 ? 32 : MX4_STEP, KQ = KS / 4;
  const int block = blockIdx.x, step = blockIdx.y, lane = threadIdx.x & 63, q = threadIdx.x >> 6, k0 = KS * step + KQ * q;
  if constexpr (FORM == FROM_CODES) F = 0;
  const int n = F > 0 ? 32 * block + (lane & 31) + (lane >> 5) * F : 64 * block + lane;
  const int row = (2 * (lane >> 5) + ((lane >> 2) & 1)) * 16 + 4 * ((lane >> 3) & 3) + (lane & 3);
  const bool in = k0 < K && (F > 0 ? 32 * block + (lane & 31) < F : n < N);
  u32x4 o = {0u, 0u, 0u, 0u};
  uint32_t code = 0u;
  if (in) {
    if constexpr (FORM == FROM_CODES) {
      o = *reinterpret_cast<const u32x4*>(static_cast<const char*>(W) + (size_t)n * (K / 2) + k0 / 2);
      code = Ws[(size_t)n * (K / 32) + k0 / 32];
    } else {
      const uint16_t* w = static_cast<const uint16_t*>(W) + blockIdx.z * w_stride + (size_t)k0 * N + n;
      u32x4 v[KQ / 8];
#pragma unroll
      for (int j = 0; j < KQ / 8; j++)
#pragma unroll
        for (int i = 0; i < 4; i++) v[j][i] = (uint32_t)w[(size_t)(8 * j + 2 * i) * N] | (uint32_t)w[(size_t)(8 * j + 2 * i + 1) * N] << 16;
      if constexpr (FORM == KEEP_BF16) {
        o = v[0];
      } else {
        uint32_t top = 0u;
#pragma unroll
        for (int j = 0; j < 4; j++) top = max(top, mx4_top8(v[j]));
        code = mx4_scale_code(top);
#pragma unroll
        for (int j = 0; j < 4; j++) o[j] = mx4_codes8(v[j], mx4_scale(code));
      }
    }
  }
  const int place = (row >> 4) * 64 + q * 16 + (row & 15);
  *reinterpret_cast<u32x4*>(codes + blockIdx.z * code_stride + ((size_t)block * steps + step) * MX4_PANEL + place * 16) = o;
  if constexpr (FORM != KEEP_BF16) {
    uint8_t* s = reinterpret_cast<uint8_t*>(scales) + blockIdx.z * scale_stride + ((size_t)block * ((steps + 3) >> 2) + (step >> 2)) * 1024 + place * 4;
    s[step & 3] = (uint8_t)code;
    // (the last four steps' scales are whole: an op never takes them, the streaming kernels read them)
    if (step == steps - 1)
      for (int j = (step & 3) + 1; j < 4; j++) s[j] = 0;
  }
}

template <class Epi, int AM, int BN>
int launch_mx4_tile(Mx4Gemm g, const typename Epi::Args& ea, int splits, int part, hipStream_t s) {
  using G = Mx4Geo<AM, BN>;
  auto kern = mx4_gemm_kernel<Epi, AM, BN>;
  static std::atomic<bool> configured[MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), G::LDS, configured)) return rc;
  const int tm = (g.M + G::BM - 1) / G::BM, tn = (g.N + G::BNT - 1) / G::BNT;
  g.first = 0;
  g.steps = g.A.steps;
  hipLaunchKernelGGL(kern, dim3((unsigned)(tm * tn * splits)), dim3(GEMM_THREADS), G::LDS, s, g, ea, tm, tn, splits > 1 ? part : 0);
  return (int)hipGetLastError();
}
template <class Epi>
int launch_mx4(const Mx4Gemm& g, const typename Epi::Args& ea, int tile, hipStream_t s) {
  switch (tile) {
    case 0: return launch_mx4_tile<Epi, 8, 8>(g, ea, 1, 0, s);
    case 1: return launch_mx4_tile<Epi, 8, 4>(g, ea, 1, 0, s);
    case 2: return launch_mx4_tile<Epi, 4, 4>(g, ea, 1, 0, s);
    default: return launch_mx4_tile<Epi, 4, 2>(g, ea, 1, 0, s);
  }
}
}  // namespace

int launch_quantise_mx4(const void* X, bool f32, int64_t T, int64_t K, void* codes, void* scales, hipStream_t s) {
  const size_t pieces = (size_t)T * (size_t)K / 8;
  const dim3 grid((unsigned)((pieces + 256 * ROUND_U - 1) / (256 * ROUND_U)));
  if (f32) hipLaunchKernelGGL((quantise_mx4_kernel<true>), grid, dim3(256), 0, s, X, pieces, static_cast<uint32_t*>(codes), static_cast<uint8_t*>(scales));
  else hipLaunchKernelGGL((quantise_mx4_kernel<false>), grid, dim3(256), 0, s, X, pieces, static_cast<uint32_t*>(codes), static_cast<uint8_t*>(scales));
  return (int)hipGetLastError();
}
int launch_dequantise_mx4(const void* codes, const void* scales, bool f32, int64_t T, int64_t K, void* Y, hipStream_t s) {
  const size_t pieces = (size_t)T * (size_t)K / 8;
  const dim3 grid((unsigned)((pieces + 256 * ROUND_U - 1) / (256 * ROUND_U)));
  if (f32) hipLaunchKernelGGL((dequantise_mx4_kernel<true>), grid, dim3(256), 0, s, static_cast<const uint32_t*>(codes), static_cast<const uint8_t*>(scales), pieces, Y);
  else hipLaunchKernelGGL((dequantise_mx4_kernel<false>), grid, dim3(256), 0, s, static_cast<const uint32_t*>(codes), static_cast<const uint8_t*>(scales), pieces, Y);
  return (int)hipGetLastError();
}

int64_t mx4_operand_size(int64_t rows, int64_t K) {
  const int64_t blocks = (rows + 63) / 64, steps = (K + MX4_STEP - 1) / MX4_STEP;
  return blocks * (steps * MX4_PANEL + (steps + 3) / 4 * 1024);
}
int64_t bf16_operand_size(int64_t rows, int64_t K) { return (rows + 63) / 64 * (K / 32) * MX4_PANEL; }
Mx4Operand mx4_operand(const void* p, int rows, int K) {
  const int steps = mx4_steps(K);
  const char* codes = static_cast<const char*>(p);
  return Mx4Operand{codes, codes + (size_t)((rows + 63) / 64) * steps * MX4_PANEL, steps};
}
int launch_mx4_weight(const void* W, int K, int N, bool halves, int count, void* out, hipStream_t s) {
  const Mx4Operand o = mx4_operand(out, N, K);
  const size_t size = (size_t)mx4_operand_size(N, K);
  hipLaunchKernelGGL((operand_weight_kernel<FROM_BF16>), dim3((unsigned)((N + 63) / 64), (unsigned)o.steps, (unsigned)count), dim3(256), 0, s, W, nullptr, K, N,
                     halves ? N / 2 : 0, o.steps, const_cast<char*>(o.codes), const_cast<char*>(o.scales), (size_t)K * N, size, size);
  return (int)hipGetLastError();
}
int launch_mx4_weight_codes(const void* codes, const void* scales, int K, int N, void* out, hipStream_t s) {
  const Mx4Operand o = mx4_operand(out, N, K);
  hipLaunchKernelGGL((operand_weight_kernel<FROM_CODES>), dim3((unsigned)((N + 63) / 64), (unsigned)o.steps), dim3(256), 0, s, codes, static_cast<const uint8_t*>(scales), K, N,
                     0, o.steps, const_cast<char*>(o.codes), const_cast<char*>(o.scales), (size_t)0, (size_t)0, (size_t)0);
  return (int)hipGetLastError();
}
int launch_bf16_weight(const void* W, int K, int N, bool halves, int count, void* out, hipStream_t s) {
  hipLaunchKernelGGL((operand_weight_kernel<KEEP_BF16>), dim3((unsigned)((N + 63) / 64), (unsigned)(K / 32), (unsigned)count), dim3(256), 0, s, W, nullptr, K, N,
                     halves ? N / 2 : 0, K / 32, static_cast<char*>(out), nullptr, (size_t)K * N, (size_t)bf16_operand_size(N, K), (size_t)0);
  return (int)hipGetLastError();
}
template <int R>
int launch_mx4_tokens_rows(const void* X, int T, int K, const Mx4Operand& o, hipStream_t s) {
  const long long waves = (long long)((T + 15) / 16) * (4 / R) * ((o.steps + 3) / 4);
  hipLaunchKernelGGL(mx4_tokens_kernel<R>, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, static_cast<const uint16_t*>(X), T, K, o.steps, const_cast<char*>(o.codes),
                     const_cast<char*>(o.scales));
  return (int)hipGetLastError();
}
int launch_mx4_tokens(const void* X, int T, int K, const Mx4Operand& o, hipStream_t s) {
  return mx4_tokens_rows(T, o.steps) == 1 ? launch_mx4_tokens_rows<1>(X, T, K, o, s) : launch_mx4_tokens_rows<4>(X, T, K, o, s);
}

size_t mx4_split_scratch(int M, int N, int K) {
  const Mx4Plan p = mx4_plan(M, N, mx4_steps(K), true);
  return p.splits > 1 ? (size_t)4 * p.splits * M * up_to(N, 64) : 0;
}
int launch_mx4_product(const Mx4Operand& w, int M, const Mx4Operand& x, int T, void* Y, const Scratch& scratch, hipStream_t s) {
  const Mx4Gemm g{w, x, M, T, 0, 0};
  const Mx4Plan p = mx4_plan(M, T, w.steps, true);
  if (p.splits == 1 || mx4_split_scratch(M, T, w.steps * MX4_STEP) > scratch.bytes)
    return launch_mx4<Mx4Rows>(g, Mx4Rows::Args{static_cast<uint16_t*>(Y), M, T}, p.tile, s);
  uint32_t* parts = static_cast<uint32_t*>(scratch.p);
  if (int rc = launch_mx4_tile<Mx4Part, 4, 2>(g, Mx4Part::Args{parts, M, T}, p.splits, p.part, s)) return rc;
  hipLaunchKernelGGL((edge_sum_kernel<false>), dim3((unsigned)(((size_t)M / 4 * T + 255) / 256)), dim3(256), 0, s, parts, p.splits, M, T, I8Scales{}, static_cast<uint16_t*>(Y));
  return (int)hipGetLastError();
}
int launch_mx4_gated_up(const Mx4Operand& w, int F, const Mx4Operand& x, int T, float c1, float c3, const Mx4Operand& h, hipStream_t s) {
  const Mx4Gemm g{w, x, 2 * F, T, 0, 0};
  const int tile = mx4_plan(2 * F, T, w.steps, false).tile;
  const auto go = [&](auto epi) {
    using Epi = decltype(epi);
    return launch_mx4<Epi>(g, typename Epi::Args{const_cast<char*>(h.codes), reinterpret_cast<uint8_t*>(const_cast<char*>(h.scales)), F, T, h.steps, Gate{c1, c3}}, tile, s);
  };
  return c3 == 0.f && c1 == 1.f ? go(Mx4Gated<false>{}) : go(Mx4Gated<true>{});
}

}  // namespace ffn24
