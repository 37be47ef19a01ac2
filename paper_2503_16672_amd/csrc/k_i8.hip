// Products of 8-bit integers with a scale for each token and each output channel, and the quantisation that makes their operands.
//
//   scale = max |row| * (1 / 127), the factor and the product rounded to fp32 (1 if the row is all zero; infinite or NaN if a value is, and with it every result of the row);  code = rint(x / scale)
//   Y[t][n] = bf16(sum_k X8[t][k] W8[k][n] * (sx[t] * sw[n])), the sum in 32-bit integers: exact up to K = 133144 ((2^31 - 1) / 127^2; 2^17 is the most a call takes), so results do not depend on its order
//
// The weights are laid out once: transposed, K-contiguous, in the A panel form of gemm_core.hpp (64-byte pieces), K filled up to 128 and the channels to 256 with
// zeros, then the scales of the panel's rows, then the words the largest magnitudes are found in.
//
// The quantisation is a pass over the data (8192 x 4096 26 us, 3.8 TB/s; the hidden layer 8192 x 16384, whose maxima the epilogue before it collects, 84 us, 4.8 TB/s); the
// products run at 2.2 (gated, with the gate in the epilogue) and 2.6 POP/s (plain) at 8192 x 4096 x 16384, 2.3 and 2.8 at best: twice the rate of bf16 on the same tiles.
#include "launch_block.hpp"
#include "launch_edge.hpp"
#include "i8_codes.hpp"

namespace ffn24 {
namespace {

// Where the codes of row r from value k on (a multiple of 8) go: row-major, or (panels > 0) the B panel form of gemm_core.hpp, which the large GEMMs read in whole lines:
// 8192 tokens at 4096 x 16384 gated 1411 -> 1366 us.
__device__ __forceinline__ size_t code_at(int r, int k, int K, int panels) {
  return panels ? a24_piece(b_panel_pos(r), k >> 6, panels) * 64 + (k & 63) : (size_t)r * K + k;
}

// Rows of K values (a multiple of 8) to codes, W waves a row, P pieces of 8 values a lane in registers; P = 0: any K, the row read twice (the second time from
// the caches).  zero: a word a row to be cleared, for what a later kernel collects there.
template <int P, int W>
__global__ void __launch_bounds__(256) quantise_i8_kernel(const uint16_t* __restrict__ X, int T, int K, int panels, uint8_t* __restrict__ codes,
                                                          float* __restrict__ scales, uint32_t* __restrict__ zero) {
  constexpr int LANES = 64 * W;
  __shared__ uint32_t part[4];
  const int wave = threadIdx.x >> 6, l = threadIdx.x & (LANES - 1), row = blockIdx.x * (4 / W) + wave / W;
  if (W == 1 && row >= T) return;
  const uint16_t* x = X + (size_t)row * K;
  u32x4 w[P ? P : 1];
  uint32_t top = 0u;
  if constexpr (P > 0) {
#pragma unroll
    for (int p = 0; p < P; p++) {
      const int i = 8 * (p * LANES + l);
      w[p] = i < K ? *reinterpret_cast<const u32x4*>(x + i) : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int p = 0; p < P; p++) top = i8_top8(w[p], top);
  } else {
    for (int i = 8 * l; i < K; i += 8 * LANES) top = i8_top8(*reinterpret_cast<const u32x4*>(x + i), top);
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s, 64));
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) part[wave] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; i++) top = max(top, part[(wave & ~(W - 1)) + i]);
  }
  const float s = i8_scale(top);
  if (l == 0) {
    scales[row] = s;
    if (zero) zero[row] = 0u;
  }
  if constexpr (P > 0) {
#pragma unroll
    for (int p = 0; p < P; p++) {
      const int i = 8 * (p * LANES + l);
      if (i < K) *reinterpret_cast<u32x2*>(codes + code_at(row, i, K, panels)) = i8_codes8(w[p], s);
    }
  } else {
    for (int i = 8 * l; i < K; i += 8 * LANES) *reinterpret_cast<u32x2*>(codes + code_at(row, i, K, panels)) = i8_codes8(*reinterpret_cast<const u32x4*>(x + i), s);
  }
}

// The same with the rows' largest magnitudes given (as words); F a multiple of 16.  A work item takes 16 values.
__global__ void __launch_bounds__(256) quantise_i8_given_kernel(const uint16_t* __restrict__ H, const uint32_t* __restrict__ tops, int T, int F, int panels,
                                                                uint8_t* __restrict__ codes, float* __restrict__ scales) {
  const int per = F / 16, blocks = (per + 255) / 256, row = blockIdx.x / blocks;
  const float s = i8_scale(tops[row]);
  const int i = (blockIdx.x - row * blocks) * 256 + threadIdx.x;
  if (i == 0) scales[row] = s;
  if (i >= per) return;
  const u32x4* p = reinterpret_cast<const u32x4*>(H + (size_t)row * F + 16 * i);
  const u32x2 a = i8_codes8(p[0], s), b = i8_codes8(p[1], s);
  *reinterpret_cast<u32x4*>(codes + code_at(row, 16 * i, F, panels)) = u32x4{a[0], a[1], b[0], b[1]};
}

// Weights.  Panel row of output channel n: n itself, or, with a gate half and an up half of F channels each, 8 gate channels and the 8 up channels of the same numbers in turn.
__device__ __forceinline__ int channel_row(int n, int F) { return F == 0 ? n : 16 * ((n < F ? n : n - F) >> 3) + (n & 7) + (n < F ? 0 : 8); }
__device__ __forceinline__ int row_channel(int r, int F) { return F == 0 ? r : (r >> 4) * 8 + (r & 7) + (r & 8 ? F : 0); }

__global__ void __launch_bounds__(256) i8_weight_clear_kernel(uint32_t* tops, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) tops[i] = 0u;
}
// largest magnitude of each column over TOP_ROWS rows a workgroup of 32 x 8, 8 columns a work item; tops in panel order.  One atomic a column and workgroup: with one a
// column and 8 rows 4096 x 32768 took 660 us.
constexpr int TOP_ROWS = 256;
__global__ void __launch_bounds__(256) i8_weight_top_kernel(const uint16_t* __restrict__ W, int K, int N, int F, uint32_t* tops) {
  __shared__ __attribute__((aligned(16))) uint32_t part[8][256];
  const int tid = threadIdx.x, n0 = blockIdx.x * 256, n = n0 + 8 * (tid & 31), k0 = blockIdx.y * TOP_ROWS + (tid >> 5);
  uint32_t top[8] = {};
  if (n < N) {
    const uint16_t* w = W + (size_t)k0 * N + n;
#pragma unroll 8
    for (int k = k0; k < min(K, (int)blockIdx.y * TOP_ROWS + TOP_ROWS); k += 8, w += 8 * (size_t)N) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(w);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        top[2 * j] = max(top[2 * j], v[j] << 16 & 0x7FFF0000u);
        top[2 * j + 1] = max(top[2 * j + 1], v[j] & 0x7FFF0000u);
      }
    }
  }
  u32x4* mine = reinterpret_cast<u32x4*>(&part[tid >> 5][8 * (tid & 31)]);
  mine[0] = u32x4{top[0], top[1], top[2], top[3]};
  mine[1] = u32x4{top[4], top[5], top[6], top[7]};
  __syncthreads();
  uint32_t most = part[0][tid];
#pragma unroll
  for (int i = 1; i < 8; i++) most = max(most, part[i][tid]);
  if (n0 + tid < N) atomicMax(tops + channel_row(n0 + tid, F), most);
}
// 64 panel rows x 64 k a workgroup: read along the channels, through LDS, out as one run of 64 pieces (4096 x 32768 130 us, 3.1 TB/s, once a weight)
__global__ void __launch_bounds__(256) i8_weight_codes_kernel(const uint16_t* __restrict__ W, int K, int N, int F, int panels, const uint32_t* __restrict__ tops,
                                                              uint8_t* __restrict__ out, float* __restrict__ scales) {
  __shared__ uint8_t tile[64][68];
  const int r0 = blockIdx.x * 64, kp = blockIdx.y;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int k = threadIdx.x / 8 + 32 * i, r = 8 * (threadIdx.x & 7), n = row_channel(r0 + r, F);   // (8 rows: 8 neighbouring channels)
    const bool in = 64 * kp + k < K && (F == 0 ? n < N : r0 + r < N);
    const u32x4 w = in ? *reinterpret_cast<const u32x4*>(W + (size_t)(64 * kp + k) * N + n) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const float s = i8_scale(tops[r0 + r + j]);
      tile[r + j][k] = (uint8_t)i8_code(j % 2 ? bf16_hi_to_f32(w[j / 2]) : bf16_lo_to_f32(w[j / 2]), s);
      if (kp == 0 && k == 0) scales[r0 + r + j] = s;
    }
  }
  __syncthreads();
  const int r = threadIdx.x >> 2, c = threadIdx.x & 3;
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; i++) o[i] = *reinterpret_cast<const uint32_t*>(&tile[r][16 * c + 4 * i]);
  *reinterpret_cast<u32x4*>(out + a24_piece(r0 + r, kp, panels) * 64 + 16 * c) = o;
}

int64_t pad(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
GemmArgs args(const I8Layout& w, const void* codes, int T, bool panels = false) {
  GemmArgs g{};
  g.A = w.panels; g.a_panel = 1; g.a_pitch = (int)pad(w.K, 128);
  g.B = codes; g.b_rows = T; g.b_pitch = panels ? (int)pad(w.K, 128) : w.K; g.b_panel = panels;
  g.M = w.N; g.N = T; g.K = (int)pad(w.K, 128) / 2;           // in pairs of bytes
  return g;
}
}  // namespace

int64_t i8_weight_size(int64_t K, int64_t N) { return pad(N, 256) * (pad(K, 128) + 8); }

I8Layout i8_layout(const void* p, int K, int N) {
  const char* panels = static_cast<const char*>(p);
  return I8Layout{panels, reinterpret_cast<const float*>(panels + pad(N, 256) * pad(K, 128)), K, N};
}

int launch_i8_weight(const void* W, int K, int N, bool halves, void* out, hipStream_t s) {
  const int rows = (int)pad(N, 256), panels = (int)pad(K, 128) / 64, F = halves ? N / 2 : 0;
  uint8_t* codes = static_cast<uint8_t*>(out);
  float* scales = reinterpret_cast<float*>(codes + (size_t)rows * panels * 64);
  uint32_t* tops = reinterpret_cast<uint32_t*>(scales + rows);
  hipLaunchKernelGGL(i8_weight_clear_kernel, dim3((unsigned)(rows / 256)), dim3(256), 0, s, tops, rows);
  hipLaunchKernelGGL(i8_weight_top_kernel, dim3((unsigned)((N + 255) / 256), (unsigned)((K + TOP_ROWS - 1) / TOP_ROWS)), dim3(256), 0, s, static_cast<const uint16_t*>(W), K,
                     N, F, tops);
  hipLaunchKernelGGL(i8_weight_codes_kernel, dim3((unsigned)(rows / 64), (unsigned)panels), dim3(256), 0, s, static_cast<const uint16_t*>(W), K, N, F, panels, tops, codes,
                     scales);
  return (int)hipGetLastError();
}

template <int P, int W>
static void quantise(const void* X, int T, int K, int panels, void* codes, float* scales, uint32_t* zero, hipStream_t s) {
  hipLaunchKernelGGL((quantise_i8_kernel<P, W>), dim3((unsigned)((T + 4 / W - 1) / (4 / W))), dim3(256), 0, s, static_cast<const uint16_t*>(X), T, K,
                     panels, static_cast<uint8_t*>(codes), scales, zero);
}
int64_t i8_panel_size(int64_t T, int64_t K) { return pad(T, 256) * pad(K, 128); }
int launch_quantise_i8(const void* X, int T, int K, bool panel_form, void* codes, float* scales, uint32_t* zero, hipStream_t s) {
  const int panels = panel_form ? (int)pad(K, 128) / 64 : 0;
  if (K <= 4096 && T >= 1024) {
    if (K <= 1024) quantise<2, 1>(X, T, K, panels, codes, scales, zero, s);
    else if (K <= 2048) quantise<4, 1>(X, T, K, panels, codes, scales, zero, s);
    else quantise<8, 1>(X, T, K, panels, codes, scales, zero, s);
  } else if (K <= 2048) quantise<1, 4>(X, T, K, panels, codes, scales, zero, s);
  else if (K <= 4096) quantise<2, 4>(X, T, K, panels, codes, scales, zero, s);
  else if (K <= 16384) quantise<8, 4>(X, T, K, panels, codes, scales, zero, s);
  else quantise<0, 4>(X, T, K, panels, codes, scales, zero, s);
  return (int)hipGetLastError();
}

int launch_quantise_i8_given(const void* H, const uint32_t* tops, int T, int F, void* codes, float* scales, hipStream_t s) {   // (panel form)
  hipLaunchKernelGGL(quantise_i8_given_kernel, dim3((unsigned)((F / 16 + 255) / 256) * (unsigned)T), dim3(256), 0, s, static_cast<const uint16_t*>(H), tops, T, F,
                     (int)pad(F, 128) / 64, static_cast<uint8_t*>(codes), scales);
  return (int)hipGetLastError();
}

size_t matmul_i8_scratch(int T, int K, int N) { return few_i8_tokens(T, K) ? 0 : edge_split_scratch(N, T, (int)pad(K, 128) / 2); }
size_t gated_i8_scratch(int T, int D, int F) {
  size_t most = 0;
  for (int t = 64; t <= up_to(T, 64) && (long long)D * t <= 1 << 24; t += 64) {
    const size_t y = edge_split_scratch(D, t, (int)pad(F, 128) / 2);
    if (y > most) most = y;
  }
  return most;
}
int launch_matmul_i8(const void* codes, bool panel_form, const float* sx, int T, const I8Layout& w, void* Y, const Scratch& scratch, hipStream_t s) {
  if (!panel_form && few_i8_tokens(T, w.K)) return launch_few_matmul_i8(codes, sx, T, w, Y, s);
  using Epi = EdgeColMajor<true>;
  return launch_edge_split<Epi, TR_I8>(args(w, codes, T, panel_form), Epi::Args{static_cast<__bf16*>(Y), w.N, T, I8Scales{sx, w.scales}}, scratch, s);
}

int launch_gated_up_i8(const void* codes, const float* sx, int T, const I8Layout& w, float c1, float c3, void* H, uint32_t* rowmax, hipStream_t s) {
  using Epi = EpiGateUp<true, true>;
  return launch_edge<Epi, TR_I8>(args(w, codes, T, true), Epi::Args{static_cast<__bf16*>(H), nullptr, nullptr, w.N / 2, T, Gate{c1, c3}, I8Scales{sx, w.scales}, rowmax}, s);
}

}  // namespace ffn24
