// Layer norm, forward and backward: HBM-bound, every element read once and written once.
//
//   forward   s = x + r;  mean = sum s / D;  rstd = (sum (s - mean)^2 / D + eps)^-1/2;  y = (s - mean) rstd w + b
//   backward  xh = (s - mean) rstd, p = dy w:  dx = rstd (p - sum p / D - xh sum (p xh) / D) + ds;  dw = sum_t dy xh;  db = sum_t dy
//
// A row lives in the registers of the waves that share it, so the variance is of centred values without a second read.  Lane l of the W waves of
// a row holds P pieces of 8 elements.  V = 8: a piece is 8 neighbouring elements, 16-byte accesses (D a multiple of 8); V = 1: elements 64 W apart, any D.
#include "launch_block.hpp"
#include "stream_core.hpp"

namespace ffn24 {
namespace {

template <class E> struct Elem;
template <> struct Elem<uint16_t> {                          // bf16
  static __device__ __forceinline__ float up(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
  static __device__ __forceinline__ uint16_t down(float x) { return (uint16_t)pack_bf16x2(x, 0.f); }
  static __device__ __forceinline__ float round(float x) { return up(down(x)); }
  static __device__ __forceinline__ void ld8(const uint16_t* p, float (&v)[8]) {
    const u32x4 w = ld_stream(reinterpret_cast<const u32x4*>(p));
#pragma unroll
    for (int i = 0; i < 4; i++) { v[2 * i] = bf16_lo_to_f32(w[i]); v[2 * i + 1] = bf16_hi_to_f32(w[i]); }
  }
  static __device__ __forceinline__ void st8(uint16_t* p, const float (&v)[8]) {
    st_keep(reinterpret_cast<u32x4*>(p), u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
  }
};
template <> struct Elem<float> {
  static __device__ __forceinline__ float up(float x) { return x; }
  static __device__ __forceinline__ float down(float x) { return x; }
  static __device__ __forceinline__ float round(float x) { return x; }
  static __device__ __forceinline__ void ld8(const float* p, float (&v)[8]) {
    const f32x4 a = ld_stream(reinterpret_cast<const f32x4*>(p)), b = ld_stream(reinterpret_cast<const f32x4*>(p) + 1);
#pragma unroll
    for (int i = 0; i < 4; i++) { v[i] = a[i]; v[4 + i] = b[i]; }
  }
  static __device__ __forceinline__ void st8(float* p, const float (&v)[8]) {
    st_keep(reinterpret_cast<f32x4*>(p), f32x4{v[0], v[1], v[2], v[3]});
    st_keep(reinterpret_cast<f32x4*>(p) + 1, f32x4{v[4], v[5], v[6], v[7]});
  }
};

// A row among the lanes of W waves; l: the lane's number among them.
template <int V, int W>
struct RowMap {
  static constexpr int LANES = 64 * W;
  // element j of piece p, and whether a piece (V = 8) or an element (V = 1) is inside the row
  static __device__ __forceinline__ int at(int p, int j, int l) { return V == 8 ? 8 * (p * LANES + l) + j : (8 * p + j) * LANES + l; }
  template <class E>
  static __device__ __forceinline__ void load(const E* row, int p, int l, int D, float (&v)[8]) {
    if constexpr (V == 8) {
      if (at(p, 0, l) < D) Elem<E>::ld8(row + at(p, 0, l), v);
      else {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = 0.f;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; j++) v[j] = at(p, j, l) < D ? Elem<E>::up(row[at(p, j, l)]) : 0.f;
    }
  }
  template <class E>
  static __device__ __forceinline__ void store(E* row, int p, int l, int D, const float (&v)[8]) {
    if constexpr (V == 8) {
      if (at(p, 0, l) < D) Elem<E>::st8(row + at(p, 0, l), v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; j++) if (at(p, j, l) < D) row[at(p, j, l)] = Elem<E>::down(v[j]);
    }
  }
};

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x += __shfl_xor(x, s, 64);
  return x;
}
// Sum over the W waves of a row; `part`: W floats of LDS a row, not in use by a sum whose results not every wave has read.
template <int W>
__device__ __forceinline__ float row_sum(float x, float* part, int wave) {
  x = wave_sum(x);
  if constexpr (W == 1) return x;
  if ((threadIdx.x & 63) == 0) part[wave] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < W; i++) s += part[i];
  return s;
}

constexpr int NORM_THREADS = 256;

template <class E, int V, int P, int W>
__global__ void __launch_bounds__(NORM_THREADS) norm_fwd_kernel(const E* X, const E* R, const float* weight, const float* bias, int T, int D, float eps, E* S,
                                                                E* Y, float* mean_out, float* rstd_out) {
  using M = RowMap<V, W>;
  __shared__ float part[2][4];
  const int wave = threadIdx.x >> 6, l = threadIdx.x & (M::LANES - 1), w0 = wave & ~(W - 1);
  const int row = blockIdx.x * (4 / W) + wave / W;
  if (W == 1 && row >= T) return;                            // (W = 4: the grid has T workgroups)
  const size_t o = (size_t)row * D;
  float v[P][8], sum = 0.f;
#pragma unroll
  for (int p = 0; p < P; p++) M::load(X + o, p, l, D, v[p]);
  if (R) {
#pragma unroll
    for (int p = 0; p < P; p++) {
      float r[8];
      M::load(R + o, p, l, D, r);
#pragma unroll
      for (int j = 0; j < 8; j++) v[p][j] = Elem<E>::round(v[p][j] + r[j]);
      M::store(S + o, p, l, D, v[p]);
    }
  }
#pragma unroll
  for (int p = 0; p < P; p++)
#pragma unroll
    for (int j = 0; j < 8; j++) sum += v[p][j];
  const float mean = row_sum<W>(sum, part[0] + w0, wave - w0) / (float)D;
  float sq = 0.f;
#pragma unroll
  for (int p = 0; p < P; p++)
#pragma unroll
    for (int j = 0; j < 8; j++) {
      v[p][j] = M::at(p, j, l) < D ? v[p][j] - mean : 0.f;
      sq += v[p][j] * v[p][j];
    }
  const float rstd = 1.f / sqrtf(row_sum<W>(sq, part[1] + w0, wave - w0) / (float)D + eps);
  if (l == 0 && mean_out) { mean_out[row] = mean; rstd_out[row] = rstd; }
#pragma unroll
  for (int p = 0; p < P; p++) {
    float w[8], b[8] = {};
    M::load(weight, p, l, D, w);
    if (bias) M::load(bias, p, l, D, b);
#pragma unroll
    for (int j = 0; j < 8; j++) v[p][j] = v[p][j] * rstd * w[j] + b[j];
    M::store(Y + o, p, l, D, v[p]);
  }
}

// A workgroup of R rows at a time walks rows blockIdx.x R + r, + gridDim.x R, ...; every lane adds up its columns' dy xh and dy, and at the end the workgroup's sums
// go to `parts` [gridDim.x][2][D].
template <class E, int V, int P, int W, int R>
__global__ void __launch_bounds__(64 * W * R) norm_bwd_kernel(const E* dY, const E* S, const float* weight, const float* mean, const float* rstd, const E* dS, int T,
                                                              int D, E* dX, float* parts) {
  using M = RowMap<V, W>;
  __shared__ float part[2][2][W * R];                        // [parity of the step][which sum]
  const int wave = threadIdx.x >> 6, r = wave / W, l = threadIdx.x & (M::LANES - 1), w0 = r * W;
  constexpr bool HOLD = W < 16;                              // (a workgroup of 16 waves has 128 registers a lane: the weights are read again for every row)
  float w[P][8], dw[P][8], db[P][8];
#pragma unroll
  for (int p = 0; p < P; p++) {
    if (HOLD) M::load(weight, p, l, D, w[p]);
#pragma unroll
    for (int j = 0; j < 8; j++) dw[p][j] = db[p][j] = 0.f;
  }
  const float inv = 1.f / (float)D;
  const int step = gridDim.x * R;
  int parity = 0;
  for (int row0 = blockIdx.x * R; row0 < T; row0 += step, parity ^= 1) {   // (uniform: the barriers below are met by all)
    const int row = row0 + r;
    const bool here = row < T;
    const size_t o = (size_t)(here ? row : T - 1) * D;
    float x[P][8], g[P][8], s1 = 0.f, s2 = 0.f;
    const float mu = mean[here ? row : T - 1], rs = rstd[here ? row : T - 1];
#pragma unroll
    for (int p = 0; p < P; p++) { M::load(S + o, p, l, D, x[p]); M::load(dY + o, p, l, D, g[p]); }
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
      for (int j = 0; j < 8; j++) {
        if (!HOLD && j == 0) M::load(weight, p, l, D, w[p]);
        x[p][j] = (x[p][j] - mu) * rs;                       // (outside the row the weight and dY are 0: nothing is added)
        if (here) { dw[p][j] += g[p][j] * x[p][j]; db[p][j] += g[p][j]; }
        g[p][j] *= w[p][j];
        s1 += g[p][j];
        s2 += g[p][j] * x[p][j];
      }
    s1 = wave_sum(s1); s2 = wave_sum(s2);
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) { part[parity][0][wave] = s1; part[parity][1][wave] = s2; }
      __syncthreads();
      s1 = s2 = 0.f;
#pragma unroll
      for (int i = 0; i < W; i++) { s1 += part[parity][0][w0 + i]; s2 += part[parity][1][w0 + i]; }
    }
    s1 *= inv; s2 *= inv;
    if (here) {
#pragma unroll
      for (int p = 0; p < P; p++) {
        float d[8] = {};
        if (dS) M::load(dS + o, p, l, D, d);
#pragma unroll
        for (int j = 0; j < 8; j++) d[j] += rs * (g[p][j] - s1 - x[p][j] * s2);
        M::store(dX + o, p, l, D, d);
      }
    }
  }
  // the workgroup's R rows of sums, one after the other
  float* mine = parts + (size_t)blockIdx.x * 2 * D;
  if constexpr (R == 1) {
#pragma unroll
    for (int p = 0; p < P; p++) { M::store(mine, p, l, D, dw[p]); M::store(mine + D, p, l, D, db[p]); }
  } else {
    __shared__ float sums[R][M::LANES * 8];
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
      for (int which = 0; which < 2; which++) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; j++) sums[r][j * M::LANES + l] = which ? db[p][j] : dw[p][j];
        __syncthreads();
        if (r == 0) {
          float t[8];
#pragma unroll
          for (int j = 0; j < 8; j++) {
            t[j] = sums[0][j * M::LANES + l];
#pragma unroll
            for (int i = 1; i < R; i++) t[j] += sums[i][j * M::LANES + l];
          }
          M::store(mine + which * D, p, l, D, t);
        }
      }
  }
}

// Column c of the n partial sums [n][2 D]: 16 groups of rows a workgroup, 64 columns each; dweight, then dbias.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* parts, int n, int D, float* dweight, float* dbias) {
  __shared__ float sums[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), g = threadIdx.x >> 6;
  float s = 0.f;
  if (c < 2 * D)
    for (int i = g; i < n; i += 16) s += parts[(size_t)i * 2 * D + c];
  sums[g][threadIdx.x & 63] = s;
  __syncthreads();
  if (g == 0 && c < 2 * D) {
#pragma unroll
    for (int i = 1; i < 16; i++) s += sums[i][threadIdx.x];
    if (c < D) dweight[c] = s;
    else if (dbias) dbias[c - D] = s;
  }
}

template <class E, int V, int P, int W>
void fwd(const void* X, const void* R, const float* w, const float* b, int T, int D, float eps, void* S, void* Y, float* mean, float* rstd, hipStream_t s) {
  hipLaunchKernelGGL((norm_fwd_kernel<E, V, P, W>), dim3((unsigned)((T + 4 / W - 1) / (4 / W))), dim3(NORM_THREADS), 0, s, static_cast<const E*>(X),
                     static_cast<const E*>(R), w, b, T, D, eps, static_cast<E*>(S), static_cast<E*>(Y), mean, rstd);
}
template <class E, int V>
void fwd_any(const void* X, const void* R, const float* w, const float* b, int T, int D, float eps, void* S, void* Y, float* mean, float* rstd, hipStream_t s) {
  if (D <= 4096 && T >= 1024) {
    if (D <= 512) return fwd<E, V, 1, 1>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
    if (D <= 1024) return fwd<E, V, 2, 1>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
    if (D <= 2048) return fwd<E, V, 4, 1>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
    return fwd<E, V, 8, 1>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
  }
  if (D <= 2048) return fwd<E, V, 1, 4>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
  if (D <= 4096) return fwd<E, V, 2, 4>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
  if (D <= 8192) return fwd<E, V, 4, 4>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
  return fwd<E, V, 8, 4>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
}

template <class E, int V, int P, int W, int R>
void bwd(const void* dY, const void* S, const float* w, const float* mean, const float* rstd, const void* dS, int T, int D, void* dX, float* parts, int n, hipStream_t s) {
  hipLaunchKernelGGL((norm_bwd_kernel<E, V, P, W, R>), dim3((unsigned)n), dim3(64 * W * R), 0, s, static_cast<const E*>(dY), static_cast<const E*>(S), w, mean, rstd,
                     static_cast<const E*>(dS), T, D, static_cast<E*>(dX), parts);
}
// waves a row (and pieces a lane), rows a workgroup takes at a time: at most two pieces a lane, whose columns' weights and sums stay in registers
// beside the row; with four, 220-256 registers and two waves a SIMD
int bwd_rows(int D) { return D <= 1024 ? 4 : 1; }
template <class E, int V>
void bwd_any(const void* dY, const void* S, const float* w, const float* mean, const float* rstd, const void* dS, int T, int D, void* dX, float* parts, int n, hipStream_t s) {
  if (D <= 512) return bwd<E, V, 1, 1, 4>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  if (D <= 1024) return bwd<E, V, 2, 1, 4>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  if (D <= 2048) return bwd<E, V, 1, 4, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  if (D <= 4096) return bwd<E, V, 2, 4, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  if (D <= 8192) return bwd<E, V, 2, 8, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  return bwd<E, V, 2, 16, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
}
}  // namespace

int launch_norm_fwd(const void* X, const void* R, const float* w, const float* b, int T, int D, float eps, bool f32, void* S, void* Y, float* mean, float* rstd,
                    hipStream_t s) {
  if (D % 8 == 0) f32 ? fwd_any<float, 8>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s) : fwd_any<uint16_t, 8>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
  else f32 ? fwd_any<float, 1>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s) : fwd_any<uint16_t, 1>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
  return (int)hipGetLastError();
}

// workgroups of the backward, each with its partial sums
int norm_bwd_parts(int64_t T, int D) {
  const int R = bwd_rows(D);
  const int64_t n = (T + R - 1) / R;
  return (int)(n < 512 ? n : 512);
}

int launch_norm_bwd(const void* dY, const void* S, const float* w, const float* mean, const float* rstd, const void* dS, int T, int D, bool f32, void* dX,
                    float* dweight, float* dbias, float* parts, hipStream_t s) {
  const int n = norm_bwd_parts(T, D);
  if (n > 0) {
    if (D % 8 == 0) f32 ? bwd_any<float, 8>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s) : bwd_any<uint16_t, 8>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
    else f32 ? bwd_any<float, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s) : bwd_any<uint16_t, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
    if (int rc = (int)hipGetLastError()) return rc;
  }
  hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)((2 * D + 63) / 64)), dim3(1024), 0, s, parts, n, D, dweight, dbias);
  return (int)hipGetLastError();
}

}  // namespace ffn24
