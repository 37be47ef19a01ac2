// Layer norm, forward and backward: HBM-bound, every element read once and written once.
//
//   forward   s = x + r;  mean = sum s / D;  rstd = (sum (s - mean)^2 / D + eps)^-1/2;  y = (s - mean) rstd w + b
//   backward  xh = (s - mean) rstd, p = dy w:  dx = rstd (p - sum p / D - xh sum (p xh) / D) + ds;  dw = sum_t dy xh;  db = sum_t dy
//
// A row lives in the registers of the waves that share it, so the variance is of centred values without a second read.  Lane l of the W waves of
// a row holds P pieces of 8 neighbouring elements.  EVEN: D is a multiple of 8, rows are 16-byte aligned; otherwise a row starts at any element and its last piece
// is a part of one: 16-byte accesses at the alignment of an element, which global memory takes; the part is read as the row's last 8 elements and moved into place,
// and stored element by element.
#include "launch_block.hpp"
#include "stream_core.hpp"

namespace ffn24 {
namespace {

template <class T, int ALIGN> struct Unaligned { T v; } __attribute__((packed, aligned(ALIGN)));
// 16 bytes at the alignment of an E, or (EVEN) at their own, with the streaming hint (HINT) or without
template <class T, class E, bool EVEN, bool HINT>
__device__ __forceinline__ T ld16(const void* p) {
  if constexpr (EVEN) return HINT ? ld_stream(static_cast<const T*>(p)) : *static_cast<const T*>(p);
  else return static_cast<const Unaligned<T, sizeof(E)>*>(p)->v;
}
template <class E, bool EVEN, class T>
__device__ __forceinline__ void st16(void* p, T x) {
  if constexpr (EVEN) st_keep(static_cast<T*>(p), x);
  else static_cast<Unaligned<T, sizeof(E)>*>(p)->v = x;
}

template <class E> struct Elem;
template <> struct Elem<uint16_t> {                          // bf16
  static __device__ __forceinline__ float up(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
  static __device__ __forceinline__ uint16_t down(float x) { return (uint16_t)pack_bf16x2(x, 0.f); }
  static __device__ __forceinline__ float round(float x) { return up(down(x)); }
  typedef u32x4 Raw;                                         // 8 elements as they lie in memory
  template <bool EVEN, bool HINT> static __device__ __forceinline__ Raw ld8(const uint16_t* p) { return ld16<u32x4, uint16_t, EVEN, HINT>(p); }
  static __device__ __forceinline__ void put(Raw& w, int j, uint16_t x) { w[j / 2] |= (uint32_t)x << (16 * (j % 2)); }
  static __device__ __forceinline__ void up8(const Raw& w, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; i++) { v[2 * i] = bf16_lo_to_f32(w[i]); v[2 * i + 1] = bf16_hi_to_f32(w[i]); }
  }
  template <bool EVEN> static __device__ __forceinline__ void st8(uint16_t* p, const float (&v)[8]) {
    st16<uint16_t, EVEN>(p, u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
  }
};
template <> struct Elem<float> {
  static __device__ __forceinline__ float up(float x) { return x; }
  static __device__ __forceinline__ float down(float x) { return x; }
  static __device__ __forceinline__ float round(float x) { return x; }
  struct Raw { f32x4 a, b; };
  template <bool EVEN, bool HINT> static __device__ __forceinline__ Raw ld8(const float* p) { return Raw{ld16<f32x4, float, EVEN, HINT>(p), ld16<f32x4, float, EVEN, HINT>(p + 4)}; }
  static __device__ __forceinline__ void put(Raw& w, int j, float x) { if (j < 4) w.a[j] = x; else w.b[j - 4] = x; }
  static __device__ __forceinline__ void up8(const Raw& w, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; i++) { v[i] = w.a[i]; v[4 + i] = w.b[i]; }
  }
  template <bool EVEN> static __device__ __forceinline__ void st8(float* p, const float (&v)[8]) {
    st16<float, EVEN>(p, f32x4{v[0], v[1], v[2], v[3]});
    st16<float, EVEN>(p + 4, f32x4{v[4], v[5], v[6], v[7]});
  }
};

// A row among the lanes of W waves; l: the lane's number among them.
template <bool EVEN, int W>
struct RowMap {
  static constexpr int LANES = 64 * W;
  static __device__ __forceinline__ int at(int p, int l) { return 8 * (p * LANES + l); }   // the first element of piece p
  // a piece as it lies in memory, on its way; zeros outside the row
  template <bool HINT = false, class E>
  static __device__ __forceinline__ void fetch(typename Elem<E>::Raw& x, const E* row, int p, int l, int D) {
    const int i = at(p, l);
    x = typename Elem<E>::Raw{};
    if (i >= D) return;
    if (EVEN || D >= 8) x = Elem<E>::template ld8<EVEN, HINT>(row + (EVEN ? i : min(i, D - 8)));
    else {
#pragma unroll
      for (int j = 0; j < 7; j++) if (i + j < D) Elem<E>::put(x, j, row[i + j]);
    }
  }
  template <class E>
  static __device__ __forceinline__ void unpack(const typename Elem<E>::Raw& x, int p, int l, int D, float (&v)[8]) {
    Elem<E>::up8(x, v);
    const int over = at(p, l) + 8 - D;
    if (!EVEN && over > 0 && D >= 8) {                       // (only the wave that has the row's end comes here)
#pragma unroll
      for (int by = 4; by >= 1; by /= 2)
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = over & by ? (j + by < 8 ? v[j + by] : 0.f) : v[j];
    }
  }
  template <class E>
  static __device__ __forceinline__ void load(const E* row, int p, int l, int D, float (&v)[8]) {
    typename Elem<E>::Raw x;
    fetch(x, row, p, l, D);
    unpack<E>(x, p, l, D, v);
  }
  template <class E>
  static __device__ __forceinline__ void store(E* row, int p, int l, int D, const float (&v)[8]) {
    const int i = at(p, l);
    if (EVEN ? i < D : i + 8 <= D) Elem<E>::template st8<EVEN>(row + i, v);
    else if (!EVEN && i < D) {
#pragma unroll
      for (int j = 0; j < 7; j++) if (i + j < D) row[i + j] = Elem<E>::down(v[j]);
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

// Rows blockIdx.x R + r, + gridDim.x R, ...; R rows a workgroup at a time, the next ones on their way while these are worked on.
template <class E, bool EVEN, bool HINT, int P, int W, int R>
__global__ void __launch_bounds__(64 * W * R) norm_fwd_kernel(const E* X, const E* res, const float* weight, const float* bias, int T, int D, float eps, E* S, E* Y,
                                                              float* mean_out, float* rstd_out) {
  using M = RowMap<EVEN, W>;
  constexpr bool HOLD = W < 16;                              // weights and bias stay in registers (a workgroup of 16 waves has 128 of them a lane)
  __shared__ float part[2][W * R];
  const int wave = threadIdx.x >> 6, r = wave / W, l = threadIdx.x & (M::LANES - 1), w0 = r * W;
  float w[P][8], b[P][8];
  auto weights = [&](int p) {
    M::load(weight, p, l, D, w[p]);
    if (bias) M::load(bias, p, l, D, b[p]);
    else {
#pragma unroll
      for (int j = 0; j < 8; j++) b[p][j] = 0.f;
    }
  };
  typename Elem<E>::Raw sx[P], sr[P];
  auto ask = [&](int row) {
    const size_t o = (size_t)min(row, T - 1) * D;
#pragma unroll
    for (int p = 0; p < P; p++) {
      M::template fetch<HINT>(sx[p], X + o, p, l, D);
      if (res) M::template fetch<HINT>(sr[p], res + o, p, l, D);
    }
  };
  const int step = gridDim.x * R;
  ask(blockIdx.x * R + r);
  if constexpr (HOLD) {
#pragma unroll
    for (int p = 0; p < P; p++) weights(p);
  }
  for (int row0 = blockIdx.x * R; row0 < T; row0 += step) {  // (uniform: the barriers below are met by all)
    const int row = row0 + r;
    const bool here = row < T;
    const size_t o = (size_t)row * D;
    float v[P][8], sum = 0.f;
#pragma unroll
    for (int p = 0; p < P; p++) M::template unpack<E>(sx[p], p, l, D, v[p]);
    if (res) {
#pragma unroll
      for (int p = 0; p < P; p++) {
        float x[8];
        M::template unpack<E>(sr[p], p, l, D, x);
#pragma unroll
        for (int j = 0; j < 8; j++) v[p][j] = Elem<E>::round(v[p][j] + x[j]);
      }
    }
    if (row0 + step < T) ask(row + step);
#pragma unroll
    for (int p = 0; p < P; p++) {
      if (res && here) M::store(S + o, p, l, D, v[p]);
#pragma unroll
      for (int j = 0; j < 8; j++) sum += v[p][j];
    }
    const float mean = row_sum<W>(sum, part[0] + w0, wave - w0) / (float)D;
    float sq = 0.f;
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
      for (int j = 0; j < 8; j++) {
        v[p][j] = M::at(p, l) + (EVEN ? 0 : j) < D ? v[p][j] - mean : 0.f;
        sq += v[p][j] * v[p][j];
      }
    const float rstd = 1.f / sqrtf(row_sum<W>(sq, part[1] + w0, wave - w0) / (float)D + eps);
    if (l == 0 && here && mean_out) { mean_out[row] = mean; rstd_out[row] = rstd; }
#pragma unroll
    for (int p = 0; p < P; p++) {
      if constexpr (!HOLD) weights(p);
#pragma unroll
      for (int j = 0; j < 8; j++) v[p][j] = v[p][j] * rstd * w[p][j] + b[p][j];
      if (here) M::store(Y + o, p, l, D, v[p]);
    }
  }
}

constexpr int NORM_FWD_WAVES = 16;                           // a CU

// A workgroup of R rows at a time walks rows blockIdx.x R + r, + gridDim.x R, ...; every lane adds up its columns' dy xh and dy, and at the end the workgroup's sums
// go to `parts` [gridDim.x][2][D].
template <class E, bool EVEN, bool HINT, int P, int W, int R>
__global__ void __launch_bounds__(64 * W * R) norm_bwd_kernel(const E* dY, const E* S, const float* weight, const float* mean, const float* rstd, const E* dS, int T,
                                                              int D, E* dX, float* parts) {
  using M = RowMap<EVEN, W>;
  __shared__ float part[2][2][W * R];                        // [parity of the step][which sum]
  const int wave = threadIdx.x >> 6, r = wave / W, l = threadIdx.x & (M::LANES - 1), w0 = r * W;
  constexpr bool ROOM = W < 16;                              // (a workgroup of 16 waves has 128 registers a lane: no weights and no next row in them)
  float w[P][8], dw[P][8], db[P][8];
#pragma unroll
  for (int p = 0; p < P; p++) {
    if (ROOM) M::load(weight, p, l, D, w[p]);
#pragma unroll
    for (int j = 0; j < 8; j++) dw[p][j] = db[p][j] = 0.f;
  }
  const float inv = 1.f / (float)D;
  const int step = gridDim.x * R, row_first = blockIdx.x * R + r;
  // The next row is on its way while this one is worked on: a workgroup has a barrier a row, and without it every row waited out a round trip to memory.
  typename Elem<E>::Raw sx[P], sg[P], sd[P];
  float mu, rs;
  auto ask = [&](int row, bool tokens) {
    const size_t o = (size_t)min(row, T - 1) * D;
#pragma unroll
    for (int p = 0; p < P; p++) {
      if (tokens) { M::template fetch<HINT>(sx[p], S + o, p, l, D); M::template fetch<HINT>(sg[p], dY + o, p, l, D); }
      else if (dS) M::template fetch<HINT>(sd[p], dS + o, p, l, D);
    }
    if (tokens) { mu = mean[min(row, T - 1)]; rs = rstd[min(row, T - 1)]; }
  };
  if (ROOM) {
    ask(row_first, true);
    ask(row_first, false);
  }
  int parity = 0;
  for (int row0 = blockIdx.x * R; row0 < T; row0 += step, parity ^= 1) {   // (uniform: the barriers below are met by all)
    const int row = row0 + r;
    const bool here = row < T;
    float x[P][8], g[P][8], s1 = 0.f, s2 = 0.f;
    if (!ROOM) ask(row, true);
    const float scale = rs, center = mu;
#pragma unroll
    for (int p = 0; p < P; p++) { M::template unpack<E>(sx[p], p, l, D, x[p]); M::template unpack<E>(sg[p], p, l, D, g[p]); }
    if (ROOM && row0 + step < T) ask(row + step, true);
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
      for (int j = 0; j < 8; j++) {
        if (!ROOM && j == 0) M::load(weight, p, l, D, w[p]);
        x[p][j] = (x[p][j] - center) * scale;                // (outside the row the weight and dY are 0: nothing is added)
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
    if (!ROOM) ask(row, false);
#pragma unroll
    for (int p = 0; p < P; p++) {
      float d[8] = {};
      if (dS) M::template unpack<E>(sd[p], p, l, D, d);
#pragma unroll
      for (int j = 0; j < 8; j++) d[j] += scale * (g[p][j] - s1 - x[p][j] * s2);
      if (here) M::store(dX + (size_t)row * D, p, l, D, d);
    }
    if (ROOM && row0 + step < T) ask(row + step, false);
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

// Column c of the n partial sums [n][2 D]: 32 groups of rows a workgroup, 32 columns each; dweight, then dbias.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* __restrict__ parts, int n, int D, float* dweight, float* dbias) {
  __shared__ float sums[32][33];
  const int x = threadIdx.x & 31, c = blockIdx.x * 32 + x, g = threadIdx.x >> 5;
  float s = 0.f;
  if (c < 2 * D) {
    const float* p = parts + c;
    const size_t row = 2 * (size_t)D;
    int i = g;
    for (; i + 96 < n; i += 128) {                           // four rows on their way at a time
      const float a = p[i * row], b = p[(i + 32) * row], d = p[(i + 64) * row], e = p[(i + 96) * row];
      s += (a + b) + (d + e);
    }
    for (; i < n; i += 32) s += p[i * row];
  }
  sums[g][x] = s;
  __syncthreads();
  if (g == 0 && c < 2 * D) {
#pragma unroll
    for (int i = 1; i < 32; i++) s += sums[i][x];
    if (c < D) dweight[c] = s;
    else if (dbias) dbias[c - D] = s;
  }
}

// The streaming hint from tensors of 128 MiB on, four of which the caches do not hold (T x D, with / without, whole calls, us: forward bf16 16384 x 4096 83.8, 105.9; 8192 x 8192 81.0, 98.6;
// 32768 x 2048 90, 100; 4096 x 8192 43.6, 43.1; 16384 x 1024 23.2, 22.8; 2000 x 16384 49.2, 48.1; fp32 8192 x 4096 94, 100; 16384 x 4096 207, 199; backward in that order 91, 106; 89.5, 101.6; 97, 101;
// 50.0, 49.7; 30.2, 29.1; 68, 76; 101, 103; 198, 200).
template <class E> bool hint(int T, int D) { return sizeof(E) * (size_t)T * (size_t)D >= (size_t)1 << 27; }

// Workgroups: 16 waves a CU, each with rows to walk (T x D, bf16, 12 / 16 / 32 / 64 waves: 16384 x 4096 82.6, 83.8, 85.3, 82.9 us; 4096 x 8192 47.6, 43.1, 43.7, 45.8; a row a workgroup and
// no prefetch 114 at the first).  fp32 16384 x 4096: 208 us, 5.2 TB/s.
template <class E, bool EVEN, int P, int W, int R>
void fwd(const void* X, const void* res, const float* w, const float* b, int T, int D, float eps, void* S, void* Y, float* mean, float* rstd, hipStream_t s) {
  constexpr int most = 256 * NORM_FWD_WAVES / (W * R);
  const int n = (T + R - 1) / R;
  const auto kern = EVEN && hint<E>(T, D) ? norm_fwd_kernel<E, EVEN, EVEN, P, W, R> : norm_fwd_kernel<E, EVEN, false, P, W, R>;
  hipLaunchKernelGGL(kern, dim3((unsigned)(n < most ? n : most)), dim3(64 * W * R), 0, s, static_cast<const E*>(X),
                     static_cast<const E*>(res), w, b, T, D, eps, static_cast<E*>(S), static_cast<E*>(Y), mean, rstd);
}
template <class E, bool EVEN>
void fwd_any(const void* X, const void* res, const float* w, const float* b, int T, int D, float eps, void* S, void* Y, float* mean, float* rstd, hipStream_t s) {
  if (D <= 512) return fwd<E, EVEN, 1, 1, 4>(X, res, w, b, T, D, eps, S, Y, mean, rstd, s);
  if (D <= 1024) return fwd<E, EVEN, 2, 1, 4>(X, res, w, b, T, D, eps, S, Y, mean, rstd, s);
  if (D <= 2048) return fwd<E, EVEN, 1, 4, 1>(X, res, w, b, T, D, eps, S, Y, mean, rstd, s);
  if (D <= 4096) return fwd<E, EVEN, 2, 4, 1>(X, res, w, b, T, D, eps, S, Y, mean, rstd, s);
  if (D <= 8192) return fwd<E, EVEN, 2, 8, 1>(X, res, w, b, T, D, eps, S, Y, mean, rstd, s);
  return fwd<E, EVEN, 2, 16, 1>(X, res, w, b, T, D, eps, S, Y, mean, rstd, s);
}

template <class E, bool EVEN, int P, int W, int R>
void bwd(const void* dY, const void* S, const float* w, const float* mean, const float* rstd, const void* dS, int T, int D, void* dX, float* parts, int n, hipStream_t s) {
  const auto kern = EVEN && hint<E>(T, D) ? norm_bwd_kernel<E, EVEN, EVEN, P, W, R> : norm_bwd_kernel<E, EVEN, false, P, W, R>;
  hipLaunchKernelGGL(kern, dim3((unsigned)n), dim3(64 * W * R), 0, s, static_cast<const E*>(dY), static_cast<const E*>(S), w, mean, rstd,
                     static_cast<const E*>(dS), T, D, static_cast<E*>(dX), parts);
}
// waves a row (and pieces a lane), rows a workgroup takes at a time: at most two pieces a lane, whose columns' weights and sums stay in registers
// beside the row; with four, 220-256 registers and two waves a SIMD
int bwd_rows(int D) { return D <= 1024 ? 4 : 1; }
template <class E, bool EVEN>
void bwd_any(const void* dY, const void* S, const float* w, const float* mean, const float* rstd, const void* dS, int T, int D, void* dX, float* parts, int n, hipStream_t s) {
  if (D <= 512) return bwd<E, EVEN, 1, 1, 4>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  if (D <= 1024) return bwd<E, EVEN, 2, 1, 4>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  if (D <= 2048) return bwd<E, EVEN, 1, 4, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  if (D <= 4096) return bwd<E, EVEN, 2, 4, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  if (D <= 8192) return bwd<E, EVEN, 2, 8, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
  return bwd<E, EVEN, 2, 16, 1>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
}
}  // namespace

int launch_norm_fwd(const void* X, const void* R, const float* w, const float* b, int T, int D, float eps, bool f32, void* S, void* Y, float* mean, float* rstd,
                    hipStream_t s) {
  if (D % 8 == 0) f32 ? fwd_any<float, true>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s) : fwd_any<uint16_t, true>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
  else f32 ? fwd_any<float, false>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s) : fwd_any<uint16_t, false>(X, R, w, b, T, D, eps, S, Y, mean, rstd, s);
  return (int)hipGetLastError();
}

// Workgroups of the backward, each with its partial sums: the chip's CUs, twice from 1025 to 4096 columns, where a workgroup is four waves (T x D, bf16, 256 / 512 / 1024,
// whole calls: 16384 x 4096 115, 93, 100 us; 8192 x 2048 45, 30.4, 32.6; 4096 x 8192 50, 58, 76; 16384 x 1024 29.3, 27.8, 31.5; 2000 x 16384 76, 90, 121; fp32 16384 x 4096 198, 200, 204).
int norm_bwd_parts(int64_t T, int D) {
  const int R = bwd_rows(D);
  const int64_t n = (T + R - 1) / R;
  const int most = D > 1024 && D <= 4096 ? 512 : 256;
  return (int)(n < most ? n : most);
}

int launch_norm_bwd(const void* dY, const void* S, const float* w, const float* mean, const float* rstd, const void* dS, int T, int D, bool f32, void* dX,
                    float* dweight, float* dbias, float* parts, hipStream_t s) {
  const int n = norm_bwd_parts(T, D);
  if (n > 0) {
    if (D % 8 == 0) f32 ? bwd_any<float, true>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s) : bwd_any<uint16_t, true>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
    else f32 ? bwd_any<float, false>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s) : bwd_any<uint16_t, false>(dY, S, w, mean, rstd, dS, T, D, dX, parts, n, s);
    if (int rc = (int)hipGetLastError()) return rc;
  }
  hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)((2 * D + 31) / 32)), dim3(1024), 0, s, parts, n, D, dweight, dbias);
  return (int)hipGetLastError();
}

}  // namespace ffn24
