// Epilogues of the gated block's and the int8 products' GEMMs, whose results may end anywhere inside a tile: what lies beyond M or N is not stored.
// The lane's part of the accumulators as in epilogues.hpp.  M (along the rows) is a multiple of 8.
#pragma once
#include "epilogues.hpp"

namespace ffn24 {

// Two-factor scaling of an int8 product: the 32-bit sums times the token's and the output channel's scale.  A is the weight, its rows the channels; `sw` is as
// long as the weight's panel form (whole blocks of 256 rows).
struct I8Scales { const float* sx; const float* sw; };

// the accumulators as results: their float values, or the integers in them scaled
template <bool I8, int MI, int NI, class Acc>
__device__ __forceinline__ void scale_i8(const I8Scales& sc, Acc& acc, int m_lane, int n_lane, int N) {
  if constexpr (!I8) return;
  LaneVec<MI> w;
  w.load(sc.sw, m_lane, 1.f);
#pragma unroll
  for (int ni = 0; ni < NI; ni++) {
    const float sx = sc.sx[min(n_lane + ni, N - 1)];
#pragma unroll
    for (int mi = 0; mi < MI; mi++)
#pragma unroll
      for (int v = 0; v < 16; v++) acc[mi][ni][v] = (float)__builtin_bit_cast(int, (float)acc[mi][ni][v]) * (sx * w.at(16 * mi + v));
  }
}

// A descriptor of rows [from, count) of a row-major matrix: offsets beyond its last row read zeros and store nothing.  (from: the same for the whole wave.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const void* p, int from, int count, uint32_t row_bytes) {
  const int64_t left = (int64_t)(count - from) * row_bytes;
  return __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(const_cast<void*>(p)) + (int64_t)from * row_bytes, 0, (int)(left < 0 ? 0 : left < 0x7FFFFFFF ? left : 0x7FFFFFFF),
                                           0x00020000);
}
constexpr uint32_t OUTSIDE = 0x80000000u;   // an offset that no descriptor holds

// out[n][m], m contiguous, through LDS (ColMajorStage)
template <bool I8>
struct EdgeColMajor {
  static constexpr bool STAGED = true, INTEGER = I8;
  struct Args { __bf16* C; int M, N; I8Scales sc; };
  template <int MI, int NI, class Acc>
  static __device__ __forceinline__ void run(const Args& e, Acc& acc, int m_lane, int n_lane, char* wbuf) {
    using S = ColMajorStage<MI, NI>;
    using LT = LaneTile<MI, NI>;
    scale_i8<I8, MI, NI>(e.sc, acc, m_lane, n_lane, e.N);
#pragma unroll
    for (int ni = 0; ni < NI; ni++)
#pragma unroll
      for (int mi = 0; mi < MI; mi++)
#pragma unroll
        for (int q = 0; q < 2; q++) {
          u32x4 o;
#pragma unroll
          for (int d = 0; d < 4; d++) o[d] = pack_bf16x2(acc[mi][ni][8 * q + 2 * d], acc[mi][ni][8 * q + 2 * d + 1]);
          S::put(wbuf, ni, 2 * mi + q, o);
        }
    const int n0 = n_lane - NI * LT::rho(), m0 = m_lane - 16 * MI * LT::h();
    const int lane = lane_id(), c = lane & (S::PIECES - 1), sub = lane / S::PIECES;
    constexpr int PER = 64 / S::PIECES;
    __bf16* out = e.C + (size_t)n0 * e.M + m0 + 8 * c;
    const int rows = m0 + 8 * c < e.M ? e.N - n0 : 0;
#pragma unroll
    for (int j = 0; j < LT::COLS / PER; j++) {
      const int r = PER * j + sub;
      if (r < rows) *reinterpret_cast<u32x4*>(out + (size_t)r * e.M) = *reinterpret_cast<const u32x4*>(wbuf + S::at(r, c));
    }
  }
};

// The accumulators as they are (fp32, or 32-bit integers), out[n][m]: the sums of a part of the reduction
struct EdgePart {
  struct Args { uint32_t* parts; int M, N; };
  template <int MI, int NI, class Acc>
  static __device__ __forceinline__ void run(const Args& e, Acc& acc, int m_lane, int n_lane) {
#pragma unroll
    for (int ni = 0; ni < NI; ni++) {
      if (n_lane + ni >= e.N) continue;
      uint32_t* out = e.parts + (size_t)(n_lane + ni) * e.M + m_lane;
#pragma unroll
      for (int mi = 0; mi < MI; mi++)
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
          u32x4 o;
#pragma unroll
          for (int d = 0; d < 4; d++) o[d] = __builtin_bit_cast(uint32_t, (float)acc[mi][ni][v + d]);
          if (m_lane + 16 * mi + v < e.M) *reinterpret_cast<u32x4*>(out + 16 * mi + v) = o;
        }
    }
  }
};
// The sums of `splits` parts, four values a work item; integers are scaled
template <bool I8>
__global__ void __launch_bounds__(256) edge_sum_kernel(const uint32_t* __restrict__ parts, int splits, int M, int N, I8Scales sc, uint16_t* __restrict__ out) {
  const size_t n = (size_t)M * N;
  const unsigned i = blockIdx.x * 256 + threadIdx.x, per = (unsigned)M / 4, t = i / per, col = 4 * (i - t * per);
  if (t >= (unsigned)N) return;
  const uint32_t* p = parts + (size_t)t * M + col;
  float y[4];
  if constexpr (I8) {
    i32x4 a = *reinterpret_cast<const i32x4*>(p);
    for (int s = 1; s < splits; s++) a += *reinterpret_cast<const i32x4*>(p + s * n);
#pragma unroll
    for (int j = 0; j < 4; j++) y[j] = (float)a[j] * (sc.sx[t] * sc.sw[col + j]);
  } else {
    f32x4 a = *reinterpret_cast<const f32x4*>(p);
    for (int s = 1; s < splits; s++) a += *reinterpret_cast<const f32x4*>(p + s * n);
#pragma unroll
    for (int j = 0; j < 4; j++) y[j] = a[j];
  }
  *reinterpret_cast<u32x2*>(out + (size_t)t * M + col) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
}

// out[m][n], n contiguous, N a multiple of 8
struct EdgeRowMajor {
  struct Args { __bf16* C; int M, N; };
  template <int MI, int NI, class Acc>
  static __device__ __forceinline__ void run(const Args& e, Acc& acc, int m_lane, int n_lane) {
    const int h = LaneTile<MI, NI>::h(), m0 = __builtin_amdgcn_readfirstlane(m_lane - 16 * MI * h);
    const uint32_t row = 2u * (uint32_t)e.N;
    const auto out = rows_from(e.C, m0, e.M, row);
    const uint32_t at = n_lane < e.N ? (uint32_t)(16 * MI * h) * row + 2u * (uint32_t)n_lane : OUTSIDE;
#pragma unroll
    for (int mi = 0; mi < MI; mi++)
#pragma unroll
      for (int v = 0; v < 16; v++) {
        uint32_t o[(NI + 1) / 2];
#pragma unroll
        for (int i = 0; i < (NI + 1) / 2; i++) o[i] = pack_bf16x2(acc[mi][2 * i][v], NI == 1 ? 0.f : acc[mi][NI == 1 ? 0 : 2 * i + 1][v]);
        const uint32_t to = at + (uint32_t)(16 * mi + v) * row;   // (beyond OUTSIDE by less than 2^31)
        if constexpr (NI == 8) __builtin_amdgcn_raw_buffer_store_b128(u32x4{o[0], o[1], o[2], o[3]}, out, (int)to, 0, 0);
        else if constexpr (NI == 2) __builtin_amdgcn_raw_buffer_store_b32(o[0], out, (int)to, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b16((unsigned short)o[0], out, (int)to, 0, 0);
      }
  }
};

// The gate's activation a(x) = x s, s = sigmoid(c1 x + c3 x^3): SiLU with (1, 0), GELU in its tanh form with (2 sqrt(2 / pi), 0.044715 times that).
// sigmoid(p) = 1 / (1 + 2^(-p log2 e)); 2^x is infinite for p < -88 and s then 0.  In p, and in the slope s + x s (1 - s) (c1 + 3 c3 x^2), x is held to +-1e4,
// where s is 0 or 1 long since and x^2 stays finite (SiLU: 0 times infinity otherwise, from 1.8e19 on).
struct Gate { float c1, c3; };
__device__ __forceinline__ float sigmoid(float p) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * p)); }
__device__ __forceinline__ float gate_hold(float x) { return fminf(fmaxf(x, -1e4f), 1e4f); }   // (takes NaN for a number)
__device__ __forceinline__ float gate_act(const Gate& g, float x) {
  const float y = gate_hold(x);
  return x * sigmoid(y * (g.c1 + g.c3 * (y * y)));
}
__device__ __forceinline__ void gate_act_slope(const Gate& g, float x, float& a, float& slope) {
  const float y = gate_hold(x), y2 = y * y, s = sigmoid(y * (g.c1 + g.c3 * y2));
  a = x * s;
  slope = s + y * (s - s * s) * (g.c1 + 3.f * g.c3 * y2);
  if (x != x) slope = x;                                      // (y is a number)
}

// What the backward needs of G and U is kept in 24 bits of the fp32 value: its upper 16 as a row-major [T][2 F], its next 8 as bytes [T][F / 8][16], 8 of G and
// 8 of U.  In bf16 alone (16 bits, 2 T F bytes less) dX and dWgu would carry the rounding of U and of the gate's slope besides that of dG and dU:
// 0.0030 of their norm off instead of 0.0024 (an exact result rounded to bf16: 0.0017).
__device__ __forceinline__ uint32_t upper2(float lo, float hi) { return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u); }
__device__ __forceinline__ uint32_t next4(float a, float b, float c, float d) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x0C0C0501u) |
         __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, d), __builtin_bit_cast(uint32_t, c), 0x05010C0Cu);
}
// value I (of 8) of the upper halves w and the next bytes b
template <int I> __device__ __forceinline__ float kept24(const u32x4& w, uint32_t b0, uint32_t b1) {
  return __builtin_bit_cast(float, __builtin_amdgcn_perm(w[I / 2], I < 4 ? b0 : b1, (I % 2 ? 0x0706000Cu : 0x0504000Cu) | (I % 4) << 8));
}

// Gate and up projections: rows m are features, 8 gate features and the 8 up features of the same numbers in turn, columns n are tokens.
// H[t][f] = bf16(a(G) U).  GU and GUx, if given, receive G and U for the backward (training).  ROWMAX: raises rowmax[t] to the
// bits of max_f |a(G) U| before it is rounded (as unsigned integers they order like the magnitudes, NaN above all).
template <bool I8, bool ROWMAX>
struct EpiGateUp {
  static constexpr bool STAGED = true;
  struct Args { __bf16* H; __bf16* GU; uint8_t* GUx; int F, T; Gate gate; I8Scales sc; uint32_t* rowmax; };
  template <int MI, int NI, class Acc>
  static __device__ __forceinline__ void run(const Args& e, Acc& acc, int m_lane, int n_lane, char* wbuf) {
    using S = ColMajorStage<MI, NI>;
    using LT = LaneTile<MI, NI>;
    constexpr int HALF = S::PIECES / 2;                       // pieces of 8 features that the wave has of a token
    scale_i8<I8, MI, NI>(e.sc, acc, m_lane, n_lane, e.T);
    const int h = LT::h(), rho = LT::rho();
    const int t0 = n_lane - NI * rho, f0 = (m_lane - 16 * MI * h) / 2;   // the wave's
    const int lane = lane_id();
    if (e.GU) {
#pragma unroll
      for (int ni = 0; ni < NI; ni++)
#pragma unroll
        for (int mi = 0; mi < MI; mi++)
#pragma unroll
          for (int q = 0; q < 2; q++) {
            u32x4 o;
#pragma unroll
            for (int d = 0; d < 4; d++) o[d] = upper2(acc[mi][ni][8 * q + 2 * d], acc[mi][ni][8 * q + 2 * d + 1]);
            *reinterpret_cast<u32x4*>(wbuf + S::at(NI * rho + ni, HALF * q + MI * h + mi)) = o;
          }
      const int c = lane & (S::PIECES - 1), sub = lane / S::PIECES, f = f0 + 8 * (c & (HALF - 1));
      constexpr int PER = 64 / S::PIECES;
      __bf16* out = e.GU + (size_t)t0 * (2 * (size_t)e.F) + (c >= HALF ? e.F : 0) + f;
      const int rows = f < e.F ? e.T - t0 : 0;
#pragma unroll
      for (int j = 0; j < LT::COLS / PER; j++) {
        const int r = PER * j + sub;
        if (r < rows) *reinterpret_cast<u32x4*>(out + (size_t)r * (2 * (size_t)e.F)) = *reinterpret_cast<const u32x4*>(wbuf + S::at(r, c));
      }
    }
    // two images of half the size: H, and the bytes
    auto at = [](int r, int c) { return (r * HALF + (c ^ ((r / NI) & (HALF - 1)))) << 4; };
    char* xbuf = wbuf + LT::COLS * HALF * 16;
#pragma unroll
    for (int ni = 0; ni < NI; ni++) {
      uint32_t top = 0u;
#pragma unroll
      for (int mi = 0; mi < MI; mi++) {
        u32x4 o;
#pragma unroll
        for (int d = 0; d < 4; d++) {
          const float x = gate_act(e.gate, acc[mi][ni][2 * d]) * acc[mi][ni][8 + 2 * d], y = gate_act(e.gate, acc[mi][ni][2 * d + 1]) * acc[mi][ni][9 + 2 * d];
          if constexpr (ROWMAX) top = max(top, max(__builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu, __builtin_bit_cast(uint32_t, y) & 0x7FFFFFFFu));
          o[d] = pack_bf16x2(x, y);
        }
        *reinterpret_cast<u32x4*>(wbuf + at(NI * rho + ni, MI * h + mi)) = o;
        if (e.GU) {
          const auto x = [&](int i) { return next4(acc[mi][ni][4 * i], acc[mi][ni][4 * i + 1], acc[mi][ni][4 * i + 2], acc[mi][ni][4 * i + 3]); };
          *reinterpret_cast<u32x4*>(xbuf + at(NI * rho + ni, MI * h + mi)) = u32x4{x(0), x(1), x(2), x(3)};
        }
      }
      if constexpr (ROWMAX) {                                 // (features beyond F are zero: the weight's rows there are)
#pragma unroll
        for (int s = LT::LANES; s < 64; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s, 64));
        if (h == 0 && n_lane + ni < e.T) atomicMax(e.rowmax + n_lane + ni, top);
      }
    }
    const int c = lane & (HALF - 1), sub = lane / HALF, f = f0 + 8 * c;
    constexpr int PER = 64 / HALF;
    __bf16* out = e.H + (size_t)t0 * e.F + f;
    const int rows = f < e.F ? e.T - t0 : 0;
#pragma unroll
    for (int j = 0; j < LT::COLS / PER; j++) {
      const int r = PER * j + sub;
      if (r < rows) *reinterpret_cast<u32x4*>(out + (size_t)r * e.F) = *reinterpret_cast<const u32x4*>(wbuf + at(r, c));
    }
    if (e.GU) {
      uint8_t* ox = e.GUx + 2 * ((size_t)t0 * e.F + f);
#pragma unroll
      for (int j = 0; j < LT::COLS / PER; j++) {
        const int r = PER * j + sub;
        if (r < rows) *reinterpret_cast<u32x4*>(ox + 2 * ((size_t)r * e.F)) = *reinterpret_cast<const u32x4*>(xbuf + at(r, c));
      }
    }
  }
};

// dH and the gate's derivative: rows m are features, columns n tokens, the accumulators dH.  G and U of the forward come by DMA, CH of the lane's tokens at
// a time, into a wave-private image (row: a token's G features, then its U features, 16-byte pieces at their place XOR the lane column; their next 8 bits, whose pieces
// have both of a feature, straight into registers), are replaced there by dG = dH U a'(G) and dU = dH a(G), and leave as whole runs of dGU [T][2 F].
struct EpiDGate {
  static constexpr bool STAGED = true;
  template <int NI> static constexpr int IMAGES = NI == 1 ? 2 : 1;   // (one column a lane: G and U of all of them at once)
  struct Args { const __bf16* GU; const uint8_t* GUx; __bf16* dGU; int F, T; Gate gate; };
  template <int MI, int NI, class Acc>
  static __device__ __forceinline__ void run(const Args& e, Acc& acc, int m_lane, int n_lane, char* wbuf) {
    using LT = LaneTile<MI, NI>;
    constexpr int CH = NI == 8 ? 2 : 1, BUFS = NI == 8 ? 2 : 1, CHUNKS = NI / CH, MB = MI == 4 ? 2 : MI;
    constexpr int P = LT::ROWS / 8, ROW = 2 * P, ROWS = LT::LANES * CH, BYTES = ROWS * ROW * 16, MOVES = ROWS * ROW / 64;
    const int lane = lane_id(), h = LT::h(), rho = LT::rho();
    const int t0 = __builtin_amdgcn_readfirstlane(n_lane - NI * rho), f0 = __builtin_amdgcn_readfirstlane(m_lane - 16 * MI * h);
    // Buffer accesses from the wave's first token on: tokens beyond T are outside the descriptor, features beyond F get an offset that is; both read zeros and
    // store nothing.
    const uint32_t row = 4u * (uint32_t)e.F;                  // bytes of a token's 2 F values
    const auto in = rows_from(e.GU, t0, e.T, row), out = rows_from(e.dGU, t0, e.T, row);
    // offset of what place 64 j + lane of the image of tokens ni0 .. holds
    auto place = [&](int j, int ni0) {
      const int at = 64 * j + lane, r = at / ROW, k = (at % ROW) ^ ((r / CH) & (ROW - 1)), f = f0 + 8 * (k & (P - 1));
      return f < e.F ? (uint32_t)(NI * (r / CH) + ni0 + r % CH) * row + (uint32_t)((k >= P ? e.F : 0) + f) * 2u : OUTSIDE;
    };
    auto fetch = [&](char* buf, int ni0) {
#pragma unroll
      for (int j = 0; j < MOVES; j++) __builtin_amdgcn_raw_ptr_buffer_load_lds(in, (lds_char*)(buf + j * 1024), 16, (int)place(j, ni0), 0, 0, 0);
    };
    fetch(wbuf, 0);
#pragma unroll
    for (int k = 0; k < CHUNKS; k++) {
      char* buf = wbuf + (k % BUFS) * BYTES;
      u32x4 x[CH][MB][2];
      auto bytes = [&](int m0) {
#pragma unroll
        for (int i = 0; i < CH; i++) {
          const uint8_t* p = e.GUx + 2 * (size_t)min(n_lane + CH * k + i, e.T - 1) * e.F;
#pragma unroll
          for (int mi = 0; mi < MB; mi++)
#pragma unroll
            for (int q = 0; q < 2; q++) x[i][mi][q] = *reinterpret_cast<const u32x4*>(p + 2 * min(m_lane + 16 * (m0 + mi) + 8 * q, e.F - 8));
        }
      };
      bytes(0);
      wait_vmcnt<0>();
      asm volatile("" ::: "memory");                          // (the compiler does not see the DMA write what is read here)
      if (BUFS > 1 && k + 1 < CHUNKS) fetch(wbuf + ((k + 1) % BUFS) * BYTES, CH * (k + 1));
#pragma unroll
      for (int mi = 0; mi < MI; mi++)
#pragma unroll
        for (int i = 0; i < CH; i++)
#pragma unroll
          for (int q = 0; q < 2; q++) {
            if (mi > 0 && mi % MB == 0 && i == 0 && q == 0) {    // (256 x 128: the bytes of half the features at a time, or 77 registers are spilled)
              FFN24_FENCE();
              bytes(mi);
            }
            const int r = CH * rho + i, c = 2 * MI * h + 2 * mi + q, key = rho & (ROW - 1);
            u32x4* pg = reinterpret_cast<u32x4*>(buf + ((r * ROW + (c ^ key)) << 4));
            u32x4* pu = reinterpret_cast<u32x4*>(buf + ((r * ROW + ((P + c) ^ key)) << 4));
            const u32x4 g = *pg, u = *pu;
            const u32x4 b = x[i][mi % MB][q];
            u32x4 dg, du;
            static_for<4>([&](auto D2) {
              constexpr int d = decltype(D2)::value;
              const float h0 = acc[mi][CH * k + i][8 * q + 2 * d], h1 = acc[mi][CH * k + i][8 * q + 2 * d + 1];
              float a0, a1, s0, s1;
              gate_act_slope(e.gate, kept24<2 * d>(g, b[0], b[1]), a0, s0);
              gate_act_slope(e.gate, kept24<2 * d + 1>(g, b[0], b[1]), a1, s1);
              dg[d] = pack_bf16x2(h0 * kept24<2 * d>(u, b[2], b[3]) * s0, h1 * kept24<2 * d + 1>(u, b[2], b[3]) * s1);
              du[d] = pack_bf16x2(h0 * a0, h1 * a1);
            });
            *pg = dg;
            *pu = du;
          }
#pragma unroll
      for (int j = 0; j < MOVES; j++)
        __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u32x4*>(buf + j * 1024 + 16 * lane), out, (int)place(j, CH * k), 0, 0);
      if (BUFS == 1 && k + 1 < CHUNKS) {
        wait_lgkmcnt0();                                      // the image has been read
        fetch(wbuf, CH * (k + 1));
      }
    }
  }
};

}  // namespace ffn24
