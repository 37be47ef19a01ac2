// Microscaled 4-bit numbers (mx4: e2m1 values, a power of two for every 32 of them along k) as operands of the matrix ops, and the GEMM on them.
//
//   Y[n][m] = sum_k A[m][k] B[n][k],   A the weights (rows: output channels), B the tokens
//
// Operand form.  The op is the 16 x 16 x 128 one: lane l (q = l / 16, c = l % 16) holds row c, k 32 q .. 32 q + 31 of the step's 128 in 16 bytes (low nibble first) and
// takes their scale from a byte of a register (measured with random operands).  An operand is stored as the ops read it:
//   codes   [block of 64 rows][step of 128 k][group of 16 rows][lane][16 bytes]
//   scales  [block of 64 rows][4 steps][group of 16 rows][lane][4 bytes]      byte j: step 4 S + j
// Rows are filled up to 64, k to 128 with zeros (scales to 4 steps).  A KiB is then one wave-wide access everywhere: from memory into registers (few tokens), by DMA
// into LDS, from LDS into registers, without bank conflicts and without a swizzle; a block's step is a run of 4 KiB, which covers all 16 channels of an L2.
// Which channel a row is: row 4 q + v of group 2 b + t of a block is channel 8 q + 4 t + v of its b-th 32, so a lane's accumulators of two groups are 8 neighbouring
// channels.  Of a gated block's weights [gate | up] a block has 32 features: b = 0 their gate, b = 1 their up channels.  Tokens are in their order.
#pragma once
#include "block_epilogues.hpp"
#include "i8_codes.hpp"
#include "launch_block.hpp"

namespace ffn24 {

constexpr int MX4_STEP = 128, MX4_BLOCK_ROWS = 64, MX4_PANEL = 4096;
__host__ __device__ __forceinline__ int mx4_steps(int k) { return (k + MX4_STEP - 1) / MX4_STEP; }

// ------------------------------------------------------------------------------------------------ numbers
// top: the bits of a block's largest magnitude as fp32, sign cleared.  The largest value lands in [4, 8) scales (beyond 6 it is held to 6); with an infinity or a NaN
// the code is the NaN of the scales, and so is every product of the block.
__device__ __forceinline__ uint32_t mx4_scale_code(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
__device__ __forceinline__ float mx4_scale(uint32_t code) { return __builtin_bit_cast(float, code ? code << 23 : 0x00400000u); }
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// 8 values to a dword of codes; the instruction divides by the scale, rounds to nearest even and holds to 6 (measured: every border between neighbours, scales 2^-127 .. 2^125)
__device__ __forceinline__ bf16x2 two_bf16(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }   // (of a vector's element itself the compiler takes the first)
__device__ __forceinline__ uint32_t mx4_codes8(const u32x4& w, float s) {
  uint32_t o = 0u;
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, two_bf16(w[0]), s, 0);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, two_bf16(w[1]), s, 1);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, two_bf16(w[2]), s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, two_bf16(w[3]), s, 3);
}
__device__ __forceinline__ uint32_t mx4_codes8(const float (&x)[8], float s) {
  uint32_t o = 0u;
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[0], x[1], s, 0);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[2], x[3], s, 1);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, x[6], x[7], s, 3);
}
// the bits of the largest magnitude of 8 bf16 values, as an fp32's
__device__ __forceinline__ uint32_t mx4_top8(const u32x4& w) {
  const uint32_t m = pk_max16(pk_max16(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), pk_max16(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
  return max(m << 16, m & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu; }

template <int P> __device__ __forceinline__ uint32_t quad_max(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, P, 0xF, 0xF, true)); }
__device__ __forceinline__ uint32_t quad_max(uint32_t x) { return quad_max<quad_perm(2, 3, 0, 1)>(quad_max<quad_perm(1, 0, 3, 2)>(x)); }   // over the lanes of a quad

// Where row r's codes of the 32 k [32 kb, ...) start, and the byte of their scale
__device__ __forceinline__ size_t mx4_code_at(int r, int kb, int steps) {
  return ((size_t)(r >> 6) * steps + (kb >> 2)) * MX4_PANEL + ((r >> 4) & 3) * 1024 + (((kb & 3) << 4) + (r & 15)) * 16;
}
__device__ __forceinline__ size_t mx4_scale_at(int r, int kb, int steps) {
  return ((size_t)(r >> 6) * ((steps + 3) >> 2) + (kb >> 4)) * 1024 + ((r >> 4) & 3) * 256 + (((kb & 3) << 4) + (r & 15)) * 4 + ((kb >> 2) & 3);
}

// ------------------------------------------------------------------------------------------------ GEMM
struct Mx4Gemm {
  Mx4Operand A, B;
  int M, N;                 // what is really there of A's and B's rows
  int first, steps;         // the part of the reduction
};

// Bound by the matrix units where there is work for them: the op takes 18 cycles in a loop of nothing else (7.16 PFLOP/s with random bits at the 1.98 GHz that the power leaves;
// 8.9 with zeros), a step of the 256 x 256 tile 1300-1390 for 64 of them (1152), 5.1-5.25 PFLOP/s at K 16384.  A tile's results cost as much as six steps (bf16, all CUs' stores
// at once) or ten (the gate), so at K 4096 two 256 x 128 tiles a CU win, whose results and ops overlap: 8192 x 4096 x 16384 253 us (4.35 PFLOP/s, units busy 63 %), gate and up
// 8192 x 4096 x 32768 487 (4.5, 69 %); down 8192 x 16384 x 4096 on 256 x 256 220 (5.0, 73 %).  Small products are bound by launches and latency: 333 x 1088 x 4168 5.5 us.
// The block tile: 2 x 2 waves of 16 AM x 16 BN.  The ring holds RING stages of one step; the scales of four steps come beside them.  256 x 128 tiles have a ring of three, so that
// two share a CU: one's results go out while the other's matrix ops run.
template <int AM, int BN>
struct Mx4Geo {
  static constexpr int BM = 32 * AM, BNT = 32 * BN, RING = AM * BN == 32 ? 3 : 4;
  static constexpr int STAGE = (2 * AM + 2 * BN) * 1024, SCALES = (AM + BN) / 2;   // scales: KiB (instructions) for four steps
  static constexpr int LDS = RING * STAGE + SCALES * 1024;
  static constexpr int NDMA = AM / 2 + BN / 2, NSC = (SCALES + 3) / 4;              // instructions a wave: a stage's, four steps' scales
  static constexpr int PER_CU = LDS <= 80 * 1024 ? 2 : 1;
  static constexpr int UNROLL = RING == 4 ? 4 : 12;                                 // steps until ring and scales' bytes come round together
};

// The accumulator tied in place: through the builtin the compiler moves accumulators round the scaled op and runs at half its rate (5.2 against 7.16 PFLOP/s in a loop of nothing
// else).  J: the byte of the scales' registers, the step's number of four.
template <int J>
__device__ __forceinline__ void op16_mx4(const u32x4& a, const u32x4& b, uint32_t sa, uint32_t sb, f32x4& c) {
#define FFN24_OP(lo, hi) \
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[" lo "," lo ",0] op_sel_hi:[" hi "," hi ",0] cbsz:4 blgp:4" : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb))
  if constexpr (J == 0) FFN24_OP("0", "0");
  else if constexpr (J == 1) FFN24_OP("1", "0");
  else if constexpr (J == 2) FFN24_OP("0", "1");
  else FFN24_OP("1", "1");
#undef FFN24_OP
}

// item I of N on slots 1, 2, 5, 6, ... (of few slots: from the first one on)
template <int N, int SLOTS, int M, class F>
__device__ __forceinline__ void mx4_early(F&& f) {
  if constexpr (SLOTS >= 2 * N + 2) {
    constexpr int i = M % 4 == 1 ? M / 4 * 2 : M % 4 == 2 ? M / 4 * 2 + 1 : N;
    if constexpr (i < N) f(std::integral_constant<int, i>{});
  } else if constexpr (M < N) {
    f(std::integral_constant<int, M>{});
  }
}
// item I of N spread over SLOTS slots
template <int N, int SLOTS, int M, class F>
__device__ __forceinline__ void mx4_ride(F&& f) {
  constexpr int lo = (M * N + SLOTS - 1) / SLOTS, hi = ((M + 1) * N + SLOTS - 1) / SLOTS;
  static_for<hi - lo>([&](auto i) { f(std::integral_constant<int, lo + decltype(i)::value>{}); });
}

template <class Epi, int AM, int BN>
__device__ __forceinline__ void mx4_tile(const Mx4Gemm& g, const typename Epi::Args& ea, char* smem, int tm, int tn) {
  using G = Mx4Geo<AM, BN>;
  constexpr int D = G::NDMA, H1 = (D + 1) / 2, HB = BN / 2, HO = AM * HB, R = G::RING;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wy = wave >> 1, wx = wave & 1;
  const int a_blocks = (g.M + 63) >> 6, b_blocks = (g.N + 63) >> 6, am = tm * (AM / 2), bm = tn * (BN / 2);   // in blocks of 64 rows
  const int all = (g.A.steps + 3) >> 2, n = g.steps, last = (n - 1) >> 2;   // steps; the last four steps' number
  const auto rsrc = [](const char* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, -1, 0x00020000); };
  // (a block beyond the last one is read as the last: its results are not stored)
  const __amdgpu_buffer_rsrc_t ra = rsrc(g.A.codes + ((size_t)am * g.A.steps + g.first) * MX4_PANEL), rb = rsrc(g.B.codes + ((size_t)bm * g.B.steps + g.first) * MX4_PANEL);
  const __amdgpu_buffer_rsrc_t sa_r = rsrc(g.A.scales + ((size_t)am * all + (g.first >> 2)) * 1024), sb_r = rsrc(g.B.scales + ((size_t)bm * all + (g.first >> 2)) * 1024);
  uint32_t oa[AM / 2], ob[BN / 2];
#pragma unroll
  for (int j = 0; j < AM / 2; j++) {
    const int i = wave * (AM / 2) + j;
    oa[j] = (uint32_t)(min(am + (i >> 2), a_blocks - 1) - am) * (uint32_t)g.A.steps * MX4_PANEL + (i & 3) * 1024;
  }
#pragma unroll
  for (int j = 0; j < BN / 2; j++) {
    const int i = wave * (BN / 2) + j;
    ob[j] = (uint32_t)(min(bm + (i >> 2), b_blocks - 1) - bm) * (uint32_t)g.B.steps * MX4_PANEL + (i & 3) * 1024;
  }
  char* const sc = smem + R * G::STAGE;
  // the wave's part of the scales of the four steps from 4 S on, a KiB an instruction (where there are fewer of them than waves, some are fetched twice)
  auto issue_scales = [&](int S) {
#pragma unroll
    for (int j = 0; j < G::NSC; j++) {
      const int i = (wave + 4 * j) % G::SCALES;
      const bool isb = i >= AM / 2;
      const int blk = isb ? min(bm + i - AM / 2, b_blocks - 1) - bm : min(am + i, a_blocks - 1) - am;
      const uint32_t off = ((uint32_t)blk * (uint32_t)all + (uint32_t)min(S, last)) * 1024;
      if (isb) __builtin_amdgcn_raw_ptr_buffer_load_lds(sb_r, (lds_char*)(sc + i * 1024), 16, lane * 16, (int)off, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(sa_r, (lds_char*)(sc + i * 1024), 16, lane * 16, (int)off, 0, 0);
    }
  };
  // instruction J of stage kt into place `slot` of the ring
  auto issue = [&](auto J, int kt, int slot) {
    constexpr int j = decltype(J)::value;
    char* const buf = smem + slot * G::STAGE;
    if constexpr (j < AM / 2) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_char*)(buf + (wave * (AM / 2) + j) * 1024), 16, lane * 16, (int)(oa[j < AM / 2 ? j : 0] + (uint32_t)kt * MX4_PANEL), 0, 0);
    } else {
      constexpr int i = j - AM / 2;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_char*)(buf + (2 * AM + wave * (BN / 2) + i) * 1024), 16, lane * 16, (int)(ob[i] + (uint32_t)kt * MX4_PANEL), 0, 0);
    }
  };

  const bool full = n >= R;
  issue_scales(0);
  for (int s = 0; s < min(n, R - 1); s++) static_for<D>([&](auto J) { issue(J, s, s); });
  if (full) static_for<H1>([&](auto J) { issue(J, R - 1, R - 1); });

  f32x4 acc[AM][BN];
#pragma unroll
  for (int i = 0; i < AM; i++)
#pragma unroll
    for (int j = 0; j < BN; j++) {
      acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      asm volatile("" : "+a"(acc[i][j]));
    }
  u32x4 a[AM], b[2][HB];
  uint32_t sa[AM], sb[BN];
  const char *la = smem + wy * AM * 1024 + lane * 16, *lb = smem + (2 * AM + wx * BN) * 1024 + lane * 16;
  const char *lsa = sc + wy * AM * 256 + lane * 4, *lsb = sc + (AM / 2) * 1024 + wx * BN * 256 + lane * 4;
  auto read_scales = [&](uint32_t (&xa)[AM], uint32_t (&xb)[BN]) {
#pragma unroll
    for (int t = 0; t < AM; t++) xa[t] = *reinterpret_cast<const uint32_t*>(lsa + t * 256);
#pragma unroll
    for (int t = 0; t < BN; t++) xb[t] = *reinterpret_cast<const uint32_t*>(lsb + t * 256);
  };
  if (full) wait_vmcnt<(R - 2) * D + H1>(); else wait_vmcnt<0>();
  __builtin_amdgcn_s_barrier();
  FFN24_FENCE();
  static_for<AM>([&](auto T) { a[T] = *reinterpret_cast<const u32x4*>(la + T * 1024); });
  static_for<HB>([&](auto T) { b[0][T] = *reinterpret_cast<const u32x4*>(lb + T * 1024); });
  read_scales(sa, sb);
  FFN24_FENCE();
  asm volatile("s_nop 4" ::: "memory");

  // The step of stage kt (kt % UNROLL = J), in two halves as the 256 x 256 tile of gemm_core.hpp: the other half's B fragments are read during the first; then one barrier,
  // behind which this stage's buffer is free; during the second the next step's fragments are read and the stage that reuses the buffer is asked for (the rest of
  // it during the next step's first half).  The scales of four steps are read into registers during the last step before them; behind the next barrier their place is
  // free, and the next four's are asked for.  TAIL: there may be no stage left to ask for, or to read (what is read then is not used).
  auto step = [&](int kt, auto j, auto tail) {
    constexpr int J = decltype(j)::value, S = J % 4, cur = J % R * G::STAGE, nxt = (J + 1) % R * G::STAGE;
    constexpr bool TAIL = decltype(tail)::value != 0;
    // instructions behind the next stage's that may be in flight at the barrier: the scales went out with the stages 4 i + R
    constexpr int LEFT = (R - 2) * D + ((S + 2) % 4 == R % 4 || (R == 4 && (S + 3) % 4 == 0) ? G::NSC : 0);
    const bool rest = !TAIL || kt + R - 1 < n, ask = !TAIL || kt + R < n;
    FFN24_FENCE();
    static_for<HO>([&](auto M) {
      constexpr int mi = M / HB, ni = M % HB;
      op16_mx4<S>(a[mi], b[0][ni], sa[mi], sb[ni], acc[mi][ni]);
      mx4_early<HB, HO, M>([&](auto I) { b[1][I] = *reinterpret_cast<const u32x4*>(lb + cur + (HB + I) * 1024); });
      mx4_ride<D - H1, HO, M>([&](auto I) { if (rest) issue(std::integral_constant<int, H1 + decltype(I)::value>{}, kt + R - 1, (J + R - 1) % R); });
      FFN24_FENCE();
    });
    if (rest && ask) wait_vmcnt<LEFT>(); else wait_vmcnt<0>();
    wait_lgkmcnt0();
    __builtin_amdgcn_s_barrier();
    FFN24_FENCE();
    uint32_t na[AM], nb[BN];
    if constexpr (S == 3) read_scales(na, nb);
    if constexpr (S == 0) { if (ask) issue_scales((kt >> 2) + 1); }
    FFN24_FENCE();
    static_for<HO>([&](auto M) {
      constexpr int mi = M / HB, ni = M % HB;
      op16_mx4<S>(a[mi], b[1][ni], sa[mi], sb[HB + ni], acc[mi][HB + ni]);
      mx4_early<HB, HO, M>([&](auto I) { b[0][I] = *reinterpret_cast<const u32x4*>(lb + nxt + I * 1024); });
      if constexpr (ni == HB - 1) a[mi] = *reinterpret_cast<const u32x4*>(la + nxt + mi * 1024);
      mx4_ride<H1, HO, M>([&](auto I) { if (ask) issue(I, kt + R, J % R); });
      FFN24_FENCE();
    });
    if constexpr (S == 3) {
      // (a vector instruction may write an operand two states before its op at the latest)
#pragma unroll
      for (int t = 0; t < AM; t++) sa[t] = na[t];
#pragma unroll
      for (int t = 0; t < BN; t++) sb[t] = nb[t];
      FFN24_FENCE();
      asm volatile("s_nop 1" ::: "memory");
    }
  };
  using I0 = std::integral_constant<int, 0>; using I1 = std::integral_constant<int, 1>;
  int kt = 0;
  for (; kt + G::UNROLL + R <= n; kt += G::UNROLL) static_for<G::UNROLL>([&](auto J) { step(kt + J, J, I0{}); });
  while (kt < n) static_for<G::UNROLL>([&](auto J) {
    if (kt < n) {
      step(kt, J, I1{});
      kt++;
    }
  });

  asm volatile("s_nop 15\n s_nop 15\n s_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < AM; i++)
#pragma unroll
    for (int j = 0; j < BN; j++) asm volatile("" : "+a"(acc[i][j]));
  Epi::template run<AM, BN>(ea, acc, tm * G::BM + wy * 16 * AM, tn * G::BNT + wx * 16 * BN, fresh_lane());
}

template <class Epi, int AM, int BN>
__global__ void __launch_bounds__(GEMM_THREADS, (Mx4Geo<AM, BN>::PER_CU)) mx4_gemm_kernel(Mx4Gemm g, typename Epi::Args ea, int tiles_m, int tiles_n, int part) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int pid = blockIdx.x, tm, tn;
  if (part > 0) {                                              // part `split` of the reduction
    const int split = pid / (tiles_m * tiles_n);
    pid -= split * tiles_m * tiles_n;
    g.first = split * part;
    g.steps = min(part, g.A.steps - g.first);
    Epi::part(ea, split);
  }
  tile_coords<0, AM == 2 * BN>(tiles_m, tiles_n, pid, tm, tn);
  mx4_tile<Epi, AM, BN>(g, ea, smem, tm, tn);
}

// ------------------------------------------------------------------------------------------------ epilogues
// m: the wave's first row of A, n: its first row of B.  acc[2 i], acc[2 i + 1] of a lane: channels m + 32 i + 8 q .. + 7 of token n + 16 j + c.
struct Mx4Rows {   // out[n][m] in bf16
  struct Args { uint16_t* out; int M, N; };
  static __device__ __forceinline__ void part(Args&, int) {}
  template <int AM, int BN>
  static __device__ __forceinline__ void run(const Args& e, f32x4 (&acc)[AM][BN], int m, int n, int lane) {
    const int q = lane >> 4, c = lane & 15;
#pragma unroll
    for (int j = 0; j < BN; j++) {
      const int t = n + 16 * j + c;
#pragma unroll
      for (int i = 0; i < AM / 2; i++) {
        const int ch = m + 32 * i + 8 * q;
        const f32x4 x = acc[2 * i][j], y = acc[2 * i + 1][j];
        if (t < e.N && ch < e.M)
          *reinterpret_cast<u32x4*>(e.out + (size_t)t * e.M + ch) = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
      }
    }
  }
};

struct Mx4Part {   // the sums of a part of the reduction, [part][n][m]
  struct Args { uint32_t* parts; int M, N; };
  static __device__ __forceinline__ void part(Args& e, int split) { e.parts += (size_t)split * e.M * e.N; }
  template <int AM, int BN>
  static __device__ __forceinline__ void run(const Args& e, f32x4 (&acc)[AM][BN], int m, int n, int lane) {
    const int q = lane >> 4, c = lane & 15;
#pragma unroll
    for (int j = 0; j < BN; j++) {
      const int t = n + 16 * j + c;
#pragma unroll
      for (int i = 0; i < AM / 2; i++) {
        const int ch = m + 32 * i + 8 * q;
        if (t < e.N && ch < e.M) {
          f32x4* p = reinterpret_cast<f32x4*>(e.parts + (size_t)t * e.M + ch);
          p[0] = acc[2 * i][j];
          p[1] = acc[2 * i + 1][j];
        }
      }
    }
  }
};

// h is rounded once, to mx4, from 32 bits: the down product takes nothing wider.  The gate's arithmetic is what this epilogue costs (12500-15000 cycles of a 256 x 256 tile).
// The gated block: h = a(G) U of 32 features of a token lies in four lanes, 8 each; their largest magnitude gives the scale, and the codes go out as the down product reads
// them: 16 tokens' 32 features are 256 bytes in a row.
template <bool CUBIC>
struct Mx4Gated {
  struct Args { char* codes; uint8_t* scales; int F, N, steps; Gate gate; };
  static __device__ __forceinline__ void part(Args&, int) {}
  // without the cubic term the argument needs no hold: the exponential ends at 0 and infinity by itself
  static __device__ __forceinline__ float act(const Gate& g, float x) { return CUBIC ? gate_act(g, x) : x * sigmoid(x); }
  template <int AM, int BN>
  static __device__ __forceinline__ void run(const Args& e, f32x4 (&acc)[AM][BN], int m, int n, int lane) {
    static_assert(AM % 4 == 0, "whole blocks of 64 rows a wave");
    const int q = lane >> 4, c = lane & 15;
#pragma unroll
    for (int j = 0; j < BN; j++) {
      const int t = n + 16 * j + c;
#pragma unroll
      for (int i = 0; i < AM / 4; i++) {
        const int kb = (m >> 6) + i;                           // the block of 32 features
        float h[8];
        uint32_t top = 0u;
#pragma unroll
        for (int v = 0; v < 8; v++) {
          h[v] = act(e.gate, acc[4 * i + v / 4][j][v % 4]) * acc[4 * i + 2 + v / 4][j][v % 4];
          top = max(top, magnitude(h[v]));
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
        const uint32_t code = mx4_scale_code(top);
        if (t < e.N && 32 * kb < e.F) {
          *reinterpret_cast<uint32_t*>(e.codes + mx4_code_at(t, kb, e.steps) + 4 * q) = mx4_codes8(h, mx4_scale(code));
          if (q == 0) e.scales[mx4_scale_at(t, kb, e.steps)] = (uint8_t)code;
        }
      }
    }
  }
};

}  // namespace ffn24
