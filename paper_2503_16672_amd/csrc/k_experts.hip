// Few tokens: products with weights in the operand form of mx4_core.hpp (mx4, or bf16 in the same order), and the mixture of experts made of them.
//
//   Y[t][n] = sum_k X[t][k] W[k][n];   h = a(X Wg) (X Wu);   y = sum over the chosen experts of p_e (h_e Wd_e)
//
// Bound by the weights' bytes: up to 64 tokens a weight meets few products.  A wave streams weights from memory straight into operands of the 16 x 16 matrix ops (rows: output
// channels, columns: tokens, 16 at a time), for which they lie in the ops' own order: no LDS, no swizzle, whole lines.  The waves of a workgroup share the reduction of a strip of
// channels and add up through LDS in a fixed order.  A wave has 8 KiB of weights on their way while it works on 8 KiB, a CU 128 KiB.
//
// Mixture of experts, four launches and a fifth where strips are shared (a single token: three or four):
//   router   logits X Wr in 64 bits, a part of D a workgroup (a product of two bf16 is exact in fp32; in 64 bits the choice between near experts is the definition's)
//   pick     a token's k largest by their rank, ties to the lowest index; shares; and the plan, which expert has which tokens (a single token's: in `up`)
//   up       a workgroup a strip of 32 features of a chosen expert: h = a(G) U for the tokens that chose it; a row of H for each (token, choice), in the experts' order
//   down     a workgroup a strip of 16 to 64 channels and all chosen experts one after the other: the shares' sum stays in LDS, in the order of the experts
//   sum      where several workgroups share a strip's experts (moe_down_splits): their sums, in a fixed order
// us, kernel by kernel (in brackets weights' bytes a second): 64 tokens, 4096 x 2048, all of 64 bf16 experts 4.8, 5.6, up 319 (6.7 TB/s), down 160 (6.7), 4.8; 8 tokens of 64 mx4
// experts 5.0, 6.0, 62.4 (5.8), 34.6 (5.2); 37 tokens, 1088 x 704, 24 bf16 experts 4.3, 5.8, 16.4 (4.5), 11.7, 3.9; 1 token, 2048 x 1024, 4 of 32 3.8, -, 7.9 (with the choice),
// 7.8.  The large ones run at 0.95 of the rate of reads alone (7.1 TB/s of 4 GiB); what bounds the small ones is the launches and each one's way through memory and LDS.
#include "mx4_core.hpp"
#include "mx4_rule.hpp"
#include "stream_core.hpp"

namespace ffn24 {
namespace {

constexpr int WAVES = 8, THREADS = 64 * WAVES, RED = 17;   // RED: pitch of the sums' image [channel][16 tokens]

// Workgroup ids go round the 8 XCDs; an XCD gets a run of neighbouring strips instead (a strip of 16 channels is a KiB of every 4: a quarter of an L2's channels)
__device__ __forceinline__ unsigned run_of(unsigned id, unsigned n) {
  const unsigned per = n >> 3, more = n & 7u, xcd = id & 7u;
  return xcd * per + min(xcd, more) + (id >> 3);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }   // what is the same for the whole wave, in a scalar register

// Where a wave's weights are: the strip's codes and scales, bytes from a step (four steps' scales) to the next
struct Strip { const char* codes; const char* scales; int steps; };

// The scaled op with its accumulator in place, as in mx4_core.hpp (the builtin also keeps 32 bytes of registers for an operand of 16).  The compiler does not see what it needs:
// two states behind the vector instructions that make its operands, and where the same accumulator comes round at once (RG 1), the op before it; settle() before results are read.
template <int RG>
__device__ __forceinline__ void op16_mx4_few(const u32x4& a, const u32x4& b, uint32_t sa, uint32_t sb, f32x4& c) {
  if constexpr (RG == 1) asm volatile("s_nop 7\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+v"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
  else asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+v"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
}
template <int RG, int NT>
__device__ __forceinline__ void settle(f32x4 (&acc)[RG][NT]) {
  asm volatile("s_nop 15" ::: "memory");
#pragma unroll
  for (int g = 0; g < RG; g++)
#pragma unroll
    for (int i = 0; i < NT; i++) asm volatile("" : "+v"(acc[g][i]));
}

// Sums, shares and the gate are fp32.  Between the products h of mx4 experts is rounded to mx4, which their definition says; of bf16 experts it is the sum of two bf16, its upper
// 16 bits and the rest rounded, which leaves 2^-16 of it: the op takes no fp32, and rounded to one bf16 h would cost as much accuracy as Y's own rounding.
__device__ __forceinline__ uint32_t two_parts(float h) {          // the first in the low half; an infinity or a NaN has no rest
  const float first = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, h) & 0xFFFF0000u);
  const float rest = magnitude(h) < 0x7F800000u ? h - first : 0.f;
  return __builtin_bit_cast(uint32_t, first) >> 16 | pack_bf16x2(0.f, rest);
}

// Tokens of a product: rows of bf16 [..][K]; the mx4 operand form; (a small T K) rows of bf16 that the workgroup brings to mx4 in its LDS, codes [K / 32][T][16 bytes] and
// scales [K / 32][T], while its first weights are on their way; or values in two parts as the bf16 op reads them, [16 rows][step of 32 k][part][lane][16 bytes]
enum { ROWS_BF16 = 0, OPERAND_MX4 = 1, LDS_MX4 = 2, OPERAND_PARTS = 3 };
__device__ __forceinline__ size_t parts_at(int r, int s, int q, int K) { return ((size_t)(r >> 4) * (K >> 5) + s) * 2048 + q * 256 + (r & 15) * 16; }   // row r, k 32 s + 8 q
struct Tokens { const char* p; const char* scales; int K, steps, T; };
constexpr int LDS_PIECES = MX4_FUSED_VALUES / 8 / THREADS;     // of 8 values a work item

struct StagedTokens {
  u32x4 w[LDS_PIECES];
  __device__ __forceinline__ void load(const char* X, int pieces) {
#pragma unroll
    for (int j = 0; j < LDS_PIECES; j++) {
      const int i = j * THREADS + (int)threadIdx.x;
      if (j * THREADS < pieces) w[j] = i < pieces ? reinterpret_cast<const u32x4*>(X)[i] : u32x4{0u, 0u, 0u, 0u};
    }
  }
  // (a row is a whole number of blocks, so the four lanes of a block are all there or none)
  __device__ __forceinline__ void store(char* codes, char* scales, int pieces, int K, int T) const {
    const int per = K / 8, p = threadIdx.x & 3;
    const uint32_t inverse = 0xFFFFFFFFu / (uint32_t)per + 1u;   // (i / per = the upper half of i * inverse for i, per up to 2^13)
#pragma unroll
    for (int j = 0; j < LDS_PIECES; j++) {
      const int i = j * THREADS + (int)threadIdx.x;
      if (j * THREADS >= pieces) break;
      const uint32_t code = mx4_scale_code(quad_max(mx4_top8(w[j])));
      const int t = (int)__umulhi((uint32_t)i, inverse), at = ((i - t * per) >> 2) * T + t;
      if (i < pieces) {
        *reinterpret_cast<uint32_t*>(codes + at * 16 + 4 * p) = mx4_codes8(w[j], mx4_scale(code));
        if (p == 0) scales[at] = (char)code;
      }
    }
  }
};

// U steps of RG groups of 16 channels, and of the first NP groups of 16 tokens, on their way.  The tokens are asked for first: loads come back in order, so what is asked
// for behind the weights would wait for them.
template <int SRC, int RG, int U, int NP, int GS = 1>   // GS: from a group to the next of the strip's
struct Unit {
  static constexpr bool MX4 = SRC == OPERAND_MX4 || SRC == LDS_MX4;
  static constexpr int SU = MX4 ? (U + 3) / 4 : 1, XU = SRC == LDS_MX4 ? 1 : U;
  static constexpr int P = SRC == OPERAND_PARTS ? 2 : 1, C = P == 2 && RG == 1 ? U / 2 : U;   // parts of a value; steps of a later group at once (eight in parts would not fit the registers)
  u32x4 w[U][RG], x[XU][NP][P];
  uint32_t sw[SU][RG], sx[SRC == OPERAND_MX4 ? SU : 1][NP];

  // the lane's 16 bytes of token row `row` in step s (part p of its values), and its scales of the four steps of s
  static __device__ __forceinline__ u32x4 token(const Tokens& t, int row, bool on, int s, int q, int p) {
    if constexpr (SRC == OPERAND_PARTS) return *reinterpret_cast<const u32x4*>(t.p + parts_at(row, s, q, t.K) + 1024 * p);   // (`row` is one that is there)
    if (!on) return u32x4{0u, 0u, 0u, 0u};
    if constexpr (SRC == OPERAND_MX4) return *reinterpret_cast<const u32x4*>(t.p + mx4_code_at(row, 4 * s + q, t.steps));
    return *reinterpret_cast<const u32x4*>(t.p + ((size_t)row * t.K + 32 * s + 8 * q) * 2);
  }
  static __device__ __forceinline__ uint32_t token_scales(const Tokens& t, int row, bool on, int s, int q) {
    return on ? *reinterpret_cast<const uint32_t*>(t.scales + (mx4_scale_at(row, 4 * s + q, t.steps) & ~(size_t)3)) : 0u;
  }
  // from step s0 (a multiple of U) on; steps beyond the last read the last one and are not used
  __device__ __forceinline__ void load(const Strip& p, const Tokens& t, const int (&row)[NP], const bool (&on)[NP], int s0, int lane) {
    const int q = lane >> 4;
    if constexpr (SRC != LDS_MX4) {
#pragma unroll
      for (int j = 0; j < U; j++)
#pragma unroll
        for (int i = 0; i < NP; i++)
#pragma unroll
          for (int a = 0; a < P; a++) x[j][i][a] = token(t, row[i], on[i], min(s0 + j, p.steps - 1), q, a);
    }
    if constexpr (SRC == OPERAND_MX4) {
#pragma unroll
      for (int j = 0; j < SU; j++)
#pragma unroll
        for (int i = 0; i < NP; i++) sx[j][i] = token_scales(t, row[i], on[i], min(s0 + 4 * j, p.steps - 1), q);
    }
    if constexpr (MX4) {
#pragma unroll
      for (int j = 0; j < SU; j++) {
        const char* at = p.scales + (size_t)(min(s0 + 4 * j, p.steps - 1) >> 2) * 1024 + lane * 4;
#pragma unroll
        for (int g = 0; g < RG; g++) sw[j][g] = *reinterpret_cast<const uint32_t*>(at + g * GS * 256);
      }
    }
#pragma unroll
    for (int j = 0; j < U; j++) {
      const char* at = p.codes + (size_t)min(s0 + j, p.steps - 1) * MX4_PANEL + lane * 16;
#pragma unroll
      for (int g = 0; g < RG; g++) w[j][g] = ld_stream(reinterpret_cast<const u32x4*>(at + g * GS * 1024));
    }
  }
  // sx: the scale in the low byte
  template <int NT>
  __device__ __forceinline__ void op(int j, int i, int s0, const u32x4& v, uint32_t sx, f32x4 (&acc)[RG][NT]) const {
#pragma unroll
    for (int g = 0; g < RG; g++) {
      if constexpr (MX4) op16_mx4_few<RG>(w[j][g], v, sw[j / 4][g] >> (8 * ((s0 + j) & 3)), sx, acc[g][i]);
      else acc[g][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[j][g]), __builtin_bit_cast(bf16x8, v), acc[g][i], 0, 0, 0);
    }
  }
  // the ops of the unit for `groups` groups of tokens; those from NP on are asked for here, C steps of a group together
  template <int NT>
  __device__ __forceinline__ void ops(const Tokens& t, const int (&row)[NT], const bool (&on)[NT], int groups, int s0, int steps, int q, f32x4 (&acc)[RG][NT]) const {
#pragma unroll
    for (int i = 0; i < NT; i++) {
      if (i > 0 && i >= groups) break;
      uint32_t sv[SU];
#pragma unroll
      for (int j = 0; j < SU; j++) {
        sv[j] = 0u;
        if constexpr (SRC == OPERAND_MX4) sv[j] = i < NP ? sx[j][i < NP ? i : 0] : token_scales(t, row[i], on[i], min(s0 + 4 * j, steps - 1), q);
      }
#pragma unroll
      for (int j0 = 0; j0 < U; j0 += C) {
        u32x4 v[C][P];
#pragma unroll
        for (int j = 0; j < C; j++)
#pragma unroll
          for (int a = 0; a < P; a++) {
            if constexpr (SRC == LDS_MX4) {
              v[j][a] = u32x4{0u, 0u, 0u, 0u};
            } else {
              v[j][a] = i < NP ? x[j0 + j][i < NP ? i : 0][a] : token(t, row[i], on[i], min(s0 + j0 + j, steps - 1), q, a);
            }
          }
#pragma unroll
        for (int c = 0; c < C; c++) {
          const int j = j0 + c;
          if (s0 + j >= steps) break;
          if constexpr (SRC == LDS_MX4) {
            const int kb = 4 * (s0 + j) + q, at = kb * t.T + row[i];
            const bool there = on[i] && 32 * kb < t.K;
            op(j, i, s0, there ? *reinterpret_cast<const u32x4*>(t.p + at * 16) : u32x4{0u, 0u, 0u, 0u}, there ? (uint32_t)(uint8_t)t.scales[at] : 0u, acc);
          } else {
#pragma unroll
            for (int a = 0; a < P; a++) op(j, i, s0, v[c][a], sv[MX4 ? j / 4 : 0] >> (8 * ((s0 + j) & 3)), acc);
          }
        }
      }
      if constexpr (NT > 1 && MX4) {                           // (where the groups' paths part, the compiler may move accumulators)
        asm volatile("s_nop 15" ::: "memory");
#pragma unroll
        for (int g = 0; g < RG; g++) asm volatile("" : "+v"(acc[g][i]));
      }
    }
  }
};

// The channel of a strip's row r (0 .. 16 RG - 1) from the strip's block of 64 on; g0: the strip's first group in its block
__device__ __forceinline__ int channel_of(int g, int r) { return 32 * (g >> 1) + 8 * (r >> 2) + 4 * (g & 1) + (r & 3); }

// ------------------------------------------------------------------------------------------------ experts' lists
constexpr int MOE_E = MOE_MAX_E, MOE_PAIRS = MOE_TOKENS * MOE_MAX_K;   // most experts; most (token, choice) pairs
// The chosen experts in ascending order; the pairs of the i-th are list[start[i]] .. list[start[i + 1] - 1], with their shares beside them.  (The order of an expert's pairs
// is as it comes: it says which column of an op a token is, which no result depends on.)
struct MoePlan {
  int ticket, n_active, expert[MOE_E], start[MOE_E + 2], list[MOE_PAIRS];
  float share[MOE_PAIRS];
  int picks[MOE_PAIRS];                // on their way to the plan
  float shares[MOE_PAIRS];
};
// Words that workgroups of a launch hand to each other go past the XCDs' own L2s (agent scope); what was stored so is there once the storing wave has waited for it.
template <class T> __device__ __forceinline__ void put(T* p, T x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class T> __device__ __forceinline__ T get(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A value as an integer of the same order; NaN below all
__device__ __forceinline__ unsigned long long order_of(double x) {
  const unsigned long long b = __builtin_bit_cast(unsigned long long, x + 0.0);   // (-0 is 0)
  return x != x ? 1ull : b >> 63 ? ~b : b | 1ull << 63;
}

// The choice of one token by a workgroup of THREADS: its k experts by falling logit, and their shares.  Several work items have an expert, each a part of its logit's sum and of
// the comparisons that give its rank.  p: the token's parts of the logits, `stride` values from a part to the next.
struct Choice {
  double sums[THREADS], logit[MOE_MAX_K];
  unsigned long long order[MOE_E];
  int rank[MOE_E], which[MOE_MAX_K];
  float share[MOE_MAX_K], part[4];
};
__device__ __forceinline__ void moe_choose(const double* __restrict__ p, size_t stride, int n_parts, int E, int k, bool renormalise, Choice& c) {
  const int e = threadIdx.x, ways = THREADS / E, way = e / E, ex = e - way * E;
  double s = 0.0;
  if (way < ways)
    for (int i = way; i < n_parts; i += 8 * ways) {            // eight on their way at once
      double v[8];
#pragma unroll
      for (int j = 0; j < 8; j++) v[j] = i + j * ways < n_parts ? p[(size_t)(i + j * ways) * stride + ex] : 0.0;
#pragma unroll
      for (int j = 0; j < 8; j++) s += v[j];
    }
  c.sums[e] = s;
  __syncthreads();
  s = 0.0;
  if (e < E) {
    for (int i = 0; i < ways; i++) s += c.sums[i * E + e];
    c.order[e] = order_of(s);
    c.rank[e] = 0;
  }
  __syncthreads();
  if (way < ways) {
    const unsigned long long mine = c.order[ex];
    int before = 0;
#pragma unroll 4
    for (int i = way; i < E; i += ways) before += c.order[i] > (i < ex ? mine - 1 : mine);   // (an equal one of a lower index is before it; no order is 0)
    atomicAdd(&c.rank[ex], before);
  }
  __syncthreads();
  int rank = MOE_E;
  if (e < E) {
    rank = c.rank[e];
    if (rank < k) {
      c.logit[rank] = s;
      c.which[rank] = e;
    }
  }
  __syncthreads();
  // shares: exp(l - largest) over its sum, of the chosen or of all
  const float x = e < E && (rank < k || !renormalise) ? expf((float)(s - c.logit[0])) : 0.f;
  float sum = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
  if (e < MOE_E && (e & 63) == 0) c.part[e >> 6] = sum;
  __syncthreads();
  if (rank < k) c.share[rank] = x / (c.part[0] + c.part[1] + c.part[2] + c.part[3]);
  __syncthreads();
}
// Work item j < k of a single token: its expert's place among the chosen ones
__device__ __forceinline__ int place_of(const Choice& c, int j, int k) {
  int at = 0;
  for (int i = 0; i < k; i++) at += c.which[i] < c.which[j];
  return at;
}

// ------------------------------------------------------------------------------------------------ up
struct UpArgs {
  const char* w; size_t w_stride;      // weights of an expert (operand form, codes then scales) and bytes to the next expert's
  size_t scales_at;                    // where an expert's scales start
  int steps, K, F, T;                  // steps of K; features
  Gate gate;
  const char* x; const char* x_scales; // bf16 [T][K], or the operand form
  char* h; char* h_scales; int h_steps;   // the operand form, of values in two parts or of mx4
  const MoePlan* plan; int k;          // MOE
  MoePlan* plan_out; const double* logits; int n_parts, E, renormalise; int* picks; float* shares;   // MOE_ONE: parts of the logits, where the choice goes
};

// Gate and up of a feature are rows 16 apart of a strip, so h is made where the waves' sums are added up, and an mx4 block's largest magnitude is over 32 neighbouring lanes.
// grid (strips, slots).  A slot is a chosen expert; without MOE there is one, and it has all tokens.  A strip is 8 RG features: a block of 64 rows, or (RG 2, bf16, whose result
// needs no 32 features together) every other group of one.
// MOE_ONE: a single token of the experts, whose choice every workgroup makes by itself; the first one stores it.  PASSES: over the weights, one for every 16 NT tokens of the
// expert (otherwise it has no more than those).
enum { ALL_TOKENS = 0, MOE = 1, MOE_ONE = 2 };
template <int SRC, int NT, int WHO, int RG, int W, bool PASSES = false>
__global__ void __launch_bounds__(64 * W, NT == 1 && WHO != MOE_ONE ? 4 : 2) few_up_kernel(UpArgs e) {
  constexpr bool MX4 = SRC != ROWS_BF16;
  constexpr int U = PASSES && MX4 ? 1 : 8 / RG, NP = 1, FEATS = 8 * RG;   // (more would not fit the registers)
  static_assert(RG == 4 || (RG == 2 && !MX4), "whole blocks of 32 features");
  static_assert(WHO != MOE_ONE || W == WAVES, "chosen by all work items");
  __shared__ __attribute__((aligned(16))) float red[W * 16 * RG * RED];
  extern __shared__ __attribute__((aligned(16))) char staged_lds[];   // LDS_MX4: T K 17 / 32 bytes
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // whole blocks are 4 KiB a step and cover an L2's channels by themselves: they go round the XCDs, which then share the experts that were chosen (the last slots may have none)
  const unsigned at = blockIdx.y * gridDim.x + blockIdx.x, id = RG == 4 ? at : run_of(at, gridDim.x * gridDim.y), slot = id / gridDim.x;
  const int strip = (int)(id - slot * gridDim.x), block = RG == 4 ? strip : strip >> 1, half = RG == 4 ? 0 : strip & 1;
  int expert = 0, n = e.T, first = 0;
  if constexpr (WHO == MOE_ONE) {
    __shared__ Choice one;
    __shared__ int mine;
    moe_choose(e.logits, (size_t)e.E, e.n_parts, e.E, e.k, e.renormalise != 0, one);
    if (tid < e.k) {
      const int to = place_of(one, tid, e.k);
      if (to == (int)slot) mine = tid;
      if (at == 0) {
        e.picks[tid] = one.which[tid];
        e.shares[tid] = one.share[tid];
        e.plan_out->expert[to] = one.which[tid];
        e.plan_out->start[to] = to;
        e.plan_out->list[to] = tid;
        e.plan_out->share[to] = one.share[tid];
        if (tid == 0) {
          e.plan_out->n_active = e.k;
          e.plan_out->start[e.k] = e.k;
        }
      }
    }
    __syncthreads();
    first = (int)slot;
    expert = uniform(one.which[uniform(mine)]);
  }
  if constexpr (WHO == MOE) {
    if ((int)slot >= e.plan->n_active) return;
    expert = e.plan->expert[slot];
    first = e.plan->start[slot];
    n = e.plan->start[slot + 1] - first;
  }
  const char* codes = e.w + (size_t)expert * e.w_stride;
  const Strip w{codes + (size_t)block * e.steps * MX4_PANEL + half * 1024, codes + e.scales_at + (size_t)block * ((e.steps + 3) >> 2) * 1024, e.steps};
  Tokens x{e.x, e.x_scales, e.K, e.steps, e.T};
  const int pieces = e.T * e.K / 8;
  StagedTokens staged;
  if constexpr (SRC == LDS_MX4) staged.load(e.x, pieces);

  for (int t0 = 0; t0 < (PASSES ? n : 1); t0 += 16 * NT) {
  int row[NT], row_p[NP];
  bool on[NT], on_p[NP];
#pragma unroll
  for (int i = 0; i < NT; i++) {
    const int at = t0 + 16 * i + c;
    on[i] = at < n;
    row[i] = !on[i] || WHO == MOE_ONE ? 0 : WHO == MOE ? e.plan->list[first + at] / e.k : at;
  }
  row_p[0] = row[0];
  on_p[0] = on[0];
  const int groups = min((n - t0 + 15) >> 4, NT);
  f32x4 acc[RG][NT];
#pragma unroll
  for (int g = 0; g < RG; g++)
#pragma unroll
    for (int i = 0; i < NT; i++) acc[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  Unit<SRC, RG, U, NP, RG == 4 ? 1 : 2> now, next;
  int s = wave * U;
  if (s < e.steps) now.load(w, x, row_p, on_p, s, lane);
  if constexpr (SRC == LDS_MX4) {
    static_assert(W == WAVES, "staged by all work items");
    x.p = staged_lds;
    x.scales = staged_lds + e.T * e.K / 2;
    staged.store(staged_lds, staged_lds + e.T * e.K / 2, pieces, e.K, e.T);
    __syncthreads();
  }
  for (; s < e.steps; s += W * U) {
    const bool more = s + W * U < e.steps;
    if (more) next.load(w, x, row_p, on_p, s + W * U, lane);
    now.ops(x, row, on, groups, s, e.steps, q, acc);
    if (more) now = next;
  }
  settle(acc);
  for (int i = 0; i < groups; i++) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NT; j++)
      if (j == i) {
#pragma unroll
        for (int g = 0; g < RG; g++)
#pragma unroll
          for (int v = 0; v < 4; v++) red[(wave * 16 * RG + 16 * g + 4 * q + v) * RED + c] = acc[g][j][v];
      }
    __syncthreads();
    // neighbouring lanes have the features of a token
    for (int o = tid; o < FEATS * 16; o += 64 * W) {
      const int f = o % FEATS, tok = o / FEATS, at = t0 + 16 * i + tok;
      const int r = RG == 4 ? ((f >> 2) & 1) * 16 + 4 * (f >> 3) + (f & 3) : f;
      float gate = 0.f, up = 0.f;
#pragma unroll
      for (int k = 0; k < W; k++) {
        gate += red[(k * 16 * RG + r) * RED + tok];
        up += red[(k * 16 * RG + 8 * RG + r) * RED + tok];
      }
      const float h = gate_act(e.gate, gate) * up;
      const int dest = first + at;                                 // (H's rows are in the plan's order: an expert's one after the other)
      if constexpr (MX4) {
        uint32_t top = magnitude(h);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
        const uint32_t code = mx4_scale_code(top);
        uint32_t word = (__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, h, 0.f, mx4_scale(code), 0) & 15u) << (4 * (f & 7));
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) word |= (uint32_t)__shfl_xor((int)word, d, 64);
        if (at < n && (f & 7) == 0) *reinterpret_cast<uint32_t*>(e.h + mx4_code_at(dest, block, e.h_steps) + (f >> 1)) = word;
        if (at < n && f == 0) e.h_scales[mx4_scale_at(dest, block, e.h_steps)] = (char)code;
      } else {
        const int feat = 32 * block + (RG == 4 ? f : 8 * (f >> 2) + 4 * half + (f & 3));
        // two neighbours' first parts go out from the even lane, their rests from the odd one
        const uint32_t mine = two_parts(h), other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mine, quad_perm(1, 0, 3, 2), 0xF, 0xF, true);
        const uint32_t two = f & 1 ? other >> 16 | (mine & 0xFFFF0000u) : (mine & 0xFFFFu) | other << 16;
        if (at < n) *reinterpret_cast<uint32_t*>(e.h + parts_at(dest, block, (feat >> 3) & 3, e.F) + 1024 * (f & 1) + 2 * (feat & 6)) = two;
      }
    }
  }
  }   // passes
}

// ------------------------------------------------------------------------------------------------ a product by itself
struct RowsArgs {
  const char* w; const char* w_scales; int steps, K, N, T;
  const char* x; const char* x_scales; int x_steps;
  uint16_t* out;
};
// Few channels and a long reduction want narrow strips, for there to be workgroups, a short one wide strips, for eight waves to have loads (mx4_few_groups).  1 token of 2048 x
// 8192 3.6 us (8.9 MB: the launch and one way through memory, LDS and back); down of 16 tokens, 16384 x 4096, 8.3 us (4.3 TB/s: two rounds of loads a wave).
template <int RG, int NT, int SRC>
__global__ void __launch_bounds__(THREADS, NT == 1 && (RG > 1 || SRC == LDS_MX4) ? 4 : 2) few_rows_kernel(RowsArgs e) {
  constexpr int U = 8 / RG;
  __shared__ __attribute__((aligned(16))) float red[WAVES * 16 * RG * RED];
  extern __shared__ __attribute__((aligned(16))) char staged_lds[];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int strip = (int)run_of(blockIdx.x, gridDim.x), block = strip / (4 / RG), g0 = strip % (4 / RG) * RG;
  const Strip w{e.w + (size_t)block * e.steps * MX4_PANEL + g0 * 1024, e.w_scales + (size_t)block * ((e.steps + 3) >> 2) * 1024 + g0 * 256, e.steps};
  Tokens x{e.x, e.x_scales, e.K, e.x_steps, e.T};
  const int pieces = e.T * e.K / 8;
  StagedTokens staged;
  if constexpr (SRC == LDS_MX4) staged.load(e.x, pieces);
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
  Unit<SRC, RG, U, NT> now, next;
  int s = wave * U;
  if (s < e.steps) now.load(w, x, row, on, s, lane);
  if constexpr (SRC == LDS_MX4) {
    x.p = staged_lds;
    x.scales = staged_lds + e.T * e.K / 2;
    staged.store(staged_lds, staged_lds + e.T * e.K / 2, pieces, e.K, e.T);
    __syncthreads();
  }
  for (; s < e.steps; s += WAVES * U) {
    const bool more = s + WAVES * U < e.steps;
    if (more) next.load(w, x, row, on, s + WAVES * U, lane);
    now.ops(x, row, on, NT, s, e.steps, q, acc);
    if (more) now = next;
  }
  settle(acc);
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
  const char* h; const char* h_scales; int h_steps;   // rows in the order of the plan
  const MoePlan* plan;
  float* parts;                        // [splits][T][D]
  uint16_t* out;
};
constexpr int down_pitch(int groups) { return 16 * groups + 4; }   // of a token's channels of a strip
constexpr int down_lds(int T, int groups) { return WAVES * T * down_pitch(groups) * 4; }

// A wave takes units of 8 KiB of any expert's weights; an op's 16 tokens go to their rows of the wave's sums with their shares (a read and a write of LDS, no atomics: the wave has
// its own), so that neither a row of Y for each expert nor its sum over the experts goes through memory.  The waves' sums are added up in the waves' order.
// A strip reads the activations of all its experts' tokens, 4 bytes a value in parts, from L2, and a CU takes in weights and activations at 39 KB a us together: with 16 channels a
// strip, 64 tokens of 64 experts of 4096 x 2048, each meant as many bytes, 215 us; 32 channels (RG 2) 175, 64 (RG 4) 160 (moe_down_groups).
// grid (D / (16 RG), splits).  Where the strips are few, several workgroups share one's experts, and a second kernel adds up (tickets instead, with sums past the L2s: 21 -> 24.8 us
// for 1 token of 2048 x 1024).
template <bool MX4, int NT, int RG>
__global__ void __launch_bounds__(THREADS, 2) moe_down_kernel(DownArgs e) {
  constexpr int U = 8 / RG, SUM = down_pitch(RG), SRC = MX4 ? OPERAND_MX4 : OPERAND_PARTS;
  extern __shared__ __attribute__((aligned(16))) float sums[];   // [wave][token][SUM]
  __shared__ int active[MOE_E], start[MOE_E + 1], list[MOE_PAIRS];
  __shared__ float share[MOE_PAIRS];
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned id = run_of(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y), splits = gridDim.y;
  const int strip = (int)(id / splits), split = (int)(id - strip * splits), block = strip / (4 / RG), g0 = strip % (4 / RG) * RG, stride = WAVES * (int)splits;
  for (int i = tid; i < WAVES * e.T * SUM; i += THREADS) sums[i] = 0.f;
  const int n_active = e.plan->n_active;
  for (int i = tid; i < e.T * e.k; i += THREADS) {
    list[i] = e.plan->list[i];
    share[i] = e.plan->share[i];
  }
  if (tid < n_active) active[tid] = e.plan->expert[tid];
  if (tid <= n_active) start[tid] = e.plan->start[tid];
  __syncthreads();
  float* mine = sums + wave * e.T * SUM;
  const Tokens x{e.h, e.h_scales, e.F, e.h_steps, 0};
  const int units = (e.steps + U - 1) / U, total = n_active * units;   // units of U steps, the experts' one after the other, dealt out to the waves
  auto strip_of = [&](int i) {
    const char* codes = e.w + (size_t)uniform(active[i / units]) * e.w_stride;
    return Strip{codes + (size_t)block * e.steps * MX4_PANEL + g0 * 1024, codes + e.scales_at + (size_t)block * ((e.steps + 3) >> 2) * 1024 + g0 * 256, e.steps};
  };
  using Piece = Unit<SRC, RG, U, 1>;
  struct Rows { int row[1]; bool on[1]; };
  // (lanes without a token read the expert's first: a column of an op is a token's alone, and theirs are not used)
  auto load = [&](Piece& u, Rows& rows, int i) {
    const int first = start[i / units];
    rows.on[0] = first + c < start[i / units + 1];
    rows.row[0] = first + (rows.on[0] ? c : 0);
    u.load(strip_of(i), x, rows.row, rows.on, i % units * U, lane);
  };
  auto work = [&](const Piece& u, const Rows& rows, int i) {
    const int first = uniform(start[i / units]), n = uniform(start[i / units + 1]) - first, groups = (n + 15) >> 4;
    int row[NT];
    bool on[NT];
    row[0] = rows.row[0];
    on[0] = rows.on[0];
#pragma unroll
    for (int g = 1; g < NT; g++) {
      on[g] = 16 * g + c < n;
      row[g] = first + (on[g] ? 16 * g + c : 0);
    }
    f32x4 acc[RG][NT];
#pragma unroll
    for (int r = 0; r < RG; r++)
#pragma unroll
      for (int g = 0; g < NT; g++) acc[r][g] = f32x4{0.f, 0.f, 0.f, 0.f};
    u.ops(x, row, on, groups, i % units * U, e.steps, q, acc);
    settle(acc);
#pragma unroll
    for (int g = 0; g < NT; g++)
      if (on[g]) {                                         // (a token chooses an expert once: no two lanes of a quarter have the same one)
        const float p = share[row[g]];
        f32x4* to = reinterpret_cast<f32x4*>(mine + list[row[g]] / e.k * SUM + 4 * q);
#pragma unroll
        for (int r = 0; r < RG; r++) {
          f32x4 y = to[4 * r];
#pragma unroll
          for (int v = 0; v < 4; v++) y[v] += p * acc[r][g][v];
          to[4 * r] = y;
        }
      }
  };
  // (two units in turn, and the last apart: where paths with and without loads under way meet, the compiler waits for all of them)
  int i = split * WAVES + wave;
  if (i < total) {
    Piece one, two;
    Rows rows1, rows2;
    load(one, rows1, i);
    for (;;) {
      if (i + stride >= total) {
        work(one, rows1, i);
        break;
      }
      load(two, rows2, i + stride);
      work(one, rows1, i);
      i += stride;
      if (i + stride >= total) {
        work(two, rows2, i);
        break;
      }
      load(one, rows1, i + stride);
      work(two, rows2, i);
      i += stride;
    }
  }
  __syncthreads();
  for (int o = tid; o < 16 * RG * e.T; o += THREADS) {
    const int r = o % (16 * RG), t = o / (16 * RG);
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < WAVES; k++) y += sums[(k * e.T + t) * SUM + r];
    const size_t at = (size_t)t * e.D + 64 * block + channel_of(g0 + r / 16, r % 16);
    if (splits == 1) e.out[at] = (uint16_t)pack_bf16x2(y, 0.f);
    else e.parts[(size_t)split * e.T * e.D + at] = y;
  }
}

// ------------------------------------------------------------------------------------------------ router
// In 64 bits on the matrix ops too: op j of a step of 32 d takes d 8 q + j from lane quarter q.  A: 16 tokens, B: 16 experts (Wr in the order of the bf16 operands).
// grid (parts of 128 d, groups of 16 tokens); parts [part][T][E].  steps > 0: the tokens go out as mx4 too, in the operand form.
typedef double f64x4 __attribute__((ext_vector_type(4)));
constexpr int ROUTE_D = 128, ROUTE_STEPS = ROUTE_D / 32;
__device__ __forceinline__ double bf16_of(const u32x4& w, int j) { return (double)(j % 2 ? bf16_hi_to_f32(w[j / 2]) : bf16_lo_to_f32(w[j / 2])); }
__global__ void __launch_bounds__(256) moe_router_kernel(const uint16_t* __restrict__ X, const char* __restrict__ Wr, int T, int D, int E, double* __restrict__ parts, int steps,
                                                         char* __restrict__ codes, char* __restrict__ scales) {
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int s0 = blockIdx.x * ROUTE_STEPS, all = D / 32, n = min(all - s0, ROUTE_STEPS), t0 = 16 * blockIdx.y;
  const int groups = 4 * (E / 64) + (E % 64 > 32 ? 4 : E % 64 ? 2 : 0);    // of 16 rows that have an expert
  u32x4 x[ROUTE_STEPS];
#pragma unroll
  for (int s = 0; s < ROUTE_STEPS; s++)
    x[s] = t0 + c < T && s < n ? *reinterpret_cast<const u32x4*>(X + (size_t)(t0 + c) * D + 32 * (s0 + s) + 8 * q) : u32x4{0u, 0u, 0u, 0u};
  for (int g = wave; g < groups; g += 4) {
    const char* w = Wr + ((size_t)(g >> 2) * all + s0) * MX4_PANEL + (g & 3) * 1024 + lane * 16;
    u32x4 y[ROUTE_STEPS];
#pragma unroll
    for (int s = 0; s < ROUTE_STEPS; s++) y[s] = s < n ? *reinterpret_cast<const u32x4*>(w + (size_t)s * MX4_PANEL) : u32x4{0u, 0u, 0u, 0u};
    f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int s = 0; s < ROUTE_STEPS; s++)
#pragma unroll
      for (int j = 0; j < 8; j++) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(bf16_of(x[s], j), bf16_of(y[s], j), acc, 0, 0, 0);
    const int e = 64 * (g >> 2) + channel_of(g & 3, c);                    // result v of a lane: token 4 v + q, column c
#pragma unroll
    for (int v = 0; v < 4; v++) {
      const int t = t0 + 4 * v + q;
      if (t < T && e < E) parts[((size_t)blockIdx.x * T + t) * E + e] = acc[v];
    }
  }
  const int t = t0 + (tid >> 4), d = 32 * s0 + 8 * (tid & 15), p = tid & 3;    // four lanes have a block of 32
  if (steps > 0 && t < T && d < D) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(X + (size_t)t * D + d);
    const uint32_t code = mx4_scale_code(quad_max(mx4_top8(w)));
    *reinterpret_cast<uint32_t*>(codes + mx4_code_at(t, d >> 5, steps) + 4 * p) = mx4_codes8(w, mx4_scale(code));
    if (p == 0) scales[mx4_scale_at(t, d >> 5, steps)] = (char)code;
  }
}

// A workgroup a token; the one that comes last makes the plan (a launch less than a kernel for it; in every workgroup of `up` the lists took longer than this does).
__global__ void __launch_bounds__(THREADS) moe_pick_kernel(const double* __restrict__ parts, int n_parts, int T, int E, int k, int renormalise, int* __restrict__ picks,
                                                       float* __restrict__ shares, MoePlan* __restrict__ plan) {
  __shared__ Choice c;
  __shared__ int count[MOE_E], cursor[MOE_E], come;
  const int t = blockIdx.x, tid = threadIdx.x;
  moe_choose(parts + (size_t)t * E, (size_t)T * E, n_parts, E, k, renormalise != 0, c);
  if (tid < k) {
    picks[t * k + tid] = c.which[tid];
    shares[t * k + tid] = c.share[tid];
    put(&plan->picks[t * k + tid], c.which[tid]);
    put(&plan->shares[t * k + tid], c.share[tid]);
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (tid == 0) come = __hip_atomic_fetch_add(&plan->ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (tid < MOE_E) count[tid] = 0;
  __syncthreads();
  if (come != T - 1) return;

  const int pairs = T * k;
  int mine[MOE_PAIRS / THREADS];
  float p[MOE_PAIRS / THREADS];
#pragma unroll
  for (int j = 0; j < MOE_PAIRS / THREADS; j++) {
    const int i = THREADS * j + tid;
    if (i < pairs) {
      mine[j] = get(&plan->picks[i]);
      p[j] = get(&plan->shares[i]);
    }
  }
#pragma unroll
  for (int j = 0; j < MOE_PAIRS / THREADS; j++)
    if (THREADS * j + tid < pairs) atomicAdd(&count[mine[j]], 1);
  __syncthreads();
  if (tid < 64) {                                              // four experts a lane: pairs before them below, chosen ones above
    int n[4], all = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      n[i] = count[4 * tid + i];
      all += n[i] | (n[i] > 0 ? 1 << 16 : 0);
    }
    int upto = all;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(upto, d, 64);
      if (tid >= d) upto += y;
    }
    int run = upto - all;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      cursor[4 * tid + i] = run & 0xFFFF;
      if (n[i] > 0) {
        plan->expert[run >> 16] = 4 * tid + i;
        plan->start[run >> 16] = run & 0xFFFF;
      }
      run += n[i] | (n[i] > 0 ? 1 << 16 : 0);
    }
    if (tid == 63) {
      plan->start[run >> 16] = run & 0xFFFF;
      plan->n_active = run >> 16;
      put(&plan->ticket, 0);
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < MOE_PAIRS / THREADS; j++)
    if (THREADS * j + tid < pairs) {
      const int at = atomicAdd(&cursor[mine[j]], 1);
      plan->list[at] = THREADS * j + tid;
      plan->share[at] = p[j];
    }
}

int staged_bytes(int T, int K) { return T * K / 2 + T * K / 32; }

template <int SRC, int NT, int WHO, int RG, int W, bool PASSES = false>
int launch_up_one(const UpArgs& a, int slots, hipStream_t s) {
  auto kern = few_up_kernel<SRC, NT, WHO, RG, W, PASSES>;
  int lds = 0;
  if constexpr (SRC == LDS_MX4) {
    static std::atomic<bool> configured[MAX_DEVICES] = {};
    if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), staged_bytes(1, MX4_FUSED_VALUES), configured)) return rc;
    lds = staged_bytes(a.T, a.K);
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.F / (8 * RG)), (unsigned)slots), dim3(64 * W), lds, s, a);
  return (int)hipGetLastError();
}
template <int SRC, int WHO, bool PASSES = false>
int launch_up_tokens(const UpArgs& a, int slots, hipStream_t s) {
  if constexpr (SRC == OPERAND_MX4 && WHO == MOE)
    if (few_up_waves(a.F / 32 * slots, a.steps) == 4) return launch_up_one<SRC, 1, WHO, 4, 4, PASSES>(a, slots, s);
  if constexpr (SRC == ROWS_BF16 && !PASSES)
    if (few_up_halves(a.F / 32 * slots)) return launch_up_one<SRC, 1, WHO, 2, 8>(a, slots, s);
  return launch_up_one<SRC, 1, WHO, 4, 8, PASSES>(a, slots, s);
}
template <int SRC>
int launch_moe_up(const UpArgs& a, int slots, hipStream_t s) {
  if (a.T == 1) return launch_up_tokens<SRC, MOE_ONE>(a, slots, s);
  if (a.T <= 16) return launch_up_tokens<SRC, MOE>(a, slots, s);
  return moe_crowded(a.T, a.k, a.E) ? launch_up_one<SRC, 4, MOE, 4, 8>(a, slots, s) : launch_up_tokens<SRC, MOE, true>(a, slots, s);
}
template <bool MX4, int NT, int RG>
int launch_down(const DownArgs& a, int splits, hipStream_t s) {
  auto kern = moe_down_kernel<MX4, NT, RG>;
  static std::atomic<bool> configured[MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), down_lds(MOE_TOKENS, RG), configured)) return rc;
  hipLaunchKernelGGL(kern, dim3((unsigned)(a.D / (16 * RG)), (unsigned)splits), dim3(THREADS), down_lds(a.T, RG), s, a);
  return (int)hipGetLastError();
}
template <int NT>
int launch_down_groups(const DownArgs& a, int groups, int splits, hipStream_t s) {
  switch (groups) {
    case 4: return launch_down<false, NT, 4>(a, splits, s);
    case 2: return launch_down<false, NT, 2>(a, splits, s);
    default: return launch_down<false, NT, 1>(a, splits, s);
  }
}
template <int RG, int SRC, int NT>
int launch_rows_tokens(const RowsArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(RG == 1 ? (a.N + 31) / 32 * 2 : (a.N + 16 * RG - 1) / (16 * RG)));   // (two groups of 16 share 32 channels)
  auto kern = few_rows_kernel<RG, NT, SRC>;
  int lds = 0;
  if constexpr (SRC == LDS_MX4) {
    static std::atomic<bool> configured[MAX_DEVICES] = {};
    if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), staged_bytes(1, MX4_FUSED_VALUES), configured)) return rc;
    lds = staged_bytes(a.T, a.K);
  }
  hipLaunchKernelGGL(kern, grid, dim3(THREADS), lds, s, a);
  return (int)hipGetLastError();
}
template <int RG>
int launch_rows(const RowsArgs& a, bool staged, hipStream_t s) {
  if (staged) return launch_rows_tokens<RG, LDS_MX4, 1>(a, s);
  if constexpr (RG == 1)
    if (a.T > 16) return launch_rows_tokens<RG, OPERAND_MX4, 2>(a, s);
  return launch_rows_tokens<RG, OPERAND_MX4, 1>(a, s);
}
}  // namespace

size_t moe_plan_size() { return sizeof(MoePlan); }
size_t moe_parts_size(int T, int D, int E) { return (size_t)((D + ROUTE_D - 1) / ROUTE_D) * T * E * sizeof(double); }

int launch_moe_route(const MoeCall& m, const Mx4Operand* x, hipStream_t s) {
  const int n = (m.D + ROUTE_D - 1) / ROUTE_D;
  hipLaunchKernelGGL(moe_router_kernel, dim3((unsigned)n, (unsigned)((m.T + 15) / 16)), dim3(256), 0, s, static_cast<const uint16_t*>(m.X), static_cast<const char*>(m.Wr), m.T, m.D,
                     m.E, static_cast<double*>(m.logits), x ? x->steps : 0, x ? const_cast<char*>(x->codes) : nullptr, x ? const_cast<char*>(x->scales) : nullptr);
  if (m.T > 1)
    hipLaunchKernelGGL(moe_pick_kernel, dim3((unsigned)m.T), dim3(THREADS), 0, s, static_cast<const double*>(m.logits), n, m.T, m.E, m.k, (int)m.renormalise, m.picks, m.shares,
                       static_cast<MoePlan*>(m.plan));
  return (int)hipGetLastError();
}

int launch_moe_experts(const MoeCall& m, const MoeWeights& w, const Mx4Operand* x, float c1, float c3, hipStream_t s) {
  const int T = m.T, D = m.D, F = m.F, E = m.E, k = m.k;
  UpArgs up{};
  up.w = static_cast<const char*>(w.up); up.w_stride = w.up_stride; up.scales_at = w.up_scales;
  up.K = D; up.F = F; up.T = T; up.steps = w.mx4 ? mx4_steps(D) : D / 32; up.gate = Gate{c1, c3};
  up.x = w.mx4 ? x->codes : static_cast<const char*>(m.X); up.x_scales = w.mx4 ? x->scales : nullptr;
  const Mx4Operand h = mx4_operand(m.H, m.h_rows, F);
  up.h = const_cast<char*>(w.mx4 ? h.codes : static_cast<const char*>(m.H));
  up.h_scales = const_cast<char*>(h.scales);
  up.h_steps = h.steps;
  up.plan = up.plan_out = static_cast<MoePlan*>(m.plan); up.k = k;
  up.logits = static_cast<const double*>(m.logits); up.n_parts = (D + ROUTE_D - 1) / ROUTE_D; up.E = E; up.renormalise = m.renormalise;
  up.picks = m.picks; up.shares = m.shares;
  const int slots = T * k < E ? T * k : E;
  if (const int rc = w.mx4 ? launch_moe_up<OPERAND_MX4>(up, slots, s) : launch_moe_up<ROWS_BF16>(up, slots, s)) return rc;
  DownArgs d{};
  d.w = static_cast<const char*>(w.down); d.w_stride = w.down_stride; d.scales_at = w.down_scales;
  d.steps = w.mx4 ? mx4_steps(F) : F / 32; d.F = F; d.D = D; d.T = T; d.k = k;
  d.h = up.h; d.h_scales = h.scales; d.h_steps = h.steps;
  d.plan = up.plan; d.out = static_cast<uint16_t*>(m.Y);
  d.parts = static_cast<float*>(m.parts);
  const int groups = w.mx4 ? 1 : moe_down_groups(T * k, D, F), splits = moe_down_splits(D / (16 * groups), slots * ((d.steps * groups + 7) / 8));
  const int rc = T <= 16 ? (w.mx4 ? launch_down<true, 1, 1>(d, splits, s) : launch_down_groups<1>(d, groups, splits, s))
                         : (w.mx4 ? launch_down<true, 4, 1>(d, splits, s) : launch_down_groups<4>(d, groups, splits, s));
  if (rc || splits == 1) return rc;
  hipLaunchKernelGGL((edge_sum_kernel<false>), dim3((unsigned)((D / 4 * T + 255) / 256)), dim3(256), 0, s, static_cast<const uint32_t*>(m.parts), splits, D, T, I8Scales{},
                     static_cast<uint16_t*>(m.Y));
  return (int)hipGetLastError();
}

// X: bf16 rows; x: instead of them
int launch_few_mx4_up(const Mx4Operand& w, const void* X, const Mx4Operand* x, int T, int D, int F, float c1, float c3, const Mx4Operand& h, hipStream_t s) {
  UpArgs up{};
  up.w = w.codes; up.scales_at = (size_t)(w.scales - w.codes);
  up.K = D; up.F = F; up.T = T; up.steps = w.steps; up.gate = Gate{c1, c3};
  up.x = x ? x->codes : static_cast<const char*>(X); up.x_scales = x ? x->scales : nullptr;
  up.h = const_cast<char*>(h.codes); up.h_scales = const_cast<char*>(h.scales); up.h_steps = h.steps;
  if (!x) return launch_up_tokens<LDS_MX4, ALL_TOKENS>(up, 1, s);
  return launch_up_tokens<OPERAND_MX4, ALL_TOKENS>(up, 1, s);
}
int launch_few_mx4_rows(const Mx4Operand& w, int K, int N, const void* X, const Mx4Operand* x, int T, void* Y, hipStream_t s) {
  RowsArgs a{w.codes, w.scales, w.steps, K, N, T, static_cast<const char*>(X), nullptr, 0, static_cast<uint16_t*>(Y)};
  if (x) { a.x = x->codes; a.x_scales = x->scales; a.x_steps = x->steps; }
  switch (T > 16 ? 1 : mx4_few_groups(N, w.steps)) {
    case 4: return launch_rows<4>(a, !x, s);
    case 2: return launch_rows<2>(a, !x, s);
    default: return launch_rows<1>(a, !x, s);
  }
}

}  // namespace ffn24
