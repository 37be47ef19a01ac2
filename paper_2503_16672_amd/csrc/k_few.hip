// Products for few tokens (up to 64): bound by the weights, which pass through once.
//
// A wave takes a strip of output channels and every n-th step of the reduction, straight from memory into registers as the A operand of the 16 x 16 matrix ops (rows:
// channels, columns: tokens, 16 at a time); the waves of a workgroup add their results up through LDS in a fixed order.  Compute is a tenth of the time the bytes take.
//
// bf16: the weights are k-major.  Lane (c, q) of a wave loads 16 bytes, 8 neighbouring channels, of rows k 8 q .. 8 q + 7 of a step of 32 k; transposed in
// registers (byte permutes), channel t of every lane's eight is the row c of matrix op t.  16 lanes are 256 bytes of a row: 128 channels, or 64 gate channels and the
// 64 up channels of the same numbers.
// 8-bit integers: the panel form (gemm_core.hpp) has the 16 bytes of k that a lane of the 16 x 16 x 64 op takes next to each other: 16 rows are a contiguous KiB.
#include "launch_block.hpp"
#include "launch_edge.hpp"

namespace ffn24 {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int FEW_TOKENS = 64;
constexpr int RED = 17;                     // pitch of the sums' image: [channel][16 tokens]

__device__ __forceinline__ uint16_t to_bf16(float x) { return (uint16_t)pack_bf16x2(x, 0.f); }

// ------------------------------------------------------------------------------------------------ bf16
constexpr int few_waves(int nt) { return nt == 1 ? 16 : 8; }

// grid: (strips, splits).  GATED: H = bf16(a(G) U), cols = F, a row of W 2 F; else out [T][cols].  splits > 1: the sums of split y go to parts [y][T][row].
template <bool GATED, int NT>
__global__ void __launch_bounds__(64 * few_waves(NT)) few_bf16_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, int T, int K, int cols, Gate gate,
                                                                      uint16_t* __restrict__ out, float* __restrict__ parts) {
  constexpr int KS = few_waves(NT), STEPS = 2;
  extern __shared__ __attribute__((aligned(16))) float red[];   // [KS][128][RED]
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = GATED ? 2 * cols : cols;
  const int n0 = blockIdx.x * (GATED ? 64 : 128);
  // the lane's piece of a row; beyond the last column (a strip of 64) the first one again, whose results are not stored
  const int n = GATED ? (c < 8 ? n0 + 8 * c : cols + n0 + 8 * (c - 8)) : (n0 + 8 * c < cols ? n0 + 8 * c : n0);
  const uint16_t* w = W + (size_t)(8 * q) * row + n;
  const uint16_t* x[NT];
#pragma unroll
  for (int i = 0; i < NT; i++) x[i] = X + (size_t)min(16 * i + c, T - 1) * K + 8 * q;
  f32x4 acc[8][NT];
#pragma unroll
  for (int t = 0; t < 8; t++)
#pragma unroll
    for (int i = 0; i < NT; i++) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int total = K / 32, stride = KS * gridDim.y;
  for (int s = blockIdx.y * KS + wave; s < total; s += STEPS * stride) {
    u32x4 a[STEPS][8];
    bf16x8 b[STEPS][NT];
#pragma unroll
    for (int j = 0; j < STEPS; j++) {
      const int at = s + j * stride < total ? s + j * stride : s;
      const uint16_t* p = w + (size_t)at * 32 * row;
#pragma unroll
      for (int r = 0; r < 8; r++) a[j][r] = ld_stream(reinterpret_cast<const u32x4*>(p + (size_t)r * row));
#pragma unroll
      for (int i = 0; i < NT; i++) b[j][i] = *reinterpret_cast<const bf16x8*>(x[i] + at * 32);
    }
#pragma unroll
    for (int j = 0; j < STEPS; j++) {
      if (j > 0 && s + j * stride >= total) break;
#pragma unroll
      for (int t = 0; t < 8; t++) {
        u32x4 f;
#pragma unroll
        for (int d = 0; d < 4; d++) f[d] = __builtin_amdgcn_perm(a[j][2 * d + 1][t / 2], a[j][2 * d][t / 2], t % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int i = 0; i < NT; i++) acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), b[j][i], acc[t][i], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NT; i++) {
    const int tokens = min(T - 16 * i, 16);
    if (i > 0) __syncthreads();
    if (c < tokens) {
#pragma unroll
      for (int t = 0; t < 8; t++)
#pragma unroll
        for (int v = 0; v < 4; v++) red[(wave * 128 + 8 * (4 * q + v) + t) * RED + c] = acc[t][i][v];   // row 4 q + v of op t: that lane's channel t
    }
    __syncthreads();
    auto sum = [&](int ch, int tok) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < KS; k++) s += red[(k * 128 + ch) * RED + tok];
      return s;
    };
    if (GATED && !parts) {
      for (int o = tid; o < 64 * tokens; o += 64 * KS) {
        const int f = o & 63, tok = o >> 6;
        out[(size_t)(16 * i + tok) * cols + n0 + f] = to_bf16(gate_act(gate, sum(f, tok)) * sum(64 + f, tok));
      }
    } else {
      for (int o = tid; o < 128 * tokens; o += 64 * KS) {
        const int f = o & 127, tok = o >> 7, col = GATED ? (f < 64 ? n0 + f : cols + n0 + f - 64) : n0 + f;
        if (col >= row) continue;
        const float s = sum(f, tok);
        if (parts) parts[((size_t)blockIdx.y * T + 16 * i + tok) * row + col] = s;
        else out[(size_t)(16 * i + tok) * row + col] = to_bf16(s);
      }
    }
  }
}

// The sums of `splits` parts [T][row], four columns a work item; GATED: of both halves, and the gate.
template <bool GATED>
__global__ void __launch_bounds__(256) few_sum_kernel(const float* __restrict__ parts, int splits, int T, int cols, Gate gate, uint16_t* __restrict__ out) {
  const int row = GATED ? 2 * cols : cols;
  const size_t n = (size_t)T * row;
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= T * (cols / 4)) return;
  const int t = i / (cols / 4), col = 4 * (i - t * (cols / 4));
  const float* p = parts + (size_t)t * row + col;
  f32x4 a = *reinterpret_cast<const f32x4*>(p), u = GATED ? *reinterpret_cast<const f32x4*>(p + cols) : a;
  for (int s = 1; s < splits; s++) {
    a += *reinterpret_cast<const f32x4*>(p + s * n);
    if (GATED) u += *reinterpret_cast<const f32x4*>(p + s * n + cols);
  }
  if constexpr (GATED) {
#pragma unroll
    for (int j = 0; j < 4; j++) a[j] = gate_act(gate, a[j]) * u[j];
  }
  *reinterpret_cast<u32x2*>(out + (size_t)t * cols + col) = u32x2{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3])};
}

// Workgroups stream about 60 GB/s each, so fewer than 128 strips are split along the reduction until there are that many, each wave with a step at least.
template <bool GATED>
int few_splits(int T, int K, int cols) {
  const int strips = GATED ? cols / 64 : (cols + 127) / 128, waves = few_waves(T <= 16 ? 1 : 2);
  int s = 1;
  while (s < 16 && strips * s < 128 && K / 32 >= 4 * s * waves) s *= 2;
  return s;
}

template <bool GATED, int NT>
int launch_few_bf16_tokens(const void* X, const void* W, int T, int K, int cols, Gate gate, int splits, void* out, float* parts, hipStream_t s) {
  constexpr int KS = few_waves(NT), LDS = KS * 128 * RED * 4;
  auto kern = few_bf16_kernel<GATED, NT>;
  static std::atomic<bool> configured[MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), LDS, configured)) return rc;
  hipLaunchKernelGGL(kern, dim3((unsigned)(GATED ? cols / 64 : (cols + 127) / 128), (unsigned)splits), dim3(64 * KS), LDS, s, static_cast<const uint16_t*>(X),
                     static_cast<const uint16_t*>(W), T, K, cols, gate, static_cast<uint16_t*>(out), splits > 1 ? parts : nullptr);
  if (splits > 1)
    hipLaunchKernelGGL((few_sum_kernel<GATED>), dim3((unsigned)((T * (cols / 4) + 255) / 256)), dim3(256), 0, s, parts, splits, T, cols, gate, static_cast<uint16_t*>(out));
  return (int)hipGetLastError();
}
template <bool GATED>
int launch_few_bf16(const void* X, const void* W, int T, int K, int cols, Gate gate, void* out, float* parts, hipStream_t s) {
  const int splits = few_splits<GATED>(T, K, cols);
  if (T <= 16) return launch_few_bf16_tokens<GATED, 1>(X, W, T, K, cols, gate, splits, out, parts, s);
  if (T <= 32) return launch_few_bf16_tokens<GATED, 2>(X, W, T, K, cols, gate, splits, out, parts, s);
  return launch_few_bf16_tokens<GATED, 4>(X, W, T, K, cols, gate, splits, out, parts, s);
}
}  // namespace

bool few_tokens(int T) { return T <= FEW_TOKENS; }

size_t few_gated_scratch(int T, int D, int F) {
  size_t most = 0;
  for (int t : {16, 64}) {                    // (the splits depend on T through this only)
    const int n = T < t ? T : t;
    const size_t up = (size_t)few_splits<true>(t, D, F) * n * 2 * F, down = (size_t)few_splits<false>(t, F, D) * n * D;
    most = up > most ? up : most;
    most = down > most ? down : most;
  }
  return 4 * most;
}
int launch_few_gated_up(const void* X, const void* Wgu, int T, int D, int F, float c1, float c3, void* H, float* parts, hipStream_t s) {
  return launch_few_bf16<true>(X, Wgu, T, D, F, Gate{c1, c3}, H, parts, s);
}
int launch_few_gated_down(const void* H, const void* Wd, int T, int D, int F, void* Y, float* parts, hipStream_t s) {
  return launch_few_bf16<false>(H, Wd, T, F, D, Gate{}, Y, parts, s);
}

}  // namespace ffn24
