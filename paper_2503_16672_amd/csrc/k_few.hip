// Products for few tokens (up to 64): bound by the weights, which pass through once.
//
// A wave takes a strip of output channels and every n-th step of the reduction, straight from memory into registers as the A operand of the 16 x 16 matrix ops (rows:
// channels, columns: tokens, 16 at a time); the waves of a workgroup add their results up through LDS in a fixed order.  Compute is a tenth of the time the bytes take.
//
// bf16: the weights are k-major.  Lane (c, q) of a wave loads 16 bytes, 8 neighbouring channels, of rows k 8 q .. 8 q + 7 of a step of 32 k; transposed in
// registers (byte permutes), channel t of every lane's eight is the row c of matrix op t.  16 lanes are 256 bytes of a row: 128 channels, or 64 gate channels and the
// 64 up channels of the same numbers.
// Measured, one token at 4096 x 16384: gate and up 48 us (268 MB, 5.6 TB/s), down 23.5 (134 MB, 5.7) and 4.6 for the sums of its 8 splits.
// 8-bit integers: the panel form (gemm_core.hpp) has the 16 bytes of k that a lane of the 16 x 16 x 64 op takes next to each other: 16 rows are a contiguous KiB.
// 16 tokens at 4096 x 16384: 22.4 us (134 MB, 6.0 TB/s), 16.5 (67 MB, 4.1), and 4.6 and 5.1 for the two quantisations.
#include "launch_block.hpp"
#include "launch_edge.hpp"
#include "i8_codes.hpp"

namespace ffn24 {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int I8_FUSE_BYTES = 17 * 1024;   // of codes that a workgroup makes itself
constexpr int RED = 17;                     // pitch of the sums' image: [channel][16 tokens]

// Workgroup ids go round the 8 XCDs; an XCD gets a run of neighbouring strips instead.  Its L2 has 16 channels of 256 bytes in turn, and a strip's pieces are 128 to 1024
// bytes at a stride that is mostly a multiple of the 4 KiB they span: every eighth strip would be 2 to 4 channels' work.
__device__ __forceinline__ unsigned strip_of(unsigned id, unsigned n) {
  const unsigned per = n >> 3, more = n & 7u, xcd = id & 7u;
  return xcd * per + min(xcd, more) + (id >> 3);
}

__device__ __forceinline__ uint16_t to_bf16(float x) { return (uint16_t)pack_bf16x2(x, 0.f); }

// ------------------------------------------------------------------------------------------------ bf16
constexpr int few_waves(int nt) { return nt <= 2 ? 16 : 8; }

// grid: (strips, splits).  GATED: H = bf16(a(G) U), cols = F, a row of W 2 F; else out [T][cols].  splits > 1: the sums of split y go to parts [y][T][row].
template <bool GATED, int NT, bool STREAM>
__global__ void __launch_bounds__(64 * few_waves(NT)) few_bf16_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, int T, int K, int cols, Gate gate,
                                                                      uint16_t* __restrict__ out, float* __restrict__ parts) {
  constexpr int KS = few_waves(NT), STEPS = 2;
  extern __shared__ __attribute__((aligned(16))) float red[];   // [KS][128][RED]
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = GATED ? 2 * cols : cols;
  const unsigned id = strip_of(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y), split = id / gridDim.x;
  const int n0 = (int)(id - split * gridDim.x) * (GATED ? 64 : 128);
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
  for (int s = (int)split * KS + wave; s < total; s += STEPS * stride) {
    u32x4 a[STEPS][8];
    bf16x8 b[STEPS][NT];
#pragma unroll
    for (int j = 0; j < STEPS; j++) {
      const int at = s + j * stride < total ? s + j * stride : s;
      const uint16_t* p = w + (size_t)at * 32 * row;
#pragma unroll
      for (int r = 0; r < 8; r++) {
        const u32x4* at_row = reinterpret_cast<const u32x4*>(p + (size_t)r * row);
        a[j][r] = STREAM ? ld_stream(at_row) : *at_row;
      }
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
        if (parts) parts[((size_t)split * T + 16 * i + tok) * row + col] = s;
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

// Over how many workgroups the reduction of a strip is split: the least of (rounds of the chip) x (a workgroup's bytes at the rate so many of them reach) + (for the
// sums: a launch, the parts written and read).  A workgroup streams 24 GB/s and more, the chip 6 TB/s.
constexpr int FEW_SPLITS = 16;
template <bool GATED> int few_strips(int cols) { return GATED ? cols / 64 : (cols + 127) / 128; }
template <bool GATED>
int few_splits(int T, int K, int cols) {
  const int waves = few_waves((T + 15) / 16), slots = 256, one = 24;   // (workgroups at once: one a CU; bytes a ns)
  const long long strips = few_strips<GATED>(cols), row = GATED ? 2 * cols : cols, bytes = 2LL * K * row;
  int best = 1;
  long long best_time = 0;
  for (int s = 1; s <= FEW_SPLITS && (s == 1 || K / 32 >= s * waves); s++) {
    const long long n = strips * s, at_once = n < slots ? n : slots, rate = at_once * one < 6000 ? at_once * one : 6000;
    const long long time = (n + slots - 1) / slots * (bytes / n * at_once / rate) + (s > 1 ? 6000 + 16LL * s * T * row / 6000 : 0);
    if (s == 1 || time < best_time) { best = s; best_time = time; }
  }
  return best;
}

constexpr size_t FEW_STREAM = 16 << 20;      // values of a weight from which on it is read with the streaming hint
template <bool GATED, int NT>
int launch_few_bf16_tokens(const void* X, const void* W, int T, int K, int cols, Gate gate, int splits, void* out, float* parts, hipStream_t s) {
  constexpr int KS = few_waves(NT), LDS = KS * 128 * RED * 4;
  const bool stream = (size_t)K * (GATED ? 2 * cols : cols) > FEW_STREAM;
  auto kern = stream ? few_bf16_kernel<GATED, NT, true> : few_bf16_kernel<GATED, NT, false>;
  static std::atomic<bool> configured[2][MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), LDS, configured[stream])) return rc;
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
  if (T <= 48) return launch_few_bf16_tokens<GATED, 3>(X, W, T, K, cols, gate, splits, out, parts, s);
  return launch_few_bf16_tokens<GATED, 4>(X, W, T, K, cols, gate, splits, out, parts, s);
}

// ------------------------------------------------------------------------------------------------ 8-bit integers
// What a workgroup's tokens are: codes and scales in memory; bf16 tokens that it quantises itself (OWN_MAX); or bf16 activations whose largest magnitudes are the
// largest of `n_tops` words a token (GIVEN_MAX).  The last two bring the codes into LDS and save a launch, where a workgroup's work on them is small (few_i8_fuses).
enum { I8_CODES = 0, I8_OWN_MAX = 1, I8_GIVEN_MAX = 2 };
constexpr int I8_WAVES = 8, I8_THREADS = 64 * I8_WAVES;
struct FewI8Args {
  const void* X; const float* sx; const uint32_t* tops; int n_tops;   // tops [n_tops][T]
  const char* panels; const float* sw; int T, K, N, npanels;
  Gate gate;
  uint16_t* out; uint32_t* tops_out;                                  // GATED: tops_out [workgroup][T]
};

// The largest of this work item's word over the workgroup.
__device__ __forceinline__ uint32_t group_max(uint32_t x, uint32_t* part) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, s, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < I8_WAVES; i++) x = max(x, part[i]);
  return x;
}

// RG: groups of 16 panel rows a workgroup; NT: groups of 16 tokens
template <bool GATED, int NT, int RG, int SOURCE>
__global__ void __launch_bounds__(I8_THREADS) few_i8_kernel(FewI8Args e) {
  constexpr int STEPS = 8 / RG;                               // 8 KiB a wave in flight
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ uint32_t part[I8_WAVES];
  __shared__ float scale[16 * NT];
  int* red = reinterpret_cast<int*>(smem);                    // [wave][16 RG][RED]
  char* xs = smem + I8_WAVES * 16 * RG * RED * 4;             // codes [T][pitch]
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int total = (e.K + 63) / 64, pitch = total * 64 + 16;
  const int strip = (int)strip_of(blockIdx.x, gridDim.x), r0 = strip * 16 * RG;
  const char* a0 = e.panels + (size_t)(r0 >> 8) * e.npanels * 16384 + (r0 & 255) * 64 + c * 64 + q * 16;
  i32x4 acc[RG][NT];
#pragma unroll
  for (int g = 0; g < RG; g++)
#pragma unroll
    for (int i = 0; i < NT; i++) acc[g][i] = i32x4{0, 0, 0, 0};

  u32x4 a[STEPS][RG];
  auto load_a = [&](int s) {
#pragma unroll
    for (int j = 0; j < STEPS; j++) {
      const int at = s + j * I8_WAVES < total ? s + j * I8_WAVES : s;
#pragma unroll
      for (int g = 0; g < RG; g++) a[j][g] = ld_stream(reinterpret_cast<const u32x4*>(a0 + (size_t)at * 16384 + g * 1024));
    }
  };
  if (wave < total) load_a(wave);                             // on its way while the tokens are quantised

  if constexpr (SOURCE != I8_CODES) {
    const int pieces = total * 8;                             // of 8 values, zeros behind K
    for (int t = 0; t < e.T; t++) {
      const u32x4* x = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(e.X) + (size_t)t * e.K);
      uint32_t top = 0u;
      if constexpr (SOURCE == I8_OWN_MAX) {
        for (int i = tid; i < e.K / 8; i += I8_THREADS) top = i8_top8(x[i], top);
      } else {
        for (int i = tid; i < e.n_tops; i += I8_THREADS) top = max(top, e.tops[(size_t)i * e.T + t]);
      }
      const float s = i8_scale(group_max(top, part));
      if (tid == 0) scale[t] = s;
      for (int i = tid; i < pieces; i += I8_THREADS) *reinterpret_cast<u32x2*>(xs + t * pitch + 8 * i) = i < e.K / 8 ? i8_codes8(x[i], s) : u32x2{0u, 0u};
    }
    __syncthreads();
  } else {
    for (int t = tid; t < e.T; t += I8_THREADS) scale[t] = e.sx[t];   // (read behind the barriers below)
  }

  for (int s = wave; s < total; s += STEPS * I8_WAVES) {
    u32x4 b[STEPS][NT];
#pragma unroll
    for (int j = 0; j < STEPS; j++) {
      const int at = s + j * I8_WAVES < total ? s + j * I8_WAVES : s;
#pragma unroll
      for (int i = 0; i < NT; i++) {
        const int t = min(16 * i + c, e.T - 1), k = 64 * at + 16 * q;
        if constexpr (SOURCE == I8_CODES) b[j][i] = k < e.K ? *reinterpret_cast<const u32x4*>(static_cast<const char*>(e.X) + (size_t)t * e.K + k) : u32x4{0u, 0u, 0u, 0u};
        else b[j][i] = *reinterpret_cast<const u32x4*>(xs + t * pitch + k);
      }
    }
#pragma unroll
    for (int j = 0; j < STEPS; j++) {
      if (j > 0 && s + j * I8_WAVES >= total) break;
#pragma unroll
      for (int g = 0; g < RG; g++)
#pragma unroll
        for (int i = 0; i < NT; i++)
          acc[g][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a[j][g]), __builtin_bit_cast(i32x4, b[j][i]), acc[g][i], 0, 0, 0);
    }
    if (s + STEPS * I8_WAVES < total) load_a(s + STEPS * I8_WAVES);
  }

#pragma unroll
  for (int i = 0; i < NT; i++) {
    const int tokens = min(e.T - 16 * i, 16);
    if (i > 0) __syncthreads();
    if (c < tokens) {
#pragma unroll
      for (int g = 0; g < RG; g++)
#pragma unroll
        for (int v = 0; v < 4; v++) red[(wave * 16 * RG + 16 * g + 4 * q + v) * RED + c] = acc[g][i][v];
    }
    __syncthreads();
    auto sum = [&](int r, int tok) {
      int s = 0;
#pragma unroll
      for (int k = 0; k < I8_WAVES; k++) s += red[(k * 16 * RG + r) * RED + tok];
      return (float)s * (scale[16 * i + tok] * e.sw[r0 + r]);
    };
    if constexpr (GATED) {
      constexpr int FEATS = 8 * RG;
      for (int o = tid; o < FEATS * tokens; o += I8_THREADS) {   // (FEATS neighbouring lanes have a token: all of them here, or none)
        const int f = o % FEATS, tok = o / FEATS, r = 16 * (f >> 3) + (f & 7), n = strip * FEATS + f;
        const float y = gate_act(e.gate, sum(r, tok)) * sum(r + 8, tok);
        uint32_t top = __builtin_bit_cast(uint32_t, y) & 0x7FFFFFFFu;
        if (n < e.N / 2) e.out[(size_t)(16 * i + tok) * (e.N / 2) + n] = to_bf16(y);
#pragma unroll
        for (int s = 1; s < FEATS; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s, 64));
        if (f == 0) e.tops_out[(size_t)strip * e.T + 16 * i + tok] = top;
      }
    } else {
      for (int o = tid; o < 16 * RG * tokens; o += I8_THREADS) {
        const int r = o % (16 * RG), tok = o / (16 * RG);
        if (r0 + r < e.N) e.out[(size_t)(16 * i + tok) * e.N + r0 + r] = to_bf16(sum(r, tok));
      }
    }
  }
}

// Activations to codes, a workgroup a token, with the largest magnitude of n_tops words a token
__global__ void __launch_bounds__(I8_THREADS) few_i8_quantise_kernel(const uint16_t* __restrict__ H, const uint32_t* __restrict__ tops, int n_tops, int T, int F,
                                                                     uint8_t* __restrict__ codes, float* __restrict__ scales) {
  __shared__ uint32_t part[I8_WAVES];
  const int t = blockIdx.x;
  uint32_t top = 0u;
  for (int i = threadIdx.x; i < n_tops; i += I8_THREADS) top = max(top, tops[(size_t)i * T + t]);
  const float s = i8_scale(group_max(top, part));
  if (threadIdx.x == 0) scales[t] = s;
  const u32x4* h = reinterpret_cast<const u32x4*>(H + (size_t)t * F);
  for (int i = threadIdx.x; i < F / 8; i += I8_THREADS) *reinterpret_cast<u32x2*>(codes + (size_t)t * F + 8 * i) = i8_codes8(h[i], s);
}

// Rows a workgroup: at least 512 workgroups if there are that many groups of 16.
int few_i8_groups(int N) { return N >= 512 * 64 ? 4 : N >= 512 * 32 ? 2 : 1; }

template <bool GATED, int NT, int RG, int SOURCE>
int launch_few_i8_one(const FewI8Args& e, hipStream_t s) {
  const int lds = I8_WAVES * 16 * RG * RED * 4 + (SOURCE == I8_CODES ? 0 : e.T * (up_to(e.K, 64) + 16));
  constexpr int MOST = I8_WAVES * 16 * RG * RED * 4 + (SOURCE == I8_CODES ? 0 : I8_FUSE_BYTES);
  auto kern = few_i8_kernel<GATED, NT, RG, SOURCE>;
  static std::atomic<bool> configured[MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), MOST, configured)) return rc;
  hipLaunchKernelGGL(kern, dim3((unsigned)((e.N + 16 * RG - 1) / (16 * RG))), dim3(I8_THREADS), lds, s, e);
  return (int)hipGetLastError();
}
template <bool GATED, int NT, int SOURCE>
int launch_few_i8_rows(const FewI8Args& e, hipStream_t s) {
  switch (few_i8_groups(e.N)) {
    case 4: return launch_few_i8_one<GATED, NT, 4, SOURCE>(e, s);
    case 2: return launch_few_i8_one<GATED, NT, 2, SOURCE>(e, s);
    default: return launch_few_i8_one<GATED, NT, 1, SOURCE>(e, s);
  }
}
template <bool GATED>
int launch_few_i8(const FewI8Args& e, int source, hipStream_t s) {
  if (source == I8_OWN_MAX) return launch_few_i8_rows<GATED, 1, I8_OWN_MAX>(e, s);
  if (source == I8_GIVEN_MAX) return GATED ? 1 : launch_few_i8_rows<false, 1, I8_GIVEN_MAX>(e, s);
  if (e.T <= 16) return launch_few_i8_rows<GATED, 1, I8_CODES>(e, s);
  return launch_few_i8_rows<GATED, 2, I8_CODES>(e, s);
}
FewI8Args few_i8_args(const void* X, const float* sx, int T, const I8Layout& w, void* out) {
  FewI8Args e{};
  e.X = X; e.sx = sx;
  e.panels = w.panels; e.sw = w.scales; e.T = T; e.K = w.K; e.N = w.N; e.npanels = up_to(w.K, 128) / 64;
  e.out = static_cast<uint16_t*>(out);
  return e;
}
}  // namespace

size_t few_gated_scratch(int T, int D, int F) {
  size_t most = 0;
  for (int t = 1; t <= (T < FEW_TOKENS ? T : FEW_TOKENS); t++) {
    const size_t up = (size_t)few_splits<true>(t, D, F) * t * 2 * F, down = (size_t)few_splits<false>(t, F, D) * t * D;
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

bool few_i8_fuses(int T, int K) { return T <= 16 && T * (up_to(K, 64) + 16) <= I8_FUSE_BYTES; }
size_t few_i8_tops(int T, int F) { return 4 * (size_t)(T < FEW_I8_TOKENS ? T : FEW_I8_TOKENS) * (size_t)((2 * F + 15) / 16); }

int launch_few_linear_i8(const void* X, int T, const I8Layout& w, void* Y, hipStream_t s) { return launch_few_i8<false>(few_i8_args(X, nullptr, T, w, Y), I8_OWN_MAX, s); }
int launch_few_matmul_i8(const void* codes, const float* sx, int T, const I8Layout& w, void* Y, hipStream_t s) {
  return launch_few_i8<false>(few_i8_args(codes, sx, T, w, Y), I8_CODES, s);
}
int launch_few_gated_i8(const void* X, int T, const I8Layout& wgu, const I8Layout& wd, float c1, float c3, void* X8, float* sx, void* H, uint32_t* tops, void* H8, float* sh,
                        void* Y, hipStream_t s) {
  const bool fused = few_i8_fuses(T, wgu.K);
  if (!fused)
    if (int rc = launch_quantise_i8(X, T, wgu.K, false, X8, sx, nullptr, s)) return rc;
  FewI8Args up = few_i8_args(fused ? X : X8, sx, T, wgu, H);
  up.gate = Gate{c1, c3};
  up.tops_out = tops;
  if (int rc = launch_few_i8<true>(up, fused ? I8_OWN_MAX : I8_CODES, s)) return rc;
  const int rows = 16 * few_i8_groups(wgu.N), n_tops = (wgu.N + rows - 1) / rows;
  if (few_i8_fuses(T, wd.K)) {
    FewI8Args down = few_i8_args(H, nullptr, T, wd, Y);
    down.tops = tops;
    down.n_tops = n_tops;
    return launch_few_i8<false>(down, I8_GIVEN_MAX, s);
  }
  hipLaunchKernelGGL(few_i8_quantise_kernel, dim3((unsigned)T), dim3(I8_THREADS), 0, s, static_cast<const uint16_t*>(H), tops, n_tops, T, wd.K, static_cast<uint8_t*>(H8), sh);
  if (int rc = (int)hipGetLastError()) return rc;
  return launch_few_matmul_i8(H8, sh, T, wd, Y, s);
}

}  // namespace ffn24
