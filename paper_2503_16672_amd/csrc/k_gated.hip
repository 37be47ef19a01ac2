// The gated feed-forward block in bf16, many tokens: five GEMMs on the core, forward two, backward three launches.  X, H, dY, dGU are [T][...] row-major; the
// weights Wgu [D][2 F] (gate | up) and Wd [F][D] are read where they lie.
//
//   [G|U] = X Wgu, H = a(G) U      A = Wgu, k-major, gate and up features interleaved by 8 (TR_GATE); B = X
//   Y = H Wd                       A = Wd, k-major; B = H
//   dH = dY Wd^T -> dG, dU         A = Wd; B = dY
//   dX = [dG|dU] Wgu^T             A = Wgu; B = dGU (K = 2 F)
//   dWd = H^T dY, dWgu = X^T dGU   both operands k-major (K = T), one launch
//
// Bound by the matrix ops (and the power they draw) from some thousand tokens on.  Kernels at T 16384 D 4096 F 16384, ms (PFLOP/s; a library product of these
// sizes 1.29 - 1.38): up 3.53 (1.24), down 1.57 (1.40), dH 2.11 (1.04), dX 3.08 (1.43) + 0.12 for Wgu's panels, weight gradients 4.94 (1.33).  Up and dH have what their epilogues
// move besides, 2.1 and 2.7 GB that one workgroup a CU does not overlap with its matrix ops.  Tiles come from the rule of tile_rule.hpp on the result's extent and K.
#include "launch_block.hpp"
#include "launch_edge.hpp"

namespace ffn24 {
namespace {

GemmArgs args(const void* A, int a_rows, int a_cols, const void* B, int b_rows, int b_cols, int M, int N, int K) {
  GemmArgs g{};
  g.A = A; g.B = B;
  g.M = M; g.N = N; g.K = K;
  g.a_rows = a_rows; g.a_pitch = 2 * a_cols;
  g.b_rows = b_rows; g.b_pitch = 2 * b_cols;
  return g;
}

// dWd and dWgu: workgroups [0, n_first) take the tiles of the first
template <int MI, int NI>
__global__ void __launch_bounds__(GEMM_THREADS, (Geo<false, false, MI, NI>::PER_CU)) gated_wgrad_kernel(GemmArgs ga, EdgeRowMajor::Args ea, int n_first, GemmArgs gb,
                                                                                                        EdgeRowMajor::Args eb) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const bool second = (int)blockIdx.x >= n_first;
  const GemmArgs g = second ? gb : ga;
  const EdgeRowMajor::Args e = second ? eb : ea;
  gemm_tile<false, EdgeRowMajor, false, 0, MI, NI, TR_A | TR_B | TR_EDGE>(g, e, smem, second ? (int)blockIdx.x - n_first : (int)blockIdx.x);
}
template <int MI, int NI>
int launch_wgrad_tile(GemmArgs ga, const EdgeRowMajor::Args& ea, GemmArgs gb, const EdgeRowMajor::Args& eb, hipStream_t s) {
  using G = Geo<false, false, MI, NI>;
  auto kern = gated_wgrad_kernel<MI, NI>;
  static std::atomic<bool> configured[MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), G::LDS_TOTAL, configured)) return rc;
  ga.M = up_to(ga.M, G::BM); ga.N = up_to(ga.N, G::BN);
  gb.M = up_to(gb.M, G::BM); gb.N = up_to(gb.N, G::BN);
  const int na = (ga.M / G::BM) * (ga.N / G::BN), nb = (gb.M / G::BM) * (gb.N / G::BN);
  hipLaunchKernelGGL(kern, dim3((unsigned)(na + nb)), dim3(GEMM_THREADS), G::LDS_TOTAL, s, ga, ea, na, gb, eb);
  return (int)hipGetLastError();
}

// dX and both weight gradients, which do not need one another, in one launch: the long reductions of dX (K = 2 F) first, the others fill what they leave of the chip.
template <int MI, int NI>
__global__ void __launch_bounds__(GEMM_THREADS, (Geo<false, false, MI, NI>::PER_CU)) gated_grads_kernel(GemmArgs gx, EdgeColMajor<false>::Args ex, int n_x, GemmArgs ga,
                                                                                                        EdgeRowMajor::Args ea, int n_first, GemmArgs gb, EdgeRowMajor::Args eb) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int id = (int)blockIdx.x - n_x;
  if (id < 0) { gemm_tile<false, EdgeColMajor<false>, false, 0, MI, NI, TR_EDGE>(gx, ex, smem, (int)blockIdx.x); return; }
  const bool second = id >= n_first;
  const GemmArgs g = second ? gb : ga;
  const EdgeRowMajor::Args e = second ? eb : ea;
  gemm_tile<false, EdgeRowMajor, false, 0, MI, NI, TR_A | TR_B | TR_EDGE>(g, e, smem, second ? id - n_first : id);
}
template <int MI, int NI>
int launch_grads_tile(GemmArgs gx, const EdgeColMajor<false>::Args& ex, GemmArgs ga, const EdgeRowMajor::Args& ea, GemmArgs gb, const EdgeRowMajor::Args& eb, hipStream_t s) {
  using G = Geo<false, false, MI, NI>;
  auto kern = gated_grads_kernel<MI, NI>;
  static std::atomic<bool> configured[MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), G::LDS_TOTAL, configured)) return rc;
  int n[3], i = 0;
  for (GemmArgs* g : {&gx, &ga, &gb}) {
    g->M = up_to(g->M, G::BM);
    g->N = up_to(g->N, G::BN);
    n[i++] = (g->M / G::BM) * (g->N / G::BN);
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)(n[0] + n[1] + n[2])), dim3(GEMM_THREADS), G::LDS_TOTAL, s, gx, ex, n[0], ga, ea, n[1], gb, eb);
  return (int)hipGetLastError();
}

__global__ void __launch_bounds__(256) zero_kernel(u32x4* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = u32x4{0u, 0u, 0u, 0u};
}
// A row-major matrix (K a multiple of 32) into the dense A panel form, 16 bytes a work item in the order of the output; rows beyond the last one are not written.
__global__ void __launch_bounds__(256) gated_panelise_kernel(const u32x4* __restrict__ in, u32x4* __restrict__ out, int rows, int panels) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  const unsigned block = (unsigned)(i >> 10), kp = block % (unsigned)panels, r = block / (unsigned)panels * 256 + ((unsigned)(i >> 2) & 255u);
  if ((int)r < rows) out[i] = ld_stream(in + ((size_t)r * (unsigned)panels + kp) * 4 + (i & 3));
}
}  // namespace

// for any token count up to T: what the splits of Y and dX need (beyond 2^24 values a result has 4096 of the smallest tiles)
size_t gated_scratch(int T, int D, int F, bool training) {
  size_t most = 0;
  for (int t = 64; t <= up_to(T, 64) && (long long)D * t <= 1 << 24; t += 64) {
    const size_t y = edge_split_scratch(D, t, F), x = training ? edge_split_scratch(D, t, 2 * F) : 0, top = y > x ? y : x;
    if (top > most) most = top;
  }
  return most;
}
size_t gated_panel_bytes(int rows, int K) { return 2 * (size_t)up_to(rows, 256) * (size_t)K; }
int launch_gated_panels(const void* Wgu, int D, int F, void* panels, hipStream_t s) {
  const size_t items = gated_panel_bytes(D, 2 * F) / 16;
  hipLaunchKernelGGL(gated_panelise_kernel, dim3((unsigned)(items / 256)), dim3(256), 0, s, static_cast<const u32x4*>(Wgu), static_cast<u32x4*>(panels), D, 2 * F / 32);
  return (int)hipGetLastError();
}

int launch_zero(void* p, size_t bytes, hipStream_t s) {
  hipLaunchKernelGGL(zero_kernel, dim3(1024), dim3(256), 0, s, static_cast<u32x4*>(p), bytes / 16);
  return (int)hipGetLastError();
}

int launch_gated_up(const void* X, const void* Wgu, int T, int D, int F, float c1, float c3, void* H, void* GU, void* GUx, hipStream_t s) {
  GemmArgs g = args(Wgu, D, 2 * F, X, T, D, 2 * F, T, D);
  g.gate = 2u * (uint32_t)F;
  using Epi = EpiGateUp<false, false>;
  return launch_edge<Epi, TR_A | TR_GATE>(g, Epi::Args{static_cast<__bf16*>(H), static_cast<__bf16*>(GU), static_cast<uint8_t*>(GUx), F, T, Gate{c1, c3}, I8Scales{}, nullptr}, s);
}

int launch_gated_down(const void* H, const void* Wd, int T, int D, int F, void* Y, const Scratch& scratch, hipStream_t s) {
  using Epi = EdgeColMajor<false>;
  return launch_edge_split<Epi, TR_A>(args(Wd, F, D, H, T, F, D, T, F), Epi::Args{static_cast<__bf16*>(Y), D, T, I8Scales{}}, scratch, s);
}

int launch_gated_dgate(const void* dY, const void* Wd, const void* GU, const void* GUx, int T, int D, int F, float c1, float c3, void* dGU, hipStream_t s) {
  const GemmArgs g = args(Wd, F, D, dY, T, D, F, T, D);
  const EpiDGate::Args e{static_cast<const __bf16*>(GU), static_cast<const uint8_t*>(GUx), static_cast<__bf16*>(dGU), F, T, Gate{c1, c3}};
  // (no 128 x 64: 64 x 64 was faster wherever the rule took it, us, T D F: 128 4096 12288 39.3, 27.8; 256 4096 12288 67.8, 54.8; 1000 1088 2944 20.2, 18.3)
  switch (pick_edge_tile(F, T, D)) {
    case 0: return launch_edge_tile<EpiDGate, TR_EDGE, 4, 4>(g, e, s);
    case 1: return launch_edge_tile<EpiDGate, TR_EDGE, 4, 2>(g, e, s);
    case 2: return launch_edge_tile<EpiDGate, TR_EDGE, 2, 2>(g, e, s);
    default: return launch_edge_tile<EpiDGate, TR_EDGE, 1, 1>(g, e, s);
  }
}

int launch_gated_grads(const void* X, const void* dY, const void* H, const void* dGU, const void* Wgu, bool panels, int T, int D, int F, void* dX, void* dWgu, void* dWd,
                       const Scratch& scratch, hipStream_t s) {
  using EpiX = EdgeColMajor<false>;
  const int K = up_to(T, 64);
  GemmArgs gx = args(Wgu, D, 2 * F, dGU, T, 2 * F, D, T, 2 * F);
  gx.a_panel = panels;
  const GemmArgs ga = args(X, T, D, dGU, T, 2 * F, D, 2 * F, K), gb = args(H, T, F, dY, T, D, F, D, K);
  const EpiX::Args ex{static_cast<__bf16*>(dX), D, T, I8Scales{}};
  const EdgeRowMajor::Args ea{static_cast<__bf16*>(dWgu), D, 2 * F}, eb{static_cast<__bf16*>(dWd), F, D};
  switch (panels ? 0 : pick_grads_tile(T, D, F, K)) {
    case 1: return launch_grads_tile<4, 2>(gx, ex, ga, ea, gb, eb, s);
    case 2: return launch_grads_tile<2, 2>(gx, ex, ga, ea, gb, eb, s);
    case 3: return launch_grads_tile<2, 1>(gx, ex, ga, ea, gb, eb, s);
    case 4: return launch_grads_tile<1, 1>(gx, ex, ga, ea, gb, eb, s);
    default: break;                        // apart
  }
  if (int rc = launch_edge_split<EpiX, 0>(gx, ex, scratch, s)) return rc;
  switch (pick_edge_tile(D, 2 * F, K, F, D)) {
    case 0: return launch_wgrad_tile<4, 4>(ga, ea, gb, eb, s);
    case 1: return launch_wgrad_tile<4, 2>(ga, ea, gb, eb, s);
    case 2: return launch_wgrad_tile<2, 2>(ga, ea, gb, eb, s);
    case 3: return launch_wgrad_tile<2, 1>(ga, ea, gb, eb, s);
    default: return launch_wgrad_tile<1, 1>(ga, ea, gb, eb, s);
  }
}

}  // namespace ffn24
