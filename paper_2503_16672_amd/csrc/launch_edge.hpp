// Launches of the GEMM core on operands of any extent (TR_EDGE); included by the units that instantiate them.
#pragma once
#include "block_epilogues.hpp"
#include "launch_block.hpp"
#include "launch_impl.hpp"

namespace ffn24 {

inline int up_to(int x, int m) { return (x + m - 1) / m * m; }

template <class Epi, int TR, int MI, int NI>
static int launch_edge_tile(GemmArgs g, const typename Epi::Args& ea, hipStream_t s) {
  using G = Geo<false, false, MI, NI>;
  g.M = up_to(g.M, G::BM);
  g.N = up_to(g.N, G::BN);
  return launch_tile<false, Epi, false, 0, MI, NI, TR>(g, ea, s);
}

// g.M, g.N: the result's real size; g.K: a multiple of 64
template <class Epi, int TR>
static int launch_edge(const GemmArgs& g, const typename Epi::Args& ea, hipStream_t s) {
  switch (pick_edge_tile(g.M, g.N, g.K)) {
    case 0: return launch_edge_tile<Epi, TR | TR_EDGE, 4, 4>(g, ea, s);
    case 1: return launch_edge_tile<Epi, TR | TR_EDGE, 4, 2>(g, ea, s);
    case 2: return launch_edge_tile<Epi, TR | TR_EDGE, 2, 2>(g, ea, s);
    case 3: return launch_edge_tile<Epi, TR | TR_EDGE, 2, 1>(g, ea, s);
    default: return launch_edge_tile<Epi, TR | TR_EDGE, 1, 1>(g, ea, s);
  }
}

// Where the result has few tiles and the reduction is long, it is split over several workgroups a tile, whose sums a second kernel adds up in a fixed order.
template <int TR, int MI, int NI>
__global__ void __launch_bounds__(GEMM_THREADS, (Geo<false, false, MI, NI>::PER_CU)) gemm_split_kernel(GemmArgs g, EdgePart::Args ea, int tiles, int part) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int split = (int)blockIdx.x / tiles, k0 = split * part;
  constexpr bool TRA = (TR & TR_A) != 0;
  g.K = min(part, g.K - k0);
  // (K-contiguous: a row's part starts 2 k0 bytes on; rows beyond the last one still start behind the tensor's extent.  Panel form: k0 / 32 panels of 256 rows x 64 bytes on)
  g.A = static_cast<const char*>(g.A) + (TRA ? (size_t)k0 * g.a_pitch : g.a_panel ? (size_t)k0 * (2 * 256) : (size_t)k0 * 2);
  if constexpr (TRA) g.a_rows -= k0;
  g.B = static_cast<const char*>(g.B) + (g.b_panel ? (size_t)k0 * (2 * 256) : (size_t)k0 * 2);
  ea.parts += (size_t)split * ea.M * ea.N;
  gemm_tile<false, EdgePart, false, 0, MI, NI, TR>(g, ea, smem, (int)blockIdx.x - split * tiles);
}
template <int TR, int MI, int NI>
static int launch_split_tile(GemmArgs g, const EdgePart::Args& ea, int splits, int part, hipStream_t s) {
  using G = Geo<false, false, MI, NI>;
  auto kern = gemm_split_kernel<TR, MI, NI>;
  static std::atomic<bool> configured[MAX_DEVICES] = {};
  if (int rc = ensure_dynamic_lds(reinterpret_cast<const void*>(kern), G::LDS_TOTAL, configured)) return rc;
  g.M = up_to(g.M, G::BM);
  g.N = up_to(g.N, G::BN);
  const int tiles = (g.M / G::BM) * (g.N / G::BN);
  hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * splits)), dim3(GEMM_THREADS), G::LDS_TOTAL, s, g, ea, tiles, part);
  return (int)hipGetLastError();
}
inline size_t edge_split_scratch(int M, int N, int K) {
  const EdgeSplit p = pick_edge_split(M, N, K);
  return p.splits > 1 ? 4 * (size_t)p.splits * (size_t)M * (size_t)up_to(N, 64) : 0;
}
// launch_edge for a plain product stored as out[n][m] (Epi: EdgeColMajor), split if the scratch holds edge_split_scratch bytes
template <class Epi, int TR>
static int launch_edge_split(const GemmArgs& g, const typename Epi::Args& ea, const Scratch& scratch, hipStream_t s) {
  const EdgeSplit p = pick_edge_split(g.M, g.N, g.K);
  if (p.splits == 1 || edge_split_scratch(g.M, g.N, g.K) > scratch.bytes) return launch_edge<Epi, TR>(g, ea, s);
  const EdgePart::Args parts{static_cast<uint32_t*>(scratch.p), g.M, g.N};
  int rc;
  switch (p.tile) {
    case 2: rc = launch_split_tile<TR | TR_EDGE, 2, 2>(g, parts, p.splits, p.part, s); break;
    case 3: rc = launch_split_tile<TR | TR_EDGE, 2, 1>(g, parts, p.splits, p.part, s); break;
    default: rc = launch_split_tile<TR | TR_EDGE, 1, 1>(g, parts, p.splits, p.part, s); break;
  }
  if (rc) return rc;
  hipLaunchKernelGGL((edge_sum_kernel<Epi::INTEGER>), dim3((unsigned)(((size_t)g.M / 4 * g.N + 255) / 256)), dim3(256), 0, s, parts.parts, p.splits, g.M, g.N, ea.sc,
                     reinterpret_cast<uint16_t*>(ea.C));
  return (int)hipGetLastError();
}

}  // namespace ffn24
