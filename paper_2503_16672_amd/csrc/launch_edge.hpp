// Launches of the GEMM core on operands of any extent (TR_EDGE); included by the units that instantiate them.
#pragma once
#include "block_epilogues.hpp"
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

}  // namespace ffn24
