// C ABI of the operators around the feed-forward block (ffn24_block.h): argument checks, workspaces, and the kernel sequences.
#include <hip/hip_runtime.h>
#include <new>
#include "../../include/ffn24_block.h"
#include "launch_block.hpp"

using namespace ffn24;

namespace {
constexpr int64_t MAX_TOKENS = 1 << 24;   // (row counts and grids stay within 32 bits)

template <class... P> bool misaligned(const P*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 15u) != 0; }
int done(int rc) { return rc ? FFN24_ERR_HIP : FFN24_OK; }
}  // namespace

extern "C" {

int layer_norm_fwd(const void* X, const void* R, const float* weight, const float* bias, int64_t T, int64_t D, float eps, ffn24_norm_dtype dtype, void* S,
                   void* Y, float* mean, float* rstd, void* stream) {
  if (dtype != FFN24_NORM_BF16 && dtype != FFN24_NORM_F32) return FFN24_ERR_DTYPE;
  if (T < 0 || T > MAX_TOKENS || D < 1 || D > NORM_MAX_D || !(eps > 0.f)) return FFN24_ERR_SHAPE;
  if (T == 0) return FFN24_OK;
  if (!X || !weight || !Y || (R == nullptr) != (S == nullptr) || (mean == nullptr) != (rstd == nullptr)) return FFN24_ERR_NULL;
  if (misaligned(X, R, S, Y, weight, bias, mean, rstd)) return FFN24_ERR_ALIGN;
  return done(launch_norm_fwd(X, R, weight, bias, (int)T, (int)D, eps, dtype == FFN24_NORM_F32, S, Y, mean, rstd, static_cast<hipStream_t>(stream)));
}

int64_t layer_norm_bwd_scratch(int64_t T, int64_t D) {
  if (T < 0 || T > MAX_TOKENS || D < 1 || D > NORM_MAX_D) return -1;
  return (int64_t)norm_bwd_parts(T, (int)D) * 2 * D * 4;
}

int layer_norm_bwd(const void* dY, const void* S, const float* weight, const float* mean, const float* rstd, const void* dS, int64_t T, int64_t D,
                   ffn24_norm_dtype dtype, void* dX, float* dweight, float* dbias, void* scratch, void* stream) {
  if (dtype != FFN24_NORM_BF16 && dtype != FFN24_NORM_F32) return FFN24_ERR_DTYPE;
  if (T < 0 || T > MAX_TOKENS || D < 1 || D > NORM_MAX_D) return FFN24_ERR_SHAPE;
  if (!dweight || (T > 0 && (!dY || !S || !weight || !mean || !rstd || !dX || !scratch))) return FFN24_ERR_NULL;
  if (misaligned(dY, S, weight, mean, rstd, dS, dX, dweight, dbias, scratch)) return FFN24_ERR_ALIGN;
  return done(launch_norm_bwd(dY, S, weight, mean, rstd, dS, (int)T, (int)D, dtype == FFN24_NORM_F32, dX, dweight, dbias, static_cast<float*>(scratch),
                              static_cast<hipStream_t>(stream)));
}

}  // extern "C"
