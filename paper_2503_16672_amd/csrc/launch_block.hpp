// Host-side launchers of the operators around the feed-forward block (definitions in k_norm.hip, ...).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ffn24 {

constexpr int NORM_MAX_D = 16384;

// k_norm.hip
int launch_norm_fwd(const void* X, const void* R, const float* w, const float* b, int T, int D, float eps, bool f32, void* S, void* Y, float* mean, float* rstd,
                    hipStream_t s);
int norm_bwd_parts(int64_t T, int D);   // partial sums [2][D] that a backward keeps in its scratch
int launch_norm_bwd(const void* dY, const void* S, const float* w, const float* mean, const float* rstd, const void* dS, int T, int D, bool f32, void* dX,
                    float* dweight, float* dbias, float* parts, hipStream_t s);

}  // namespace ffn24
