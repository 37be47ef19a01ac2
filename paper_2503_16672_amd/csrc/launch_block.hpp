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

// k_gated.hip: T >= 1, D and F multiples of 64; GU NULL in a forward without a backward
int launch_gated_up(const void* X, const void* Wgu, int T, int D, int F, float c1, float c3, void* H, void* GU, hipStream_t s);
int launch_gated_down(const void* H, const void* Wd, int T, int D, int F, void* Y, hipStream_t s);
int launch_gated_dgate(const void* dY, const void* Wd, const void* GU, int T, int D, int F, float c1, float c3, void* dGU, hipStream_t s);
int launch_gated_dx(const void* dGU, const void* Wgu, int T, int D, int F, void* dX, hipStream_t s);
int launch_gated_wgrad(const void* X, const void* dY, const void* H, const void* dGU, int T, int D, int F, void* dWgu, void* dWd, hipStream_t s);
int launch_zero(void* p, size_t bytes, hipStream_t s);   // 16-byte aligned, a multiple of 16 bytes

}  // namespace ffn24
