// Host-side launchers of the operators around the feed-forward block (definitions in k_norm.hip, ...).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "tile_rule.hpp"

namespace ffn24 {

constexpr int NORM_MAX_D = 16384;

struct Scratch { void* p; size_t bytes; };   // device memory of a call or a context

// k_norm.hip
int launch_norm_fwd(const void* X, const void* R, const float* w, const float* b, int T, int D, float eps, bool f32, void* S, void* Y, float* mean, float* rstd,
                    hipStream_t s);
int norm_bwd_parts(int64_t T, int D);   // partial sums [2][D] that a backward keeps in its scratch
int launch_norm_bwd(const void* dY, const void* S, const float* w, const float* mean, const float* rstd, const void* dS, int T, int D, bool f32, void* dX,
                    float* dweight, float* dbias, float* parts, hipStream_t s);

// k_gated.hip: T >= 1, D and F multiples of 64; GU, GUx (EpiGateUp) NULL in a forward without a backward
int launch_gated_up(const void* X, const void* Wgu, int T, int D, int F, float c1, float c3, void* H, void* GU, void* GUx, hipStream_t s);
int launch_gated_down(const void* H, const void* Wd, int T, int D, int F, void* Y, const Scratch& scratch, hipStream_t s);
size_t gated_scratch(int T, int D, int F, bool training);   // bytes of `scratch` for any token count up to T (with less, reductions are not split)
size_t gated_panel_bytes(int rows, int K);
int launch_gated_panels(const void* Wgu, int D, int F, void* panels, hipStream_t s);   // for dX (gated_dx_panels; `panels` below: it reads Wgu so)
int launch_gated_dgate(const void* dY, const void* Wd, const void* GU, const void* GUx, int T, int D, int F, float c1, float c3, void* dGU, hipStream_t s);
int launch_gated_grads(const void* X, const void* dY, const void* H, const void* dGU, const void* Wgu, bool panels, int T, int D, int F, void* dX, void* dWgu, void* dWd,
                       const Scratch& scratch, hipStream_t s);
int launch_zero(void* p, size_t bytes, hipStream_t s);   // 16-byte aligned, a multiple of 16 bytes

// k_i8.hip: K a multiple of 16, N of 8 (with two halves: of 16); T >= 1
struct I8Layout { const char* panels; const float* scales; int K, N; };   // weights as i8_weight lays them out
int64_t i8_weight_size(int64_t K, int64_t N);
I8Layout i8_layout(const void* p, int K, int N);
int launch_i8_weight(const void* W, int K, int N, bool halves, void* out, hipStream_t s);
int64_t i8_panel_size(int64_t T, int64_t K);     // bytes of codes in panel form
int launch_quantise_i8(const void* X, int T, int K, bool panel_form, void* codes, float* scales, uint32_t* zero, hipStream_t s);
int launch_quantise_i8_given(const void* H, const uint32_t* tops, int T, int F, void* codes, float* scales, hipStream_t s);
size_t matmul_i8_scratch(int T, int K, int N);
size_t gated_i8_scratch(int T, int D, int F);    // for any token count up to T
int launch_matmul_i8(const void* codes, bool panel_form, const float* sx, int T, const I8Layout& w, void* Y, const Scratch& scratch, hipStream_t s);
// (codes in panel form)
int launch_gated_up_i8(const void* codes, const float* sx, int T, const I8Layout& w, float c1, float c3, void* H, uint32_t* rowmax, hipStream_t s);

// k_few.hip: few tokens, where the weights are what counts (few_tokens, few_i8_tokens, few_gated_i8_tokens)
size_t few_gated_scratch(int T, int D, int F);   // bytes of `parts` for any token count up to T
int launch_few_gated_up(const void* X, const void* Wgu, int T, int D, int F, float c1, float c3, void* H, float* parts, hipStream_t s);
int launch_few_gated_down(const void* H, const void* Wd, int T, int D, int F, void* Y, float* parts, hipStream_t s);

bool few_i8_fuses(int T, int K);                 // whether the product's workgroups quantise the tokens themselves
size_t few_i8_tops(int T, int F);                // bytes of the gated block's `tops`
int launch_few_linear_i8(const void* X, int T, const I8Layout& w, void* Y, hipStream_t s);   // few_i8_fuses
int launch_few_matmul_i8(const void* codes, const float* sx, int T, const I8Layout& w, void* Y, hipStream_t s);
int launch_few_gated_i8(const void* X, int T, const I8Layout& wgu, const I8Layout& wd, float c1, float c3, void* X8, float* sx, void* H, uint32_t* tops, void* H8, float* sh,
                        void* Y, hipStream_t s);

}  // namespace ffn24
