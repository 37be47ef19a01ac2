// Quantisation to 8-bit integers (ffn24_block.h): a row's scale from the bits of its largest magnitude, and codes.
#pragma once
#include "gemm_core.hpp"

namespace ffn24 {

__device__ __forceinline__ float i8_scale(uint32_t top) { return top ? __builtin_bit_cast(float, top) * (1.f / 127.f) : 1.f; }
__device__ __forceinline__ uint32_t i8_code(float x, float s) { return (uint32_t)(int)fminf(fmaxf(rintf(x / s), -127.f), 127.f) & 0xFFu; }
// of 8 bf16 values: the larger of `top` and their largest magnitude (as the bits of an fp32), and their codes
__device__ __forceinline__ uint32_t i8_top8(const u32x4& w, uint32_t top) {
#pragma unroll
  for (int i = 0; i < 4; i++) top = max(top, max(w[i] << 16 & 0x7FFF0000u, w[i] & 0x7FFF0000u));
  return top;
}
__device__ __forceinline__ u32x2 i8_codes8(const u32x4& w, float s) {
  u32x2 o;
#pragma unroll
  for (int i = 0; i < 2; i++)
    o[i] = i8_code(bf16_lo_to_f32(w[2 * i]), s) | i8_code(bf16_hi_to_f32(w[2 * i]), s) << 8 | i8_code(bf16_lo_to_f32(w[2 * i + 1]), s) << 16 |
           i8_code(bf16_hi_to_f32(w[2 * i + 1]), s) << 24;
  return o;
}

}  // namespace ffn24
