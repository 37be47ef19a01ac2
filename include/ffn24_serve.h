/* ffn24_serve -- serving with 4-bit weights and with experts: mx4 numbers, products and the gated block on mx4 weights, the mixture of experts for few tokens.
 *
 * C ABI of libffn24.so, the third part.  The conventions of ffn24.h and ffn24_block.h hold: device pointers owned by the caller, row-major, contiguous and 16-byte
 * aligned; `stream` a hipStream_t; calls only enqueue kernels (the *_ctx_create calls allocate, and wait for what they clear); FFN24_OK or a negative FFN24_ERR_*
 * code; bad arguments are rejected before anything is launched; kernels run on the current device; an output must not overlap an input or another output.  T == 0
 * is a no-op.  All of them are forward only.
 */
#ifndef FFN24_SERVE_H
#define FFN24_SERVE_H

#include "ffn24_block.h"

#ifdef __cplusplus
extern "C" {
#endif

/* mx4: 4-bit values (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, codes 0 .. 7 and 8 .. 15) that share a power of two with the other 31 of their block, 32
 * neighbours of a row.  With e = floor(log2 max |block|):
 *   scale code = max(e - 2 + 127, 0), its value 2^(code - 127);  255, the NaN, if the block has an infinity or a NaN (the block's values are then NaN, whatever their codes)
 *   value code = x / scale to the nearest value, ties to the even code, beyond 6 held to 6
 * Codes [T][K / 2], two a byte, the lower k in the low nibble; scale codes [T][K / 32].  K a multiple of 32, at most 2^17; T at most 2^24.  X and Y bf16 or fp32. */
FFN24_API int quantise_mx4(const void* X, int64_t T, int64_t K, ffn24_norm_dtype dtype, void* codes, void* scales, void* stream);
/* Y = value * scale, exact in both types (a bf16 or fp32 below its normal range as its subnormal) */
FFN24_API int dequantise_mx4(const void* codes, const void* scales, int64_t T, int64_t K, ffn24_norm_dtype dtype, void* Y, void* stream);

/* Weights W [K][N] for the products, blocks along K, laid out once: mx4_weight_bytes(K, N) bytes at `out`, to be used with the same K and N.  mx4_weight quantises bf16;
 * mx4_weight_codes takes codes [N][K / 2] and scales [N][K / 32] that are mx4 already.  reserved: 0, anything else is FFN24_ERR_SHAPE (the contexts below lay out their own
 * weights).  K a multiple of 32, at most 2^17; N a multiple of 8, at most 2^20. */
/* ceil(N / 64) (4096 s + 1024 ceil(s / 4)) with s = ceil(K / 128): 17/32 of a byte a value where N is a multiple of 64 and K of 512, more where blocks are filled up;
 * -1 for sizes out of range */
FFN24_API int64_t mx4_weight_bytes(int64_t K, int64_t N);
FFN24_API int mx4_weight(const void* W, int64_t K, int64_t N, int reserved, void* out, void* stream);
FFN24_API int mx4_weight_codes(const void* codes, const void* scales, int64_t K, int64_t N, int reserved, void* out, void* stream);
/* Y [T][N] = bf16(X4 W4): bf16 X [T][K] to mx4 on the way, sums in fp32.  T at most 2^20.  scratch: linear_mx4_scratch(T, K, N) bytes, used until the call's last
 * kernel has run. */
FFN24_API int64_t linear_mx4_scratch(int64_t T, int64_t K, int64_t N);   /* or -1 */
FFN24_API int linear_mx4(const void* X, int64_t T, const void* weight, int64_t K, int64_t N, void* Y, void* scratch, void* stream);

/* The gated block on mx4 weights: G, U from such products of X and [Wg | Wu], in fp32;  h = a(G) U;  H4 = mx4(h), blocks along F;  Y = bf16(H4 Wd4).  T, D, F, gate as
 * for gated_ctx_create, D and F at most 2^17.  Workspace: mx4_weight_bytes(D, 2 F) + (F, D) for the weights, mx4_weight_bytes(D, T) for X, (F, T) for H (T filled up to 8s), and what a
 * split reduction takes (some tens of MiB at most).  gated_mx4_set_weights quantises Wgu [D][2 F] and Wd [F][D] (bf16) into the context, which does not need them afterwards;
 * gated_mx4_fwd before it returns FFN24_ERR_STATE. */
typedef struct gated_mx4_ctx gated_mx4_ctx;
FFN24_API int gated_mx4_ctx_create(gated_mx4_ctx** out, int64_t T, int64_t D, int64_t F, ffn24_gate gate);
FFN24_API int gated_mx4_ctx_destroy(gated_mx4_ctx* ctx);
FFN24_API int gated_mx4_set_weights(gated_mx4_ctx* ctx, const void* Wgu, const void* Wd, void* stream);
FFN24_API int gated_mx4_fwd(gated_mx4_ctx* ctx, const void* X, int64_t T, void* Y, void* stream);

/* A mixture of E gated blocks for few tokens.  For each token x (bf16):
 *   l = x Wr  (Wr bf16 [D][E]; in 64 bits);  its k experts: the largest l, among equals the lowest index (a NaN counts as the lowest);
 *   shares p = exp(l) over the sum of exp(l), of the chosen ones (renormalise != 0) or of all E;
 *   y = bf16(sum over the chosen of p_e (h_e Wd_e)),  h_e = a(x Wg_e) (x Wu_e), sums in fp32;
 * FFN24_EXPERTS_BF16: h_e is held to 2^-16 of it, as two bf16;  FFN24_EXPERTS_MX4: x, h_e and the weights are mx4 (the router is not).
 * 1 <= T <= 64 (every call says how many it has), D and F multiples of 64, D at most 2^14, F at most 2^16, 1 <= E <= 256, 1 <= k <= min(E, 16).  moe_set_weights lays out Wr,
 * Wgu [E][D][2 F] and Wd [E][F][D] in the context (their size, Wr's with E filled up to 64s; in mx4 E (mx4_weight_bytes(D, 2 F) + mx4_weight_bytes(F, D))), which does not need
 * them afterwards.  Workspace besides: at most 49 MiB + 4 KiB F.  moe_fwd stores the choice too where experts (int32 [T][k], by falling l) and shares (fp32 [T][k]) are given: both or
 * neither.  No other token's values enter a token's result, and results repeat bit for bit; the order of its sums may depend on how many tokens
 * there are and which experts they chose.  The contexts' other rules are those of gated_ctx. */
typedef enum { FFN24_EXPERTS_BF16 = 0, FFN24_EXPERTS_MX4 = 1 } ffn24_experts;
typedef struct moe_ctx moe_ctx;
FFN24_API int moe_ctx_create(moe_ctx** out, int64_t T, int64_t D, int64_t F, int64_t E, int64_t k, ffn24_gate gate, int renormalise, ffn24_experts type);
FFN24_API int moe_ctx_destroy(moe_ctx* ctx);
FFN24_API int moe_set_weights(moe_ctx* ctx, const void* Wr, const void* Wgu, const void* Wd, void* stream);
FFN24_API int moe_fwd(moe_ctx* ctx, const void* X, int64_t T, void* Y, void* experts, void* shares, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FFN24_SERVE_H */
