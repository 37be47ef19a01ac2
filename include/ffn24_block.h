/* ffn24_block -- the operators around the feed-forward block: layer norm, the gated feed-forward block, int8 products.
 *
 * C ABI of libffn24.so, the second half.  ffn24.h has the conventions that hold here too: device pointers owned by the caller, row-major,
 * contiguous and 16-byte aligned; `stream` a hipStream_t (NULL = the default stream); calls only enqueue kernels, they neither synchronise nor
 * allocate device memory (the *_ctx_create calls allocate); return values FFN24_OK or a negative FFN24_ERR_* code; bad arguments are rejected
 * before anything is launched; kernels run on the current device, whose memory every pointer has to be; outputs are overwritten.  No call keeps a tensor's address: a backward is handed what it needs again.  An output must not
 * overlap an input or another output unless the call says so.  T == 0 is a no-op everywhere (gradients of weights are then zero).
 *
 * Together they are the pre-norm gated feed-forward sublayer, the baseline that the paper's Table 1 compares 2:4 activation sparsity with
 * (SwiGLU): layer_norm_fwd, gated_fwd, gated_bwd, layer_norm_bwd in training, layer_norm_fwd and gated_i8_fwd in int8 serving.
 */
#ifndef FFN24_BLOCK_H
#define FFN24_BLOCK_H

#include "ffn24.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of a norm's tokens. */
typedef enum { FFN24_NORM_BF16 = 0, FFN24_NORM_F32 = 1 } ffn24_norm_dtype;

/* Layer norm of T tokens of D values, 1 <= D <= 16384, with an optional residual in front:
 *   S = X + R, rounded to the element type (R == NULL: S is X itself, and the S argument must be NULL);
 *   mean[t] = sum_d S / D;  rstd[t] = 1 / sqrt(sum_d (S - mean)^2 / D + eps);  Y = (S - mean) rstd weight + bias.
 * weight, bias fp32 [D], bias may be NULL (no bias); mean, rstd fp32 [T], both may be NULL (a forward without a backward).  Statistics in fp32, the
 * variance from the centred values.  eps > 0.  S may be X or R (in place); Y may be S's or X's buffer if the caller needs neither. */
FFN24_API int layer_norm_fwd(const void* X, const void* R, const float* weight, const float* bias, int64_t T, int64_t D, float eps,
                             ffn24_norm_dtype dtype, void* S, void* Y, float* mean, float* rstd, void* stream);

/* Its backward.  With xh = (S - mean) rstd and p = dY weight:
 *   dX = rstd (p - sum_d p / D - xh sum_d (p xh) / D) + dS;   dweight[d] = sum_t dY xh;   dbias[d] = sum_t dY.
 * S is what the forward normalised.  dS, the gradient that reaches S along the residual stream, may be NULL (0); dX is the gradient of X and of R.  dX
 * may be dS's buffer.  dbias may be NULL.  scratch: layer_norm_bwd_scratch(T, D) bytes of device memory, used until the call's last kernel has run.  The sums over tokens
 * are added in an order that depends on T and D alone: results repeat bit for bit. */
FFN24_API int64_t layer_norm_bwd_scratch(int64_t T, int64_t D);   /* bytes, or -1 for sizes out of range */
FFN24_API int layer_norm_bwd(const void* dY, const void* S, const float* weight, const float* mean, const float* rstd, const void* dS, int64_t T,
                             int64_t D, ffn24_norm_dtype dtype, void* dX, float* dweight, float* dbias, void* scratch, void* stream);

/* Gated feed-forward block, bf16 with fp32 accumulation: with Wgu [D][2 F] = [Wg | Wu] (a row of it: F gate columns, then F up columns) and Wd [F][D],
 *   [G | U] = X Wgu;   H = bf16(a(G) U);   Y = H Wd.
 * Gate activations: a(x) = x / (1 + exp(-x)) (SwiGLU), and GELU in its tanh form, a(x) = x / (1 + exp(-2 sqrt(2/pi) (x + 0.044715 x^3))) (GEGLU). */
typedef enum { FFN24_GATE_SILU = 0, FFN24_GATE_GELU_TANH = 1 } ffn24_gate;
typedef struct gated_ctx gated_ctx; /* opaque; owns only its device workspace */

/* A context for up to T tokens (1 <= T <= 2^20; every call says how many it has, any number up to T), D and F multiples of 64, at most 2^18.
 * flags: 0 or FFN24_TRAINING (gated_bwd).  Workspace, allocated on the current device: 2 T F bytes, 12 T F with FFN24_TRAINING, and besides
 * what a split reduction takes (some tens of MiB at most) and, in training, the size of Wgu.  A context belongs to that
 * device and to one thread at a time; calls on different streams are the caller's to order.  *out is untouched on error. */
FFN24_API int gated_ctx_create(gated_ctx** out, int64_t T, int64_t D, int64_t F, ffn24_gate gate, int flags);
/* The caller must have synchronised every stream that used the context.  NULL is allowed. */
FFN24_API int gated_ctx_destroy(gated_ctx* ctx);

/* X [T][D] -> Y [T][D], 0 <= T <= the context's.  The weights are read where they lie.  A training context keeps H in bf16 and G, U in 24
 * bits for gated_bwd. */
FFN24_API int gated_fwd(gated_ctx* ctx, const void* X, int64_t T, const void* Wgu, const void* Wd, void* Y, void* stream);

/* Backward of the context's last gated_fwd (FFN24_ERR_STATE without one, or without FFN24_TRAINING): dY [T][D] with that call's T, and its X, Wgu, Wd again:
 *   dH = dY Wd^T;  dG = bf16(dH U a'(G));  dU = bf16(dH a(G));
 *   dX = dG Wg^T + dU Wu^T;  dWgu = X^T [dG | dU];  dWd = H^T dY        (bf16 [T][D], [D][2 F], [F][D])
 * It may be called more than once for a forward. */
FFN24_API int gated_bwd(gated_ctx* ctx, const void* dY, const void* X, const void* Wgu, const void* Wd, void* dX, void* dWgu, void* dWd, void* stream);

/* Products of 8-bit integers with a scale for each token and each output channel (serving).  A row x (a token; a channel's weights) becomes
 *   scale = max |x| * (1 / 127), factor and product rounded to fp32 (1 if all zero);  code = rint(x / scale), in -127 .. 127 (an IEEE division);
 * and the product of X [T][K] and W [K][N] is Y[t][n] = bf16(sx[t] sw[n] sum_k X8[t][k] W8[k][n]), the sum in 32-bit integers, exact.  A token with an infinite or NaN
 * value gets such a scale and NaN or infinite results; the others do not see it.  K a multiple of 16, at most 2^17; N a multiple of 8, at most 2^20; T at most 2^20.
 *
 * i8_weight quantises W (bf16 [K][N]) and lays it out as the products read it: i8_weight_bytes(K, N) bytes at `out`, to be used with the same K and N.  halves != 0:
 * W is [Wg | Wu] of a gated block (N a multiple of 16), laid out for gated_i8 (not for matmul_i8). */
FFN24_API int64_t i8_weight_bytes(int64_t K, int64_t N);   /* or -1 for sizes out of range */
FFN24_API int i8_weight(const void* W, int64_t K, int64_t N, int halves, void* out, void* stream);
/* X (bf16 [T][K]) -> codes [T][K], scales fp32 [T] */
FFN24_API int quantise_i8(const void* X, int64_t T, int64_t K, void* codes, float* scales, void* stream);
/* Y [T][N] (bf16) from codes and scales of quantise_i8 and weights of i8_weight.  It has no scratch, so a long reduction whose result has few tiles is not split over workgroups
 * as linear_i8 splits it; the results are the same, the time is not (64 tokens, K 16384, N 4096: 39 us, linear_i8 with its quantisation 26). */
FFN24_API int matmul_i8(const void* codes, const float* scales, int64_t T, const void* weight, int64_t K, int64_t N, void* Y, void* stream);
/* The two in one call: Y from bf16 X.  scratch: linear_i8_scratch(T, K, N) bytes, used until the call's last kernel has run. */
FFN24_API int64_t linear_i8_scratch(int64_t T, int64_t K, int64_t N);   /* or -1 */
FFN24_API int linear_i8(const void* X, int64_t T, const void* weight, int64_t K, int64_t N, void* Y, void* scratch, void* stream);

/* The gated block on int8 weights: G, U in fp32 from such products of X and [Wg | Wu];  h = a(G) U;  sh[t] = max_f |h[t][f]| * (1 / 127) (1 if zero);
 * H8 = rint(bf16(h) / sh), held to -127 .. 127;  Y = bf16(sh[t] sw[d] sum_f H8 Wd8).  T, D, F, gate as for gated_ctx_create, F at most 2^17.
 * Workspace: T (D + 3 F + 12) bytes, the weights (3 D F and a little) and what a split reduction takes (some tens of MiB at most).  gated_i8_set_weights quantises Wgu [D][2 F] and Wd [F][D] (bf16) into the context, which
 * does not need them afterwards; gated_i8_fwd before it returns FFN24_ERR_STATE. */
typedef struct gated_i8_ctx gated_i8_ctx;
FFN24_API int gated_i8_ctx_create(gated_i8_ctx** out, int64_t T, int64_t D, int64_t F, ffn24_gate gate);
FFN24_API int gated_i8_ctx_destroy(gated_i8_ctx* ctx);
FFN24_API int gated_i8_set_weights(gated_i8_ctx* ctx, const void* Wgu, const void* Wd, void* stream);
FFN24_API int gated_i8_fwd(gated_i8_ctx* ctx, const void* X, int64_t T, void* Y, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FFN24_BLOCK_H */
