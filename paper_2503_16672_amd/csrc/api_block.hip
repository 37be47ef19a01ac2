// C ABI of the operators around the feed-forward block (ffn24_block.h): argument checks, workspaces, and the kernel sequences.
#include <hip/hip_runtime.h>
#include <new>
#include "../../include/ffn24_block.h"
#include "launch_block.hpp"

using namespace ffn24;

namespace {
constexpr int64_t MAX_TOKENS = 1 << 24;   // (row counts and grids stay within 32 bits)
constexpr int64_t MAX_CTX_TOKENS = 1 << 20, MAX_WIDTH = 1 << 18;

template <class... P> bool misaligned(const P*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 15u) != 0; }
int done(int rc) { return rc ? FFN24_ERR_HIP : FFN24_OK; }

struct GateCoefficients { float c1, c3; };
constexpr float GELU_C1 = 1.5957691216057308f;   // 2 sqrt(2 / pi)
GateCoefficients coefficients(ffn24_gate g) { return g == FFN24_GATE_SILU ? GateCoefficients{1.f, 0.f} : GateCoefficients{GELU_C1, GELU_C1 * 0.044715f}; }

// the checks that the contexts share
int check_sizes(int64_t T, int64_t D, int64_t F, ffn24_gate gate) {
  if (gate != FFN24_GATE_SILU && gate != FFN24_GATE_GELU_TANH) return FFN24_ERR_DTYPE;
  if (T < 1 || T > MAX_CTX_TOKENS || D < 64 || D > MAX_WIDTH || D % 64 || F < 64 || F > MAX_WIDTH || F % 64) return FFN24_ERR_SHAPE;
  return FFN24_OK;
}
int check_device(int device) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return FFN24_ERR_HIP;
  return dev == device ? FFN24_OK : FFN24_ERR_STATE;
}
}  // namespace

struct gated_ctx {
  int64_t T, D, F;
  GateCoefficients gate;
  int training, device;
  int64_t fwd_T;               // tokens of the last forward, -1: none yet
  void *H, *GU, *GUx, *dGU;    // [T][F] bf16; in training G and U ([T][2 F] bf16 and bytes) and their gradients [T][2 F]
  void *Wgu_p;                 // in training: Wgu in panel form, made by a backward that reads it so
  Scratch scratch;             // sums over parts of a reduction
};

struct gated_i8_ctx {
  int64_t T, D, F;
  GateCoefficients gate;
  int device, have_weights;
  void *Wgu, *Wd;              // laid out by i8_weight
  void *X8, *H, *H8;           // [T][D] codes, [T][F] bf16, [T][F] codes
  float *sx, *sh; uint32_t* tops;
  Scratch scratch;             // sums over parts of a reduction
};

namespace {
constexpr int64_t MAX_I8_K = 1 << 17, MAX_I8_N = 1 << 20;
bool i8_sizes(int64_t K, int64_t N) { return K >= 16 && K <= MAX_I8_K && K % 16 == 0 && N >= 8 && N <= MAX_I8_N && N % 8 == 0; }
bool i8_rows(int64_t T, int64_t K) { return T >= 0 && T <= MAX_CTX_TOKENS && K >= 16 && K <= MAX_I8_K && K % 16 == 0; }
int64_t up16(int64_t x) { return (x + 15) & ~(int64_t)15; }
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

int gated_ctx_create(gated_ctx** out, int64_t T, int64_t D, int64_t F, ffn24_gate gate, int flags) {
  if (!out) return FFN24_ERR_NULL;
  if (int rc = check_sizes(T, D, F, gate)) return rc;
  if (flags & ~FFN24_TRAINING) return FFN24_ERR_STATE;
  gated_ctx* c = new (std::nothrow) gated_ctx();
  if (!c) return FFN24_ERR_HIP;
  c->T = T; c->D = D; c->F = F; c->gate = coefficients(gate);
  c->training = flags & FFN24_TRAINING; c->fwd_T = -1;
  const size_t tf = (size_t)T * (size_t)F;
  bool ok = hipGetDevice(&c->device) == hipSuccess && hipMalloc(&c->H, 2 * tf) == hipSuccess;
  if (ok && c->training) ok = hipMalloc(&c->GU, 4 * tf) == hipSuccess && hipMalloc(&c->GUx, 2 * tf) == hipSuccess && hipMalloc(&c->dGU, 4 * tf) == hipSuccess;
  if (ok && c->training && gated_dx_panels((int)T, (int)D, (int)F)) ok = hipMalloc(&c->Wgu_p, gated_panel_bytes((int)D, (int)(2 * F))) == hipSuccess;
  const size_t few = few_gated_scratch((int)T, (int)D, (int)F), most = gated_scratch((int)T, (int)D, (int)F, c->training);
  c->scratch.bytes = few > most ? few : most;
  if (ok) ok = hipMalloc(&c->scratch.p, c->scratch.bytes) == hipSuccess;
  if (!ok) {
    (void)hipGetLastError();
    gated_ctx_destroy(c);
    return FFN24_ERR_HIP;
  }
  *out = c;
  return FFN24_OK;
}

int gated_ctx_destroy(gated_ctx* c) {
  if (!c) return FFN24_OK;
  int bad = 0;
  for (void* p : {c->H, c->GU, c->GUx, c->dGU, c->Wgu_p, c->scratch.p}) if (p && hipFree(p) != hipSuccess) bad = 1;
  delete c;
  return bad ? FFN24_ERR_HIP : FFN24_OK;
}

int gated_fwd(gated_ctx* c, const void* X, int64_t T, const void* Wgu, const void* Wd, void* Y, void* stream) {
  if (!c) return FFN24_ERR_NULL;
  if (T < 0 || T > c->T) return FFN24_ERR_SHAPE;
  if (T > 0 && (!X || !Wgu || !Wd || !Y)) return FFN24_ERR_NULL;
  if (misaligned(X, Wgu, Wd, Y)) return FFN24_ERR_ALIGN;
  if (int rc = check_device(c->device)) return rc;
  c->fwd_T = -1;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int t = (int)T, D = (int)c->D, F = (int)c->F;
  if (T > 0) {
    const bool few = few_tokens(t, D, F);        // (the kernel for few tokens keeps nothing for a backward)
    float* parts = static_cast<float*>(c->scratch.p);
    if (few && !c->training ? launch_few_gated_up(X, Wgu, t, D, F, c->gate.c1, c->gate.c3, c->H, parts, s)
                            : launch_gated_up(X, Wgu, t, D, F, c->gate.c1, c->gate.c3, c->H, c->GU, c->GUx, s)) return FFN24_ERR_HIP;
    if (few ? launch_few_gated_down(c->H, Wd, t, D, F, Y, parts, s) : launch_gated_down(c->H, Wd, t, D, F, Y, c->scratch, s)) return FFN24_ERR_HIP;
  }
  c->fwd_T = T;
  return FFN24_OK;
}

int gated_bwd(gated_ctx* c, const void* dY, const void* X, const void* Wgu, const void* Wd, void* dX, void* dWgu, void* dWd, void* stream) {
  if (!c) return FFN24_ERR_NULL;
  if (!c->training || c->fwd_T < 0) return FFN24_ERR_STATE;
  if (!dWgu || !dWd || (c->fwd_T > 0 && (!dY || !X || !Wgu || !Wd || !dX))) return FFN24_ERR_NULL;
  if (misaligned(dY, X, Wgu, Wd, dX, dWgu, dWd)) return FFN24_ERR_ALIGN;
  if (int rc = check_device(c->device)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int t = (int)c->fwd_T, D = (int)c->D, F = (int)c->F;
  if (t == 0) return done(launch_zero(dWgu, (size_t)4 * D * F, s) || launch_zero(dWd, (size_t)2 * D * F, s));
  const bool panels = c->Wgu_p && gated_dx_panels(t, D, F);
  if (panels) {
    if (launch_gated_panels(Wgu, D, F, c->Wgu_p, s)) return FFN24_ERR_HIP;
    Wgu = c->Wgu_p;
  }
  if (launch_gated_dgate(dY, Wd, c->GU, c->GUx, t, D, F, c->gate.c1, c->gate.c3, c->dGU, s)) return FFN24_ERR_HIP;
  return done(launch_gated_grads(X, dY, c->H, c->dGU, Wgu, panels, t, D, F, dX, dWgu, dWd, c->scratch, s));
}

int64_t i8_weight_bytes(int64_t K, int64_t N) { return i8_sizes(K, N) ? i8_weight_size(K, N) : -1; }

int i8_weight(const void* W, int64_t K, int64_t N, int halves, void* out, void* stream) {
  if (!i8_sizes(K, N) || (halves && N % 16)) return FFN24_ERR_SHAPE;
  if (!W || !out) return FFN24_ERR_NULL;
  if (misaligned(W, out)) return FFN24_ERR_ALIGN;
  return done(launch_i8_weight(W, (int)K, (int)N, halves != 0, out, static_cast<hipStream_t>(stream)));
}

int quantise_i8(const void* X, int64_t T, int64_t K, void* codes, float* scales, void* stream) {
  if (!i8_rows(T, K)) return FFN24_ERR_SHAPE;
  if (T == 0) return FFN24_OK;
  if (!X || !codes || !scales) return FFN24_ERR_NULL;
  if (misaligned(X, codes, scales)) return FFN24_ERR_ALIGN;
  return done(launch_quantise_i8(X, (int)T, (int)K, false, codes, scales, nullptr, static_cast<hipStream_t>(stream)));
}

int matmul_i8(const void* codes, const float* scales, int64_t T, const void* weight, int64_t K, int64_t N, void* Y, void* stream) {
  if (!i8_rows(T, K) || !i8_sizes(K, N)) return FFN24_ERR_SHAPE;
  if (T == 0) return FFN24_OK;
  if (!codes || !scales || !weight || !Y) return FFN24_ERR_NULL;
  if (misaligned(codes, scales, weight, Y)) return FFN24_ERR_ALIGN;
  return done(launch_matmul_i8(codes, false, scales, (int)T, i8_layout(weight, (int)K, (int)N), Y, Scratch{}, static_cast<hipStream_t>(stream)));
}

int64_t linear_i8_scratch(int64_t T, int64_t K, int64_t N) {
  return i8_rows(T, K) && i8_sizes(K, N) ? T * K + up16(4 * T) + (T > 0 ? (int64_t)matmul_i8_scratch((int)T, (int)K, (int)N) : 0) : -1;
}

int linear_i8(const void* X, int64_t T, const void* weight, int64_t K, int64_t N, void* Y, void* scratch, void* stream) {
  if (!i8_rows(T, K) || !i8_sizes(K, N)) return FFN24_ERR_SHAPE;
  if (T == 0) return FFN24_OK;
  if (!X || !weight || !Y || !scratch) return FFN24_ERR_NULL;
  if (misaligned(X, weight, Y, scratch)) return FFN24_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (few_i8_fuses((int)T, (int)K)) return done(launch_few_linear_i8(X, (int)T, i8_layout(weight, (int)K, (int)N), Y, s));
  float* sx = reinterpret_cast<float*>(static_cast<char*>(scratch) + T * K);
  if (launch_quantise_i8(X, (int)T, (int)K, false, scratch, sx, nullptr, s)) return FFN24_ERR_HIP;
  const Scratch rest{static_cast<char*>(scratch) + T * K + up16(4 * T), matmul_i8_scratch((int)T, (int)K, (int)N)};
  return done(launch_matmul_i8(scratch, false, sx, (int)T, i8_layout(weight, (int)K, (int)N), Y, rest, s));
}

int gated_i8_ctx_create(gated_i8_ctx** out, int64_t T, int64_t D, int64_t F, ffn24_gate gate) {
  if (!out) return FFN24_ERR_NULL;
  if (int rc = check_sizes(T, D, F, gate)) return rc;
  if (D > MAX_I8_K || F > MAX_I8_K) return FFN24_ERR_SHAPE;
  gated_i8_ctx* c = new (std::nothrow) gated_i8_ctx();
  if (!c) return FFN24_ERR_HIP;
  c->T = T; c->D = D; c->F = F; c->gate = coefficients(gate);
  const size_t tf = (size_t)T * (size_t)F, t4 = 4 * (size_t)T, few = few_i8_tops((int)T, (int)F), tops = few > t4 ? few : t4;
  c->scratch.bytes = gated_i8_scratch((int)T, (int)D, (int)F);
  const bool ok = hipGetDevice(&c->device) == hipSuccess && (!c->scratch.bytes || hipMalloc(&c->scratch.p, c->scratch.bytes) == hipSuccess) &&
                  hipMalloc(&c->Wgu, (size_t)i8_weight_size(D, 2 * F)) == hipSuccess &&
                  hipMalloc(&c->Wd, (size_t)i8_weight_size(F, D)) == hipSuccess && hipMalloc(&c->X8, (size_t)i8_panel_size(T, D)) == hipSuccess && hipMalloc(&c->H, 2 * tf) == hipSuccess &&
                  hipMalloc(&c->H8, (size_t)i8_panel_size(T, F)) == hipSuccess && hipMalloc(reinterpret_cast<void**>(&c->sx), t4) == hipSuccess &&
                  hipMalloc(reinterpret_cast<void**>(&c->sh), t4) == hipSuccess && hipMalloc(reinterpret_cast<void**>(&c->tops), tops) == hipSuccess;
  if (!ok) {
    (void)hipGetLastError();
    gated_i8_ctx_destroy(c);
    return FFN24_ERR_HIP;
  }
  *out = c;
  return FFN24_OK;
}

int gated_i8_ctx_destroy(gated_i8_ctx* c) {
  if (!c) return FFN24_OK;
  int bad = 0;
  void* bufs[] = {c->Wgu, c->Wd, c->X8, c->H, c->H8, c->sx, c->sh, c->tops, c->scratch.p};
  for (void* p : bufs) if (p && hipFree(p) != hipSuccess) bad = 1;
  delete c;
  return bad ? FFN24_ERR_HIP : FFN24_OK;
}

int gated_i8_set_weights(gated_i8_ctx* c, const void* Wgu, const void* Wd, void* stream) {
  if (!c || !Wgu || !Wd) return FFN24_ERR_NULL;
  if (misaligned(Wgu, Wd)) return FFN24_ERR_ALIGN;
  if (int rc = check_device(c->device)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  c->have_weights = 0;
  if (launch_i8_weight(Wgu, (int)c->D, (int)(2 * c->F), true, c->Wgu, s) || launch_i8_weight(Wd, (int)c->F, (int)c->D, false, c->Wd, s)) return FFN24_ERR_HIP;
  c->have_weights = 1;
  return FFN24_OK;
}

int gated_i8_fwd(gated_i8_ctx* c, const void* X, int64_t T, void* Y, void* stream) {
  if (!c) return FFN24_ERR_NULL;
  if (T < 0 || T > c->T) return FFN24_ERR_SHAPE;
  if (!c->have_weights) return FFN24_ERR_STATE;
  if (T == 0) return FFN24_OK;
  if (!X || !Y) return FFN24_ERR_NULL;
  if (misaligned(X, Y)) return FFN24_ERR_ALIGN;
  if (int rc = check_device(c->device)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int t = (int)T, D = (int)c->D, F = (int)c->F;
  if (few_gated_i8_tokens(t, D, F))
    return done(launch_few_gated_i8(X, t, i8_layout(c->Wgu, D, 2 * F), i8_layout(c->Wd, F, D), c->gate.c1, c->gate.c3, c->X8, c->sx, c->H, c->tops, c->H8, c->sh, Y, s));
  if (launch_quantise_i8(X, t, D, true, c->X8, c->sx, c->tops, s)) return FFN24_ERR_HIP;
  if (launch_gated_up_i8(c->X8, c->sx, t, i8_layout(c->Wgu, D, 2 * F), c->gate.c1, c->gate.c3, c->H, c->tops, s)) return FFN24_ERR_HIP;
  if (launch_quantise_i8_given(c->H, c->tops, t, F, c->H8, c->sh, s)) return FFN24_ERR_HIP;
  return done(launch_matmul_i8(c->H8, true, c->sh, t, i8_layout(c->Wd, F, D), Y, c->scratch, s));
}

}  // extern "C"
