// C ABI of serving with mx4 weights and with experts (ffn24_serve.h): argument checks, workspaces, and the kernel sequences.
#include <hip/hip_runtime.h>
#include <new>
#include "../../include/ffn24_serve.h"
#include "launch_block.hpp"
#include "mx4_rule.hpp"

using namespace ffn24;

namespace {
constexpr int64_t MAX_ROWS = 1 << 24, MAX_TOKENS = 1 << 20, MAX_K = 1 << 17, MAX_N = 1 << 20, MAX_WIDTH = 1 << 17, MAX_MOE_D = 1 << 14, MAX_MOE_F = 1 << 16;

template <class... P> bool misaligned(const P*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 15u) != 0; }
int done(int rc) { return rc ? FFN24_ERR_HIP : FFN24_OK; }
int64_t up16(int64_t x) { return (x + 15) / 16 * 16; }

struct GateCoefficients { float c1, c3; };
constexpr float GELU_C1 = 1.5957691216057308f;   // 2 sqrt(2 / pi)
GateCoefficients coefficients(ffn24_gate g) { return g == FFN24_GATE_SILU ? GateCoefficients{1.f, 0.f} : GateCoefficients{GELU_C1, GELU_C1 * 0.044715f}; }
bool gate_known(ffn24_gate g) { return g == FFN24_GATE_SILU || g == FFN24_GATE_GELU_TANH; }
bool dtype_known(ffn24_norm_dtype d) { return d == FFN24_NORM_BF16 || d == FFN24_NORM_F32; }
bool sizes(int64_t K, int64_t N) { return K >= 32 && K <= MAX_K && K % 32 == 0 && N >= 8 && N <= MAX_N && N % 8 == 0; }
bool tokens(int64_t T) { return T >= 0 && T <= MAX_TOKENS; }
bool width(int64_t x, int64_t most) { return x >= 64 && x <= most && x % 64 == 0; }

int check_device(int device) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return FFN24_ERR_HIP;
  return dev == device ? FFN24_OK : FFN24_ERR_STATE;
}
bool cleared(void** p, int64_t bytes) { return hipMalloc(p, (size_t)bytes) == hipSuccess && hipMemset(*p, 0, (size_t)bytes) == hipSuccess; }
}  // namespace

struct gated_mx4_ctx {
  int64_t T, D, F;
  GateCoefficients gate;
  int device, have_weights;
  void *Wgu, *Wd, *X, *H;      // in the operand form
  Scratch scratch;             // sums over parts of a reduction
};

struct moe_ctx {
  int64_t T, D, F, E, k;
  GateCoefficients gate;
  int renormalise, device, have_weights;
  MoeWeights w;
  void *Wr, *up, *down, *X, *parts, *plan, *sums, *H, *picks, *shares;   // X, H: tokens and activations as mx4 (H: or two bf16 a value)
};

extern "C" {

int quantise_mx4(const void* X, int64_t T, int64_t K, ffn24_norm_dtype dtype, void* codes, void* scales, void* stream) {
  if (!dtype_known(dtype)) return FFN24_ERR_DTYPE;
  if (T < 0 || T > MAX_ROWS || !sizes(K, 8)) return FFN24_ERR_SHAPE;
  if (T == 0) return FFN24_OK;
  if (!X || !codes || !scales) return FFN24_ERR_NULL;
  if (misaligned(X, codes, scales)) return FFN24_ERR_ALIGN;
  return done(launch_quantise_mx4(X, dtype == FFN24_NORM_F32, T, K, codes, scales, static_cast<hipStream_t>(stream)));
}

int dequantise_mx4(const void* codes, const void* scales, int64_t T, int64_t K, ffn24_norm_dtype dtype, void* Y, void* stream) {
  if (!dtype_known(dtype)) return FFN24_ERR_DTYPE;
  if (T < 0 || T > MAX_ROWS || !sizes(K, 8)) return FFN24_ERR_SHAPE;
  if (T == 0) return FFN24_OK;
  if (!codes || !scales || !Y) return FFN24_ERR_NULL;
  if (misaligned(codes, scales, Y)) return FFN24_ERR_ALIGN;
  return done(launch_dequantise_mx4(codes, scales, dtype == FFN24_NORM_F32, T, K, Y, static_cast<hipStream_t>(stream)));
}

int64_t mx4_weight_bytes(int64_t K, int64_t N) { return sizes(K, N) ? mx4_operand_size(N, K) : -1; }

int mx4_weight(const void* W, int64_t K, int64_t N, int reserved, void* out, void* stream) {
  if (!sizes(K, N) || reserved) return FFN24_ERR_SHAPE;
  if (!W || !out) return FFN24_ERR_NULL;
  if (misaligned(W, out)) return FFN24_ERR_ALIGN;
  return done(launch_mx4_weight(W, (int)K, (int)N, false, 1, out, static_cast<hipStream_t>(stream)));
}

int mx4_weight_codes(const void* codes, const void* scales, int64_t K, int64_t N, int reserved, void* out, void* stream) {
  if (!sizes(K, N) || reserved) return FFN24_ERR_SHAPE;
  if (!codes || !scales || !out) return FFN24_ERR_NULL;
  if (misaligned(codes, scales, out)) return FFN24_ERR_ALIGN;
  return done(launch_mx4_weight_codes(codes, scales, (int)K, (int)N, out, static_cast<hipStream_t>(stream)));
}

int64_t linear_mx4_scratch(int64_t T, int64_t K, int64_t N) {
  if (!tokens(T) || !sizes(K, N)) return -1;
  if (T == 0 || mx4_few_fused((int)T, (int)K)) return 0;
  return up16(mx4_operand_size(T, K)) + (mx4_few((int)T, (int)K, (int)N) ? 0 : (int64_t)mx4_split_scratch((int)N, (int)T, (int)K));
}

int linear_mx4(const void* X, int64_t T, const void* weight, int64_t K, int64_t N, void* Y, void* scratch, void* stream) {
  if (!tokens(T) || !sizes(K, N)) return FFN24_ERR_SHAPE;
  if (T == 0) return FFN24_OK;
  const bool fused = mx4_few_fused((int)T, (int)K);
  if (!X || !weight || !Y || (!scratch && !fused)) return FFN24_ERR_NULL;
  if (misaligned(X, weight, Y, scratch)) return FFN24_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int t = (int)T, k = (int)K, n = (int)N;
  const Mx4Operand w = mx4_operand(weight, n, k);
  if (fused) return done(launch_few_mx4_rows(w, k, n, X, nullptr, t, Y, s));
  const Mx4Operand x = mx4_operand(scratch, t, k);
  if (launch_mx4_tokens(X, t, k, x, s)) return FFN24_ERR_HIP;
  if (mx4_few(t, k, n)) return done(launch_few_mx4_rows(w, k, n, nullptr, &x, t, Y, s));
  return done(launch_mx4_product(w, n, x, t, Y, Scratch{static_cast<char*>(scratch) + up16(mx4_operand_size(T, K)), mx4_split_scratch(n, t, k)}, s));
}

int gated_mx4_ctx_create(gated_mx4_ctx** out, int64_t T, int64_t D, int64_t F, ffn24_gate gate) {
  if (!out) return FFN24_ERR_NULL;
  if (!gate_known(gate)) return FFN24_ERR_DTYPE;
  if (T < 1 || T > MAX_TOKENS || !width(D, MAX_WIDTH) || !width(F, MAX_WIDTH)) return FFN24_ERR_SHAPE;
  gated_mx4_ctx* c = new (std::nothrow) gated_mx4_ctx();
  if (!c) return FFN24_ERR_HIP;
  c->T = T; c->D = D; c->F = F; c->gate = coefficients(gate);
  for (int64_t t = 64; t <= (T + 63) / 64 * 64 && t * D <= MX4_SPLIT_MOST; t += 64) {
    const size_t y = mx4_split_scratch((int)D, (int)t, (int)F);
    if (y > c->scratch.bytes) c->scratch.bytes = y;
  }
  // (H's k beyond F are zero for good: no kernel writes them)
  const bool ok = hipGetDevice(&c->device) == hipSuccess && hipMalloc(&c->Wgu, (size_t)mx4_operand_size(2 * F, D)) == hipSuccess &&
                  hipMalloc(&c->Wd, (size_t)mx4_operand_size(D, F)) == hipSuccess && hipMalloc(&c->X, (size_t)mx4_operand_size(T, D)) == hipSuccess &&
                  (!c->scratch.bytes || hipMalloc(&c->scratch.p, c->scratch.bytes) == hipSuccess) && cleared(&c->H, mx4_operand_size(T, F)) && hipDeviceSynchronize() == hipSuccess;
  if (!ok) {
    (void)hipGetLastError();
    gated_mx4_ctx_destroy(c);
    return FFN24_ERR_HIP;
  }
  *out = c;
  return FFN24_OK;
}

int gated_mx4_ctx_destroy(gated_mx4_ctx* c) {
  if (!c) return FFN24_OK;
  int bad = 0;
  for (void* p : {c->Wgu, c->Wd, c->X, c->H, c->scratch.p}) if (p && hipFree(p) != hipSuccess) bad = 1;
  delete c;
  return bad ? FFN24_ERR_HIP : FFN24_OK;
}

int gated_mx4_set_weights(gated_mx4_ctx* c, const void* Wgu, const void* Wd, void* stream) {
  if (!c || !Wgu || !Wd) return FFN24_ERR_NULL;
  if (misaligned(Wgu, Wd)) return FFN24_ERR_ALIGN;
  if (int rc = check_device(c->device)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  c->have_weights = 0;
  if (launch_mx4_weight(Wgu, (int)c->D, (int)(2 * c->F), true, 1, c->Wgu, s) || launch_mx4_weight(Wd, (int)c->F, (int)c->D, false, 1, c->Wd, s)) return FFN24_ERR_HIP;
  c->have_weights = 1;
  return FFN24_OK;
}

int gated_mx4_fwd(gated_mx4_ctx* c, const void* X, int64_t T, void* Y, void* stream) {
  if (!c) return FFN24_ERR_NULL;
  if (T < 0 || T > c->T) return FFN24_ERR_SHAPE;
  if (!c->have_weights) return FFN24_ERR_STATE;
  if (T == 0) return FFN24_OK;
  if (!X || !Y) return FFN24_ERR_NULL;
  if (misaligned(X, Y)) return FFN24_ERR_ALIGN;
  if (int rc = check_device(c->device)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int t = (int)T, D = (int)c->D, F = (int)c->F;
  const Mx4Operand wgu = mx4_operand(c->Wgu, 2 * F, D), wd = mx4_operand(c->Wd, D, F), x = mx4_operand(c->X, (int)c->T, D), h = mx4_operand(c->H, (int)c->T, F);
  const bool few = mx4_few_gated(t), fused = few && mx4_few_fused(t, D);
  if (!fused && launch_mx4_tokens(X, t, D, x, s)) return FFN24_ERR_HIP;
  if (few ? launch_few_mx4_up(wgu, X, fused ? nullptr : &x, t, D, F, c->gate.c1, c->gate.c3, h, s)
          : launch_mx4_gated_up(wgu, F, x, t, c->gate.c1, c->gate.c3, h, s)) return FFN24_ERR_HIP;
  if (mx4_few(t, F, D)) return done(launch_few_mx4_rows(wd, F, D, nullptr, &h, t, Y, s));
  return done(launch_mx4_product(wd, D, h, t, Y, c->scratch, s));
}

int moe_ctx_create(moe_ctx** out, int64_t T, int64_t D, int64_t F, int64_t E, int64_t k, ffn24_gate gate, int renormalise, ffn24_experts type) {
  if (!out) return FFN24_ERR_NULL;
  if (!gate_known(gate) || (type != FFN24_EXPERTS_BF16 && type != FFN24_EXPERTS_MX4)) return FFN24_ERR_DTYPE;
  if (T < 1 || T > MOE_TOKENS || !width(D, MAX_MOE_D) || !width(F, MAX_MOE_F) || E < 1 || E > MOE_MAX_E || k < 1 || k > E || k > MOE_MAX_K) return FFN24_ERR_SHAPE;
  moe_ctx* c = new (std::nothrow) moe_ctx();
  if (!c) return FFN24_ERR_HIP;
  c->T = T; c->D = D; c->F = F; c->E = E; c->k = k; c->gate = coefficients(gate); c->renormalise = renormalise != 0;
  const bool mx4 = type == FFN24_EXPERTS_MX4;
  const int64_t up = mx4 ? mx4_operand_size(2 * F, D) : bf16_operand_size(2 * F, D), down = mx4 ? mx4_operand_size(D, F) : bf16_operand_size(D, F);
  // (of mx4 rows the k beyond D and F are zero for good: no kernel writes them)
  const bool ok = hipGetDevice(&c->device) == hipSuccess && hipMalloc(&c->Wr, (size_t)bf16_operand_size(E, D)) == hipSuccess && hipMalloc(&c->up, (size_t)(E * up)) == hipSuccess &&
                  hipMalloc(&c->down, (size_t)(E * down)) == hipSuccess && hipMalloc(&c->parts, moe_parts_size((int)T, (int)D, (int)E)) == hipSuccess &&
                  hipMalloc(&c->picks, (size_t)(4 * T * k)) == hipSuccess && hipMalloc(&c->shares, (size_t)(4 * T * k)) == hipSuccess &&
                  hipMalloc(&c->sums, (size_t)(4 * MOE_SPLITS * T * D)) == hipSuccess && cleared(&c->plan, (int64_t)moe_plan_size()) &&
                  (!mx4 || cleared(&c->X, mx4_operand_size(T, D))) && cleared(&c->H, mx4 ? mx4_operand_size(T * k, F) : 4 * ((T * k + 15) / 16 * 16) * F) && hipDeviceSynchronize() == hipSuccess;
  if (!ok) {
    (void)hipGetLastError();
    moe_ctx_destroy(c);
    return FFN24_ERR_HIP;
  }
  const Mx4Operand u = mx4_operand(c->up, (int)(2 * F), (int)D), d = mx4_operand(c->down, (int)D, (int)F);
  c->w = MoeWeights{mx4, c->up, c->down, (size_t)up, (size_t)down, (size_t)(u.scales - u.codes), (size_t)(d.scales - d.codes)};
  *out = c;
  return FFN24_OK;
}

int moe_ctx_destroy(moe_ctx* c) {
  if (!c) return FFN24_OK;
  int bad = 0;
  for (void* p : {c->Wr, c->up, c->down, c->X, c->parts, c->plan, c->sums, c->H, c->picks, c->shares}) if (p && hipFree(p) != hipSuccess) bad = 1;
  delete c;
  return bad ? FFN24_ERR_HIP : FFN24_OK;
}

int moe_set_weights(moe_ctx* c, const void* Wr, const void* Wgu, const void* Wd, void* stream) {
  if (!c || !Wr || !Wgu || !Wd) return FFN24_ERR_NULL;
  if (misaligned(Wr, Wgu, Wd)) return FFN24_ERR_ALIGN;
  if (int rc = check_device(c->device)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int D = (int)c->D, F = (int)c->F, E = (int)c->E;
  c->have_weights = 0;
  const auto lay_out = c->w.mx4 ? launch_mx4_weight : launch_bf16_weight;
  if (launch_bf16_weight(Wr, D, E, false, 1, c->Wr, s) || lay_out(Wgu, D, 2 * F, true, E, c->up, s) || lay_out(Wd, F, D, false, E, c->down, s)) return FFN24_ERR_HIP;
  c->have_weights = 1;
  return FFN24_OK;
}

int moe_fwd(moe_ctx* c, const void* X, int64_t T, void* Y, void* experts, void* shares, void* stream) {
  if (!c) return FFN24_ERR_NULL;
  if (T < 0 || T > c->T) return FFN24_ERR_SHAPE;
  if (!c->have_weights) return FFN24_ERR_STATE;
  if (T == 0) return FFN24_OK;
  if (!X || !Y || (experts == nullptr) != (shares == nullptr)) return FFN24_ERR_NULL;
  if (misaligned(X, Y, experts, shares)) return FFN24_ERR_ALIGN;
  if (int rc = check_device(c->device)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const MoeCall m{X, c->Wr, (int)T, (int)c->D, (int)c->F, (int)c->E, (int)c->k, c->renormalise != 0, c->parts, c->plan, static_cast<int*>(experts ? experts : c->picks),
                  static_cast<float*>(experts ? shares : c->shares), c->H, (int)(c->T * c->k), c->sums, Y};
  const Mx4Operand x = mx4_operand(c->X, (int)c->T, (int)c->D);
  if (launch_moe_route(m, c->w.mx4 ? &x : nullptr, s)) return FFN24_ERR_HIP;
  return done(launch_moe_experts(m, c->w, &x, c->gate.c1, c->gate.c3, s));
}

}  // extern "C"
