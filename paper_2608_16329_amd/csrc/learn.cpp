// C ABI of the learning operators (declared in include/mlip.h): contexts,
// argument checks, workspace, and the launches of their kernels.
#include <algorithm>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "learn_host.h"

using namespace mlip;

namespace {

mlip_status check_route(mlip_learn* ctx, const mlip_route_params* p, int64_t n, const void* logits,
                        const int32_t* kinds, const uint8_t* allowed) {
  if (!p) return fail(ctx, MLIP_E_ARG, "NULL parameters");
  if (p->n_experts < 1 || p->n_experts > kMaxExperts) return fail(ctx, MLIP_E_ARG, "n_experts must be in 1..256");
  if (p->top_k < 1 || p->top_k > kMaxTopK || p->top_k > p->n_experts)
    return fail(ctx, MLIP_E_ARG, "top_k must be in 1..16 and at most n_experts");
  if (p->gates != MLIP_GATES_CHOSEN && p->gates != MLIP_GATES_ALL) return fail(ctx, MLIP_E_ARG, "unknown gates");
  if (p->dtype != MLIP_F32 && p->dtype != MLIP_BF16) return fail(ctx, MLIP_E_ARG, "unknown dtype");
  if (n < 0 || n >= (int64_t(1) << 31) / p->top_k) return fail(ctx, MLIP_E_ARG, "n outside [0, 2^31 / top_k)");
  if (p->row_stride < p->n_experts || p->row_stride > (int64_t(1) << 31))
    return fail(ctx, MLIP_E_ARG, "row_stride must be in n_experts..2^31");
  if (!kinds != !allowed) return fail(ctx, MLIP_E_ARG, "kinds and allowed go together");
  if (kinds ? p->n_kinds < 1 : p->n_kinds != 0) return fail(ctx, MLIP_E_ARG, "n_kinds must fit allowed");
  if (n > 0 && !logits) return fail(ctx, MLIP_E_ARG, "NULL logits");
  return MLIP_OK;
}

RouteArgs route_args(const mlip_route_params* p, int64_t n, const void* logits, const int32_t* kinds,
                     const uint8_t* allowed) {
  RouteArgs a{};
  a.n = n;
  a.stride = p->row_stride;
  a.E = p->n_experts;
  a.K = p->top_k;
  a.n_kinds = p->n_kinds;
  a.bf16 = p->dtype == MLIP_BF16;
  a.all = p->gates == MLIP_GATES_ALL;
  a.logits = logits;
  a.kinds = kinds;
  a.allowed = allowed;
  return a;
}

bool heads_valid(const mlip_heads_params* p) {
  return p->n_experts >= 1 && p->n_experts <= kMaxExperts && p->width >= 1 && p->width <= kMaxHeadInputs &&
         p->hidden >= 1 && p->hidden <= kMaxHeadLayers;
}

int64_t head_values(const mlip_heads_params* p) {
  return 64 * int64_t(p->width) + 64 + int64_t(p->hidden - 1) * (64 * 64 + 64) + 64 + 1;
}

// The state arrays of a call: both moments, and exponents with 8 bits.
bool state_given(const mlip_adamw* h, const mlip_adamw_state* s) {
  return s && (h->elements == 0 || (s->m_dev && s->v_dev && (h->bits == 32 || (s->m_exp_dev && s->v_exp_dev))));
}

AdamArgs adam_args(const mlip_adamw* h, const mlip_adamw_state* from, const mlip_adamw_state* into) {
  AdamArgs a{};
  a.piece = h->d_pieces;
  a.pieces = h->pieces;
  a.bits = h->bits;
  a.m = from->m_dev;
  a.v = from->v_dev;
  a.m_exp = from->m_exp_dev;
  a.v_exp = from->v_exp_dev;
  a.new_m = into->m_dev;
  a.new_v = into->v_dev;
  a.new_m_exp = into->m_exp_dev;
  a.new_v_exp = into->v_exp_dev;
  return a;
}

}  // namespace

extern "C" {

mlip_status mlip_learn_create(void* hip_stream, mlip_learn** out) {
  t_learn_err.clear();
  if (!out) return fail<mlip_learn>(nullptr, MLIP_E_ARG, "NULL output pointer");
  *out = nullptr;
  mlip_learn* ctx = new (std::nothrow) mlip_learn();
  if (!ctx) return fail<mlip_learn>(nullptr, MLIP_E_OOM, "host allocation failed");
  ctx->stream = reinterpret_cast<hipStream_t>(hip_stream);
  if (hipGetDevice(&ctx->device) != hipSuccess ||
      hipDeviceGetAttribute(&ctx->n_cu, hipDeviceAttributeMultiprocessorCount, ctx->device) != hipSuccess) {
    (void)hipGetLastError();
    delete ctx;
    return fail<mlip_learn>(nullptr, MLIP_E_HIP, "no current HIP device");
  }
  *out = ctx;
  return MLIP_OK;
}

const char* mlip_learn_last_error(const mlip_learn* ctx) { return ctx ? ctx->err.c_str() : t_learn_err.c_str(); }

mlip_status mlip_learn_memory_bytes(const mlip_learn* ctx, size_t* bytes) {
  if (!ctx || !bytes) return MLIP_E_ARG;
  *bytes = ctx->cap_ws + ctx->kept_bytes;
  return MLIP_OK;
}

void mlip_learn_destroy(mlip_learn* ctx) {
  if (!ctx) return;
  (void)hipStreamSynchronize(ctx->stream);
  if (ctx->d_ws) (void)hipFree(ctx->d_ws);
  for (unsigned char* ws : ctx->kept) (void)hipFree(ws);
  (void)hipGetLastError();
  delete ctx;
}

mlip_status mlip_route(mlip_learn* ctx, const mlip_route_params* p, int64_t n, const void* logits_dev,
                       const int32_t* kinds_dev, const uint8_t* allowed_dev, int32_t* experts_dev, float* gates_dev,
                       int32_t* counts_dev, float* loss_dev) {
  if (!ctx) return MLIP_E_ARG;
  ctx->err.clear();
  if (elsewhere(ctx)) return fail(ctx, MLIP_E_ARG, kElsewhere);
  const mlip_status st = check_route(ctx, p, n, logits_dev, kinds_dev, allowed_dev);
  if (st != MLIP_OK) return st;
  if (!counts_dev || !loss_dev || (n > 0 && (!experts_dev || !gates_dev))) return fail(ctx, MLIP_E_ARG, "NULL output");
  RouteArgs a = route_args(p, n, logits_dev, kinds_dev, allowed_dev);
  a.experts = experts_dev;
  a.gates = gates_dev;
  a.counts = counts_dev;
  a.loss = loss_dev;
  const int blocks = route_blocks(n, a.E, ctx->n_cu);
  if (blocks > 1) {
    const mlip_status w = workspace(ctx, size_t(blocks) * size_t(2 * a.E + 1) * sizeof(float));
    if (w != MLIP_OK) return w;
    a.part_p = reinterpret_cast<float*>(ctx->d_ws);
    a.part_c = reinterpret_cast<int32_t*>(ctx->d_ws) + size_t(blocks) * size_t(a.E);
  }
  LEARN_HIP(ctx, launch_route(a, blocks, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_route_backward(mlip_learn* ctx, const mlip_route_params* p, int64_t n, const void* logits_dev,
                                const int32_t* kinds_dev, const uint8_t* allowed_dev, const int32_t* experts_dev,
                                const int32_t* counts_dev, const float* dgates_dev, const float* dloss_dev,
                                void* dlogits_dev) {
  if (!ctx) return MLIP_E_ARG;
  ctx->err.clear();
  if (elsewhere(ctx)) return fail(ctx, MLIP_E_ARG, kElsewhere);
  const mlip_status st = check_route(ctx, p, n, logits_dev, kinds_dev, allowed_dev);
  if (st != MLIP_OK) return st;
  if (n == 0) return MLIP_OK;
  if (!experts_dev || !counts_dev || !dlogits_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  RouteArgs a = route_args(p, n, logits_dev, kinds_dev, allowed_dev);
  a.experts = const_cast<int32_t*>(experts_dev);
  a.counts = const_cast<int32_t*>(counts_dev);
  a.dgates = dgates_dev;
  a.dloss = dloss_dev;
  a.dlogits = dlogits_dev;
  LEARN_HIP(ctx, launch_route_backward(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_group(mlip_learn* ctx, int64_t n_entries, int32_t n_experts, const int32_t* experts_dev,
                       int32_t* offsets_dev, int32_t* order_dev) {
  if (!ctx) return MLIP_E_ARG;
  ctx->err.clear();
  if (elsewhere(ctx)) return fail(ctx, MLIP_E_ARG, kElsewhere);
  if (n_experts < 1 || n_experts > kMaxExperts) return fail(ctx, MLIP_E_ARG, "n_experts must be in 1..256");
  if (n_entries < 0 || n_entries >= (int64_t(1) << 31)) return fail(ctx, MLIP_E_ARG, "n_entries outside [0, 2^31)");
  if (!offsets_dev || (n_entries > 0 && (!experts_dev || !order_dev))) return fail(ctx, MLIP_E_ARG, "NULL argument");
  const mlip_status w = workspace(ctx, group_ws_bytes(n_entries, n_experts));
  if (w != MLIP_OK) return w;
  LEARN_HIP(ctx, launch_group(experts_dev, n_entries, n_experts, offsets_dev, order_dev, ctx->d_ws, ctx->stream));
  return MLIP_OK;
}

size_t mlip_heads_weight_count(const mlip_heads_params* p) {
  return p && heads_valid(p) ? size_t(p->n_experts) * size_t(head_values(p)) : 0;
}

mlip_status mlip_heads(mlip_learn* ctx, const mlip_heads_params* p, int64_t n, const void* x_dev,
                       const float* weights_dev, const int32_t* offsets_dev, const int32_t* order_dev,
                       const float* gates_dev, const float* denergy_dev, float* energy_dev, void* dx_dev,
                       float* dweights_dev, float* dgates_dev) {
  if (!ctx) return MLIP_E_ARG;
  ctx->err.clear();
  if (elsewhere(ctx)) return fail(ctx, MLIP_E_ARG, kElsewhere);
  if (!p) return fail(ctx, MLIP_E_ARG, "NULL parameters");
  if (!heads_valid(p)) return fail(ctx, MLIP_E_ARG, "n_experts must be in 1..256, width in 1..1024, hidden in 1..8");
  if (p->top_k < 1 || p->top_k > kMaxTopK) return fail(ctx, MLIP_E_ARG, "top_k must be in 1..16");
  if (p->dtype != MLIP_F32 && p->dtype != MLIP_BF16) return fail(ctx, MLIP_E_ARG, "unknown dtype");
  if (n < 0 || n >= (int64_t(1) << 31) / p->top_k) return fail(ctx, MLIP_E_ARG, "n outside [0, 2^31 / top_k)");
  if (p->row_stride < p->width || p->row_stride > (int64_t(1) << 31))
    return fail(ctx, MLIP_E_ARG, "row_stride must be in width..2^31");
  if (n > 0 && !energy_dev && !dx_dev && !dweights_dev && !dgates_dev) return fail(ctx, MLIP_E_ARG, "no output");
  if (!weights_dev || !offsets_dev || (n > 0 && (!x_dev || !order_dev))) return fail(ctx, MLIP_E_ARG, "NULL argument");
  HeadsArgs a{};
  a.n = n;
  a.m = n * p->top_k;
  a.stride = p->row_stride;
  a.E = p->n_experts;
  a.D = p->width;
  a.H = p->hidden;
  a.K = p->top_k;
  a.bf16 = p->dtype == MLIP_BF16;
  a.values = head_values(p);
  a.x = x_dev;
  a.weights = weights_dev;
  a.offsets = offsets_dev;
  a.order = order_dev;
  a.gates = gates_dev;
  a.denergy = denergy_dev;
  a.energy = energy_dev;
  a.dx = dx_dev;
  a.dweights = dweights_dev;
  a.dgates = dgates_dev;
  const size_t need = heads_plan(&a, ctx->n_cu);
  const mlip_status w = workspace(ctx, need);
  if (w != MLIP_OK) return w;
  heads_workspace(&a, ctx->d_ws);
  LEARN_HIP(ctx, launch_heads(a, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_adamw_create(const mlip_adamw_tensor* tensors, int64_t n_tensors, int32_t state_bits,
                              void* hip_stream, mlip_adamw** out) {
  t_learn_err.clear();
  mlip_adamw* const none = nullptr;
  if (!out) return fail(none, MLIP_E_ARG, "NULL output pointer");
  *out = nullptr;
  if (!tensors || n_tensors < 1) return fail(none, MLIP_E_ARG, "no tensors");
  if (state_bits != 32 && state_bits != 8) return fail(none, MLIP_E_ARG, "state_bits must be 32 or 8");
  mlip_adamw* h = nullptr;
  try {
    std::vector<AdamPiece> pp;
    int64_t at = 0, block = 0, into = 0, filled = 0;
    for (int64_t k = 0; k < n_tensors; ++k) {
      const mlip_adamw_tensor& t = tensors[k];
      if (t.n < 0 || t.n > (int64_t(1) << 40) - at) return fail(none, MLIP_E_ARG, "more than 2^40 elements");
      if (t.n > 0 && (!t.param_dev || !t.grad_dev)) return fail(none, MLIP_E_ARG, "NULL parameter or gradient");
      if ((t.param_dtype != MLIP_F32 && t.param_dtype != MLIP_BF16) || (t.grad_dtype != MLIP_F32 && t.grad_dtype != MLIP_BF16))
        return fail(none, MLIP_E_ARG, "unknown dtype");
      filled += t.n > 0 ? 1 : 0;   // an empty tensor may be nowhere
      into += t.n > 0 && t.into_dev ? 1 : 0;
      const int64_t size = t.param_dtype == MLIP_BF16 ? 2 : 4, grad_size = t.grad_dtype == MLIP_BF16 ? 2 : 4;
      for (int64_t i = 0; i < t.n; i += kAdamPiece) {
        AdamPiece p{};
        p.param = static_cast<char*>(t.param_dev) + size * i;
        p.into = static_cast<char*>(t.into_dev ? t.into_dev : t.param_dev) + size * i;
        p.grad = static_cast<const char*>(t.grad_dev) + grad_size * i;
        p.at = at + i;
        p.block = block + i / 256;
        p.n = int32_t(std::min<int64_t>(t.n - i, kAdamPiece));
        p.param_bf16 = t.param_dtype == MLIP_BF16;
        p.grad_bf16 = t.grad_dtype == MLIP_BF16;
        p.decay = t.decay != 0;
        pp.push_back(p);
      }
      at += t.n;
      block += (t.n + 255) / 256;
    }
    if (into != 0 && into != filled) return fail(none, MLIP_E_ARG, "into_dev is for all tensors or for none");
    h = new mlip_adamw();
    h->stream = reinterpret_cast<hipStream_t>(hip_stream);
    h->bits = state_bits;
    h->into = into != 0;
    h->elements = at;
    h->blocks = block;
    h->pieces = int64_t(pp.size());
    if (hipGetDevice(&h->device) != hipSuccess ||
        hipDeviceGetAttribute(&h->n_cu, hipDeviceAttributeMultiprocessorCount, h->device) != hipSuccess) {
      (void)hipGetLastError();
      delete h;
      return fail(none, MLIP_E_HIP, "no current HIP device");
    }
    const size_t bytes = std::max<size_t>(1, pp.size()) * sizeof(AdamPiece);
    if (hipMalloc(reinterpret_cast<void**>(&h->d_pieces), bytes) != hipSuccess) {
      (void)hipGetLastError();
      delete h;
      return fail(none, MLIP_E_OOM, "device allocation failed: table of pieces");
    }
    const hipError_t e = pp.empty() ? hipSuccess
                                    : hipMemcpy(h->d_pieces, pp.data(), pp.size() * sizeof(AdamPiece), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
      (void)hipFree(h->d_pieces);
      delete h;
      return fail_hip(none, e);
    }
  } catch (...) {
    delete h;
    return fail(none, MLIP_E_OOM, "host allocation failed");
  }
  *out = h;
  return MLIP_OK;
}

const char* mlip_adamw_last_error(const mlip_adamw* plan) { return plan ? plan->err.c_str() : t_learn_err.c_str(); }

mlip_status mlip_adamw_state_count(const mlip_adamw* plan, int64_t* elements, int64_t* blocks) {
  if (!plan || !elements || !blocks) return MLIP_E_ARG;
  *elements = plan->elements;
  *blocks = plan->bits == 8 ? plan->blocks : 0;
  return MLIP_OK;
}

void mlip_adamw_destroy(mlip_adamw* plan) {
  if (!plan) return;
  (void)hipStreamSynchronize(plan->stream);
  if (plan->d_pieces) (void)hipFree(plan->d_pieces);
  (void)hipGetLastError();
  delete plan;
}

mlip_status mlip_adamw_step(mlip_adamw* plan, const mlip_adamw_params* p, const mlip_adamw_state* from,
                            const mlip_adamw_state* into, int32_t reverse) {
  if (!plan) return MLIP_E_ARG;
  plan->err.clear();
  if (elsewhere(plan)) return fail(plan, MLIP_E_ARG, kElsewhere);
  if (!p) return fail(plan, MLIP_E_ARG, "NULL parameters");
  if (p->step < 1) return fail(plan, MLIP_E_ARG, "step must be 1 or more");
  if (!(p->beta1 >= 0.0 && p->beta1 < 1.0) || !(p->beta2 >= 0.0 && p->beta2 < 1.0))
    return fail(plan, MLIP_E_ARG, "beta1 and beta2 must be in [0, 1)");
  if (!(p->eps >= 0.0) || !std::isfinite(p->eps) || !std::isfinite(p->lr) || !std::isfinite(p->weight_decay) ||
      !std::isfinite(p->grad_scale))
    return fail(plan, MLIP_E_ARG, "eps must be at least 0, and lr, weight_decay and grad_scale finite");
  if (reverse && !plan->into) return fail(plan, MLIP_E_ARG, "reverse needs a plan with into_dev");
  if (!state_given(plan, from) || (into && !state_given(plan, into))) return fail(plan, MLIP_E_ARG, "NULL state");
  if (plan->pieces == 0) return MLIP_OK;
  AdamArgs a = adam_args(plan, from, into ? into : from);
  a.reverse = reverse != 0;
  AdamStep h{};
  h.lr = p->lr;
  h.beta1 = p->beta1;
  h.beta2 = p->beta2;
  h.eps = p->eps;
  h.weight_decay = p->weight_decay;
  h.grad_scale = p->grad_scale;
  h.correction1 = 1.0 - std::pow(p->beta1, double(p->step));
  h.root_correction2 = std::sqrt(1.0 - std::pow(p->beta2, double(p->step)));
  h.seed = p->seed;
  LEARN_HIP(plan, launch_adamw(a, h, plan->n_cu, plan->stream));
  return MLIP_OK;
}

mlip_status mlip_adamw_moments(mlip_adamw* plan, const mlip_adamw_state* state, float* m_out_dev, float* v_out_dev) {
  if (!plan) return MLIP_E_ARG;
  plan->err.clear();
  if (elsewhere(plan)) return fail(plan, MLIP_E_ARG, kElsewhere);
  if (plan->bits != 8) return fail(plan, MLIP_E_ARG, "the moments are values already");
  if (!state_given(plan, state)) return fail(plan, MLIP_E_ARG, "NULL state");
  if (plan->pieces == 0) return MLIP_OK;
  if (!m_out_dev || !v_out_dev) return fail(plan, MLIP_E_ARG, "NULL output");
  const AdamArgs a = adam_args(plan, state, state);
  LEARN_HIP(plan, launch_moments(a, m_out_dev, v_out_dev, plan->n_cu, plan->stream));
  return MLIP_OK;
}

}  // extern "C"
