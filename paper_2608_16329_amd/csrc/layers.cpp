// C ABI of the operators of wide layers of experts (declared in include/mlip.h):
// argument checks, workspace, and the launches of their kernels.
#include <algorithm>

#include "layers.h"
#include "learn_host.h"

using namespace mlip;

namespace {

constexpr int64_t kMaxStride = int64_t(1) << 31;
constexpr int64_t kMaxBlocks = (int64_t(1) << 22) - 1;      // work-groups of up to 1024 in a launch

mlip_status check_rows(mlip_learn* ctx, const mlip_rows_params* p, int64_t n) {
  if (!p) return fail(ctx, MLIP_E_ARG, "NULL parameters");
  if (p->n_experts < 1 || p->n_experts > kMaxExperts) return fail(ctx, MLIP_E_ARG, "n_experts must be in 1..256");
  if (p->top_k < 1 || p->top_k > kMaxTopK) return fail(ctx, MLIP_E_ARG, "top_k must be in 1..16");
  if (p->width < 1 || p->width > kMaxLayerWidth) return fail(ctx, MLIP_E_ARG, "width must be in 1..65536");
  if (p->dtype != MLIP_F32 && p->dtype != MLIP_BF16) return fail(ctx, MLIP_E_ARG, "unknown dtype");
  if (n < 0 || n >= (int64_t(1) << 31) / p->top_k) return fail(ctx, MLIP_E_ARG, "n outside [0, 2^31 / top_k)");
  return MLIP_OK;
}
bool stride_fits(int64_t stride, int64_t width) { return stride >= width && stride <= kMaxStride; }
constexpr const char* kStride = "a row stride must be in width..2^31";

// Codes are read and written 16 bytes at a time, exponents four.
bool placed(const void* codes, const void* exps) {
  return reinterpret_cast<uintptr_t>(codes) % 16 == 0 && reinterpret_cast<uintptr_t>(exps) % 4 == 0;
}
constexpr const char* kPlaced = "codes must be aligned to 16 bytes and exponents to 4";

mlip_status check_product(mlip_learn* ctx, const mlip_product8_params* p, int64_t m) {
  if (!p) return fail(ctx, MLIP_E_ARG, "NULL parameters");
  if (p->n_experts < 1 || p->n_experts > kMaxExperts) return fail(ctx, MLIP_E_ARG, "n_experts must be in 1..256");
  if (p->inputs < 1 || p->inputs > kMaxLayerWidth || p->outputs < 1 || p->outputs > kMaxLayerWidth)
    return fail(ctx, MLIP_E_ARG, "inputs and outputs must be in 1..65536");
  if (p->dtype != MLIP_F32 && p->dtype != MLIP_BF16) return fail(ctx, MLIP_E_ARG, "unknown dtype");
  if (m < 0 || m >= (int64_t(1) << 31)) return fail(ctx, MLIP_E_ARG, "m outside [0, 2^31)");
  return MLIP_OK;
}
int64_t tiles_of(int64_t v) { return (v + 127) / 128; }

RowsArgs rows_args(const mlip_rows_params* p, int64_t n) {
  RowsArgs a{};
  a.n = n;
  a.m = n * p->top_k;
  a.E = p->n_experts;
  a.K = p->top_k;
  a.width = p->width;
  a.bf16 = p->dtype == MLIP_BF16;
  return a;
}
Pack8Args pack_args(const mlip_rows_params* p, int64_t n) {
  Pack8Args a{};
  a.n = n;
  a.E = p->n_experts;
  a.K = p->top_k;
  a.width = p->width;
  a.bf16 = p->dtype == MLIP_BF16;
  return a;
}

// What every call begins with.
#define LAYER_BEGIN(check)                                             \
  if (!ctx) return MLIP_E_ARG;                                         \
  ctx->err.clear();                                                    \
  if (elsewhere(ctx)) return fail(ctx, MLIP_E_ARG, kElsewhere);        \
  {                                                                    \
    const mlip_status st_ = (check);                                   \
    if (st_ != MLIP_OK) return st_;                                    \
  }

}  // namespace

extern "C" {

mlip_status mlip_sort(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* x_dev, int64_t x_stride,
                      const int32_t* offsets_dev, const int32_t* order_dev, void* sorted_dev, int32_t* places_dev) {
  LAYER_BEGIN(check_rows(ctx, p, n));
  if (!stride_fits(x_stride, p->width)) return fail(ctx, MLIP_E_ARG, kStride);
  if (n == 0) return MLIP_OK;
  if ((sorted_dev && !x_dev) || !offsets_dev || !order_dev || !places_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  RowsArgs a = rows_args(p, n);
  if (!sorted_dev) a.width = 1;                               // (no lanes for values)
  a.x = x_dev;
  a.x_stride = x_stride;
  a.offsets = offsets_dev;
  a.order = order_dev;
  a.out = sorted_dev;
  a.places = places_dev;
  LEARN_HIP(ctx, launch_sort(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_combine(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* y_dev, int64_t y_stride,
                         const int32_t* places_dev, const float* gates_dev, void* out_dev) {
  LAYER_BEGIN(check_rows(ctx, p, n));
  if (!stride_fits(y_stride, p->width)) return fail(ctx, MLIP_E_ARG, kStride);
  if (n == 0) return MLIP_OK;
  if (!y_dev || !places_dev || !out_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  RowsArgs a = rows_args(p, n);
  a.x = y_dev;
  a.x_stride = y_stride;
  a.places = const_cast<int32_t*>(places_dev);
  a.gates = gates_dev;
  a.out = out_dev;
  LEARN_HIP(ctx, launch_combine(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_combine_backward(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* dout_dev,
                                  int64_t dout_stride, const void* y_dev, int64_t y_stride, const int32_t* places_dev,
                                  const float* gates_dev, void* dy_dev, float* dgates_dev) {
  LAYER_BEGIN(check_rows(ctx, p, n));
  if (!stride_fits(dout_stride, p->width) || (dgates_dev && !stride_fits(y_stride, p->width)))
    return fail(ctx, MLIP_E_ARG, kStride);
  if (n == 0) return MLIP_OK;
  if (!dout_dev || !places_dev || !dy_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  if (dgates_dev && !y_dev) return fail(ctx, MLIP_E_ARG, "dgates needs y");
  RowsArgs a = rows_args(p, n);
  a.x = dout_dev;
  a.x_stride = dout_stride;
  a.y = y_dev;
  a.y_stride = y_stride;
  a.places = const_cast<int32_t*>(places_dev);
  a.gates = gates_dev;
  a.out = dy_dev;
  a.dgates = dgates_dev;
  LEARN_HIP(ctx, launch_combine_backward(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

int64_t mlip_row8_codes(int32_t width) { return width >= 1 && width <= kMaxLayerWidth ? codes8(width) : 0; }
int64_t mlip_row8_exps(int32_t width) { return width >= 1 && width <= kMaxLayerWidth ? exps8(width) : 0; }

mlip_status mlip_pack8(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* x_dev, int64_t x_stride,
                       const int32_t* offsets_dev, const int32_t* order_dev, uint8_t* codes_dev, uint8_t* exps_dev) {
  LAYER_BEGIN(check_rows(ctx, p, n));
  if (!stride_fits(x_stride, p->width)) return fail(ctx, MLIP_E_ARG, kStride);
  if (!offsets_dev != !order_dev) return fail(ctx, MLIP_E_ARG, "offsets and order go together");
  if (!order_dev && p->top_k != 1) return fail(ctx, MLIP_E_ARG, "top_k is 1 without an order");
  if (n == 0) return MLIP_OK;
  if (!x_dev || !codes_dev || !exps_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  if (!placed(codes_dev, exps_dev)) return fail(ctx, MLIP_E_ARG, kPlaced);
  Pack8Args a = pack_args(p, n);
  a.n = n * p->top_k;
  a.x = x_dev;
  a.x_stride = x_stride;
  a.offsets = offsets_dev;
  a.order = order_dev;
  a.codes = codes_dev;
  a.exps = exps_dev;
  LEARN_HIP(ctx, launch_pack8(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_unpack8(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const uint8_t* codes_dev,
                         const uint8_t* exps_dev, void* x_dev) {
  LAYER_BEGIN(check_rows(ctx, p, n));
  if (n == 0) return MLIP_OK;
  if (!codes_dev || !exps_dev || !x_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  if (!placed(codes_dev, exps_dev)) return fail(ctx, MLIP_E_ARG, kPlaced);
  Pack8Args a = pack_args(p, n);
  a.kept = codes_dev;
  a.kept_exps = exps_dev;
  a.out = x_dev;
  LEARN_HIP(ctx, launch_unpack8(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_activate8(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const void* z_dev, int64_t z_stride,
                           const void* residual_dev, int64_t residual_stride, void* h_dev, uint8_t* h_codes_dev,
                           uint8_t* h_exps_dev, uint8_t* kept_codes_dev, uint8_t* kept_exps_dev) {
  LAYER_BEGIN(check_rows(ctx, p, n));
  if (!stride_fits(z_stride, p->width) || (residual_dev && !stride_fits(residual_stride, p->width)))
    return fail(ctx, MLIP_E_ARG, kStride);
  if (!h_codes_dev != !h_exps_dev || !kept_codes_dev != !kept_exps_dev) return fail(ctx, MLIP_E_ARG, "codes and exponents go together");
  if (n == 0) return MLIP_OK;
  if (!z_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  if (!h_dev && !h_codes_dev && !kept_codes_dev) return fail(ctx, MLIP_E_ARG, "no output");
  if (!placed(h_codes_dev, h_exps_dev) || !placed(kept_codes_dev, kept_exps_dev)) return fail(ctx, MLIP_E_ARG, kPlaced);
  Pack8Args a = pack_args(p, n);
  a.x = z_dev;
  a.x_stride = z_stride;
  a.residual = residual_dev;
  a.residual_stride = residual_stride;
  a.out = h_dev;
  a.out_codes = h_codes_dev;
  a.out_exps = h_exps_dev;
  a.codes = kept_codes_dev;
  a.exps = kept_exps_dev;
  LEARN_HIP(ctx, launch_activate8(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_activate8_backward(mlip_learn* ctx, const mlip_rows_params* p, int64_t n, const uint8_t* kept_codes_dev,
                                    const uint8_t* kept_exps_dev, const void* dh_dev, int64_t dh_stride, void* dz_dev,
                                    uint8_t* dz_codes_dev, uint8_t* dz_exps_dev) {
  LAYER_BEGIN(check_rows(ctx, p, n));
  if (!stride_fits(dh_stride, p->width)) return fail(ctx, MLIP_E_ARG, kStride);
  if (!dz_codes_dev != !dz_exps_dev) return fail(ctx, MLIP_E_ARG, "codes and exponents go together");
  if (n == 0) return MLIP_OK;
  if (!kept_codes_dev || !kept_exps_dev || !dh_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  if (!dz_dev && !dz_codes_dev) return fail(ctx, MLIP_E_ARG, "no output");
  if (!placed(kept_codes_dev, kept_exps_dev) || !placed(dz_codes_dev, dz_exps_dev)) return fail(ctx, MLIP_E_ARG, kPlaced);
  Pack8Args a = pack_args(p, n);
  a.kept = kept_codes_dev;
  a.kept_exps = kept_exps_dev;
  a.x = dh_dev;
  a.x_stride = dh_stride;
  a.out = dz_dev;
  a.out_codes = dz_codes_dev;
  a.out_exps = dz_exps_dev;
  LEARN_HIP(ctx, launch_activate8_backward(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_pack8_weights(mlip_learn* ctx, const mlip_product8_params* p, const void* w_dev, uint8_t* codes_dev,
                               uint8_t* exps_dev, uint8_t* t_codes_dev, uint8_t* t_exps_dev) {
  LAYER_BEGIN(check_product(ctx, p, 0));
  if (!w_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  if (!codes_dev != !exps_dev || !t_codes_dev != !t_exps_dev) return fail(ctx, MLIP_E_ARG, "codes and exponents go together");
  if (!codes_dev && !t_codes_dev) return fail(ctx, MLIP_E_ARG, "no output");
  if (!placed(codes_dev, exps_dev) || !placed(t_codes_dev, t_exps_dev)) return fail(ctx, MLIP_E_ARG, kPlaced);
  Weights8Args a{};
  a.E = p->n_experts;
  a.N = p->outputs;
  a.K = p->inputs;
  a.bf16 = p->dtype == MLIP_BF16;
  a.w = w_dev;
  a.codes = codes_dev;
  a.exps = exps_dev;
  a.codes_t = t_codes_dev;
  a.exps_t = t_exps_dev;
  LEARN_HIP(ctx, launch_pack8_weights(a, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_product8(mlip_learn* ctx, const mlip_product8_params* p, int64_t m, const uint8_t* x_codes_dev,
                          const uint8_t* x_exps_dev, const uint8_t* w_codes_dev, const uint8_t* w_exps_dev,
                          const int32_t* offsets_dev, const float* bias_dev, void* y_dev) {
  LAYER_BEGIN(check_product(ctx, p, m));
  if (!offsets_dev && p->n_experts != 1) return fail(ctx, MLIP_E_ARG, "several experts need offsets");
  if ((tiles_of(m) + p->n_experts) * tiles_of(p->outputs) > kMaxBlocks) return fail(ctx, MLIP_E_ARG, "m outputs exceeds 2^36");
  if (m == 0) return MLIP_OK;
  if (!x_codes_dev || !x_exps_dev || !w_codes_dev || !w_exps_dev || !y_dev) return fail(ctx, MLIP_E_ARG, "NULL argument");
  if (!placed(x_codes_dev, x_exps_dev) || !placed(w_codes_dev, w_exps_dev)) return fail(ctx, MLIP_E_ARG, kPlaced);
  Product8Args a{};
  a.m = m;
  a.E = p->n_experts;
  a.N = p->outputs;
  a.K = p->inputs;
  a.bf16 = p->dtype == MLIP_BF16;
  a.x = x_codes_dev;
  a.x_exps = x_exps_dev;
  a.w = w_codes_dev;
  a.w_exps = w_exps_dev;
  a.offsets = offsets_dev;
  a.bias = bias_dev;
  a.y = y_dev;
  LEARN_HIP(ctx, launch_product8(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

mlip_status mlip_product8_weights(mlip_learn* ctx, const mlip_product8_params* p, int64_t m, const uint8_t* dy_codes_dev,
                                  const uint8_t* dy_exps_dev, const uint8_t* x_codes_dev, const uint8_t* x_exps_dev,
                                  const int32_t* offsets_dev, float* dweights_dev, float* dbias_dev) {
  LAYER_BEGIN(check_product(ctx, p, m));
  if (!offsets_dev && p->n_experts != 1) return fail(ctx, MLIP_E_ARG, "several experts need offsets");
  if (!dweights_dev || (m > 0 && (!dy_codes_dev || !dy_exps_dev || !x_codes_dev || !x_exps_dev)))
    return fail(ctx, MLIP_E_ARG, "NULL argument");
  if (!placed(dy_codes_dev, dy_exps_dev) || !placed(x_codes_dev, x_exps_dev)) return fail(ctx, MLIP_E_ARG, kPlaced);
  Product8Args a{};
  a.m = m;
  a.E = p->n_experts;
  a.N = p->outputs;
  a.K = p->inputs;
  a.x = x_codes_dev;
  a.x_exps = x_exps_dev;
  a.w = dy_codes_dev;
  a.w_exps = dy_exps_dev;
  a.offsets = offsets_dev;
  a.dweights = dweights_dev;
  a.dbias = dbias_dev;
  const size_t need = product8_weights_plan(&a, ctx->n_cu);
  if ((m / a.slice + p->n_experts) * tiles_of(p->outputs) * tiles_of(p->inputs) > kMaxBlocks)
    return fail(ctx, MLIP_E_ARG, "n_experts inputs outputs exceeds 2^36");
  const mlip_status w = workspace(ctx, need);
  if (w != MLIP_OK) return w;
  product8_workspace(&a, ctx->d_ws);
  LEARN_HIP(ctx, launch_product8_weights(a, ctx->n_cu, ctx->stream));
  return MLIP_OK;
}

}  // extern "C"
