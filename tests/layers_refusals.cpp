// What the entries of wide layers of experts refuse, and what they pass on, with the
// HIP runtime and the kernels' launchers replaced by counters.  Prints what is wrong;
// 0: nothing.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../paper_2608_16329_amd/csrc/layers.h"
#include "../paper_2608_16329_amd/csrc/learn.h"

namespace {
int wrong = 0, launches = 0, device = 0;
bool recorded = false;
void need(bool ok, const char* what, int line) {
  if (!ok) std::printf("line %d: %s\n", line, what), ++wrong;
}
#define NEED(x) need((x), #x, __LINE__)
}  // namespace

extern "C" {
hipError_t hipMalloc(void** p, size_t n) { return *p = std::malloc(n), hipSuccess; }
hipError_t hipFree(void* p) { return std::free(p), hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  return *s = recorded ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone, hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipGetDevice(int* d) { return *d = device, hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
}

namespace mlip {
hipError_t one() { return ++launches, hipSuccess; }
hipError_t launch_sort(const RowsArgs&, int, hipStream_t) { return one(); }
hipError_t launch_combine(const RowsArgs&, int, hipStream_t) { return one(); }
hipError_t launch_combine_backward(const RowsArgs&, int, hipStream_t) { return one(); }
hipError_t launch_pack8(const Pack8Args&, int, hipStream_t) { return one(); }
hipError_t launch_unpack8(const Pack8Args&, int, hipStream_t) { return one(); }
hipError_t launch_activate8(const Pack8Args&, int, hipStream_t) { return one(); }
hipError_t launch_activate8_backward(const Pack8Args&, int, hipStream_t) { return one(); }
hipError_t launch_pack8_weights(const Weights8Args&, hipStream_t) { return one(); }
hipError_t launch_product8(const Product8Args&, int, hipStream_t) { return one(); }
size_t product8_weights_plan(Product8Args* a, int) { return a->slice = 64, size_t(1000); }
void product8_workspace(Product8Args*, unsigned char*) {}
hipError_t launch_product8_weights(const Product8Args&, int, hipStream_t) { return one(); }
}  // namespace mlip

int main() {
  mlip_learn ctx;
  ctx.n_cu = 256;
  // an address that is aligned to 256 bytes, and one that is aligned to one value alone
  void* const a = reinterpret_cast<void*>(uintptr_t(1) << 20);
  void* const odd = reinterpret_cast<void*>((uintptr_t(1) << 20) + 4);
  uint8_t* const c = static_cast<uint8_t*>(a), *const co = static_cast<uint8_t*>(odd), *const co1 = co + 1;
  int32_t* const i = static_cast<int32_t*>(a);
  float* const f = static_cast<float*>(a);
  const mlip_rows_params good = {8, 2, 100, MLIP_BF16};
  const mlip_product8_params pgood = {8, 100, 60, MLIP_F32};

  struct {
    mlip_rows_params p;
    int64_t n;
  } const bad_rows[] = {{{0, 2, 100, 0}, 5}, {{257, 2, 100, 0}, 5}, {{8, 0, 100, 0}, 5}, {{8, 17, 100, 0}, 5}, {{8, 2, 0, 0}, 5},
                        {{8, 2, 65537, 0}, 5}, {{8, 2, 100, 2}, 5}, {{8, 2, 100, 0}, -1}, {{8, 2, 100, 0}, int64_t(1) << 30}};
  for (const auto& b : bad_rows) {
    NEED(mlip_sort(&ctx, &b.p, b.n, a, 200000, i, i, a, i) == MLIP_E_ARG);
    NEED(mlip_combine(&ctx, &b.p, b.n, a, 200000, i, f, a) == MLIP_E_ARG);
    NEED(mlip_combine_backward(&ctx, &b.p, b.n, a, 200000, a, 200000, i, f, a, f) == MLIP_E_ARG);
    NEED(mlip_pack8(&ctx, &b.p, b.n, a, 200000, i, i, c, c) == MLIP_E_ARG);
    NEED(mlip_unpack8(&ctx, &b.p, b.n, c, c, a) == MLIP_E_ARG);
    NEED(mlip_activate8(&ctx, &b.p, b.n, a, 200000, nullptr, 0, a, nullptr, nullptr, c, c) == MLIP_E_ARG);
    NEED(mlip_activate8_backward(&ctx, &b.p, b.n, c, c, a, 200000, a, nullptr, nullptr) == MLIP_E_ARG);
    NEED(!ctx.err.empty());
  }
  struct {
    mlip_product8_params p;
    int64_t m;
  } const bad_products[] = {{{0, 100, 60, 0}, 5}, {{257, 100, 60, 0}, 5}, {{8, 0, 60, 0}, 5}, {{8, 65537, 60, 0}, 5}, {{8, 100, 0, 0}, 5},
                            {{8, 100, 65537, 0}, 5}, {{8, 100, 60, 2}, 5}, {{8, 100, 60, 0}, -1}, {{8, 100, 60, 0}, int64_t(1) << 31},
                            {{8, 65536, 65536, 0}, int64_t(1) << 30}};
  for (const auto& b : bad_products) {
    NEED(mlip_product8(&ctx, &b.p, b.m, c, c, c, c, i, f, a) == MLIP_E_ARG);
    NEED(mlip_product8_weights(&ctx, &b.p, b.m, c, c, c, c, i, f, f) == MLIP_E_ARG);
  }
  for (int k = 0; k < 7; ++k) NEED(mlip_pack8_weights(&ctx, &bad_products[k].p, a, c, c, c, c) == MLIP_E_ARG);
  // strides
  for (int64_t s : {int64_t(99), int64_t(-1), (int64_t(1) << 31) + 1}) {
    NEED(mlip_sort(&ctx, &good, 5, a, s, i, i, a, i) == MLIP_E_ARG);
    NEED(mlip_combine(&ctx, &good, 5, a, s, i, f, a) == MLIP_E_ARG);
    NEED(mlip_combine_backward(&ctx, &good, 5, a, s, a, 100, i, f, a, f) == MLIP_E_ARG);
    NEED(mlip_combine_backward(&ctx, &good, 5, a, 100, a, s, i, f, a, f) == MLIP_E_ARG);
    NEED(mlip_pack8(&ctx, &good, 5, a, s, i, i, c, c) == MLIP_E_ARG);
    NEED(mlip_activate8(&ctx, &good, 5, a, s, nullptr, 0, a, nullptr, nullptr, c, c) == MLIP_E_ARG);
    NEED(mlip_activate8(&ctx, &good, 5, a, 100, a, s, a, nullptr, nullptr, c, c) == MLIP_E_ARG);
    NEED(mlip_activate8_backward(&ctx, &good, 5, c, c, a, s, a, nullptr, nullptr) == MLIP_E_ARG);
  }
  // what is missing
  NEED(mlip_sort(&ctx, nullptr, 5, a, 100, i, i, a, i) == MLIP_E_ARG);
  NEED(mlip_sort(&ctx, &good, 5, nullptr, 100, i, i, a, i) == MLIP_E_ARG);
  NEED(mlip_sort(&ctx, &good, 5, a, 100, nullptr, i, a, i) == MLIP_E_ARG);
  NEED(mlip_sort(&ctx, &good, 5, a, 100, i, nullptr, a, i) == MLIP_E_ARG);
  NEED(mlip_sort(&ctx, &good, 5, a, 100, i, i, a, nullptr) == MLIP_E_ARG);
  NEED(mlip_combine(&ctx, &good, 5, nullptr, 100, i, f, a) == MLIP_E_ARG);
  NEED(mlip_combine(&ctx, &good, 5, a, 100, nullptr, f, a) == MLIP_E_ARG);
  NEED(mlip_combine(&ctx, &good, 5, a, 100, i, f, nullptr) == MLIP_E_ARG);
  NEED(mlip_combine_backward(&ctx, &good, 5, a, 100, nullptr, 100, i, f, a, f) == MLIP_E_ARG);
  NEED(mlip_combine_backward(&ctx, &good, 5, a, 100, a, 100, i, f, nullptr, f) == MLIP_E_ARG);
  NEED(mlip_pack8(&ctx, &good, 5, a, 100, i, nullptr, c, c) == MLIP_E_ARG);
  NEED(mlip_pack8(&ctx, &good, 5, a, 100, nullptr, i, c, c) == MLIP_E_ARG);
  NEED(mlip_pack8(&ctx, &good, 5, a, 100, nullptr, nullptr, c, c) == MLIP_E_ARG);   // top_k 2 without an order
  NEED(mlip_pack8(&ctx, &good, 5, a, 100, i, i, c, nullptr) == MLIP_E_ARG);
  NEED(mlip_activate8(&ctx, &good, 5, a, 100, nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr) == MLIP_E_ARG);
  NEED(mlip_activate8(&ctx, &good, 5, a, 100, nullptr, 0, a, c, nullptr, nullptr, nullptr) == MLIP_E_ARG);
  NEED(mlip_activate8(&ctx, &good, 5, a, 100, nullptr, 0, a, nullptr, nullptr, nullptr, c) == MLIP_E_ARG);
  NEED(mlip_activate8_backward(&ctx, &good, 5, c, c, a, 100, nullptr, nullptr, nullptr) == MLIP_E_ARG);
  NEED(mlip_activate8_backward(&ctx, &good, 5, c, nullptr, a, 100, a, nullptr, nullptr) == MLIP_E_ARG);
  NEED(mlip_pack8_weights(&ctx, &pgood, a, nullptr, nullptr, nullptr, nullptr) == MLIP_E_ARG);
  NEED(mlip_pack8_weights(&ctx, &pgood, a, c, nullptr, c, c) == MLIP_E_ARG);
  NEED(mlip_pack8_weights(&ctx, &pgood, nullptr, c, c, c, c) == MLIP_E_ARG);
  NEED(mlip_product8(&ctx, &pgood, 5, c, c, c, c, nullptr, f, a) == MLIP_E_ARG);     // several experts without offsets
  NEED(mlip_product8(&ctx, &pgood, 5, c, c, nullptr, c, i, f, a) == MLIP_E_ARG);
  NEED(mlip_product8_weights(&ctx, &pgood, 5, c, c, c, c, nullptr, f, f) == MLIP_E_ARG);
  NEED(mlip_product8_weights(&ctx, &pgood, 0, c, c, c, c, i, nullptr, f) == MLIP_E_ARG);
  // places
  NEED(mlip_pack8(&ctx, &good, 5, a, 100, i, i, co, c) == MLIP_E_ARG);
  NEED(mlip_pack8(&ctx, &good, 5, a, 100, i, i, c, co1) == MLIP_E_ARG);
  NEED(mlip_unpack8(&ctx, &good, 5, co, c, a) == MLIP_E_ARG);
  NEED(mlip_activate8(&ctx, &good, 5, a, 100, nullptr, 0, a, co, c, c, c) == MLIP_E_ARG);
  NEED(mlip_activate8_backward(&ctx, &good, 5, co, c, a, 100, a, nullptr, nullptr) == MLIP_E_ARG);
  NEED(mlip_pack8_weights(&ctx, &pgood, a, c, c, co, c) == MLIP_E_ARG);
  NEED(mlip_product8(&ctx, &pgood, 5, co, c, c, c, i, f, a) == MLIP_E_ARG);
  NEED(mlip_product8_weights(&ctx, &pgood, 5, c, c, co, c, i, f, f) == MLIP_E_ARG);
  // another device, and no context
  device = 1;
  NEED(mlip_sort(&ctx, &good, 5, a, 100, i, i, a, i) == MLIP_E_ARG);
  NEED(mlip_product8(&ctx, &pgood, 5, c, c, c, c, i, f, a) == MLIP_E_ARG && std::strstr(mlip_learn_last_error(&ctx), "device"));
  device = 0;
  NEED(mlip_sort(nullptr, &good, 5, a, 100, i, i, a, i) == MLIP_E_ARG);
  NEED(mlip_product8_weights(nullptr, &pgood, 5, c, c, c, c, i, f, f) == MLIP_E_ARG);
  NEED(launches == 0);

  // calls that are fine: nothing to do, and something
  NEED(mlip_sort(&ctx, &good, 0, nullptr, 100, nullptr, nullptr, nullptr, nullptr) == MLIP_OK);
  NEED(mlip_pack8(&ctx, &good, 0, nullptr, 100, nullptr, nullptr, nullptr, nullptr) == MLIP_E_ARG);   // (top_k 2 without an order)
  NEED(mlip_product8(&ctx, &pgood, 0, nullptr, nullptr, nullptr, nullptr, i, nullptr, nullptr) == MLIP_OK);
  NEED(launches == 0);
  NEED(mlip_sort(&ctx, &good, 5, nullptr, 100, i, i, nullptr, i) == MLIP_OK);                        // (places alone)
  NEED(mlip_sort(&ctx, &good, 5, odd, 101, i, i, odd, i) == MLIP_OK);
  NEED(mlip_combine(&ctx, &good, 5, odd, 101, i, nullptr, odd) == MLIP_OK);
  NEED(mlip_combine_backward(&ctx, &good, 5, odd, 101, nullptr, 0, i, f, odd, nullptr) == MLIP_OK);
  NEED(mlip_pack8(&ctx, &good, 5, odd, 101, i, i, c, c) == MLIP_OK);
  NEED(mlip_product8(&ctx, &pgood, 5, c, c, c, c, i, nullptr, odd) == MLIP_OK);
  NEED(launches == 6 && ctx.err.empty());
  // a gradient's workspace is not made while the stream is recorded
  recorded = true;
  NEED(mlip_product8_weights(&ctx, &pgood, 5, c, c, c, c, i, f, nullptr) == MLIP_E_STATE);
  recorded = false;
  NEED(mlip_product8_weights(&ctx, &pgood, 5, c, c, c, c, i, f, nullptr) == MLIP_OK);
  recorded = true;
  NEED(mlip_product8_weights(&ctx, &pgood, 5, c, c, c, c, i, f, nullptr) == MLIP_OK && launches == 8);
  NEED(mlip_row8_codes(1) == 128 && mlip_row8_codes(128) == 128 && mlip_row8_codes(129) == 256 && mlip_row8_codes(0) == 0);
  NEED(mlip_row8_exps(1) == 4 && mlip_row8_exps(512) == 4 && mlip_row8_exps(513) == 8 && mlip_row8_exps(65537) == 0);
  return wrong;
}

const char* mlip_learn_last_error(const mlip_learn* ctx) { return ctx->err.c_str(); }
