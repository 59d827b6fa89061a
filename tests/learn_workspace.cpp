// The workspace of a learning context over calls that are recorded and calls
// that are not, with the HIP runtime and the kernels' launchers replaced by
// counters: which memory is alive when.  Prints what is wrong; 0: nothing.
#include <cstdio>
#include <cstdlib>
#include <map>

#include "../paper_2608_16329_amd/csrc/learn.h"

namespace {
std::map<void*, size_t> alive;
bool recorded = false, refused = false;
int wrong = 0;

void need(bool ok, const char* what) {
  if (!ok) std::printf("%s\n", what), ++wrong;
}
size_t held() {
  size_t b = 0;
  for (const auto& a : alive) b += a.second;
  return b;
}
}  // namespace

extern "C" {
hipError_t hipMalloc(void** p, size_t n) {
  *p = std::malloc(n);
  alive[*p] = n;
  return hipSuccess;
}
hipError_t hipFree(void* p) {
  need(alive.erase(p) == 1, "freed what is not allocated");
  std::free(p);
  return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  *s = recorded ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return refused ? hipErrorStreamCaptureImplicit : hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) { return recorded ? hipErrorStreamCaptureUnsupported : hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { return *v = 256, hipSuccess; }
hipError_t hipMemcpy(void*, const void*, size_t, hipMemcpyKind) { return hipSuccess; }
}

namespace mlip {
int route_blocks(int64_t, int, int) { return 1; }
hipError_t launch_route(const RouteArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_route_backward(const RouteArgs&, int, hipStream_t) { return hipSuccess; }
size_t group_ws_bytes(int64_t m, int) { return size_t(m); }
hipError_t launch_group(const int32_t*, int64_t, int, int32_t*, int32_t*, void*, hipStream_t) { return hipSuccess; }
size_t heads_plan(HeadsArgs*, int) { return 0; }
void heads_workspace(HeadsArgs*, unsigned char*) {}
hipError_t launch_heads(const HeadsArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_adamw(const AdamArgs&, const AdamStep&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_moments(const AdamArgs&, float*, float*, int, hipStream_t) { return hipSuccess; }
}  // namespace mlip

int main() {
  mlip_learn* ctx = nullptr;
  need(mlip_learn_create(reinterpret_cast<void*>(16), &ctx) == MLIP_OK, "no context");
  int32_t x = 0;
  auto call = [&](int64_t bytes) { return mlip_group(ctx, bytes, 4, &x, &x, &x); };
  auto bytes = [&]() {
    size_t b = 0;
    need(mlip_learn_memory_bytes(ctx, &b) == MLIP_OK, "no size");
    return b;
  };
  need(call(1000) == MLIP_OK && alive.size() == 1 && bytes() == held(), "first call");
  void* const first = alive.begin()->first;
  recorded = true;
  need(call(900) == MLIP_OK && alive.size() == 1, "recorded call");
  need(call(100000) == MLIP_E_STATE && alive.count(first) == 1, "growth while recorded");
  recorded = false;
  // larger calls: the graph's workspace stays, what no graph has goes
  need(call(5000) == MLIP_OK, "larger call");
  need(alive.count(first) == 1, "a recorded call's workspace was freed by a larger call");
  need(bytes() == held(), "bytes while a graph's workspace is kept");
  need(call(50000) == MLIP_OK && alive.count(first) == 1 && alive.size() == 2, "a workspace that no graph has");
  recorded = true;
  need(call(50000) == MLIP_OK, "second recording");
  recorded = false;
  need(call(500000) == MLIP_OK && alive.size() == 3 && bytes() == held(), "two graphs' workspaces");
  // where the runtime does not say whether the stream is recorded, it may be
  refused = true;
  need(call(500000) == MLIP_OK, "call without an answer");
  refused = false;
  need(call(5000000) == MLIP_OK && alive.size() == 4, "workspace of a call that may have been recorded");
  mlip_learn_destroy(ctx);
  need(alive.empty(), "memory left after the context");
  return wrong;
}
