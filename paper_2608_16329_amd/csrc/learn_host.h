// What the C entries of the learning operators share on the host's side: error
// texts, the check of the current device, and the context's workspace.
#pragma once

#include <string>

#include "learn.h"

namespace mlip {

inline thread_local std::string t_learn_err;

template <typename Ctx>
mlip_status fail(Ctx* ctx, mlip_status st, const char* msg) {
  // no exception crosses the ABI: without memory for it the text is dropped
  try {
    (ctx ? ctx->err : t_learn_err) = msg;
  } catch (...) {
    (ctx ? ctx->err : t_learn_err).clear();
  }
  return st;
}

template <typename Ctx>
mlip_status fail_hip(Ctx* ctx, hipError_t e) {
  (void)hipGetLastError();
  return fail(ctx, MLIP_E_HIP, hipGetErrorString(e));
}

#define LEARN_HIP(ctx, expr)                          \
  do {                                                \
    const hipError_t e_ = (expr);                     \
    if (e_ != hipSuccess) return fail_hip((ctx), e_); \
  } while (0)

// A call on another device's stream would take memory and sizes of the wrong one.
template <typename Ctx>
bool elsewhere(Ctx* ctx) {
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess) (void)hipGetLastError();
  return device != ctx->device;
}
inline constexpr const char* kElsewhere = "the device of the context is not current";

// The workspace holds at least `need` bytes; it is allocated anew where it is
// smaller, and freed after the stream's work that may still use it, or, where a
// recorded call has it, with the context: the graph may be replayed at any time.
// Not while the stream is recorded: the recording would end with an error at the
// wait.
inline mlip_status workspace(mlip_learn* ctx, size_t need) {
  if (need == 0) return MLIP_OK;
  if (need <= ctx->cap_ws) {
    // (the null stream cannot be recorded; without an answer it may be)
    if (ctx->stream && !ctx->recorded_ws) {
      hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
      const bool known = hipStreamIsCapturing(ctx->stream, &status) == hipSuccess;
      if (!known) (void)hipGetLastError();
      ctx->recorded_ws = !known || status != hipStreamCaptureStatusNone;
    }
    return MLIP_OK;
  }
  hipStreamCaptureStatus recorded = hipStreamCaptureStatusNone;
  LEARN_HIP(ctx, hipStreamIsCapturing(ctx->stream, &recorded));
  if (recorded != hipStreamCaptureStatusNone)
    return fail(ctx, MLIP_E_STATE, "the workspace is too small and the stream is being recorded: make the call once before");
  if (ctx->d_ws) {
    if (ctx->recorded_ws) {
      try {
        ctx->kept.push_back(ctx->d_ws);
      } catch (...) {
        return fail(ctx, MLIP_E_OOM, "host allocation failed");
      }
      ctx->kept_bytes += ctx->cap_ws;
    } else {
      LEARN_HIP(ctx, hipStreamSynchronize(ctx->stream));
      (void)hipFree(ctx->d_ws);
    }
    ctx->d_ws = nullptr;
    ctx->cap_ws = 0;
    ctx->recorded_ws = false;
  }
  const size_t size = (need + need / 4 + 255) / 256 * 256;
  if (hipMalloc(reinterpret_cast<void**>(&ctx->d_ws), size) != hipSuccess) {
    ctx->d_ws = nullptr;
    (void)hipGetLastError();
    return fail(ctx, MLIP_E_OOM, "device allocation failed: workspace");
  }
  ctx->cap_ws = size;
  return MLIP_OK;
}

}  // namespace mlip
