// The descriptor buffer of the three-kernel configuration (by sorted slot, in
// the network's type) and the caller's rows (by atom, float32): what goes to
// heads outside the fused kernel and comes back from them.  Bound by memory:
// a wavefront copies neighbouring values of a row, four a lane.  131,072 atoms of
// 128 values, float64 network: 30 us out, 37 back (201 MB, 6.7 and 5.4 TB/s, part
// of it from the last-level cache).  Float32 rows: the heads' arithmetic is
// float32, so a wider row would only be rounded later.
#include <algorithm>

#include "learn_math.h"
#include "mlip_internal.h"

namespace mlip {
namespace {

template <typename R, bool OUT>
__global__ __launch_bounds__(256) void k_rows(R* __restrict__ slots, const int32_t* __restrict__ perm, int64_t n, int nin,
                                              float* __restrict__ rows) {
  const int groups = nin / 4;   // k is a multiple of 16
  for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < n * groups; at += int64_t(gridDim.x) * 256) {
    const int64_t slot = at / groups;
    const int c = 4 * int(at % groups);
    R* s = slots + slot * nin + c;
    float* r = rows + int64_t(perm[slot]) * nin + c;
    F4 f;
    if (OUT) {
#pragma unroll
      for (int q = 0; q < 4; ++q) f[q] = float(s[q]);
      *reinterpret_cast<F4*>(r) = f;
    } else {
      f = *reinterpret_cast<const F4*>(r);
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] = R(f[q]);
    }
  }
}

template <typename R>
hipError_t rows_of(void* slots, const int32_t* perm, int64_t n, int nin, float* rows, bool out, hipStream_t s) {
  // (fewer than 2^32 threads a launch)
  const unsigned blocks = unsigned(std::min<int64_t>((n * (nin / 4) + 255) / 256, 1 << 22));
  if (out) k_rows<R, true><<<blocks, 256, 0, s>>>(static_cast<R*>(slots), perm, n, nin, rows);
  else k_rows<R, false><<<blocks, 256, 0, s>>>(static_cast<R*>(slots), perm, n, nin, rows);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_descriptor_rows(void* slots, int precision, const int32_t* perm, int64_t n, int nin, float* rows,
                                  bool out, hipStream_t s) {
  return precision == 64 ? rows_of<double>(slots, perm, n, nin, rows, out, s)
                         : rows_of<float>(slots, perm, n, nin, rows, out, s);
}

}  // namespace mlip
