// Device helpers shared by the learning operators' kernels: 16-bit floats and
// loads of four values at their own alignment.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mlip {

// Four neighbouring values, aligned like one of them (rows and tables start
// anywhere; the hardware loads and stores them in one access all the same).
// Vectors, not arrays: of an array's four stores the compiler moves some out of
// a branch and leaves three.
typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t H4 __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float from_bf16(uint16_t h) { return __uint_as_float(uint32_t(h) << 16); }
// round to nearest even; a NaN stays one
__device__ __forceinline__ uint16_t to_bf16(float f) {
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return uint16_t((u >> 16) | 0x40u);
  return uint16_t((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// Values at, at + 1, at + 2, at + 3 of an array of either type, those from
// `left` on as zero (left <= 0: none is read).
__device__ __forceinline__ void load4(const void* p, bool bf16, int64_t at, int left, float v[4]) {
  if (left >= 4) {
    if (bf16) {
      const H4 h = *reinterpret_cast<const H4*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = from_bf16(h[q]);
    } else {
      const F4 f = *reinterpret_cast<const F4*>(static_cast<const float*>(p) + at);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = f[q];
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[q] = 0.f;
    if (q < left) v[q] = bf16 ? from_bf16(static_cast<const uint16_t*>(p)[at + q]) : static_cast<const float*>(p)[at + q];
  }
}

__device__ __forceinline__ void store4(void* p, bool bf16, int64_t at, int left, const float v[4]) {
  if (left >= 4) {
    if (bf16) {
      H4 h;
#pragma unroll
      for (int q = 0; q < 4; ++q) h[q] = to_bf16(v[q]);
      *reinterpret_cast<H4*>(static_cast<uint16_t*>(p) + at) = h;
    } else {
      F4 f;
#pragma unroll
      for (int q = 0; q < 4; ++q) f[q] = v[q];
      *reinterpret_cast<F4*>(static_cast<float*>(p) + at) = f;
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q < left) {
      if (bf16) static_cast<uint16_t*>(p)[at + q] = to_bf16(v[q]);
      else static_cast<float*>(p)[at + q] = v[q];
    }
}

}  // namespace mlip
