// Device helpers of the layers' kernels: chunks of values in either type, 8-bit
// codes, sums and maxima over groups of lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "layers.h"
#include "learn_math.h"

namespace mlip {

// 16 and 8 neighbouring bytes at the alignment of one value or byte (rows start
// anywhere; the hardware takes them in one access all the same).
typedef uint32_t U4 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t U2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));

// 16 bytes from and to memory; STREAM: past what the caches hold.
template <bool STREAM>
__device__ __forceinline__ u4v take16(const void* from) {
  if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const U4*>(from));
  else return *static_cast<const U4*>(from);
}
template <bool STREAM>
__device__ __forceinline__ void give16(void* to, u4v v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<U4*>(to));
  else *static_cast<U4*>(to) = v;
}

typedef float f2v __attribute__((ext_vector_type(2)));
typedef __bf16 b2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16x2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2v{a, b}, b2v));
}

// Four values of an array of either type from `at` on, those from `left` on as
// zero (left <= 0: none is read); and back, those before `left`.
template <bool BF, bool STREAM = false>
__device__ __forceinline__ void load4at(const void* p, int64_t at, int left, float* v) {
  if (left >= 4) {
    if (BF) {
      const u2v h = *reinterpret_cast<const U2*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        v[2 * q] = __uint_as_float(h[q] << 16);
        v[2 * q + 1] = __uint_as_float(h[q] & 0xffff0000u);
      }
    } else {
      const u4v a = take16<STREAM>(static_cast<const float*>(p) + at);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = __uint_as_float(a[q]);
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[q] = 0.f;
    if (q < left) v[q] = BF ? from_bf16(static_cast<const uint16_t*>(p)[at + q]) : static_cast<const float*>(p)[at + q];
  }
}
template <bool BF, bool STREAM>
__device__ __forceinline__ void store4at(void* p, int64_t at, int left, const float* v) {
  if (left >= 4) {
    if (BF) *reinterpret_cast<U2*>(static_cast<uint16_t*>(p) + at) = u2v{bf16x2(v[0], v[1]), bf16x2(v[2], v[3])};
    else
      give16<STREAM>(static_cast<float*>(p) + at,
                     u4v{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (q < left) {
      if (BF) static_cast<uint16_t*>(p)[at + q] = uint16_t(bf16x2(v[q], 0.f));
      else static_cast<float*>(p)[at + q] = v[q];
    }
}

// A lane's eight values of a block of 128: from `at` on, neighbours in bfloat16, in
// float32 four and the four that are 64 behind them, so that 16 lanes' 16-byte
// accesses lie side by side.  `left`: values of the row from `at` on.
template <bool BF>
constexpr int kSecond = BF ? 4 : 64;
template <bool BF, bool STREAM>
__device__ __forceinline__ void load8(const void* p, int64_t at, int left, float v[8]) {
  if (BF && left >= 8) {
    const u4v h = take16<STREAM>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[2 * q] = __uint_as_float(h[q] << 16);
      v[2 * q + 1] = __uint_as_float(h[q] & 0xffff0000u);
    }
    return;
  }
  load4at<BF, STREAM>(p, at, left, v);
  load4at<BF, STREAM>(p, at + kSecond<BF>, left - kSecond<BF>, v + 4);
}
template <bool BF, bool STREAM>
__device__ __forceinline__ void store8(void* p, int64_t at, int left, const float v[8]) {
  if (BF && left >= 8) {
    u4v h;
#pragma unroll
    for (int q = 0; q < 4; ++q) h[q] = bf16x2(v[2 * q], v[2 * q + 1]);
    give16<STREAM>(static_cast<uint16_t*>(p) + at, h);
    return;
  }
  store4at<BF, STREAM>(p, at, left, v);
  store4at<BF, STREAM>(p, at + kSecond<BF>, left - kSecond<BF>, v + 4);
}

// The largest of 16 neighbouring lanes' values, in each of them: rotations
// within the row of 16, by 8, 4, 2 and 1.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xf, 0xf, true)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xf, 0xf, true)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xf, 0xf, true)));
  return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xf, 0xf, true)));
}

// The exponent e of a block whose largest finite size has these bits: the least
// with all of it within codes up to 448, kept within -100 .. 120 so that codes'
// values and the scales are normal float32 and bfloat16 numbers.
__device__ __forceinline__ int exponent8(uint32_t bits) {
  return min(120, max(-100, int(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0)));
}
// 2^e, -126 <= e <= 127
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }
// The bits of the largest finite size among eight values.
__device__ __forceinline__ uint32_t largest8(const float v[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int q = 0; q < 8; ++q) top = max(top, __float_as_uint(v[q]) & 0x7fffffffu);
  if (top >= 0x7f800000u) {     // an infinity or a NaN is among them
    top = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const uint32_t u = __float_as_uint(v[q]) & 0x7fffffffu;
      top = max(top, u < 0x7f800000u ? u : 0u);
    }
  }
  return top;
}
// The bits of a finite value's size; 0 for an infinity or a NaN.
__device__ __forceinline__ uint32_t finite_size(float v) {
  const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
// Codes of eight values times 2^-e, to nearest even (the conversion gives the
// NaN code for infinities and NaN; nothing finite is over 448).
__device__ __forceinline__ u2v encode8(const float v[8], int e) {
  const float unit = pow2(-e);
  float t[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) t[q] = v[q] * unit;
  // 256 2^120 would be an infinity in float32: 240 is the largest code there
  if (e == 120) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (finite_size(v[q]) && fabsf(t[q]) > 240.f) t[q] = copysignf(240.f, t[q]);
  }
  u2v c;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(t[4 * q], t[4 * q + 1], 0, false);
    c[q] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(t[4 * q + 2], t[4 * q + 3], w, true));
  }
  return c;
}
__device__ __forceinline__ void decode8(u2v c, float unit, float v[8]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(c[q]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(c[q]), true);
    v[4 * q] = lo[0] * unit;
    v[4 * q + 1] = lo[1] * unit;
    v[4 * q + 2] = hi[0] * unit;
    v[4 * q + 3] = hi[1] * unit;
  }
}

}  // namespace mlip
