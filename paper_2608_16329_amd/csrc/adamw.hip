// One AdamW step over many tensors, moments in 32 or in 8 bits.
//
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2  (g scaled by grad_scale),
//   p' = p (1 - lr wd) - lr / (1 - b1^t) m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
//
// Bound by memory: 28 bytes an element in 32 bits, 16 with 8-bit moments
// (float32 parameters and gradients).  The tensors are cut into pieces of at
// most kAdamPiece elements, a table of them is laid out once, and one launch walks
// it; a tensor of one element costs a wavefront, not a launch.
//
// 8 bits: blocks of 256 elements of a tensor share a power of two 2^e > max
// |x|.  m: a sign, 4 exponent and 3 mantissa bits of |m| 2^-e, v: 4 and 4 of
// v 2^-e; exponent field E > 0 stands for 2^(E - 15) (1 + f), 0 for subnormal
// 2^-14 f.  v changes by a part of 1 - b2 a step, less than half the distance
// of its codes, so rounding to nearest would hold it where it is: both are
// rounded up or down at random, up with the probability of the part cut off (to
// 2^-16), by bits mixed from the caller's seed and the element's place.  On average
// that is the value, but for a v below the smallest code, 2^-18 2^e, which is
// raised to it.
#include <algorithm>

#include "learn.h"
#include "learn_math.h"

// results of float32 operations one by one, as written: the codes of 8-bit
// moments must not depend on which products are fused into sums
#pragma clang fp contract(off)

namespace mlip {
namespace {

constexpr int kThreads = 256;

struct __attribute__((packed, aligned(1))) B4 { uint8_t v[4]; };

__device__ __forceinline__ float pow2(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }

// 32 mixed bits from the seed and an element's place: multiplications and shifts
// with constants from a published search for mixers of low bias (C. Wellons, 2018)
__device__ __forceinline__ uint32_t dice(uint32_t seed, uint32_t at) {
  uint32_t h = at * 0x9E3779B1u + seed;
  h = (h ^ (h >> 15)) * 0x2C1B3C6Du;
  h = (h ^ (h >> 12)) * 0x297A2D39u;
  return h ^ (h >> 15);
}

template <int M>
__device__ __forceinline__ float decode(uint32_t code, int e) {
  const uint32_t c = M == 3 ? code & 127u : code;
  const int ec = int(c >> M);
  const float base = float((c & ((1u << M) - 1u)) + (ec ? 1u << M : 0u));
  float v = base * pow2((ec ? ec : 1) - 15 - M) * pow2(e);
  if (c == (M == 3 ? 127u : 255u)) v = __uint_as_float(0x7fc00000u);
  return M == 3 && (code & 128u) ? -v : v;
}

// up: rounds up where the part cut off and up, in [0, 1), reach 1 together
template <int M>
__device__ __forceinline__ uint32_t encode(float x, int e, float up) {
  const float size = fabsf(x);
  if (!(size < INFINITY)) return M == 3 ? 127u : 255u;
  const float y = size * pow2(-e);
  const int ey = max(int(__float_as_uint(y) >> 23) - 127, -14);
  uint32_t code = ((uint32_t(ey + 14)) << M) + uint32_t(floorf(y * pow2(M - ey) + up));
  code = min(code, M == 3 ? 126u : 254u);
  // a v that is not zero stays so: m / sqrt(v) would run away; a v that is too
  // large only shortens steps
  if (M == 4 && size > 0.f && code == 0) code = 1;
  return M == 3 && x < 0.f ? code | 128u : code;
}

// e with top < 2^e, from the bits of the block's largest finite size
__device__ __forceinline__ int block_exponent(float top) {
  return min(max(int(__float_as_uint(top) >> 23) - 126, -126), 126);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

struct Step {
  float b1, omb1, b2, omb2, eps, scale, lr1, bc2;   // lr1 = lr / (1 - b1^t), bc2 = 1 / sqrt(1 - b2^t)
  float keep;                                        // 1 - lr wd
  uint32_t seed;
};

__device__ __forceinline__ float update(const Step& s, float keep, float p, float g, float& m, float& v) {
  g = g * s.scale;
  m = m * s.b1 + g * s.omb1;
  v = v * s.b2 + (g * g) * s.omb2;
  return p * keep - s.lr1 * (m / (sqrtf(v) * s.bc2 + s.eps));
}

// A work-group takes a piece, a wavefront 256 elements of it, four a lane: a
// block of 8-bit moments.  11.1 M elements in 2,208 tensors, 32 bits: 54 us with
// tensors that were just used (5.8 TB/s), 61 without (5.1).  1.47 M elements in 348
// tensors, 8 bits, bfloat16 gradients: 12 us (21 MB, 1.7 TB/s), the vector pipes busy for
// 66% of it: there coding and decoding and one round of work-groups' latency
// count.  18 tensors: 3.6 us.
template <bool B8>
__global__ __launch_bounds__(kThreads) void k_adamw(AdamArgs a, Step s) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = 256 * w + 4 * lane;
  for (int64_t piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
    const AdamPiece t = a.piece[piece];
    const float keep = t.decay ? s.keep : 1.f;
    const void* const from = a.reverse ? t.into : t.param;
    void* const to = a.reverse ? t.param : t.into;
    if (256 * w < t.n) {
      const int left = min(t.n - i, 4);
      float p[4], g[4], m[4], v[4];
      load4(from, t.param_bf16, i, left, p);
      load4(t.grad, t.grad_bf16, i, left, g);
      if (!B8) {
        load4(a.m, false, t.at + i, left, m);
        load4(a.v, false, t.at + i, left, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) p[q] = update(s, keep, p[q], g[q], m[q], v[q]);
        store4(a.new_m, false, t.at + i, left, m);
        store4(a.new_v, false, t.at + i, left, v);
      } else {
        const int64_t block = t.block + w;
        const uint8_t* mc = static_cast<const uint8_t*>(a.m) + t.at + i;
        const uint8_t* vc = static_cast<const uint8_t*>(a.v) + t.at + i;
        B4 cm{}, cv{};
        if (left == 4) {
          cm = *reinterpret_cast<const B4*>(mc);
          cv = *reinterpret_cast<const B4*>(vc);
        } else {
#pragma unroll
          for (int q = 0; q < 3; ++q)
            if (q < left) cm.v[q] = mc[q], cv.v[q] = vc[q];
        }
        const int em = int(a.m_exp[block]) - 127, ev = int(a.v_exp[block]) - 127;
        float top_m = 0.f, top_v = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          m[q] = decode<3>(cm.v[q], em);
          v[q] = decode<4>(cv.v[q], ev);
          p[q] = update(s, keep, p[q], g[q], m[q], v[q]);
          const float sm = fabsf(m[q]);
          if (q < left && sm < INFINITY) top_m = fmaxf(top_m, sm);
          if (q < left && v[q] < INFINITY) top_v = fmaxf(top_v, v[q]);
        }
        const int nm = block_exponent(wave_max(top_m)), nv = block_exponent(wave_max(top_v));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t r = dice(s.seed, uint32_t(t.at + i + q));
          cm.v[q] = uint8_t(encode<3>(m[q], nm, float(r & 0xffffu) * 0x1p-16f));
          cv.v[q] = uint8_t(encode<4>(v[q], nv, float(r >> 16) * 0x1p-16f));
        }
        uint8_t* mo = static_cast<uint8_t*>(a.new_m) + t.at + i;
        uint8_t* vo = static_cast<uint8_t*>(a.new_v) + t.at + i;
        if (left == 4) {
          *reinterpret_cast<B4*>(mo) = cm;
          *reinterpret_cast<B4*>(vo) = cv;
        } else {
#pragma unroll
          for (int q = 0; q < 3; ++q)
            if (q < left) mo[q] = cm.v[q], vo[q] = cv.v[q];
        }
        if (lane == 0) a.new_m_exp[block] = uint8_t(nm + 127), a.new_v_exp[block] = uint8_t(nv + 127);
      }
      store4(to, t.param_bf16, i, left, p);
    }
  }
}

// The values that 8-bit moments stand for.  Bound by memory: 8.4 M elements 19 us
// (84 MB, 4.4 TB/s).
__global__ __launch_bounds__(kThreads) void k_moments(AdamArgs a, float* m_out, float* v_out) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = 256 * w + 4 * lane;
  for (int64_t piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
    const AdamPiece t = a.piece[piece];
    if (256 * w < t.n) {
      const int left = min(t.n - i, 4);
      const int64_t block = t.block + w;
      const int em = int(a.m_exp[block]) - 127, ev = int(a.v_exp[block]) - 127;
      const uint8_t* mc = static_cast<const uint8_t*>(a.m) + t.at + i;
      const uint8_t* vc = static_cast<const uint8_t*>(a.v) + t.at + i;
      float m[4], v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        m[q] = v[q] = 0.f;
        if (q < left) m[q] = decode<3>(mc[q], em), v[q] = decode<4>(vc[q], ev);
      }
      store4(m_out, false, t.at + i, left, m);
      store4(v_out, false, t.at + i, left, v);
    }
  }
}

}  // namespace

hipError_t launch_adamw(const AdamArgs& a, const AdamStep& h, int n_cu, hipStream_t s) {
  Step k;
  k.b1 = float(h.beta1);
  k.omb1 = float(1.0 - h.beta1);
  k.b2 = float(h.beta2);
  k.omb2 = float(1.0 - h.beta2);
  k.eps = float(h.eps);
  k.scale = float(h.grad_scale);
  k.lr1 = float(h.lr / h.correction1);
  k.bc2 = float(1.0 / h.root_correction2);
  k.keep = float(1.0 - h.lr * h.weight_decay);
  k.seed = h.seed;
  const int blocks = int(std::min<int64_t>(a.pieces, int64_t(n_cu) * 8));
  if (a.bits == 8) k_adamw<true><<<blocks, kThreads, 0, s>>>(a, k);
  else k_adamw<false><<<blocks, kThreads, 0, s>>>(a, k);
  return hipGetLastError();
}

hipError_t launch_moments(const AdamArgs& a, float* m_out, float* v_out, int n_cu, hipStream_t s) {
  const int blocks = int(std::min<int64_t>(a.pieces, int64_t(n_cu) * 8));
  k_moments<<<blocks, kThreads, 0, s>>>(a, m_out, v_out);
  return hipGetLastError();
}

}  // namespace mlip
