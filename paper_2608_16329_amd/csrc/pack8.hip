// Rows and matrices in 8 bits, and activations that keep them.
//
// A block of 128 values has a power of two 2^e and codes of 4 exponent and 3
// mantissa bits beside the sign (values up to 448, NaN, no infinity): with a =
// f 2^q its largest finite size, 1 <= f < 2, e = q - 8 if f <= 1.75 and q - 7
// otherwise, and a code is the value times 2^-e, rounded to nearest even, off
// by at most 2^-4 of the value (and by 2^(e - 10) where the value is below
// 2^(e - 6)).  A matrix shares e over 128 x 128 values, so that its transpose
// has the same values.
//
// Bound by memory, activations by vector instructions about as much.  16 lanes have a
// block, 8 values each; a wavefront has four blocks, whose exponents are one 32-bit
// word: four of a row, or one or two each of four or two rows that have no more.
// Wavefronts that run side by side have neighbouring blocks, and float32 stores of 16
// lanes are whole lines (both, and conversions in hardware: 744 to 533 us of the two
// activations below).
// 131,072 rows of 1,024 bfloat16 values in the order of 2 of 16 experts: packing 147 to
// 161 us (5.0 TB/s with each row read twice), unpacking 118 to 128 (6.3, partly from the
// last cache).  65,536 rows of 4,096 bfloat16 values, the last 50 of 100 launches on normally
// distributed values: silu that keeps its argument 237 us (225 to 250), its gradient 215
// (1.34 GB each, 5.7 and 6.3 TB/s; 458 to 466 the two in turn); the first dozen launches, before the
// clock has settled, 214 to 300.  With results in 8 bits instead, 1.07 GB, 256 and 248: the maxima
// and the encoding bring the vector instructions to 172 and 159 million, and these, at four
// cycles each, fill the SIMDs (136 and 124 million without).
#include <algorithm>

#include "layers_math.h"

namespace mlip {
namespace {

// What a lane works on: row and block, the first of its eight values and how
// many the row has from there on.
struct Spot {
  int64_t row;
  int block, at, left;
  bool there;                   // the row and the block exist (and, packing, the row's entry)
};
template <bool BF, int G>
__device__ __forceinline__ Spot spot(int64_t row0, int quad, int64_t n, int width) {
  const int group = (threadIdx.x & 63) >> 4;
  Spot s;
  s.row = row0 + group / G;
  s.block = 4 * quad + group % G;
  s.at = s.block * kBlock8 + (BF ? 8 : 4) * (threadIdx.x & 15);
  s.left = width - s.at;
  s.there = s.row < n && s.block * kBlock8 < width;
  return s;
}

// f(first row, which four blocks) for all of n rows, shared by the wavefronts.
template <int G, typename F>
__device__ __forceinline__ void each(int64_t n, int width, F f) {
  const int quads = int(exps8(width) / 4);
  const int64_t all = int64_t(gridDim.x) * 4, mine = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t rows_on = all / quads;
  const int quads_on = int(all - rows_on * quads);
  int64_t group = mine / quads;
  int quad = int(mine - group * quads);
  while (group * (4 / G) < n) {
    f(group * (4 / G), quad);
    group += rows_on;
    quad += quads_on;
    if (quad >= quads) {
      quad -= quads;
      ++group;
    }
  }
}

// Writes a block's codes and exponent where it is there: all lanes of the wavefront
// call.  The lane that writes a row's exponents has the first of its four blocks,
// which a row that is there always has.
template <bool BF, int G>
__device__ __forceinline__ void put(const Spot& s, const float v[8], uint8_t* codes, uint8_t* exps, int quad, int width) {
  const int e = exponent8(max16(largest8(v)));
  if (s.there) {
    const u2v c = encode8(v, e);
    uint8_t* const to = codes + s.row * codes8(width) + s.at;
    if (BF) *reinterpret_cast<u2v*>(to) = c;
    else {
      *reinterpret_cast<uint32_t*>(to) = c[0];
      *reinterpret_cast<uint32_t*>(to + kSecond<BF>) = c[1];
    }
  }
  uint32_t word = s.there ? uint32_t(e + 127) << (8 * (s.block & 3)) : 0u;
  if (G >= 2) word |= __shfl_xor(word, 16);
  if (G == 4) word |= __shfl_xor(word, 32);
  if ((threadIdx.x & 15) == 0 && s.block % 4 == 0 && s.there)
    *reinterpret_cast<uint32_t*>(exps + s.row * exps8(width) + 4 * quad) = word;
}
// Values of a block that was written.
template <bool BF>
__device__ __forceinline__ void get(const Spot& s, const uint8_t* codes, const uint8_t* exps, int width, float v[8]) {
  if (s.there) {
    const uint8_t* const from = codes + s.row * codes8(width) + s.at;
    u2v c;
    if (BF) c = *reinterpret_cast<const u2v*>(from);
    else c = u2v{*reinterpret_cast<const uint32_t*>(from), *reinterpret_cast<const uint32_t*>(from + kSecond<BF>)};
    const uint32_t e = exps[s.row * exps8(width) + s.block];
    decode8(c, __uint_as_float(e << 23), v);
  }
}

// The row of x that packed row p is, or -1.
__device__ __forceinline__ int64_t source(const Pack8Args& a, int64_t p, int64_t end) {
  if (!a.order) return p;
  if (p >= end) return -1;
  const uint32_t entry = uint32_t(a.order[p]);
  return int64_t(entry) < a.n ? int64_t(entry / uint32_t(a.K)) : -1;
}

template <bool BF, int G, bool STREAM>
__global__ __launch_bounds__(256) void k_pack8(Pack8Args a) {
  const int64_t end = a.order ? min(a.n, max(int64_t(0), int64_t(a.offsets[a.E]))) : a.n;
  each<G>(end, a.width, [&](int64_t row0, int quad) {
    Spot s = spot<BF, G>(row0, quad, end, a.width);
    const int64_t from = s.there ? source(a, s.row, end) : -1;
    s.there = s.there && from >= 0;
    float v[8] = {};
    if (s.there) load8<BF, STREAM>(a.x, from * a.x_stride + s.at, s.left, v);
    put<BF, G>(s, v, a.codes, a.exps, quad, a.width);
  });
}

template <bool BF, int G, bool STREAM>
__global__ __launch_bounds__(256) void k_unpack8(Pack8Args a) {
  each<G>(a.n, a.width, [&](int64_t row0, int quad) {
    const Spot s = spot<BF, G>(row0, quad, a.n, a.width);
    float v[8];
    get<BF>(s, a.kept, a.kept_exps, a.width, v);
    if (s.there) store8<BF, STREAM>(a.out, s.row * a.width + s.at, s.left, v);
  });
}

// 1 / (1 + exp(-z)) from t = exp(-|z|), which does not overflow where the quotient
// is still a number: 2^f 2^n with n + f = -|z| log2(e) in two parts, |f| <= 1/2, so
// that t is good to 2 ulp at any z, also where it is a denormal number.
__device__ __forceinline__ float sigmoid(float z) {
  const float y = fminf(fabsf(z), 200.f);                     // (t is 0 from 104 on; an infinity has no f)
  const float n = rintf(-y * 1.44269502f);
  float f = fmaf(-y, 1.44269502f, -n);
  f = fmaf(-y, 1.92596299e-8f, f);
  const float t = ldexpf(__builtin_amdgcn_exp2f(f), int(n));
  return (z < 0.f ? t : 1.f) * __builtin_amdgcn_rcpf(1.f + t);
}

// What is left of values in their type.
template <bool BF>
__device__ __forceinline__ void as_stored(float v[8]) {
  if (BF)
#pragma unroll
    for (int q = 0; q < 8; q += 2) {
      const uint32_t u = bf16x2(v[q], v[q + 1]);
      v[q] = __uint_as_float(u << 16);
      v[q + 1] = __uint_as_float(u & 0xffff0000u);
    }
}

// h = r + silu(z), and z in 8 bits for the backward pass
template <bool BF, int G, bool STREAM>
__global__ __launch_bounds__(256) void k_activate8(Pack8Args a) {
  each<G>(a.n, a.width, [&](int64_t row0, int quad) {
    const Spot s = spot<BF, G>(row0, quad, a.n, a.width);
    float z[8] = {}, h[8] = {};
    if (s.there) {
      load8<BF, STREAM>(a.x, s.row * a.x_stride + s.at, s.left, z);
      if (a.residual) load8<BF, STREAM>(a.residual, s.row * a.residual_stride + s.at, s.left, h);
    }
    if (a.codes) put<BF, G>(s, z, a.codes, a.exps, quad, a.width);
#pragma unroll
    for (int q = 0; q < 8; ++q) h[q] = fmaf(z[q], sigmoid(z[q]), h[q]);
    if (a.out && s.there) store8<BF, STREAM>(a.out, s.row * a.width + s.at, s.left, h);
    if (a.out_codes) {
      as_stored<BF>(h);
      put<BF, G>(s, h, a.out_codes, a.out_exps, quad, a.width);
    }
  });
}

// dz = dh silu'(z) of the z that was kept
template <bool BF, int G, bool STREAM>
__global__ __launch_bounds__(256) void k_activate8_backward(Pack8Args a) {
  each<G>(a.n, a.width, [&](int64_t row0, int quad) {
    const Spot s = spot<BF, G>(row0, quad, a.n, a.width);
    float z[8] = {}, d[8] = {};
    if (s.there) load8<BF, STREAM>(a.x, s.row * a.x_stride + s.at, s.left, d);
    get<BF>(s, a.kept, a.kept_exps, a.width, z);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float t = sigmoid(z[q]);
      d[q] *= t * fmaf(z[q], 1.f - t, 1.f);
    }
    if (a.out && s.there) store8<BF, STREAM>(a.out, s.row * a.width + s.at, s.left, d);
    if (a.out_codes) {
      as_stored<BF>(d);
      put<BF, G>(s, d, a.out_codes, a.out_exps, quad, a.width);
    }
  });
}

// One work-group for a block of 128 x 128 of a matrix: thread t has the 8 values
// from 8 (t % 16) on of rows t / 16, t / 16 + 16 ..  The transpose goes through LDS as
// codes.  Bound by memory: 8 matrices of 4,096 x 1,024 float32 values, both ways, 45 us
// (201 MB, 4.5 TB/s); bytes one at a time through LDS 57.
template <bool BF>
__global__ __launch_bounds__(256) void k_pack8_weights(Weights8Args a) {
  constexpr int kPitch = kBlock8 / 4 + 1;           // of a row of codes in LDS, in 32-bit words
  __shared__ uint32_t tops[4];
  __shared__ uint32_t tile[kBlock8 * kPitch];
  const int kb = blockIdx.x, nb = blockIdx.y, t = threadIdx.x;
  const int64_t e = blockIdx.z;
  const int blocks_k = (a.K + kBlock8 - 1) / kBlock8, blocks_n = (a.N + kBlock8 - 1) / kBlock8;
  const int k0 = kb * kBlock8 + 8 * (t & 15);
  float v[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int n = nb * kBlock8 + 16 * j + (t >> 4);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[j][q] = 0.f;
    if (n < a.N) {
      const int64_t at = (e * a.N + n) * a.K + k0;
      load4at<BF>(a.w, at, a.K - k0, v[j]);
      load4at<BF>(a.w, at + 4, a.K - k0 - 4, v[j] + 4);
    }
    top = max(top, largest8(v[j]));
  }
  top = max16(top);
  top = max(top, uint32_t(__shfl_xor(top, 16)));
  top = max(top, uint32_t(__shfl_xor(top, 32)));
  if ((t & 63) == 0) tops[t >> 6] = top;
  __syncthreads();
  const int x = exponent8(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int r = 16 * j + (t >> 4), n = nb * kBlock8 + r;
    const u2v c = encode8(v[j], x);
    if (a.codes && n < a.N) *reinterpret_cast<u2v*>(a.codes + (e * a.N + n) * codes8(a.K) + k0) = c;
    if (a.codes_t) {
      tile[r * kPitch + 2 * (t & 15)] = c[0];
      tile[r * kPitch + 2 * (t & 15) + 1] = c[1];
    }
  }
  // the exponent, and zeros behind the last block
  if (t < 4) {
    if (a.codes && (t == 0 || (kb == blocks_k - 1 && kb + t < exps8(a.K))))
      a.exps[(e * blocks_n + nb) * exps8(a.K) + kb + t] = t == 0 ? uint8_t(x + 127) : uint8_t(0);
    if (a.codes_t && (t == 0 || (nb == blocks_n - 1 && nb + t < exps8(a.N))))
      a.exps_t[(e * blocks_k + kb) * exps8(a.N) + nb + t] = t == 0 ? uint8_t(x + 127) : uint8_t(0);
  }
  if (!a.codes_t) return;
  __syncthreads();
  // four columns of eight rows at a time, as columns: bytes of four words change places
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r0 = 8 * (t & 15), k4 = 16 * j + (t >> 4);
    uint32_t w[8], col[4][2];
#pragma unroll
    for (int q = 0; q < 8; ++q) w[q] = tile[(r0 + q) * kPitch + k4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t* const v = w + 4 * h;
      const uint32_t a01 = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), a23 = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u);
      const uint32_t b01 = __builtin_amdgcn_perm(v[1], v[0], 0x07030602u), b23 = __builtin_amdgcn_perm(v[3], v[2], 0x07030602u);
      col[0][h] = __builtin_amdgcn_perm(a23, a01, 0x05040100u);
      col[1][h] = __builtin_amdgcn_perm(a23, a01, 0x07060302u);
      col[2][h] = __builtin_amdgcn_perm(b23, b01, 0x05040100u);
      col[3][h] = __builtin_amdgcn_perm(b23, b01, 0x07060302u);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int k = kb * kBlock8 + 4 * k4 + q;
      if (k < a.K) *reinterpret_cast<u2v*>(a.codes_t + (e * a.K + k) * codes8(a.N) + nb * kBlock8 + r0) = u2v{col[q][0], col[q][1]};
    }
  }
}

template <typename F>
hipError_t with_group(const Pack8Args& a, int n_cu, F run) {
  const int blocks = (a.width + kBlock8 - 1) / kBlock8, quads = (blocks + 3) / 4;
  const int rows = blocks == 1 ? 4 : blocks == 2 ? 2 : 1;           // of a wavefront
  const int64_t units = (a.n + rows - 1) / rows * quads;
  const unsigned g = unsigned(std::max<int64_t>(1, std::min<int64_t>((units + 3) / 4, int64_t(n_cu) * 64)));
  const auto with = [&](auto w) {
    if (pack8_streams(a)) run(w, std::true_type(), g);
    else run(w, std::false_type(), g);
  };
  if (blocks == 1) with(std::integral_constant<int, 1>());
  else if (blocks == 2) with(std::integral_constant<int, 2>());
  else with(std::integral_constant<int, 4>());
  return hipGetLastError();
}

}  // namespace

#define PACK8_LAUNCH(kernel)                                                \
  return with_group(a, n_cu, [&](auto w, auto t, unsigned g) {              \
    if (a.bf16) kernel<true, w.value, t.value><<<g, 256, 0, s>>>(a);        \
    else kernel<false, w.value, t.value><<<g, 256, 0, s>>>(a);              \
  })

hipError_t launch_pack8(const Pack8Args& a, int n_cu, hipStream_t s) { PACK8_LAUNCH(k_pack8); }
hipError_t launch_unpack8(const Pack8Args& a, int n_cu, hipStream_t s) { PACK8_LAUNCH(k_unpack8); }
hipError_t launch_activate8(const Pack8Args& a, int n_cu, hipStream_t s) { PACK8_LAUNCH(k_activate8); }
hipError_t launch_activate8_backward(const Pack8Args& a, int n_cu, hipStream_t s) { PACK8_LAUNCH(k_activate8_backward); }

hipError_t launch_pack8_weights(const Weights8Args& a, hipStream_t s) {
  const dim3 g{unsigned((a.K + kBlock8 - 1) / kBlock8), unsigned((a.N + kBlock8 - 1) / kBlock8), unsigned(a.E)};
  if (a.bf16) k_pack8_weights<true><<<g, 256, 0, s>>>(a);
  else k_pack8_weights<false><<<g, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mlip
