// Rows brought into the experts' order and back with weights, and the gradient.
//
//   xs[p] = x[order[p] / k], p < offsets[E]; places[order[p]] = p, -1 from there on
//   out_i = sum_s g_is y[places_is]
//   dy[places_is] = g_is dout_i,  dg_is = <dout_i, y[places_is]>
// and the gradient of the first in x is the second without weights.
//
// Bound by memory: each row is read once and written once, whole, in pieces of 16
// bytes a lane.  A row has a group of 8 to 64 lanes, as many as take about four
// pieces each, whose loads are under way together.  Sums are float32, in the
// order of s; nothing is added up by atomics.
// 262,144 rows of 1,024 bfloat16 values, 2 of 16 experts each: sorting 336 us (4.8 TB/s of
// what is read and written, 6.4 with a row's second reading; a copy of 1 GiB 5.15),
// combining 257 (6.3: some of it is still in the last cache), combining's gradient with
// the gates' 493 (5.4).  32,767 rows of 385 float32 values, 3 of 29 experts: 49, 50
// and 72 us, 39, 30 and 74 where the last cache has them.  Places alone, 8 lanes an entry of
// which one works: 262,144 entries 6.3 us, 524,288 9.9, 2 1.5.
#include <algorithm>

#include "layers_math.h"

namespace mlip {
namespace {

constexpr int kPieces = 4;      // 16-byte pieces a lane has under way

// A row's pieces of 16 bytes: the last one ends where the row does, and has some of
// the values of the one before it again (a row of less than 16 bytes has none, and
// its values go one a lane).
struct Shape {
  int pieces, last, few, size;  // pieces, where the last one starts, values of a short row, bytes of a value
  __device__ __forceinline__ int at(int c) const { return min(16 * c, last); }
};
__device__ __forceinline__ Shape shape(const RowsArgs& a) {
  const int size = a.bf16 ? 2 : 4, bytes = a.width * size;
  return bytes < 16 ? Shape{0, 0, a.width, size} : Shape{(bytes + 15) / 16, bytes - 16, 0, size};
}

// Where entry `e` stands: its place, or -1 for none (and for what is no place).
__device__ __forceinline__ int64_t place_of(const RowsArgs& a, int64_t e) {
  const int64_t p = a.places[e];
  return p < a.m ? p : -1;
}

template <bool BF>
__device__ __forceinline__ void add(float* sum, const u4v v, float g) {
  if (BF) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[2 * q] = fmaf(g, __uint_as_float(v[q] << 16), sum[2 * q]);
      sum[2 * q + 1] = fmaf(g, __uint_as_float(v[q] & 0xffff0000u), sum[2 * q + 1]);
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] = fmaf(g, __uint_as_float(v[q]), sum[q]);
  }
}
template <bool BF>
__device__ __forceinline__ u4v rounded(const float* v) {
  u4v u;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    u[q] = BF ? bf16x2(v[2 * q], v[2 * q + 1]) : __float_as_uint(v[q]);
  return u;
}
template <bool BF>
__device__ __forceinline__ float value(const void* p, int64_t at) {
  return BF ? from_bf16(static_cast<const uint16_t*>(p)[at]) : static_cast<const float*>(p)[at];
}
template <bool BF>
__device__ __forceinline__ void set(void* p, int64_t at, float v) {
  if (BF) static_cast<uint16_t*>(p)[at] = to_bf16(v);
  else static_cast<float*>(p)[at] = v;
}

// One group of lanes for each place in the experts' order.
template <bool BF, int L, bool STREAM>
__global__ __launch_bounds__(256) void k_sort(RowsArgs a) {
  const Shape f = shape(a);
  const int lane = threadIdx.x % L;
  const int64_t end = min(a.m, max(int64_t(0), int64_t(a.offsets[a.E])));
  for (int64_t p = int64_t(blockIdx.x) * (256 / L) + threadIdx.x / L; p < a.m; p += int64_t(gridDim.x) * (256 / L)) {
    const uint32_t entry = uint32_t(a.order[p]);
    if (entry >= a.m) continue;
    if (lane == 0) a.places[entry] = p < end ? int32_t(p) : -1;
    if (p >= end || !a.out) continue;
    const char* from = static_cast<const char*>(a.x) + int64_t(entry / uint32_t(a.K)) * a.x_stride * f.size;
    char* to = static_cast<char*>(a.out) + p * a.width * f.size;
    for (int c = lane; c < f.pieces; c += L * kPieces) {
      u4v v[kPieces];
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
        if (c + q * L < f.pieces) v[q] = *reinterpret_cast<const U4*>(from + f.at(c + q * L));
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
        if (c + q * L < f.pieces) give16<STREAM>(to + f.at(c + q * L), v[q]);
    }
    if (lane < f.few) {
      if (BF) reinterpret_cast<uint16_t*>(to)[lane] = reinterpret_cast<const uint16_t*>(from)[lane];
      else reinterpret_cast<uint32_t*>(to)[lane] = reinterpret_cast<const uint32_t*>(from)[lane];
    }
  }
}

// One group of lanes for each row.
template <bool BF, int L, bool STREAM>
__global__ __launch_bounds__(256) void k_combine(RowsArgs a) {
  constexpr int V = BF ? 8 : 4;
  const Shape f = shape(a);
  const int lane = threadIdx.x % L;
  for (int64_t i = int64_t(blockIdx.x) * (256 / L) + threadIdx.x / L; i < a.n; i += int64_t(gridDim.x) * (256 / L)) {
    char* to = static_cast<char*>(a.out) + i * a.width * f.size;
    for (int c = lane; c < f.pieces; c += L * kPieces) {
      float sum[kPieces][V] = {};
      // two entries at a time, whose rows are under way together
      for (int s = 0; s < a.K; s += 2) {
        int64_t p[2];
        float g[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          p[h] = s + h < a.K ? place_of(a, i * a.K + s + h) : -1;
          g[h] = a.gates && s + h < a.K ? a.gates[i * a.K + s + h] : 1.f;
        }
        u4v v[2][kPieces];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const char* const from = static_cast<const char*>(a.x) + p[h] * a.x_stride * f.size;
#pragma unroll
          for (int q = 0; q < kPieces; ++q)
            if (p[h] >= 0 && c + q * L < f.pieces) v[h][q] = take16<STREAM>(from + f.at(c + q * L));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int q = 0; q < kPieces; ++q)
            if (p[h] >= 0 && c + q * L < f.pieces) add<BF>(sum[q], v[h][q], g[h]);
      }
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
        if (c + q * L < f.pieces) give16<STREAM>(to + f.at(c + q * L), rounded<BF>(sum[q]));
    }
    if (lane < f.few) {
      float sum = 0.f;
      for (int s = 0; s < a.K; ++s) {
        const int64_t p = place_of(a, i * a.K + s);
        if (p >= 0) sum = fmaf(a.gates ? a.gates[i * a.K + s] : 1.f, value<BF>(a.x, p * a.x_stride + lane), sum);
      }
      set<BF>(a.out, i * a.width + lane, sum);
    }
  }
}

// One group of lanes for each row: its gradient goes to its entries' places, and
// its products with the experts' outputs there are the gates' gradients.
template <bool BF, int L, bool STREAM>
__global__ __launch_bounds__(256) void k_combine_backward(RowsArgs a) {
  constexpr int V = BF ? 8 : 4;
  const Shape f = shape(a);
  const int lane = threadIdx.x % L;
  for (int64_t i = int64_t(blockIdx.x) * (256 / L) + threadIdx.x / L; i < a.n; i += int64_t(gridDim.x) * (256 / L)) {
    const char* from = static_cast<const char*>(a.x) + i * a.x_stride * f.size;
    for (int s = 0; s < a.K; ++s) {
      const int64_t p = place_of(a, i * a.K + s);
      float dot = 0.f;
      if (p >= 0) {
        const float g = a.gates ? a.gates[i * a.K + s] : 1.f;
        const char* y = static_cast<const char*>(a.y) + p * a.y_stride * f.size;
        char* to = static_cast<char*>(a.out) + p * a.width * f.size;
        for (int c = lane; c < f.pieces; c += L * kPieces) {
          u4v d[kPieces], v[kPieces];
#pragma unroll
          for (int q = 0; q < kPieces; ++q)
            if (c + q * L < f.pieces) {
              d[q] = *reinterpret_cast<const U4*>(from + f.at(c + q * L));
              if (a.dgates) v[q] = take16<STREAM>(y + f.at(c + q * L));
            }
#pragma unroll
          for (int q = 0; q < kPieces; ++q)
            if (c + q * L < f.pieces) {
              float dv[V] = {}, out[V];
              add<BF>(dv, d[q], 1.f);
              if (a.dgates) {
                float yv[V] = {};
                add<BF>(yv, v[q], 1.f);
                // (values that the piece before has count there)
                const int again = (16 * (c + q * L) - f.at(c + q * L)) / f.size;
#pragma unroll
                for (int j = 0; j < V; ++j) dot = j >= again ? fmaf(dv[j], yv[j], dot) : dot;
              }
#pragma unroll
              for (int j = 0; j < V; ++j) out[j] = g * dv[j];
              give16<STREAM>(to + f.at(c + q * L), rounded<BF>(out));
            }
        }
        if (lane < f.few) {
          const float d = value<BF>(a.x, i * a.x_stride + lane);
          if (a.dgates) dot = fmaf(d, value<BF>(a.y, p * a.y_stride + lane), dot);
          set<BF>(a.out, p * a.width + lane, g * d);
        }
      }
      if (a.dgates) {
#pragma unroll
        for (int o = L / 2; o > 0; o /= 2) dot += __shfl_xor(dot, o);
        if (lane == 0) a.dgates[i * a.K + s] = dot;
      }
    }
  }
}

// Lanes of a row: 8 to 64, about kPieces pieces each (385 float32 values, 97 pieces,
// 32 lanes: sorting, combining twice and its gradient 220 us; 16 lanes 245, 64 lanes 224).
int lanes(const RowsArgs& a) {
  const int pieces = (a.width * (a.bf16 ? 2 : 4) + 15) / 16;
  int l = 8;
  while (l < 64 && l * kPieces < pieces) l *= 2;
  return l;
}
int grid(int64_t rows, int l, int n_cu) { return int(std::max<int64_t>(1, std::min<int64_t>((rows * l + 255) / 256, int64_t(n_cu) * 64))); }

// Rows in the experts' order that are more than the last cache, of 256 MB, holds go past
// it in and out: what comes next would not find them there, and the rows of the
// caller's order, which are read once for each expert, stay longer (262,144 rows of 1,024
// bfloat16 values, 2 experts each: sorting 394 us and 336 so, combining 294 and 261, its
// gradient 525 and 493; 32,767 rows of 385 float32 values, 3 each, 151 MB, called
// again and again: 39 and 41, 30 and 39, 74 and 82).
bool streams(const RowsArgs& a) { return a.m * a.width * (a.bf16 ? 2 : 4) > int64_t(1) << 28; }

template <typename F>
void with_lanes(int l, bool stream, F run) {
  const auto with = [&](auto w) {
    if (stream) run(w, std::true_type());
    else run(w, std::false_type());
  };
  if (l == 8) with(std::integral_constant<int, 8>());
  else if (l == 16) with(std::integral_constant<int, 16>());
  else if (l == 32) with(std::integral_constant<int, 32>());
  else with(std::integral_constant<int, 64>());
}

}  // namespace

#define ROWS_LAUNCH(kernel, rows)                                                                                      \
  const int l = lanes(a), g = grid(rows, l, n_cu);                                                                     \
  if (a.bf16) with_lanes(l, streams(a), [&](auto w, auto t) { kernel<true, w.value, t.value><<<g, 256, 0, s>>>(a); });     \
  else with_lanes(l, streams(a), [&](auto w, auto t) { kernel<false, w.value, t.value><<<g, 256, 0, s>>>(a); });          \
  return hipGetLastError()

hipError_t launch_sort(const RowsArgs& a, int n_cu, hipStream_t s) { ROWS_LAUNCH(k_sort, a.m); }
hipError_t launch_combine(const RowsArgs& a, int n_cu, hipStream_t s) { ROWS_LAUNCH(k_combine, a.n); }
hipError_t launch_combine_backward(const RowsArgs& a, int n_cu, hipStream_t s) { ROWS_LAUNCH(k_combine_backward, a.n); }

}  // namespace mlip
