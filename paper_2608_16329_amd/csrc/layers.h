// Internal declarations of the operators that wide layers of experts are made of
// (mlip_sort .. mlip_activate8_backward): arguments and host-side launchers of
// their kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mlip {

constexpr int kMaxLayerWidth = 65536;
constexpr int kBlock8 = 128;                        // values that share a power of two
// Bytes of a row's codes and of its exponents: whole blocks, whole groups of four blocks.
__host__ __device__ constexpr int64_t codes8(int64_t width) { return (width + 127) / 128 * 128; }
__host__ __device__ constexpr int64_t exps8(int64_t width) { return ((width + 127) / 128 + 3) / 4 * 4; }

// Rows in the caller's order and in the experts' (mlip_sort, mlip_combine and its gradient).
struct RowsArgs {
  int64_t n;
  int64_t m;                  // entries, n top_k
  int E, K, width;
  bool bf16;
  const void* x;              // rows of n (sort, combine_backward: dout) or of m (combine)
  int64_t x_stride;
  const void* y;              // [m], combine_backward
  int64_t y_stride;
  const int32_t* offsets;     // [E + 1]
  const int32_t* order;       // [m]
  int32_t* places;            // [n][K]
  const float* gates;         // [n][K] or null
  void* out;
  float* dgates;              // [n][K] or null
};
hipError_t launch_sort(const RowsArgs& a, int n_cu, hipStream_t s);
hipError_t launch_combine(const RowsArgs& a, int n_cu, hipStream_t s);
hipError_t launch_combine_backward(const RowsArgs& a, int n_cu, hipStream_t s);

// Rows to and from 8 bits, and activations that keep them.
struct Pack8Args {
  int64_t n;                  // rows that are written
  int E, K, width;
  bool bf16;
  const void* x;              // x, z or dh
  int64_t x_stride;
  const void* residual;
  int64_t residual_stride;
  const int32_t* offsets;     // with order
  const int32_t* order;       // [n] or null
  const uint8_t* kept;        // codes that are read
  const uint8_t* kept_exps;
  void* out;                  // values in x's type, or null
  uint8_t* codes;             // of x, or of z
  uint8_t* exps;
  uint8_t* out_codes;         // of h or dz, or null
  uint8_t* out_exps;
};
// Whether values go past the last cache, of 256 MB, in and out: where they are more
// than it holds, what comes next would not find them there, and finds the codes (65,536
// rows of 4,096 bfloat16 values: packing 148 us and 126 so, unpacking 141 and 120, the
// activation 250 and 220, its gradient 252 and 203; 16,384 rows of 2,048, which stay there
// from call to call, 19 and 22, 16 and 15, 31 and 34, 33 and 38).
// With an order each row is read again for each of its experts, so rows that stay there
// together with their codes do not go past it (1,024 bfloat16 values, through the cache and
// past it: 10,240 rows, 16 experts each, 75 us and 97, 131 and 155 with unpacking behind it;
// 45,000 rows, 3 each, 62 and 82, 111 and 131).  Where they do not fit, the codes count, which
// what comes next reads: 131,072 rows, 2 each, 153 and 149, 291 and 261 with unpacking; 65,536
// rows, 4 each, 127 and 148, 280 and 259 (but 100,000 rows of 512 float32 values, 8 each, 276
// and 390, 655 and 763: codes that do not fit by themselves gain nothing).
inline bool pack8_streams(const Pack8Args& a) {
  constexpr int64_t kCache = int64_t(1) << 28;
  const int64_t values = a.n * a.width * (a.bf16 ? 2 : 4);
  return values > kCache && (!a.order || values / a.K + a.n * (codes8(a.width) + exps8(a.width)) > kCache);
}
hipError_t launch_pack8(const Pack8Args& a, int n_cu, hipStream_t s);
hipError_t launch_unpack8(const Pack8Args& a, int n_cu, hipStream_t s);
hipError_t launch_activate8(const Pack8Args& a, int n_cu, hipStream_t s);
hipError_t launch_activate8_backward(const Pack8Args& a, int n_cu, hipStream_t s);

struct Weights8Args {
  int E, N, K;                // matrices [N][K]
  bool bf16;
  const void* w;
  uint8_t* codes;             // [E][N][codes8(K)] or null
  uint8_t* exps;              // [E][blocks of N][exps8(K)]
  uint8_t* codes_t;           // [E][K][codes8(N)] or null
  uint8_t* exps_t;            // [E][blocks of K][exps8(N)]
};
hipError_t launch_pack8_weights(const Weights8Args& a, hipStream_t s);

// y = W x + c over rows grouped by expert, and the gradients of W and c.
struct Product8Args {
  int64_t m;
  int E, N, K;                // outputs (rows of W), inputs
  bool bf16;                  // y
  const uint8_t* x;           // [m][codes8(K)]
  const uint8_t* x_exps;
  const uint8_t* w;           // [E][N][codes8(K)]; the gradient's dy [m][codes8(N)]
  const uint8_t* w_exps;
  const int32_t* offsets;     // [E + 1], or null: one expert has all rows
  const float* bias;          // [E][N] or null
  void* y;                    // [m][N]
  float* dweights;            // [E][N][K]
  float* dbias;               // [E][N] or null
  int64_t slice;              // rows of a work-group of the gradient
  float* slots;               // [items][N][K] sums of slices, or null: one slice an expert
  float* bias_slots;          // [items][N]
};
hipError_t launch_product8(const Product8Args& a, int n_cu, hipStream_t s);
// Sets slice; the workspace in bytes, which product8_workspace divides.
size_t product8_weights_plan(Product8Args* a, int n_cu);
void product8_workspace(Product8Args* a, unsigned char* ws);
hipError_t launch_product8_weights(const Product8Args& a, int n_cu, hipStream_t s);

}  // namespace mlip
