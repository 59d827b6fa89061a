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
