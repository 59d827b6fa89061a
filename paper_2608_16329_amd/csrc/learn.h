// Internal declarations of the learning operators: the context they share and
// the host-side launchers of their kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <string>
#include <vector>

#include "../../include/mlip.h"

namespace mlip {

// A piece of a tensor of an AdamW plan, as the kernels read it: up to
// kAdamPiece elements, 256 a wavefront, which are a block of 8-bit moments.
constexpr int kAdamPiece = 1024;
struct AdamPiece {
  void* param;                // at the piece's first element
  void* into;
  const void* grad;
  int64_t at;                 // its first element among the moments
  int64_t block;              // its first block of 8-bit moments
  int32_t n;
  uint8_t param_bf16, grad_bf16, decay, pad;
};

}  // namespace mlip

struct mlip_learn {
  hipStream_t stream = nullptr;
  int device = 0;
  int n_cu = 0;
  std::string err;
  unsigned char* d_ws = nullptr;  // workspace of the calls, in the order of the stream
  size_t cap_ws = 0;
  bool recorded_ws = false;       // a recorded call uses it
  std::vector<unsigned char*> kept;   // earlier workspaces that recorded calls use
  size_t kept_bytes = 0;
};

struct mlip_adamw {
  hipStream_t stream = nullptr;
  int device = 0;
  int n_cu = 0;
  int bits = 32;
  bool into = false;          // the plan has a second set of parameters
  int64_t elements = 0, blocks = 0, pieces = 0;
  std::string err;
  mlip::AdamPiece* d_pieces = nullptr;
};

namespace mlip {

constexpr int kMaxExperts = 256;   // heads a row can be routed to
constexpr int kMaxTopK = 16;
constexpr int kMaxHeadInputs = 1024;
constexpr int kMaxHeadLayers = 8;

// Arguments of the routing kernels (mlip_route, mlip_route_backward).
struct RouteArgs {
  int64_t n;
  int64_t stride;             // values between rows of the logits
  int E, K, n_kinds;
  bool bf16, all;             // logits' type; gates are the probabilities themselves
  const void* logits;
  const int32_t* kinds;       // [n] or null
  const uint8_t* allowed;     // [n_kinds][E] (with kinds)
  int32_t* experts;           // [n][K]
  float* gates;               // [n][K]
  int32_t* counts;            // [E + 1]
  float* loss;                // [1]
  const float* dgates;        // [n][K] or null
  const float* dloss;         // [1] or null
  void* dlogits;              // [n][E], the logits' type
  float* part_p;              // [blocks][E] sums of probabilities
  int32_t* part_c;            // [blocks][E + 1] counts, routed rows
};
int route_blocks(int64_t n, int E, int n_cu);
hipError_t launch_route(const RouteArgs& a, int blocks, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs& a, int n_cu, hipStream_t s);

// Stable counting sort of m entries by expert; ids outside [0, E) come last.
size_t group_ws_bytes(int64_t m, int E);
hipError_t launch_group(const int32_t* experts, int64_t m, int E, int32_t* offsets, int32_t* order, void* ws, hipStream_t s);

// Arguments of the energy heads' kernels (mlip_heads).
struct HeadsArgs {
  int64_t n;
  int64_t m;                  // entries, n top_k
  int64_t stride;             // values between rows of x
  int E, D, H, K;
  bool bf16;                  // x and dx
  int blocks;                 // work-groups that share the tiles
  int waves;                  // wavefronts of one, 16 rows of a tile each
  int64_t values;             // of one head
  const void* x;
  const float* weights;       // [E][values]
  const int32_t* offsets;     // [E + 1]
  const int32_t* order;       // [m]
  const float* gates;         // [m] or null
  const float* denergy;       // [n] or null (ones)
  float* energy;              // [n] or null
  void* dx;                   // [n][D] or null
  float* dweights;            // [E][values] or null
  float* dgates;              // [m] or null
  float* entry_energy;        // [m], with several entries a row
  float* entry_dx;            // [m][D], with several entries a row and dx
  void* padded;               // [n][4], x with fewer than four inputs
  unsigned char* split;       // the heads' matrices in limbs, split_block bytes a block
  int64_t split_block;
  float* slots;               // [blocks + E][slot] sums of a work-group for a head
  int64_t slot;
  float* kept;                // y of a tile's layers in the middle, 16 waves x 64 values each
};
// Sets waves, blocks, split_block and slot; the workspace in bytes, which
// heads_workspace divides.
size_t heads_plan(HeadsArgs* a, int n_cu);
void heads_workspace(HeadsArgs* a, unsigned char* ws);
hipError_t launch_heads(const HeadsArgs& a, hipStream_t s);

// Arguments of the AdamW kernels.
struct AdamArgs {
  const AdamPiece* piece;
  int64_t pieces;
  int bits;
  bool reverse;               // reads `into` and writes `param`
  const void* m;              // float32 or codes [elements]
  const void* v;
  const uint8_t* m_exp;       // [blocks], 8 bits: e + 127
  const uint8_t* v_exp;
  void* new_m;
  void* new_v;
  uint8_t* new_m_exp;
  uint8_t* new_v_exp;
};
struct AdamStep {
  double lr, beta1, beta2, eps, weight_decay, grad_scale;
  double correction1;         // 1 - beta1^t
  double root_correction2;    // sqrt(1 - beta2^t)
  uint32_t seed;
};
hipError_t launch_adamw(const AdamArgs& a, const AdamStep& h, int n_cu, hipStream_t s);
hipError_t launch_moments(const AdamArgs& a, float* m_out, float* v_out, int n_cu, hipStream_t s);

}  // namespace mlip
