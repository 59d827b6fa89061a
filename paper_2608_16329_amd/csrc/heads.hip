// Energy heads over rows (atoms) grouped by head: energies, and the gradients
// in the descriptors, the weights and the gates.
//
//   z_0 = A_0 x + c_0, y_0 = silu(z_0);  z_t = A_t y_{t-1} + c_t, y_t = y_{t-1} + silu(z_t);
//   v = a . y_{H-1} + c;  energy_i = sum_s gate_is v_is
//   u = d a with d = denergy_i gate_is;  down from t = H-1: g_t = u silu'(z_t),
//   dA_t += g_t y_{t-1}^T, dc_t += g_t, u += A_t^T g_t;  dA_0 += g_0 x^T, dx = A_0^T g_0;
//   da += d y_{H-1}, dc += d, dgate_is = denergy_i v_is.
//
// One kernel takes a row through all of it.  A work-group has a tile of rows
// of one head, each wavefront 16 of them as the columns of 16x16x4 matrix
// products in float32: a layer's result is, register by register, the second
// operand of the next layer's product (the products sum over inputs 16 T + 4 g
// + i in lane group g, step i, which is where results 4 g + i stand), so y, z
// and u never leave registers.  The layers' matrices go through LDS one 64x64
// block at a time, the next block loaded while one is used.  The weights'
// gradients are products over rows: g and y change places through LDS, each
// wavefront owns some of the 16 result tiles of every layer and keeps their
// sums over all of the work-group's tiles of a head, which are written once
// and added up in order by a second kernel.
#include <algorithm>

#include "learn.h"
#include "learn_math.h"

namespace mlip {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kR = 64;                 // hidden width
constexpr int kWS = kR + 4;            // LDS row of a 64x64 block: 4 mod 64 banks apart
constexpr int kWBlock = kR * kWS;
constexpr int kTStride = kR + 16;      // LDS row of g and y: four rows 16 banks apart, as the lane groups read them
constexpr int kChunksHeld = 2;         // 64-input chunks whose gradient sums stay in registers

__device__ __forceinline__ f4 mfma(float a, float b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// Tiles of each head (and of the entries without one, as head E): first tile
// and first entry, from the entries' offsets kept within [0, m].  All threads
// call; E + 2 values each.
__device__ void tile_table(const HeadsArgs& a, int rows, int32_t* first, int32_t* entry) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    int run = 0, before = 0;
    for (int e0 = 0; e0 <= a.E; e0 += 64) {
      const int e = e0 + lane;
      // offsets rise and end at m, whatever the caller has in them
      int lo = e <= a.E ? a.offsets[e] : int(a.m);
      lo = lo < 0 ? 0 : (lo > a.m ? int(a.m) : lo);
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(lo, o, 64);
        lo = lane >= o && t > lo ? t : lo;
      }
      lo = lo < before ? before : lo;
      if (e == 0) lo = 0;
      int hi = __shfl_down(lo, 1, 64);
      if (lane == 63 || e == a.E) {
        hi = e + 1 <= a.E ? a.offsets[e + 1] : int(a.m);
        hi = hi < lo ? lo : (hi > a.m ? int(a.m) : hi);
      }
      const int tiles = e <= a.E ? (hi - lo + rows - 1) / rows : 0;
      int v = tiles;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(v, o, 64);
        v += lane >= o ? t : 0;
      }
      if (e <= a.E) {
        first[e] = run + v - tiles;
        entry[e] = lo;
        if (e == a.E) first[a.E + 1] = run + v, entry[a.E + 1] = int(a.m);
      }
      run += __shfl(v, 63, 64);
      before = __shfl(lo, 63, 64);
    }
  }
  __syncthreads();
}

// First tile of work-group b of `blocks` that share `tiles`.
__device__ __forceinline__ int share(int64_t tiles, int64_t b, int blocks) { return int(tiles * b / blocks); }

__device__ __forceinline__ f4 vec4(const float* p) {
  const F4 f = *reinterpret_cast<const F4*>(p);
  f4 t;
#pragma unroll
  for (int k = 0; k < 4; ++k) t[k] = f.v[k];
  return t;
}
// The same from a place that all lanes share, and the lane's own bytes from there.
__device__ __forceinline__ f4 vec4(const float* base, uint32_t bytes) {
  return vec4(reinterpret_cast<const float*>(reinterpret_cast<const char*>(base) + bytes));
}
// The same value, not known to be: what is computed from it is computed where
// it is used and not kept in registers around the loop over tiles.
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}
// 64 values as the lanes hold a column: 16 t + 4 g + i in v[t][i].
__device__ __forceinline__ void column(const float* base, f4 v[4]) {
  const uint32_t bytes = here(threadIdx.x & 48);
#pragma unroll
  for (int t = 0; t < 4; ++t) v[t] = vec4(base, bytes + 64 * t);
}
// A value that all lanes hold, for the scalar registers.
__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A 64 x 64 block of a head's weights on its way to LDS: rows of `ld` values.
// Of a block with fewer than 64 columns the rest is what follows in the head's
// table (its rows, then the bias): it is multiplied by zeros.
template <int NW>
struct Staged {
  static constexpr int kPer = 16 / NW;   // groups of four values a thread
  f4 v[kPer];
  __device__ __forceinline__ void load(const float* src, int ld) {
    const uint32_t tid = here(threadIdx.x), r = tid / NW, q = tid % NW;
#pragma unroll
    for (int j = 0; j < kPer; ++j) v[j] = vec4(src, 4 * (r * uint32_t(ld) + 4 * q) + 16 * NW * j);
  }
  __device__ __forceinline__ void store(float* lds) const {
    const int r = threadIdx.x / NW, q = threadIdx.x % NW;
#pragma unroll
    for (int j = 0; j < kPer; ++j) *reinterpret_cast<f4*>(lds + r * kWS + 4 * (q + NW * j)) = v[j];
  }
};

// out += block in: 64 inputs from registers, 16 at a time, the next group's
// weights loaded before this one's products (and no further ahead: loads of
// the whole block at once take the registers that sums need).
__device__ __forceinline__ void product(const float* w, const f4 in[4], f4 out[4]) {
  const int c = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
  const float* row = w + here(c * kWS + 4 * g);
  f4 wa[2][4];
#pragma unroll
  for (int t = 0; t < 4; ++t) wa[0][t] = *reinterpret_cast<const f4*>(row + 16 * t * kWS);
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    __builtin_amdgcn_sched_barrier(0);
    if (T < 3) {
#pragma unroll
      for (int t = 0; t < 4; ++t) wa[(T + 1) & 1][t] = *reinterpret_cast<const f4*>(row + 16 * t * kWS + 16 * (T + 1));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t) out[t] = mfma(wa[T & 1][t][i], in[T][i], out[t]);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// out += block^T in.
__device__ __forceinline__ void product_t(const float* w, const f4 in[4], f4 out[4]) {
  const int c = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
  const float* row = w + here(4 * g * kWS + c);
  float wa[2][2][4];
  auto fetch = [&](int k) {   // inputs 16 T + 4 g + i for i = 2 (k & 1) and the next, T = k / 2
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t) wa[k & 1][j][t] = row[(16 * (k >> 1) + 2 * (k & 1) + j) * kWS + 16 * t];
  };
  fetch(0);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    __builtin_amdgcn_sched_barrier(0);
    if (k < 7) fetch(k + 1);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < 4; ++t) out[t] = mfma(wa[k & 1][j][t], in[k >> 1][2 * (k & 1) + j], out[t]);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// The row of a lane's column in a tile.
struct Row {
  int64_t entry;   // -1: none
  int64_t i;
  float gate, up;  // gate and denergy
};
__device__ __forceinline__ Row row_of(const HeadsArgs& a, int64_t at, int64_t end) {
  Row r{-1, 0, 0.f, 0.f};
  if (at < end) {
    const int64_t ent = a.order[at];
    if (ent >= 0 && ent < a.m) {
      r.entry = ent;
      r.i = a.K == 1 ? ent : ent / a.K;
      r.gate = a.gates ? a.gates[ent] : 1.f;
      r.up = a.denergy ? a.denergy[r.i] : 1.f;
    }
  }
  return r;
}

template <bool BF>
__device__ __forceinline__ f4 x4(const void* p, int64_t at) {
  f4 f;
  if (BF) {
    const H4 h = *reinterpret_cast<const H4*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = from_bf16(h.v[i]);
  } else {
    f = vec4(static_cast<const float*>(p) + at);
  }
  return f;
}

// Inputs 64 ch .. 64 ch + 63 of the lane's row: 16 T + 4 g + i in in[T][i],
// zero from the last on.  Every lane loads four values that are there; where
// they are the row's last four and not the ones asked for, they are shifted.
template <bool BF>
__device__ __forceinline__ void load_x(const HeadsArgs& a, const Row& r, int ch, f4 in[4]) {
  const int g = (threadIdx.x >> 4) & 3;
  const int64_t row = r.i * a.stride;
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    const int c = 64 * ch + 16 * T + 4 * g;
    f4 f;
    int shift = 0;
    if (a.D >= 4) {
      const int from = min(c, a.D - 4);
      f = x4<BF>(a.x, row + from);
      shift = c - from;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t at = row + min(i, a.D - 1);
        f[i] = BF ? from_bf16(static_cast<const uint16_t*>(a.x)[at]) : static_cast<const float*>(a.x)[at];
      }
      if (a.D < 4) f[3] = 0.f;
      if (a.D < 3) f[2] = 0.f;
      if (a.D < 2) f[1] = 0.f;
      shift = c;
    }
    if (a.D & 3) {
      if (shift & 1) f = f4{f[1], f[2], f[3], 0.f};
      if (shift & 2) f = f4{f[2], f[3], 0.f, 0.f};
    }
    const bool there = shift < 4 && r.entry >= 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) in[T][i] = there ? f[i] : 0.f;
  }
}

// d[T][i] to the row of `to` at inputs 64 ch + 16 T + 4 g + i, those below `D`.
template <bool BF>
__device__ __forceinline__ void store_row(void* to, int64_t row, int D, int ch, const f4 d[4]) {
  const int g = (threadIdx.x >> 4) & 3;
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    const int c = 64 * ch + 16 * T + 4 * g;
    if (c >= D) continue;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = d[T][i];
    store4(to, BF, row + c, D - c, v);
  }
}

template <bool BF>
__device__ __forceinline__ void store_dx(const HeadsArgs& a, const Row& r, int ch, const f4 d[4]) {
  if (r.entry < 0) return;
  if (a.K == 1) store_row<BF>(a.dx, r.i * a.D, a.D, ch, d);
  else store_row<false>(a.entry_dx, r.entry * a.D, a.D, ch, d);
}

// Value v of the lane's row: energy and the gate's gradient.
__device__ __forceinline__ void store_value(const HeadsArgs& a, const Row& r, float v) {
  if (r.entry < 0 || (threadIdx.x & 48)) return;
  if (a.energy) (a.K == 1 ? a.energy + r.i : a.entry_energy + r.entry)[0] = r.gate * v;
  if (a.dgates) a.dgates[r.entry] = r.up * v;
}

// Entries without a head: energies and gradients are zero.
template <int NW, bool BF>
__device__ void empty_tile(const HeadsArgs& a, int64_t at0, int64_t end) {
  const int lane = threadIdx.x & 63;
  const int64_t at = at0 + 16 * (threadIdx.x >> 6) + (lane & 15);
  Row r = row_of(a, at, end);
  r.gate = r.up = 0.f;   // the gate of such an entry may be anything
  store_value(a, r, 0.f);
  if (a.dx) {
    const f4 zero[4] = {};
    for (int ch = 0; 64 * ch < a.D; ++ch) store_dx<BF>(a, r, ch, zero);
  }
}

__device__ __forceinline__ const float* layer(const float* w, int D, int t) {
  return w + (kR * D + kR + (t - 1) * (kR * kR + kR));
}

// Energies alone.
template <int NW, bool BF>
__global__ __launch_bounds__(NW * 64) void k_energy(HeadsArgs a) {
  constexpr int kRows = 16 * NW;
  __shared__ int32_t s_first[kMaxExperts + 2], s_entry[kMaxExperts + 2];
  __shared__ __attribute__((aligned(16))) float s_w[2 * kWBlock];
  tile_table(a, kRows, s_first, s_entry);
  const int lane = threadIdx.x & 63, w = uni(threadIdx.x >> 6);
  const int tiles = uni(s_first[a.E + 1]);
  const int t_end = share(tiles, blockIdx.x + 1, a.blocks);
  const int chunks = (a.D + 63) / 64;
  int e = 0;
  for (int tile = share(tiles, blockIdx.x, a.blocks); tile < t_end; ++tile) {
    while (tile >= uni(s_first[e + 1])) ++e;
    const int64_t at0 = uni(s_entry[e]) + int64_t(tile - uni(s_first[e])) * kRows, end = uni(s_entry[e + 1]);
    if (e == a.E) {
      empty_tile<NW, BF>(a, at0, end);
      continue;
    }
    const float* wt = a.weights + e * a.values;
    const Row r = row_of(a, at0 + 16 * w + (lane & 15), end);
    Staged<NW> next;
    next.load(wt, a.D);
    f4 in[4];
    load_x<BF>(a, r, 0, in);
    __syncthreads();
    next.store(s_w);
    __syncthreads();
    int cur = 0;
    f4 z[4], y[4] = {};
      column(wt + kR * a.D, z);
    for (int ch = 0; ch < chunks; ++ch) {
      const bool more = ch + 1 < chunks;
      if (more) next.load(wt + 64 * (ch + 1), a.D);
      else if (a.H > 1) next.load(layer(wt, a.D, 1), kR);
      product(s_w + cur * kWBlock, in, z);
      if (more) load_x<BF>(a, r, ch + 1, in);
      if (more || a.H > 1) {
        next.store(s_w + (cur ^ 1) * kWBlock);
        cur ^= 1;
        __syncthreads();
      }
    }
    for (int l = 1;; ++l) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[t][i] += z[t][i] * sigmoid(z[t][i]);
      if (l == a.H) break;
      const float* bias = layer(wt, a.D, l) + kR * kR;
      column(bias, z);
      if (l + 1 < a.H) next.load(layer(wt, a.D, l + 1), kR);
      product(s_w + cur * kWBlock, y, z);
      if (l + 1 < a.H) {
        next.store(s_w + (cur ^ 1) * kWBlock);
        cur ^= 1;
        __syncthreads();
      }
    }
    const float* out = layer(wt, a.D, a.H);
    float v = 0.f;
    f4 o[4];
    column(out, o);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) v += o[t][i] * y[t][i];
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
    store_value(a, r, v + out[kR]);
  }
}

// Values of a slot: result tiles in the order of the registers (256 a tile, 16
// tiles a 64x64 block: the chunks of A_0, then A_1 ..), then dc_0 .. dc_{H-1},
// da, dc.
__host__ __device__ __forceinline__ int64_t slot_block(int D, int b) { return int64_t(b) * kR * kR; }
__host__ __device__ __forceinline__ int64_t slot_values(int D, int H) {
  return int64_t((D + 63) / 64 + H - 1) * kR * kR + int64_t(H + 1) * kR + 64;
}

// Energies, gradients in the descriptors and (TRAIN) in the weights.
template <int H, int NW, bool TRAIN, bool BF>
__global__ __launch_bounds__(NW * 64) void k_gradient(HeadsArgs a) {
  constexpr int kRows = 16 * NW;
  constexpr int kTS = kTStride;
  constexpr int kOwn = 16 / NW;          // result tiles of a wavefront in a 64x64 block
  extern __shared__ __attribute__((aligned(16))) float s_mem[];
  float* const s_w = s_mem;              // two blocks of weights
  float* const s_g = s_mem + 2 * kWBlock;
  float* const s_y = s_g + kRows * kTS;
  __shared__ int32_t s_first[kMaxExperts + 2], s_entry[kMaxExperts + 2];
  tile_table(a, kRows, s_first, s_entry);
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int w = uni(tid >> 6);
  const int tiles = uni(s_first[a.E + 1]);
  const int t_begin = share(tiles, blockIdx.x, a.blocks), t_end = share(tiles, blockIdx.x + 1, a.blocks);
  const int chunks = (a.D + 63) / 64;
  // the wavefront's tiles of a block: outputs 16 ta .., inputs 16 (tb + k) ..
  const int ta = NW == 8 ? w >> 1 : w, tb = NW == 8 ? 2 * (w & 1) : 0;

  f4 sum_h[H > 1 ? H - 1 : 1][kOwn], sum_0[kChunksHeld][kOwn];
  float sum_b[H], sum_a = 0.f, sum_c = 0.f;   // of dc_t and da, value `lane` over the wavefront's rows; of dc

  // sums of g y^T over the tile's rows into the wavefront's tiles
  auto outer = [&](f4 acc[kOwn]) {
    const int from = here(g * kTS + c);
    const float* gp = s_g + 16 * ta + from;
    const float* yp = s_y + 16 * tb + from;
    float ga[2][4], yb[2][kOwn][4];
    auto fetch = [&](int s) {   // rows 16 s + 4 i + g
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ga[s & 1][i] = gp[(16 * s + 4 * i) * kTS];
#pragma unroll
        for (int k = 0; k < kOwn; ++k) yb[s & 1][k][i] = yp[(16 * s + 4 * i) * kTS + 16 * k];
      }
    };
    fetch(0);
#pragma unroll
    for (int s = 0; s < NW; ++s) {
      __builtin_amdgcn_sched_barrier(0);
      if (s + 1 < NW) fetch(s + 1);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < kOwn; ++k) acc[k] = mfma(ga[s & 1][i], yb[s & 1][k][i], acc[k]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // v[t][i] of the lane's row, value 16 t + 4 g + i, to LDS
  auto to_lds = [&](int from, const f4 v[4]) {
    float* const mine = s_g + here((16 * w + c) * kTS + 4 * g);
#pragma unroll
    for (int t = 0; t < 4; ++t) *reinterpret_cast<f4*>(mine + from + 16 * t) = v[t];
  };
  // value `lane` of g over the wavefront's own rows, for the bias
  auto bias_sum = [&]() {
    const float* const g_own = s_g + here(16 * w * kTS + lane);
    float v = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) v += g_own[j * kTS];
    return v;
  };
  auto clear = [&]() {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
#pragma unroll
      for (int t = 0; t < (H > 1 ? H - 1 : 1); ++t) sum_h[t][k] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < kChunksHeld; ++t) sum_0[t][k] = f4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int t = 0; t < H; ++t) sum_b[t] = 0.f;
    sum_a = 0.f;
    sum_c = 0.f;
  };
  auto place = [&](float* slot, int b, int k) {
    return reinterpret_cast<f4*>(reinterpret_cast<char*>(slot + slot_block(a.D, b) + (4 * ta + tb + k) * 256) + uint32_t(16 * lane));
  };
  // the sums of head e to this work-group's slot for it; all threads call
  auto flush = [&](int e) {
    float* slot = a.slots + (int64_t(blockIdx.x) + e) * a.slot;
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
#pragma unroll
      for (int ch = 0; ch < kChunksHeld; ++ch)
        if (ch < chunks) *place(slot, ch, k) = sum_0[ch][k];
#pragma unroll
      for (int t = 1; t < H; ++t) *place(slot, chunks + t - 1, k) = sum_h[t - 1][k];
    }
    float* tail = slot + slot_block(a.D, chunks + H - 1);
    // dc_t, da and dc over the wavefronts
    constexpr int kSums = (H + 2) * kR;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < H; ++t) s_g[w * kSums + t * kR + lane] = sum_b[t];
    s_g[w * kSums + H * kR + lane] = sum_a;
    float v = sum_c;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o, 64);
    if (lane == 0) s_g[w * kSums + (H + 1) * kR] = v;
    __syncthreads();
    for (int at = tid; at <= (H + 1) * kR; at += NW * 64) {
      float v = 0.f;
#pragma unroll
      for (int u = 0; u < NW; ++u) v += s_g[u * kSums + at];
      tail[at] = v;
    }
    __syncthreads();
  };

  int e = 0;
  for (int tile = t_begin; tile < t_end;) {
    while (tile >= uni(s_first[e + 1])) ++e;
    const int stop = min(t_end, uni(s_first[e + 1]));
    const int64_t begin = uni(s_entry[e]), end = uni(s_entry[e + 1]), t0 = uni(s_first[e]);
    if (e == a.E) {
      for (; tile < stop; ++tile) empty_tile<NW, BF>(a, begin + (tile - t0) * kRows, end);
      break;
    }
    const float* wt = a.weights + e * a.values;
    if (TRAIN) clear();
    for (bool first = true; tile < stop; ++tile, first = false) {
      const int64_t at0 = begin + (tile - t0) * kRows;
      const Row r = row_of(a, at0 + 16 * w + c, end);
      Staged<NW> next;
      next.load(wt, a.D);
      f4 in[4];
      load_x<BF>(a, r, 0, in);
      __syncthreads();
      next.store(s_w);
      __syncthreads();
      int cur = 0;
      // forward: z_t of every layer and the last y stay
      f4 y[4] = {}, z[H][4];
      column(wt + kR * a.D, z[0]);
      for (int ch = 0; ch < chunks; ++ch) {
        const bool more = ch + 1 < chunks;
        if (more) next.load(wt + 64 * (ch + 1), a.D);
        else if (H > 1) next.load(layer(wt, a.D, 1), kR);
        product(s_w + cur * kWBlock, in, z[0]);
        if (more) load_x<BF>(a, r, ch + 1, in);
        if (more || H > 1) {
          next.store(s_w + (cur ^ 1) * kWBlock);
          cur ^= 1;
          __syncthreads();
        }
      }
#pragma unroll
      for (int l = 0; l < H; ++l) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) y[t][i] += z[l][t][i] * sigmoid(z[l][t][i]);
        if (l + 1 < H) {
          const float* bias = layer(wt, a.D, l + 1) + kR * kR;
      column(bias, z[l + 1]);
          if (l + 2 < H) next.load(layer(wt, a.D, l + 2), kR);
          product(s_w + cur * kWBlock, y, z[l + 1]);
          if (l + 2 < H) {
            next.store(s_w + (cur ^ 1) * kWBlock);
            cur ^= 1;
            __syncthreads();
          }
        }
      }
      const float* out = layer(wt, a.D, H);
      f4 u[4];
      const float d = r.entry >= 0 ? r.up * r.gate : 0.f;
      {
        float v = 0.f;
        column(out, u);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v += u[t][i] * y[t][i];
            u[t][i] *= d;
          }
        if (TRAIN) {
          sum_c += d;
          to_lds(kRows * kTS, y);
          const float* const y_own = s_y + here(16 * w * kTS + lane);
#pragma unroll
          for (int j = 0; j < 16; ++j)
            sum_a += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(d), j)) * y_own[j * kTS];
        }
        v += __shfl_xor(v, 16, 64);
        v += __shfl_xor(v, 32, 64);
        store_value(a, r, v + out[kR]);
      }
      // g_t = u silu'(z_t), and y_{t-1} from y_t (the sigmoid again: a tenth of the
      // products' time, where keeping y or silu' of every layer takes 16 registers
      // a layer that there are not)
      auto back = [&](f4 zl[4], f4 gz[4]) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // (so that the compiler does not keep the forward pass's sigmoids)
          asm volatile("" : "+v"(zl[t][i]));
          const float s = sigmoid(zl[t][i]);
            gz[t][i] = u[t][i] * (s * (1.f + zl[t][i] * (1.f - s)));
            if (TRAIN) y[t][i] -= zl[t][i] * s;
          }
      };
      // backward: the block in use is A_{H-1} (A_0's last chunk for H = 1)
#pragma unroll
      for (int l = H - 1; l > 0; --l) {
        f4 gz[4];
        back(z[l], gz);
        if (l > 1) next.load(layer(wt, a.D, l - 1), kR);
        else next.load(wt, a.D);
        if (TRAIN) {
          to_lds(0, gz);
          to_lds(kRows * kTS, y);
          __syncthreads();
          outer(sum_h[l - 1]);
          sum_b[l] += bias_sum();
        }
        product_t(s_w + cur * kWBlock, gz, u);
        next.store(s_w + (cur ^ 1) * kWBlock);
        cur ^= 1;
        __syncthreads();
      }
      f4 gz[4];
      back(z[0], gz);
      if (TRAIN) {
        to_lds(0, gz);
        __syncthreads();
        sum_b[0] += bias_sum();
      }
      // A_0 chunk by chunk; for H = 1 the last chunk is in use, so that one first
      for (int k = 0; k < chunks; ++k) {
        const int ch = H > 1 ? k : chunks - 1 - k;
        const int after = H > 1 ? k + 1 : chunks - 2 - k;
        const bool more = k + 1 < chunks;
        if (more) next.load(wt + 64 * after, a.D);
        if (TRAIN) {
          load_x<BF>(a, r, ch, in);
          to_lds(kRows * kTS, in);
          __syncthreads();
          if (ch == 0) outer(sum_0[0]);
          else if (ch == 1) outer(sum_0[1]);
          else {
            float* slot = a.slots + (int64_t(blockIdx.x) + e) * a.slot;
            f4 acc[kOwn];
#pragma unroll
            for (int j = 0; j < kOwn; ++j) acc[j] = first ? f4{0.f, 0.f, 0.f, 0.f} : *place(slot, ch, j);
            outer(acc);
#pragma unroll
            for (int j = 0; j < kOwn; ++j) *place(slot, ch, j) = acc[j];
          }
        }
        if (a.dx) {
          f4 dx[4] = {};
          product_t(s_w + cur * kWBlock, gz, dx);
          store_dx<BF>(a, r, ch, dx);
        }
        if (more) {
          next.store(s_w + (cur ^ 1) * kWBlock);
          cur ^= 1;
          __syncthreads();
        }
      }
    }
    if (TRAIN) flush(e);
  }
}

// A head's weight gradients: the slots of the work-groups that had tiles of
// it, added up in order.
template <int NW>
__global__ __launch_bounds__(256) void k_sum_slots(HeadsArgs a) {
  __shared__ int32_t s_first[kMaxExperts + 2], s_entry[kMaxExperts + 2];
  tile_table(a, 16 * NW, s_first, s_entry);
  const int e = blockIdx.y;
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (at >= a.slot) return;
  const int chunks = (a.D + 63) / 64;
  // where the value stands among the head's weights
  int64_t dst;
  const int64_t blocks_end = slot_block(a.D, chunks + a.H - 1);
  if (at < blocks_end) {
    const int b = int(at / (kR * kR)), in_block = int(at % (kR * kR));
    const int tile = in_block / 256, lane = (in_block % 256) / 4, i = in_block % 4;
    const int row = 16 * (tile / 4) + 4 * (lane >> 4) + i, col = 16 * (tile % 4) + (lane & 15);
    if (b < chunks) {
      if (64 * b + col >= a.D) return;
      dst = int64_t(row) * a.D + 64 * b + col;
    } else {
      dst = int64_t(kR) * a.D + kR + int64_t(b - chunks) * (kR * kR + kR) + row * kR + col;
    }
  } else {
    const int k = int(at - blocks_end), t = k / kR;
    if (k > (a.H + 1) * kR) return;
    const int64_t after = int64_t(kR) * a.D + kR + int64_t(a.H - 1) * (kR * kR + kR);
    if (t < a.H) dst = int64_t(kR) * a.D + (t ? kR + int64_t(t - 1) * (kR * kR + kR) + kR * kR : 0) + k % kR;
    else dst = after + (k - a.H * kR);
  }
  const int tiles = s_first[a.E + 1], lo = s_first[e], hi = s_first[e + 1];
  float v = 0.f;
  if (lo < hi) {
    // work-group of a tile: the last whose share starts at or before it
    auto group_of = [&](int tile) {
      int b = int(int64_t(tile) * a.blocks / tiles);
      while (b + 1 < a.blocks && share(tiles, b + 1, a.blocks) <= tile) ++b;
      while (share(tiles, b, a.blocks) > tile) --b;
      return b;
    };
    const int b0 = group_of(lo), b1 = group_of(hi - 1);
    for (int b = b0; b <= b1; ++b)
      if (share(tiles, b, a.blocks) < share(tiles, b + 1, a.blocks)) v += a.slots[(int64_t(b) + e) * a.slot + at];
  }
  a.dweights[e * a.values + dst] = v;
}

// Rows with several entries: their energies and gradients added up in order.
__global__ __launch_bounds__(256) void k_sum_entries(HeadsArgs a) {
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (a.energy && at < a.n) {
    float v = 0.f;
    for (int s = 0; s < a.K; ++s) v += a.entry_energy[at * a.K + s];
    a.energy[at] = v;
  }
  const int groups = (a.D + 3) / 4;
  if (a.dx && at < a.n * groups) {
    const int64_t i = at / groups;
    const int c = 4 * int(at % groups);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.K; ++s) {
      float t[4];
      load4(a.entry_dx, false, (i * a.K + s) * a.D + c, a.D - c, t);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += t[q];
    }
    store4(a.dx, a.bf16, i * a.D + c, a.D - c, v);
  }
}

// Wavefronts of a work-group: eight, two a SIMD; four where y and silu' of more
// than four layers and the sums of their gradients need all of a SIMD's registers.
int heads_waves(const HeadsArgs& a) { return a.dweights && a.H > 4 ? 4 : 8; }

template <int H, int NW, bool TRAIN, bool BF>
hipError_t gradient_of(const HeadsArgs& a, hipStream_t s) {
  constexpr size_t lds = (2 * kWBlock + (TRAIN ? 2 * 16 * NW * kTStride : 0)) * sizeof(float);
  const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_gradient<H, NW, TRAIN, BF>),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
  if (ready != hipSuccess) return ready;
  k_gradient<H, NW, TRAIN, BF><<<a.blocks, NW * 64, lds, s>>>(a);
  return hipGetLastError();
}

template <bool TRAIN, bool BF>
hipError_t gradient_by_layers(const HeadsArgs& a, hipStream_t s) {
  constexpr int kDeep = TRAIN ? 4 : 8;
  switch (a.H) {
    case 1: return gradient_of<1, 8, TRAIN, BF>(a, s);
    case 2: return gradient_of<2, 8, TRAIN, BF>(a, s);
    case 3: return gradient_of<3, 8, TRAIN, BF>(a, s);
    case 4: return gradient_of<4, 8, TRAIN, BF>(a, s);
    case 5: return gradient_of<5, kDeep, TRAIN, BF>(a, s);
    case 6: return gradient_of<6, kDeep, TRAIN, BF>(a, s);
    case 7: return gradient_of<7, kDeep, TRAIN, BF>(a, s);
    default: return gradient_of<8, kDeep, TRAIN, BF>(a, s);
  }
}

}  // namespace

size_t heads_plan(HeadsArgs* a, int n_cu) {
  const int rows = 16 * heads_waves(*a);
  // at most one more tile than full ones for each head and for entries without
  const int64_t tiles = a->m / rows + a->E + 1;
  a->blocks = int(std::min<int64_t>(tiles, n_cu));
  a->slot = slot_values(a->D, a->H);
  size_t b = 0;
  if (a->dweights) b += size_t(a->blocks + a->E) * size_t(a->slot) * sizeof(float);
  if (a->K > 1 && a->energy) b += size_t(a->m) * sizeof(float);
  if (a->K > 1 && a->dx) b += size_t(a->m) * size_t(a->D) * sizeof(float);
  return b;
}

hipError_t launch_heads(const HeadsArgs& a, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.m > 0) {
    if (!a.dx && !a.dweights) {
      if (a.bf16) k_energy<8, true><<<a.blocks, 512, 0, s>>>(a);
      else k_energy<8, false><<<a.blocks, 512, 0, s>>>(a);
      e = hipGetLastError();
    } else if (a.dweights) {
      e = a.bf16 ? gradient_by_layers<true, true>(a, s) : gradient_by_layers<true, false>(a, s);
    } else {
      e = a.bf16 ? gradient_by_layers<false, true>(a, s) : gradient_by_layers<false, false>(a, s);
    }
    if (e != hipSuccess) return e;
  }
  if (a.dweights) {
    const dim3 g((unsigned)((a.slot + 255) / 256), (unsigned)a.E);
    if (heads_waves(a) == 8) k_sum_slots<8><<<g, 256, 0, s>>>(a);
    else k_sum_slots<4><<<g, 256, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.K > 1 && a.m > 0 && (a.energy || a.dx)) {
    const int64_t work = std::max<int64_t>(a.n, a.dx ? a.n * ((a.D + 3) / 4) : 0);
    k_sum_entries<<<unsigned((work + 255) / 256), 256, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace mlip
