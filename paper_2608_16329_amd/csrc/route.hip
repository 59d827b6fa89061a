// Routing of rows (atoms) to experts (energy heads), its balance loss and their
// gradients, and the grouping of routed entries by expert.
//
//   p_ie = exp(z_ie) / sum_j exp(z_ij) over the experts the row may use,
//   the K largest are chosen (equal ones: the lowest first), the gates are the
//   softmax over the chosen or p itself,
//   loss = E sum_e f_e P_e,  f_e = share of the chosen entries, P_e = mean p_ie,
//   dz_ie = p_ie (h_e - sum_j p_ij h_j) + w_ie (dw_ie - sum_s w_is dw_is),
//   h_e = dloss E f_e / rows (the shares f are constants of the gradient).
#include <algorithm>
#include <type_traits>

#include "learn.h"
#include "learn_math.h"

namespace mlip {
namespace {

constexpr int kForwardThreads = 1024;   // a work-group for each CU: few sums to add up afterwards
constexpr int kRouteThreads = 256;

typedef uint32_t U4 __attribute__((aligned(1)));   // four bytes from anywhere

typedef float f4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;

// The value of another lane: CTRL names it.
template <int CTRL, typename T>
__device__ __forceinline__ T from_lane(T v) {
  return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// f over the L lanes of a row, in all of them: with lane c ^ 1, c ^ 2, and by
// mirrored halves of 8 and of 16 lanes.
template <int L, typename T, typename F>
__device__ __forceinline__ T over_row(T v, F f) {
  if (L > 1) v = f(v, from_lane<0xb1>(v));
  if (L > 2) v = f(v, from_lane<0x4e>(v));
  if (L > 4) v = f(v, from_lane<0x141>(v));
  if (L > 8) v = f(v, from_lane<0x140>(v));
  return v;
}
template <int L>
__device__ __forceinline__ float row_sum(float v) {
  return over_row<L>(v, [](float x, float y) { return x + y; });
}
template <int L>
__device__ __forceinline__ float row_max(float v) {
  return over_row<L>(v, [](float x, float y) { return fmaxf(x, y); });
}

// The expert whose logit a lane l of a row holds as its j-th.
template <int L>
__device__ __forceinline__ int expert_of(int j, int l) { return 4 * ((j >> 2) * L + l) + (j & 3); }

// What a lane has of a row, as loaded: V logits and a byte for each that
// says whether the row may use it.  Every load is one that may be made, whatever
// the row, so that none stands in a branch and the next row's are under way while
// one is worked on: rows beyond the last are the last again, quads beyond a row's
// end its last four.  unpack() puts this right.
template <int V, bool BF>
struct Raw {
  std::conditional_t<BF, H4, f4> v[V / 4];
  uint32_t ok[V / 4];
  bool live;
};
template <bool KINDS>
__device__ __forceinline__ int kind_of(const RouteArgs& a, int64_t i) {
  return KINDS ? a.kinds[i < a.n ? i : a.n - 1] : 0;
}
template <int L, int V, bool BF, bool KINDS>
__device__ __forceinline__ void load_row(const RouteArgs& a, int64_t i, int kind, int l, Raw<V, BF>& r) {
  typedef std::conditional_t<BF, uint16_t, float> T;
  typedef std::conditional_t<BF, H4, F4> Quad;
  const bool real = !KINDS || (kind >= 0 && kind < a.n_kinds);
  r.live = i < a.n && real;
  const T* row = static_cast<const T*>(a.logits) + (i < a.n ? i : a.n - 1) * a.stride;
  const uint8_t* ok = KINDS ? a.allowed + (real ? int64_t(kind) : 0) * a.E : nullptr;
  if (L == 1 && a.E < 4) {
    const int e1 = a.E > 1 ? 1 : 0, e2 = a.E > 2 ? 2 : 0;
    r.v[0][0] = row[0], r.v[0][1] = row[e1], r.v[0][2] = row[e2], r.v[0][3] = T(0);
    if (KINDS) r.ok[0] = ok[0] | uint32_t(ok[e1]) << 8 | uint32_t(ok[e2]) << 16;
    for (int c = 1; c < V / 4; ++c) r.v[c] = r.v[0], r.ok[c] = 0;
    return;
  }
#pragma unroll
  for (int c = 0; c < V / 4; ++c) {
    const int e = 4 * (c * L + l), at = e < a.E - 4 ? e : a.E - 4;
    r.v[c] = *reinterpret_cast<const Quad*>(row + at);
    if (KINDS) r.ok[c] = *reinterpret_cast<const U4*>(ok + at);
  }
}
// Its logits, what the row may not use as -inf, whatever stands there.
template <int L, int V, bool BF, bool KINDS>
__device__ __forceinline__ void unpack(const RouteArgs& a, const Raw<V, BF>& r, int l, float z[V]) {
#pragma unroll
  for (int c = 0; c < V / 4; ++c) {
    const int left = r.live ? a.E - 4 * (c * L + l) : 0;
    float t[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (BF) t[q] = from_bf16(r.v[c][q]);
      else t[q] = r.v[c][q];
    }
    uint32_t use = KINDS ? r.ok[c] : 0x01010101u;
    if (a.E & 3) {
      const int part = left > 0 && left < 4 ? 4 - left : 0, shift = a.E < 4 ? 0 : part;
      if (shift & 1) t[0] = t[1], t[1] = t[2], t[2] = t[3];
      if (shift & 2) t[0] = t[2], t[1] = t[3];
      use = KINDS ? use >> (8 * shift) & 0xffffffffu >> (8 * part) : use >> (8 * part);
    } else if (!KINDS) {
#pragma unroll
      for (int q = 0; q < 4; ++q) z[4 * c + q] = left > 0 ? t[q] : -INFINITY;
      continue;
    }
    use = left > 0 ? use : 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) z[4 * c + q] = use & (255u << (8 * q)) ? t[q] : -INFINITY;
  }
}

// Sums of v[0] .. v[N - 1] over the lanes that differ in bits O, O / 2 .. L: each
// step adds two lanes' halves of what is left, so that 16 values take 17
// exchanges over 64 lanes, not 96.  What a lane has then begins at value `first`.
template <int N, int O, int L>
__device__ __forceinline__ void fold(float* v, int& first) {
  if constexpr (O >= L) {
    constexpr int kLeft = N > 1 ? N / 2 : 1;
    const bool upper = threadIdx.x & O;
#pragma unroll
    for (int k = 0; k < kLeft; ++k) {
      const float send = N > 1 && !upper ? v[k + N - kLeft] : v[k], keep = N > 1 && upper ? v[k + N - kLeft] : v[k];
      v[k] = keep + __shfl_xor(send, O, 64);
    }
    if (N > 1) first += upper ? kLeft : 0;
    fold<kLeft, O / 2, L>(v, first);
  }
}

// The loss from a wavefront's sums over experts (lane by lane) and the routed rows.
__device__ __forceinline__ void write_loss(const RouteArgs& a, double entries, double cross, int rows) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    entries += __shfl_xor(entries, o, 64);
    cross += __shfl_xor(cross, o, 64);
  }
  if ((threadIdx.x & 63) == 0) a.loss[0] = rows > 0 ? float(a.E * cross / (entries * double(rows))) : 0.f;
}

// Forward: L lanes per row, every lane with V of its logits (16; 4 or 8 where
// there are no more experts: 1,048,576 rows of 4, one chosen, 17.3 us instead of
// 23.6), rows taken in turn by the grid.  A choice is one more maximum over the
// row and the lowest place that has it.  Each work-group's counts and sums of p go
// to its own place and are added up in order afterwards, so results do not depend
// on the order of work-groups.
// Bound by vector instructions: 2,097,152 rows of 64 float32 logits, 4 chosen, 157
// us in a series of calls (612 MB, 3.9 TB/s; the first ones 193), 37 of them a logit,
// the vector pipes busy for 93% of the time; 1,048,576 rows of 16 bfloat16, 2 chosen,
// 19 us (50 MB, 2.6 TB/s), 29 a logit and 77%.  (With one lane a row places for 16
// choices are kept whatever K is, and 52 to 96 scalar registers go through vector
// ones.)  108 rows of 4, 5.5 us, most of it the launch and the loads' latency.
// Exponentials: z - top times log2(e) is rounded to float32, so e^(z - top) is off
// by up to 4.6e-8 |z - top| of it (3.7e-6 at 80), beside what the rounding of z - top
// makes, and is 0 below 2^-126.
template <int L, int V, bool BF, bool KINDS>
__global__ __launch_bounds__(kForwardThreads) void k_route(RouteArgs a, bool only) {
  constexpr int kKept = (kMaxTopK + L - 1) / L;   // choices a lane keeps: lane s % L the s-th
  __shared__ int32_t s_count[kMaxExperts + 1];
  __shared__ float s_p[kForwardThreads / 64][L * V];
  const int tid = threadIdx.x, l = tid % L, lane = tid & 63, w = tid >> 6;
  for (int e = tid; e <= a.E; e += kForwardThreads) s_count[e] = 0;
  __syncthreads();
  float psum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) psum[j] = 0.f;
  constexpr int kRows = kForwardThreads / L;
  const int64_t step = int64_t(gridDim.x) * kRows;
  int rows = 0;
  const int64_t first = int64_t(blockIdx.x) * kRows;
  Raw<V, BF> raw;
  int kind = 0;
  if (first < a.n) {
    load_row<L, V, BF, KINDS>(a, first + tid / L, kind_of<KINDS>(a, first + tid / L), l, raw);
    kind = kind_of<KINDS>(a, first + step + tid / L);
  }
  for (int64_t i0 = first; i0 < a.n; i0 += step) {
    const int64_t i = i0 + tid / L;
    float z[V], key[V];
    unpack<L, V, BF, KINDS>(a, raw, l, z);
    if (i0 + step < a.n) {
      load_row<L, V, BF, KINDS>(a, i + step, kind, l, raw);
      kind = kind_of<KINDS>(a, i + 2 * step);
    }
    // (a NaN is not looked at here; it is in the sum)
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      key[j] = z[j];
      top = fmaxf(top, key[j]);
    }
    top = row_max<L>(top);
    const float base = top != -INFINITY ? top : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      z[j] = __builtin_amdgcn_exp2f((z[j] - base) * kLog2e);
      sum += z[j];
    }
    sum = row_sum<L>(sum);
    const bool any = sum != 0.f;
    const float inv = any ? 1.f / sum : 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) psum[j] += z[j] * inv;
    rows += any && l == 0;
    float chosen = 0.f;
    int my_id[kKept];
    float my_w[kKept];
#pragma unroll
    for (int r = 0; r < kKept; ++r) my_id[r] = -1, my_w[r] = 0.f;
    // choices r L .. r L + L - 1, each kept by a lane of the row
#pragma unroll
    for (int r = 0; r < kKept; ++r) {
#pragma unroll 1
      for (int s = r * L; s < min(a.K, r * L + L); ++s) {
        float best = top;
        if (s > 0) {
          best = -INFINITY;
#pragma unroll
          for (int j = 0; j < V; ++j) best = fmaxf(best, key[j]);
          best = row_max<L>(best);
        }
        // the lowest expert that has it
        int at = -1;
#pragma unroll
        for (int j = V - 1; j >= 0; --j) at = key[j] == best ? j : at;
        const int own = at >= 0 ? expert_of<L>(at, l) : 0x7fffffff;
        const int id = over_row<L>(own, [](int x, int y) { return x < y ? x : y; });
        const bool there = best != -INFINITY;
        if (s + 1 < a.K) {
          at = own == id ? at : -1;
#pragma unroll
          for (int j = 0; j < V; ++j) key[j] = at == j ? -INFINITY : key[j];
        }
        const float e = there ? __builtin_amdgcn_exp2f((best - base) * kLog2e) : 0.f;
        chosen += e;
        const bool mine = s == r * L + l;
        my_id[r] = mine && there ? id : my_id[r];
        my_w[r] = mine ? e : my_w[r];
        if (there && l == 0) atomicAdd(&s_count[id], 1);
      }
    }
    if (i < a.n) {
      // a NaN is in every gate of its row
      const float norm = !any ? 0.f : (a.all || sum != sum ? inv : 1.f / chosen);
#pragma unroll
      for (int r = 0; r < kKept; ++r) {
        const int s = r * L + l;
        if (s < a.K) {
          a.experts[i * a.K + s] = my_id[r];
          a.gates[i * a.K + s] = my_w[r] * norm;
        }
      }
    }
  }
  if (rows) atomicAdd(&s_count[a.E], rows);
  // lanes with the same experts, then the wavefronts, in a fixed order
  int at = 0;
  fold<V, 32, L>(psum, at);
  constexpr int kLeft = V * L > 64 ? V * L / 64 : 1;
#pragma unroll
  for (int k = 0; k < kLeft; ++k) s_p[w][expert_of<L>(at + k, l)] = psum[k];
  __syncthreads();
  auto sum_of = [&](int e) {
    float v = 0.f;
    for (int u = 0; u < kForwardThreads / 64; ++u) v += s_p[u][e];
    return v;
  };
  if (!only) {
    for (int e = tid; e <= a.E; e += kForwardThreads) {
      a.part_c[int64_t(e) * gridDim.x + blockIdx.x] = s_count[e];
      if (e < a.E) a.part_p[int64_t(e) * gridDim.x + blockIdx.x] = sum_of(e);
    }
    return;
  }
  // one work-group has everything: the loss at once
  for (int e = tid; e <= a.E; e += kForwardThreads) a.counts[e] = s_count[e];
  if (w == 0) {
    double entries = 0.0, cross = 0.0;
    for (int e = lane; e < a.E; e += 64) {
      entries += s_count[e];
      cross += double(s_count[e]) * double(sum_of(e));
    }
    write_loss(a, entries, cross, s_count[a.E]);
  }
}

// The work-groups' counts and sums added up in order, and the loss: 16 lanes for
// an expert (and for the routed rows), each with every 16th work-group, 16 loads
// of either under way at once; then a wavefront for all.  In 64 bits: the loss is a
// quotient of sums over all rows.  Latency: 4 to 5 us up to 63 experts of 256
// work-groups, 6 to 7 at 64 to 127.
__global__ __launch_bounds__(1024) void k_route_total(RouteArgs a, int blocks) {
  __shared__ double s_p[kMaxExperts + 1];
  __shared__ int32_t s_c[kMaxExperts + 1];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int e0 = 0; e0 <= a.E; e0 += 64) {
    const int e = e0 + (threadIdx.x >> 4);
    // (places that there are none of: the last expert's)
    const int32_t* pc = a.part_c + int64_t(e < a.E ? e : a.E) * blocks;
    const float* pp = a.part_p + int64_t(e < a.E ? e : a.E - 1) * blocks;
    double p = 0.0;
    int c = 0;
    for (int b0 = lane & 15; b0 < blocks; b0 += 256) {
      int32_t vc[16];
      float vp[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int b = b0 + 16 * k < blocks ? b0 + 16 * k : blocks - 1;
        vc[k] = pc[b];
        vp[k] = pp[b];
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const bool there = b0 + 16 * k < blocks;
        c += there ? vc[k] : 0;
        p += there ? double(vp[k]) : 0.0;
      }
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
      p += __shfl_xor(p, o, 64);
      c += __shfl_xor(c, o, 64);
    }
    if ((lane & 15) == 0 && e <= a.E) s_p[e] = p, s_c[e] = c, a.counts[e] = c;
  }
  __syncthreads();
  if (w == 0) {
    double entries = 0.0, cross = 0.0;
    for (int e = lane; e < a.E; e += 64) entries += s_c[e], cross += double(s_c[e]) * s_p[e];
    write_loss(a, entries, cross, s_c[a.E]);
  }
}

// Backward: the probabilities again from the logits (they are read once in any
// case, and keeping them would write and read as much again).  The lanes of a
// row take its choices in turn; what a choice adds to its logit's gradient
// goes through LDS to the lane that holds the logit.
// Bound by memory: 2,097,152 rows of 64 float32 logits, 4 chosen, 242 us (1.15 GB,
// 4.8 TB/s; a large copy reaches 5.1).
template <int L, int V, bool BF, bool KINDS>
__global__ __launch_bounds__(kRouteThreads) void k_route_backward(RouteArgs a) {
  __shared__ float s_h[L * V];
  __shared__ __attribute__((aligned(16))) float s_add[kRouteThreads * V];
  __shared__ double s_entries;
  const int tid = threadIdx.x, l = tid % L, lane = tid & 63;
  if (tid < 64) {
    double t = 0.0;
    for (int e = lane; e < a.E; e += 64) t += a.counts[e];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o, 64);
    if (lane == 0) s_entries = t;
  }
  __syncthreads();
  {
    const double rows = a.counts[a.E];
    const double f = a.dloss && rows > 0 && s_entries > 0 ? double(a.dloss[0]) * a.E / (rows * s_entries) : 0.0;
    for (int e = tid; e < L * V; e += kRouteThreads) s_h[e] = e < a.E ? float(f * a.counts[e]) : 0.f;
  }
  __syncthreads();
  float h[V];
#pragma unroll
  for (int j = 0; j < V; ++j) h[j] = s_h[expert_of<L>(j, l)];
  float* const mine = s_add + tid / L * (L * V);   // the row's
#pragma unroll
  for (int c = 0; c < V / 4; ++c) *reinterpret_cast<f4*>(mine + 4 * (c * L + l)) = f4{0.f, 0.f, 0.f, 0.f};
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  constexpr int kRows = kRouteThreads / L, kKept = (kMaxTopK + L - 1) / L;
  const int64_t step = int64_t(gridDim.x) * kRows;
  const int64_t first = int64_t(blockIdx.x) * kRows;
  Raw<V, BF> raw;
  int kind = 0;
  if (first < a.n) {
    load_row<L, V, BF, KINDS>(a, first + tid / L, kind_of<KINDS>(a, first + tid / L), l, raw);
    kind = kind_of<KINDS>(a, first + step + tid / L);
  }
  for (int64_t i0 = first; i0 < a.n; i0 += step) {
    const int64_t i = i0 + tid / L;
    float z[V];
    unpack<L, V, BF, KINDS>(a, raw, l, z);
    if (i0 + step < a.n) {
      load_row<L, V, BF, KINDS>(a, i + step, kind, l, raw);
      kind = kind_of<KINDS>(a, i + 2 * step);
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < V; ++j) top = fmaxf(top, z[j]);
    top = row_max<L>(top);
    const float base = top != -INFINITY ? top : 0.f;
    float sum = 0.f, mean = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      z[j] = __builtin_amdgcn_exp2f((z[j] - base) * kLog2e);
      sum += z[j];
      mean += z[j] * h[j];
    }
    sum = row_sum<L>(sum);
    mean = row_sum<L>(mean);
    const bool any = sum != 0.f;
    const float inv = any ? 1.f / sum : 0.f;
    mean *= inv;
    // over the chosen: their exponentials, and the gates' gradients times those
    const bool gates = a.dgates && any;
    float chosen = 0.f, cross = 0.f;
    int my_id[kKept];
    float my_e[kKept], my_g[kKept];
#pragma unroll
    for (int r = 0; r < kKept; ++r) {
      const int s = r * L + l;
      my_id[r] = -1;
      my_e[r] = my_g[r] = 0.f;
      if (gates && s < a.K) {
        const int id = a.experts[i * a.K + s];
        if (id >= 0 && id < a.E) {
          const int64_t at = i * a.stride + id;
          const float x = BF ? from_bf16(static_cast<const uint16_t*>(a.logits)[at]) : static_cast<const float*>(a.logits)[at];
          my_id[r] = id;
          my_e[r] = __builtin_amdgcn_exp2f((x - base) * kLog2e);
          my_g[r] = a.dgates[i * a.K + s];
        }
      }
      chosen += my_e[r];
      cross += my_e[r] * my_g[r];
    }
    chosen = row_sum<L>(chosen);
    cross = row_sum<L>(cross);
    if (a.all) mean += cross * inv;
    const float per = chosen != 0.f ? 1.f / chosen : 0.f;
    cross *= per;
    if (a.dgates) {
#pragma unroll
      for (int r = 0; r < kKept; ++r)
        if (my_id[r] >= 0) mine[my_id[r]] = a.all ? my_e[r] * inv * my_g[r] : my_e[r] * per * (my_g[r] - cross);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (i < a.n) {
#pragma unroll
      for (int c = 0; c < V / 4; ++c) {
        const int e = 4 * (c * L + l);
        const f4 add = *reinterpret_cast<const f4*>(mine + e);
        float t[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) t[q] = any ? z[4 * c + q] * inv * (h[4 * c + q] - mean) + add[q] : 0.f;
        store4(a.dlogits, BF, i * a.E + e, a.E - e, t);
      }
    }
    if (a.dgates) {
      // zero again for the next row
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int r = 0; r < kKept; ++r)
        if (my_id[r] >= 0) mine[my_id[r]] = 0.f;
    }
  }
}

// Lanes per row: as few as hold E logits, 16 a lane.  (Up to 8 or 4 experts a
// lane holds only so many.)
constexpr int kMost = 16;
int route_lanes(int E) {
  int L = 1;
  while (L * kMost < E) L *= 2;
  return L;
}

// ---- grouping ------------------------------------------------------------------
//
// A stable counting sort by expert: counts of chunks, places of chunks within an
// expert, order.  A wavefront has a chunk and takes 64 entries at a time; the
// lanes with the same expert find each other with a ballot for each bit of it, and
// the first of them moves the expert's place on for all, so that no atomic decides
// the order.  Bound by launches and latency: 5,000 entries by one work-group 7.1
// us; 1,048,576 by three kernels 5.9, 4.8 and 6.4 us (12.6 MB).

constexpr int kGroupWaves = 4;
// Entries one work-group sorts by itself (4,096, 8 experts: 7.6 us, by three
// kernels 10.6; 8,192: 11.0 and 10.7; 16,384: 18.8 and 10.7).
constexpr int64_t kGroupOne = 8192;
constexpr int kGroupOneWaves = 16;
constexpr int kScanThreads = 1024;

__device__ __forceinline__ int group_key(int32_t id, int E) { return id >= 0 && id < E ? id : E; }

// The lanes that hold the same key (of `bits` bits) as this one; all 64 call.
__device__ __forceinline__ uint64_t peers_of(int key, int bits, bool on) {
  uint64_t p = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const uint64_t m = __ballot((key >> b) & 1);
    p &= (key >> b) & 1 ? m : ~m;
  }
  return p;
}

constexpr int kAhead = 8;                // rounds of 64 entries loaded before the first is used

__device__ __forceinline__ void load_ids(const int32_t* __restrict__ experts, int64_t i0, int64_t hi, int32_t id[kAhead]) {
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int64_t i = i0 + 64 * k + (threadIdx.x & 63);
    id[k] = experts[i < hi ? i : hi - 1];
  }
}

// Entries [lo, hi) placed in order by one wavefront from the running places in
// pos[key].
__device__ __forceinline__ void place(const int32_t* __restrict__ experts, int64_t lo, int64_t hi, int E, int bits,
                                      volatile int32_t* pos, int32_t* __restrict__ order) {
  const int lane = threadIdx.x & 63;
  for (int64_t i0 = lo; i0 < hi; i0 += 64 * kAhead) {
    int32_t id[kAhead];
    load_ids(experts, i0, hi, id);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i0 + 64 * k >= hi) break;
      const int64_t i = i0 + 64 * k + lane;
      const bool on = i < hi;
      const int key = on ? group_key(id[k], E) : 0;
      const uint64_t peers = peers_of(key, bits, on);
      const int rank = __popcll(peers & ((uint64_t(1) << lane) - 1));
      const int at = on ? pos[key] : 0;
      __builtin_amdgcn_wave_barrier();
      if (on && rank == 0) pos[key] = at + __popcll(peers);
      __builtin_amdgcn_wave_barrier();
      if (on) order[at + rank] = int32_t(i);
    }
  }
}

// Entries [lo, hi) counted into cnt[key] by one wavefront: a key's lanes by
// the one that is first among them.
__device__ __forceinline__ void count(const int32_t* __restrict__ experts, int64_t lo, int64_t hi, int E, int bits,
                                      volatile int32_t* cnt) {
  const int lane = threadIdx.x & 63;
  for (int64_t i0 = lo; i0 < hi; i0 += 64 * kAhead) {
    int32_t id[kAhead];
    load_ids(experts, i0, hi, id);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i0 + 64 * k >= hi) break;
      const bool on = i0 + 64 * k + lane < hi;
      const int key = on ? group_key(id[k], E) : 0;
      const uint64_t peers = peers_of(key, bits, on);
      if (on && (peers & ((uint64_t(1) << lane) - 1)) == 0) cnt[key] = cnt[key] + __popcll(peers);
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Few entries: counts, places and the order by one work-group.
__global__ __launch_bounds__(kGroupOneWaves * 64) void k_group_one(const int32_t* experts, int64_t m, int E, int bits,
                                                                   int32_t* offsets, int32_t* order) {
  __shared__ int32_t pos[kGroupOneWaves][kMaxExperts + 1];
  __shared__ int32_t total[kMaxExperts + 1], base[kMaxExperts + 1];
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  for (int e = tid; e < kGroupOneWaves * (kMaxExperts + 1); e += kGroupOneWaves * 64) (&pos[0][0])[e] = 0;
  __syncthreads();
  const int64_t chunk = (m + kGroupOneWaves * 64 - 1) / (kGroupOneWaves * 64) * 64;
  const int64_t lo = w * chunk < m ? w * chunk : m, hi = lo + chunk < m ? lo + chunk : m;
  count(experts, lo, hi, E, bits, pos[w]);
  __syncthreads();
  if (tid <= E) {
    int t = 0;
    for (int v = 0; v < kGroupOneWaves; ++v) {
      const int c = pos[v][tid];
      pos[v][tid] = t;
      t += c;
    }
    total[tid] = t;
  }
  __syncthreads();
  if (w == 0) {
    int run = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
      const int e = e0 + lane;
      const int c = e <= E ? total[e] : 0;
      int v = c;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(v, o, 64);
        v += lane >= o ? t : 0;
      }
      if (e <= E) base[e] = run + v - c, offsets[e] = run + v - c;
      run += __shfl(v, 63, 64);
    }
  }
  __syncthreads();
  for (int e = lane; e <= E; e += 64) pos[w][e] += base[e];
  __syncthreads();
  place(experts, lo, hi, E, bits, pos[w], order);
}

// Many: counts of each wavefront's chunk, hist[key][chunk].
__global__ __launch_bounds__(kGroupWaves * 64) void k_group_count(const int32_t* experts, int64_t m, int E, int bits,
                                                                  int64_t chunk, int chunks, int32_t* hist) {
  __shared__ int32_t cnt[kGroupWaves][kMaxExperts + 1];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c = blockIdx.x * kGroupWaves + w;
  for (int e = lane; e <= E; e += 64) cnt[w][e] = 0;
  __syncthreads();
  const int64_t lo = c * chunk < m ? c * chunk : m, hi = lo + chunk < m ? lo + chunk : m;
  count(experts, lo, hi, E, bits, cnt[w]);
  __syncthreads();
  if (c < chunks)
    for (int e = lane; e <= E; e += 64) hist[int64_t(e) * chunks + c] = cnt[w][e];
}

// One work-group per key: its chunks' counts to places within the key.
__global__ __launch_bounds__(kScanThreads) void k_group_scan(int32_t* hist, int chunks, int32_t* total) {
  __shared__ int32_t part[kScanThreads / 64];
  int32_t* row = hist + int64_t(blockIdx.x) * chunks;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int run = 0;
  for (int c0 = 0; c0 < chunks; c0 += kScanThreads) {
    const int c = c0 + threadIdx.x;
    const int n = c < chunks ? row[c] : 0;
    int v = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int t = __shfl_up(v, o, 64);
      v += lane >= o ? t : 0;
    }
    if (lane == 63) part[w] = v;
    __syncthreads();
    int before = run, all = 0;
#pragma unroll
    for (int u = 0; u < kScanThreads / 64; ++u) {
      before += u < w ? part[u] : 0;
      all += part[u];
    }
    if (c < chunks) row[c] = before + v - n;
    run += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) total[blockIdx.x] = run;
}

__global__ __launch_bounds__(kGroupWaves * 64) void k_group_place(const int32_t* experts, int64_t m, int E, int bits,
                                                                  int64_t chunk, int chunks, const int32_t* hist,
                                                                  const int32_t* total, int32_t* offsets,
                                                                  int32_t* order) {
  __shared__ int32_t pos[kGroupWaves][kMaxExperts + 1];
  __shared__ int32_t base[kMaxExperts + 1];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c = blockIdx.x * kGroupWaves + w;
  if (w == 0) {
    int run = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
      const int e = e0 + lane;
      const int n = e <= E ? total[e] : 0;
      int v = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(v, o, 64);
        v += lane >= o ? t : 0;
      }
      if (e <= E) {
        base[e] = run + v - n;
        if (blockIdx.x == 0) offsets[e] = run + v - n;
      }
      run += __shfl(v, 63, 64);
    }
  }
  __syncthreads();
  if (c < chunks)
    for (int e = lane; e <= E; e += 64) pos[w][e] = base[e] + hist[int64_t(e) * chunks + c];
  __syncthreads();
  const int64_t lo = c * chunk < m ? c * chunk : m, hi = lo + chunk < m ? lo + chunk : m;
  if (c < chunks) place(experts, lo, hi, E, bits, pos[w], order);
}

// A wavefront's chunk: 256 entries, more where there would be over 2,048 chunks
// (1,048,576 entries, 8 experts: 15.6 us with 2,048 chunks, 20.6 with 1,024, 16.1
// with 4,096; 8,388,608 entries, 64 experts: 84, 145 and 100).
int64_t group_chunk(int64_t m) { return std::max<int64_t>(256, (m + 2048 * 64 - 1) / (2048 * 64) * 64); }

template <typename F>
hipError_t by_type(const RouteArgs& a, F f) {
  const std::true_type yes;
  const std::false_type no;
  if (a.bf16) return a.kinds ? f(yes, yes) : f(yes, no);
  return a.kinds ? f(no, yes) : f(no, no);
}

template <bool BF, bool KINDS>
hipError_t route_of(const RouteArgs& a, int blocks, hipStream_t s) {
  const dim3 g(blocks), b(kForwardThreads);
  const bool only = blocks == 1;
  switch (route_lanes(a.E)) {
    case 1:
      if (a.E <= 4) k_route<1, 4, BF, KINDS><<<g, b, 0, s>>>(a, only);
      else if (a.E <= 8) k_route<1, 8, BF, KINDS><<<g, b, 0, s>>>(a, only);
      else k_route<1, 16, BF, KINDS><<<g, b, 0, s>>>(a, only);
      break;
    case 2: k_route<2, 16, BF, KINDS><<<g, b, 0, s>>>(a, only); break;
    case 4: k_route<4, 16, BF, KINDS><<<g, b, 0, s>>>(a, only); break;
    case 8: k_route<8, 16, BF, KINDS><<<g, b, 0, s>>>(a, only); break;
    default: k_route<16, 16, BF, KINDS><<<g, b, 0, s>>>(a, only); break;
  }
  return hipGetLastError();
}

template <bool BF, bool KINDS>
hipError_t route_backward_of(const RouteArgs& a, int blocks, hipStream_t s) {
  const dim3 g(blocks), b(kRouteThreads);
  switch (route_lanes(a.E)) {
    case 1:
      if (a.E <= 4) k_route_backward<1, 4, BF, KINDS><<<g, b, 0, s>>>(a);
      else if (a.E <= 8) k_route_backward<1, 8, BF, KINDS><<<g, b, 0, s>>>(a);
      else k_route_backward<1, 16, BF, KINDS><<<g, b, 0, s>>>(a);
      break;
    case 2: k_route_backward<2, 16, BF, KINDS><<<g, b, 0, s>>>(a); break;
    case 4: k_route_backward<4, 16, BF, KINDS><<<g, b, 0, s>>>(a); break;
    case 8: k_route_backward<8, 16, BF, KINDS><<<g, b, 0, s>>>(a); break;
    default: k_route_backward<16, 16, BF, KINDS><<<g, b, 0, s>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace

// One work-group for up to two rounds of rows: several cost a launch that adds
// them up (two rounds, 512 rows of 64 experts, 4 chosen: 13.4 us by one, 15.5 by
// two; 2,048 rows of 4 experts 13.7 and 13.8; four rounds, 1,024 rows of 64
// experts: 21.2 by one, 15.4 by four).
int route_blocks(int64_t n, int E, int n_cu) {
  const int rows = kForwardThreads / route_lanes(E);
  if (n <= 2 * rows) return 1;
  return int(std::min<int64_t>((n + rows - 1) / rows, n_cu));
}

hipError_t launch_route(const RouteArgs& a, int blocks, hipStream_t s) {
  const hipError_t e = by_type(a, [&](auto bf, auto kinds) { return route_of<bf.value, kinds.value>(a, blocks, s); });
  if (e != hipSuccess || blocks == 1) return e;
  k_route_total<<<1, 1024, 0, s>>>(a, blocks);
  return hipGetLastError();
}

hipError_t launch_route_backward(const RouteArgs& a, int n_cu, hipStream_t s) {
  const int rows = kRouteThreads / route_lanes(a.E);
  const int blocks = int(std::max<int64_t>(1, std::min<int64_t>((a.n + rows - 1) / rows, 8 * n_cu)));
  return by_type(a, [&](auto bf, auto kinds) { return route_backward_of<bf.value, kinds.value>(a, blocks, s); });
}

size_t group_ws_bytes(int64_t m, int E) {
  if (m <= kGroupOne) return 0;
  const int64_t chunk = group_chunk(m), chunks = (m + chunk - 1) / chunk;
  return size_t(E + 1) * size_t(chunks + 1) * sizeof(int32_t);
}

hipError_t launch_group(const int32_t* experts, int64_t m, int E, int32_t* offsets, int32_t* order, void* ws,
                        hipStream_t s) {
  int bits = 0;
  while ((1 << bits) <= E) ++bits;
  if (m <= kGroupOne) {
    k_group_one<<<1, kGroupOneWaves * 64, 0, s>>>(experts, m, E, bits, offsets, order);
    return hipGetLastError();
  }
  const int64_t chunk = group_chunk(m);
  const int chunks = int((m + chunk - 1) / chunk);
  const int blocks = (chunks + kGroupWaves - 1) / kGroupWaves;
  int32_t* hist = static_cast<int32_t*>(ws);
  int32_t* total = hist + size_t(E + 1) * size_t(chunks);
  k_group_count<<<blocks, kGroupWaves * 64, 0, s>>>(experts, m, E, bits, chunk, chunks, hist);
  k_group_scan<<<E + 1, kScanThreads, 0, s>>>(hist, chunks, total);
  k_group_place<<<blocks, kGroupWaves * 64, 0, s>>>(experts, m, E, bits, chunk, chunks, hist, total, offsets, order);
  return hipGetLastError();
}

}  // namespace mlip
