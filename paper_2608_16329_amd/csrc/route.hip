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

#include "learn.h"
#include "learn_math.h"

namespace mlip {
namespace {

constexpr int kRouteThreads = 256;
constexpr int kV = 16;              // logits a lane holds

// Row i's logits of this lane: expert 4 (c L + l) + q at z[4 c + q]; what the
// row may not use is -inf, whatever stands there.  True if anything is left in
// this lane.
template <int L, bool BF>
__device__ __forceinline__ bool load_row(const RouteArgs& a, int64_t i, int l, float z[kV]) {
  const uint8_t* ok = nullptr;
  bool live = i < a.n;
  if (live && a.kinds) {
    const int kind = a.kinds[i];
    live = kind >= 0 && kind < a.n_kinds;
    ok = a.allowed + int64_t(live ? kind : 0) * a.E;
  }
  bool any = false;
#pragma unroll
  for (int c = 0; c < kV / 4; ++c) {
    const int e = 4 * (c * L + l);
    float t[4];
    load4(a.logits, BF, i * a.stride + e, live ? a.E - e : 0, t);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bool use = live && e + q < a.E && (!ok || ok[e + q]);
      z[4 * c + q] = use ? t[q] : -INFINITY;
      any |= use && t[q] != -INFINITY;
    }
  }
  return any;
}

template <int L>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int o = 1; o < L; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Forward: L lanes per row, every lane with up to 16 of its logits, rows taken
// in turn by the grid.  Each work-group's counts and sums of p go to its own
// place and are added up in order afterwards, so results do not depend on the
// order of work-groups.
template <int L, bool BF>
__global__ __launch_bounds__(kRouteThreads) void k_route(RouteArgs a, bool only) {
  __shared__ int32_t s_count[kMaxExperts + 1];
  __shared__ float s_p[kRouteThreads / 64][L * kV];
  const int tid = threadIdx.x, l = tid % L, lane = tid & 63, w = tid >> 6;
  for (int e = tid; e <= a.E; e += kRouteThreads) s_count[e] = 0;
  __syncthreads();
  float psum[kV];
#pragma unroll
  for (int j = 0; j < kV; ++j) psum[j] = 0.f;
  constexpr int kRows = kRouteThreads / L;
  const int64_t step = int64_t(gridDim.x) * kRows;
  for (int64_t i0 = int64_t(blockIdx.x) * kRows; i0 < a.n; i0 += step) {
    const int64_t i = i0 + tid / L;
    float z[kV];
    bool any = load_row<L, BF>(a, i, l, z);
#pragma unroll
    for (int o = 1; o < L; o <<= 1) any |= bool(__shfl_xor(int(any), o, 64));
    unsigned used = 0;
    float top = 0.f, sum = 1.f, chosen_sum = 0.f;
    float pick_v = 0.f;       // of the choice this lane keeps: lane s % L keeps s
    int my_id[(kMaxTopK + L - 1) / L];
    float my_w[(kMaxTopK + L - 1) / L];
#pragma unroll
    for (int r = 0; r < (kMaxTopK + L - 1) / L; ++r) my_id[r] = -1, my_w[r] = 0.f;
#pragma unroll 1
    for (int s = 0; s < a.K; ++s) {
      // largest of the lane's unused logits (a NaN counts as the largest)
      float best = -INFINITY;
      int id = 0x7fffffff, at = -1;
#pragma unroll
      for (int j = 0; j < kV; ++j) {
        const float key = z[j] != z[j] ? INFINITY : z[j];
        const bool take = !((used >> j) & 1u) && key > best;
        best = take ? key : best;
        at = take ? j : at;
      }
      if (at >= 0) id = 4 * ((at >> 2) * L + l) + (at & 3);
      const int own = id;
#pragma unroll
      for (int o = 1; o < L; o <<= 1) {
        const float v = __shfl_xor(best, o, 64);
        const int d = __shfl_xor(id, o, 64);
        if (v > best || (v == best && d < id)) best = v, id = d;
      }
      const bool there = id != 0x7fffffff;
      if (there && own == id) used |= 1u << at;
      if (s == 0) {
        // the first choice is the row's largest logit
        top = any ? best : 0.f;
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < kV; ++j) t += expf(z[j] - top);
        sum = row_sum<L>(t);
        sum = any ? sum : 1.f;
      }
      pick_v = there ? expf(best - top) : 0.f;
      chosen_sum += pick_v;
#pragma unroll
      for (int r = 0; r < (kMaxTopK + L - 1) / L; ++r)
        if (s == r * L + l) my_id[r] = there ? id : -1, my_w[r] = pick_v;
      if (there && l == 0) atomicAdd(&s_count[id], 1);
    }
    const float inv = 1.f / sum;
    const float norm = any ? (a.all ? inv : 1.f / chosen_sum) : 0.f;
    if (i < a.n) {
#pragma unroll
      for (int r = 0; r < (kMaxTopK + L - 1) / L; ++r) {
        const int s = r * L + l;
        if (s < a.K) {
          a.experts[i * a.K + s] = my_id[r];
          a.gates[i * a.K + s] = my_id[r] >= 0 ? my_w[r] * norm : 0.f;
        }
      }
    }
    if (any) {
#pragma unroll
      for (int j = 0; j < kV; ++j) psum[j] += expf(z[j] - top) * inv;
      if (l == 0) atomicAdd(&s_count[a.E], 1);
    }
  }
  // lanes with the same experts, then the wavefronts, in a fixed order
#pragma unroll
  for (int j = 0; j < kV; ++j) {
    float v = psum[j];
#pragma unroll
    for (int o = L; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
    if (lane < L) s_p[w][4 * ((j >> 2) * L + l) + (j & 3)] = v;
  }
  __syncthreads();
  if (!only) {
    for (int e = tid; e <= a.E; e += kRouteThreads) {
      a.part_c[int64_t(blockIdx.x) * (a.E + 1) + e] = s_count[e];
      if (e < a.E) a.part_p[int64_t(blockIdx.x) * a.E + e] = (s_p[0][e] + s_p[1][e]) + (s_p[2][e] + s_p[3][e]);
    }
    return;
  }
  // one work-group has everything: the loss at once
  __shared__ double s_sum[2];
  if (tid == 0) {
    double entries = 0.0, cross = 0.0;
    for (int e = 0; e < a.E; ++e) {
      entries += s_count[e];
      cross += double(s_count[e]) * double((s_p[0][e] + s_p[1][e]) + (s_p[2][e] + s_p[3][e]));
    }
    s_sum[0] = entries;
    s_sum[1] = cross;
  }
  __syncthreads();
  for (int e = tid; e <= a.E; e += kRouteThreads) a.counts[e] = s_count[e];
  if (tid == 0) {
    const double rows = s_count[a.E];
    a.loss[0] = rows > 0 ? float(a.E * s_sum[1] / (s_sum[0] * rows)) : 0.f;
  }
}

// The work-groups' counts and sums added up in order, and the loss: one
// wavefront per expert (and one for the routed rows), then one work-group.
__global__ __launch_bounds__(1024) void k_route_total(RouteArgs a, int blocks) {
  __shared__ double s_p[kMaxExperts + 1];
  __shared__ int32_t s_c[kMaxExperts + 1];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int e = w; e <= a.E; e += 16) {
    double p = 0.0;
    int c = 0;
    for (int b = lane; b < blocks; b += 64) {
      c += a.part_c[int64_t(b) * (a.E + 1) + e];
      if (e < a.E) p += a.part_p[int64_t(b) * a.E + e];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      p += __shfl_xor(p, o, 64);
      c += __shfl_xor(c, o, 64);
    }
    if (lane == 0) s_p[e] = p, s_c[e] = c, a.counts[e] = c;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double entries = 0.0, cross = 0.0;
    for (int e = 0; e < a.E; ++e) entries += s_c[e], cross += double(s_c[e]) * s_p[e];
    const double rows = s_c[a.E];
    a.loss[0] = rows > 0 ? float(a.E * cross / (entries * rows)) : 0.f;
  }
}

// Backward: the probabilities again from the logits (they are read once in any
// case, and keeping them would write and read as much again).
template <int L, bool BF>
__global__ __launch_bounds__(kRouteThreads) void k_route_backward(RouteArgs a) {
  const int tid = threadIdx.x, l = tid % L;
  __shared__ double s_entries;
  if (tid == 0) {
    double t = 0.0;
    for (int e = 0; e < a.E; ++e) t += a.counts[e];
    s_entries = t;
  }
  __syncthreads();
  float h0[kV];
  {
    const double rows = a.counts[a.E];
    const double f = a.dloss && rows > 0 && s_entries > 0 ? double(a.dloss[0]) * a.E / (rows * s_entries) : 0.0;
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      const int e = 4 * ((j >> 2) * L + l) + (j & 3);
      h0[j] = e < a.E ? float(f * a.counts[e]) : 0.f;
    }
  }
  constexpr int kRows = kRouteThreads / L;
  const int64_t step = int64_t(gridDim.x) * kRows;
  for (int64_t i0 = int64_t(blockIdx.x) * kRows; i0 < a.n; i0 += step) {
    const int64_t i = i0 + tid / L;
    float z[kV], h[kV], d[kV];
    bool any = load_row<L, BF>(a, i, l, z);
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < kV; ++j) top = fmaxf(top, z[j] != z[j] ? INFINITY : z[j]);
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
      any |= bool(__shfl_xor(int(any), o, 64));
      top = fmaxf(top, __shfl_xor(top, o, 64));
    }
    top = any ? top : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      z[j] = expf(z[j] - top);
      sum += z[j];
      h[j] = h0[j];
      d[j] = 0.f;
    }
    sum = row_sum<L>(sum);
    const float inv = any ? 1.f / sum : 0.f;
    if (a.dgates && any) {
      // the chosen experts' gradients, at the lanes that hold them
      float wsum = 0.f, cross = 0.f;
      if (!a.all) {
#pragma unroll 1
        for (int s = 0; s < a.K; ++s) {
          const int id = a.experts[i * a.K + s];
          if (id < 0 || id >= a.E) continue;
          float e = 0.f;
#pragma unroll
          for (int j = 0; j < kV; ++j) e += 4 * ((j >> 2) * L + l) + (j & 3) == id ? z[j] : 0.f;
          e = row_sum<L>(e);
          wsum += e;
          cross += e * a.dgates[i * a.K + s];
        }
      }
      const float winv = wsum > 0.f || wsum != wsum ? 1.f / wsum : 0.f;
      cross *= winv;
#pragma unroll 1
      for (int s = 0; s < a.K; ++s) {
        const int id = a.experts[i * a.K + s];
        if (id < 0 || id >= a.E) continue;
        const float g = a.dgates[i * a.K + s];
#pragma unroll
        for (int j = 0; j < kV; ++j) {
          const bool mine = 4 * ((j >> 2) * L + l) + (j & 3) == id;
          if (a.all) h[j] += mine ? g : 0.f;
          else d[j] += mine ? z[j] * winv * (g - cross) : 0.f;
        }
      }
    }
    float mean = 0.f;
#pragma unroll
    for (int j = 0; j < kV; ++j) {
      z[j] *= inv;
      mean += z[j] * h[j];
    }
    mean = row_sum<L>(mean);
    if (i < a.n) {
#pragma unroll
      for (int c = 0; c < kV / 4; ++c) {
        const int e = 4 * (c * L + l);
        float t[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) t[q] = any ? z[4 * c + q] * (h[4 * c + q] - mean) + d[4 * c + q] : 0.f;
        store4(a.dlogits, BF, i * a.E + e, a.E - e, t);
      }
    }
  }
}

// Lanes per row: as few as hold E logits, 16 a lane.
int route_lanes(int E) {
  int L = 1;
  while (L * kV < E) L *= 2;
  return L;
}

// ---- grouping ------------------------------------------------------------------

constexpr int kGroupWaves = 4;
constexpr int64_t kGroupOne = 8192;      // entries one work-group sorts by itself
constexpr int kGroupOneWaves = 16;

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

// Entries [lo, hi) placed in order by one wavefront from the running places in
// pos[key].
__device__ __forceinline__ void place(const int32_t* __restrict__ experts, int64_t lo, int64_t hi, int E, int bits,
                                      volatile int32_t* pos, int32_t* __restrict__ order) {
  const int lane = threadIdx.x & 63;
  for (int64_t i = lo; i < hi; i += 64) {
    const bool on = i + lane < hi;
    const int key = on ? group_key(experts[i + lane], E) : 0;
    const uint64_t peers = peers_of(key, bits, on);
    const int rank = __popcll(peers & ((uint64_t(1) << lane) - 1));
    const int at = on ? pos[key] : 0;
    __builtin_amdgcn_wave_barrier();
    if (on && rank == 0) pos[key] = at + __popcll(peers);
    __builtin_amdgcn_wave_barrier();
    if (on) order[at + rank] = int32_t(i + lane);
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
  for (int64_t i = lo + lane; i < hi; i += 64) atomicAdd(&pos[w][group_key(experts[i], E)], 1);
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
__global__ __launch_bounds__(kGroupWaves * 64) void k_group_count(const int32_t* experts, int64_t m, int E,
                                                                  int64_t chunk, int chunks, int32_t* hist) {
  __shared__ int32_t cnt[kGroupWaves][kMaxExperts + 1];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c = blockIdx.x * kGroupWaves + w;
  for (int e = lane; e <= E; e += 64) cnt[w][e] = 0;
  __syncthreads();
  const int64_t lo = c * chunk < m ? c * chunk : m, hi = lo + chunk < m ? lo + chunk : m;
  for (int64_t i = lo + lane; i < hi; i += 64) atomicAdd(&cnt[w][group_key(experts[i], E)], 1);
  __syncthreads();
  if (c < chunks)
    for (int e = lane; e <= E; e += 64) hist[int64_t(e) * chunks + c] = cnt[w][e];
}

// One work-group per key: its chunks' counts to places within the key.
__global__ __launch_bounds__(256) void k_group_scan(int32_t* hist, int chunks, int32_t* total) {
  __shared__ int32_t part[4];
  int32_t* row = hist + int64_t(blockIdx.x) * chunks;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int run = 0;
  for (int c0 = 0; c0 < chunks; c0 += 256) {
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
    int before = run;
    for (int u = 0; u < w; ++u) before += part[u];
    if (c < chunks) row[c] = before + v - n;
    run += part[0] + part[1] + part[2] + part[3];
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

// A wavefront's chunk: 1,024 entries, more where there would be over 4,096 chunks.
int64_t group_chunk(int64_t m) { return std::max<int64_t>(1024, (m + 4096 * 64 - 1) / (4096 * 64) * 64); }

template <bool BF>
hipError_t route_of(const RouteArgs& a, int blocks, hipStream_t s) {
  const dim3 g(blocks), b(kRouteThreads);
  const bool only = blocks == 1;
  switch (route_lanes(a.E)) {
    case 1: k_route<1, BF><<<g, b, 0, s>>>(a, only); break;
    case 2: k_route<2, BF><<<g, b, 0, s>>>(a, only); break;
    case 4: k_route<4, BF><<<g, b, 0, s>>>(a, only); break;
    case 8: k_route<8, BF><<<g, b, 0, s>>>(a, only); break;
    default: k_route<16, BF><<<g, b, 0, s>>>(a, only); break;
  }
  return hipGetLastError();
}

template <bool BF>
hipError_t route_backward_of(const RouteArgs& a, int blocks, hipStream_t s) {
  const dim3 g(blocks), b(kRouteThreads);
  switch (route_lanes(a.E)) {
    case 1: k_route_backward<1, BF><<<g, b, 0, s>>>(a); break;
    case 2: k_route_backward<2, BF><<<g, b, 0, s>>>(a); break;
    case 4: k_route_backward<4, BF><<<g, b, 0, s>>>(a); break;
    case 8: k_route_backward<8, BF><<<g, b, 0, s>>>(a); break;
    default: k_route_backward<16, BF><<<g, b, 0, s>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace

int route_blocks(int64_t n, int E, int n_cu) {
  const int rows = kRouteThreads / route_lanes(E);
  return int(std::max<int64_t>(1, std::min<int64_t>((n + rows - 1) / rows, 4 * n_cu)));
}

hipError_t launch_route(const RouteArgs& a, int blocks, hipStream_t s) {
  const hipError_t e = a.bf16 ? route_of<true>(a, blocks, s) : route_of<false>(a, blocks, s);
  if (e != hipSuccess || blocks == 1) return e;
  k_route_total<<<1, 1024, 0, s>>>(a, blocks);
  return hipGetLastError();
}

hipError_t launch_route_backward(const RouteArgs& a, int n_cu, hipStream_t s) {
  const int rows = kRouteThreads / route_lanes(a.E);
  const int blocks = int(std::max<int64_t>(1, std::min<int64_t>((a.n + rows - 1) / rows, 8 * n_cu)));
  return a.bf16 ? route_backward_of<true>(a, blocks, s) : route_backward_of<false>(a, blocks, s);
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
  k_group_count<<<blocks, kGroupWaves * 64, 0, s>>>(experts, m, E, chunk, chunks, hist);
  k_group_scan<<<E + 1, 256, 0, s>>>(hist, chunks, total);
  k_group_place<<<blocks, kGroupWaves * 64, 0, s>>>(experts, m, E, bits, chunk, chunks, hist, total, offsets, order);
  return hipGetLastError();
}

}  // namespace mlip
