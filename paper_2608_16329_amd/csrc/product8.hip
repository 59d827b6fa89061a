// Products of rows and matrices in 8 bits over rows grouped by expert, and the
// gradients of the matrices.
//
//   y_p = W_e x_p + c_e,  offsets[e] <= p < offsets[e + 1]
//   dW_e = sum_p dy_p x_p^T,  dc_e = sum_p dy_p
// (the gradient in x is the first with W packed transposed and dy for x).
//
// A block of 128 inputs is one 16x16x128 matrix instruction on the codes, whose
// scale operands are the blocks' powers of two: values of x are columns, each
// with its row's exponent, those of W rows with their block's.  That instruction
// adds eight neighbouring products at a time, with their bits below 2^-13 of the
// largest one cut off (rms 1.5e-5 of a sum of normally distributed values, at most
// 7 x 2^-13 of the largest product of each eight); sums from there on are float32.
// It is 2^-7 of the rounding of a bfloat16 result, so y in bfloat16 is formed that
// way.  y in float32, and the gradients of W, are formed on 16x16x32 bfloat16
// instructions (8e-9 on the same values): a code and its power of two make a
// bfloat16 without rounding, one conversion for two.
//
// Bound by the matrix instructions where there are many rows and wide matrices, by
// memory where one of the three sizes is small.  Rates on one card: the 16x16x128
// instruction from registers 3,930 TFLOP/s on random codes (4,880 on constant ones:
// the clock falls with what the bits do), products here 8,192 x 8,192 x 8,192 2,270
// to 2,390; 16x16x32 bfloat16 1,830, gradients of 8,192 x 8,192 1,240.
#include <algorithm>
#include <type_traits>

#include "layers_math.h"
#include "learn.h"

namespace mlip {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uni64(int64_t v) {
  return int64_t(uint64_t(uint32_t(uni(int(v >> 32)))) << 32 | uint32_t(uni(int(v))));
}

// The same value, of which the compiler does not know that an earlier one was: what
// is worked out from it is worked out where it is used, not kept from the loop's start.
__device__ __forceinline__ int anew(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The rows of one expert that a work-group has: expert (-1: none), first, end.
struct Part {
  int expert;
  int64_t first, end;
};
// Part t of the experts' rows in parts of `rows`, each expert's from its first
// row on.  All lanes of a wavefront call with the same t.  `whole`: every expert
// has one part at least, also one without rows.
__device__ Part find_part(const int32_t* offsets, int E, int64_t m, int64_t rows, int64_t t, bool whole) {
  if (!offsets) {
    const int64_t first = t * rows;
    if (first >= m && !(whole && t == 0)) return {-1, 0, 0};
    return {0, first, min(m, first + rows)};
  }
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int e = e0 + lane;
    int64_t from = 0, to = 0;
    if (e < E) {
      from = min(m, max(int64_t(0), int64_t(offsets[e])));
      to = min(m, max(from, int64_t(offsets[e + 1])));
    }
    // (fewer than 2^31 parts: their number is at most m + E)
    int parts = int((to - from + rows - 1) / rows);
    if (whole && e < E && parts == 0) parts = 1;
    int sum = parts;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int up = __shfl_up(sum, o);
      if (lane >= o) sum += up;
    }
    const int64_t upto = before + sum;
    const uint64_t mine = __ballot(t < upto && t >= upto - parts);
    if (mine) {
      const int l = __ffsll(static_cast<unsigned long long>(mine)) - 1;
      const int64_t k = t - (before + __shfl(sum, l) - __shfl(parts, l));
      const int64_t f = __shfl(int(from), l), g = __shfl(int(to), l);
      return {uni(e0 + l), uni64(f + k * rows), uni64(min(g, f + (k + 1) * rows))};
    }
    before += __shfl(sum, 63);
  }
  return {-1, 0, 0};
}

// All rows of the expert that is the rank-th largest, for at most 64 experts: long
// parts first leave the work-groups that come last short ones (65,536 rows, 8 experts
// of rising sizes, gradients of 4,096 x 1,024: 620 us against 678 in their order).
__device__ Part sized_part(const int32_t* offsets, int E, int64_t m, int rank) {
  const int lane = threadIdx.x & 63;
  int from = 0, to = -1;
  if (lane < E) {
    from = int(min(m, int64_t(max(0, offsets[lane]))));
    to = int(min(m, int64_t(max(from, offsets[lane + 1]))));
  }
  const int mine = to - from;
  int larger = 0;
  for (int f = 0; f < E; ++f) {
    const int other = __builtin_amdgcn_readlane(mine, f);
    larger += other > mine || (other == mine && f < lane) ? 1 : 0;
  }
  const int l = uni(int(__ffsll(static_cast<unsigned long long>(__ballot(lane < E && larger == rank))) - 1));
  return {l, __builtin_amdgcn_readlane(from, l), __builtin_amdgcn_readlane(to, l)};
}

// One operand's 32 codes of a lane as four bfloat16 operands.
__device__ __forceinline__ void widen(const i8 c, float unit, bf8 v[4]) {
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s], unit, false);
    const bf2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s], unit, true);
    const bf2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s + 1], unit, false);
    const bf2 f = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s + 1], unit, true);
    v[s] = bf8{a[0], a[1], b[0], b[1], d[0], d[1], f[0], f[1]};
  }
}

__device__ __forceinline__ u4v bf16x8(const f4 a, const f4 b) {
  return u4v{bf16x2(a[0], a[1]), bf16x2(a[2], a[3]), bf16x2(b[0], b[1]), bf16x2(b[2], b[3])};
}

// Four neighbouring outputs of a row, at the alignment of one.
template <bool F32>
__device__ __forceinline__ void put4(void* y, int64_t at, int left, const f4 v) {
  if (F32) {
    float* p = static_cast<float*>(y) + at;
    if (left >= 4) *reinterpret_cast<U4*>(p) = __builtin_bit_cast(u4v, v);
    else {
#pragma unroll
      for (int q = 0; q < 3; ++q)
        if (q < left) p[q] = v[q];
    }
  } else {
    uint16_t* p = static_cast<uint16_t*>(y) + at;
    if (left >= 4) *reinterpret_cast<U2*>(p) = u2v{bf16x2(v[0], v[1]), bf16x2(v[2], v[3])};
    else {
#pragma unroll
      for (int q = 0; q < 3; ++q)
        if (q < left) p[q] = to_bf16(v[q]);
    }
  }
}

// ---- many rows: tiles of WR x 16 RF rows and WC x 16 CF outputs ---------------------
//
// A work-group takes tiles in turn.  A step is one block of 128 inputs: its codes
// come to LDS as they are, without registers, while the block before is multiplied;
// the next tile's first block comes during a tile's last step, so that only the stores
// of the results stand between two tiles, and those of a full tile are not waited for
// until the next one's first step ends.
// 65,536 rows, 8 experts, 1,024 inputs to 4,096 outputs, bfloat16: 306 to 357 us (1,540
// to 1,800 TFLOP/s, the cards differ), 339 MB read past L2 and 538 written, the matrix instructions
// busy for 35% of the cycles: a tile has eight steps only, and its results take 60 us of
// stores; 4,096 to 1,024: 326 to 350, four rounds of tiles and a fifth of a few.
// Four or sixteen tiles of rows beside each other instead of eight, and a higher priority
// of wavefronts while they multiply, are within 2% (the gradients below get 8% slower
// by that priority).

// Which of a wavefront's outputs row r of its operand i of W is: the four that a
// lane gets of each of two neighbouring operands (rows 4 g .. 4 g + 3) are eight
// neighbouring outputs, so bfloat16 results are stored 16 bytes a lane; float32
// results are that with one operand.
template <bool F32>
__device__ __forceinline__ int output_of(int i, int r) {
  return F32 ? 16 * i + r : 32 * (i >> 1) + 8 * (r >> 2) + 4 * (i & 1) + (r & 3);
}
// Where 16-byte piece c of row r of a block stands in LDS: at c ^ key, such that
// the 16 rows that lanes read together spread over the banks.
template <bool PAIRS>
__device__ __forceinline__ int key(int r) {
  return PAIRS ? (r & 3) | ((r >> 3) & 1) << 2 : r & 7;
}

// Brings one block of 128 codes of a tile's rows to LDS, 8 rows an instruction, N
// instructions a wavefront; a row behind the last one is the last one again.
template <int N, bool PAIRS>
struct Stage {
  const uint8_t* base;
  uint32_t at[N];               // of a lane's piece, from the tile's first row on
  __device__ __forceinline__ Stage(const uint8_t* first, int64_t pitch, int rows) : base(first) {
    const int w = uni(int(threadIdx.x >> 6)), lane = anew(threadIdx.x & 63);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int r = 8 * (N * w + k) + (lane >> 3);
      at[k] = uint32_t(min(r, rows - 1)) * uint32_t(pitch) + 16u * ((lane & 7) ^ key<PAIRS>(r));
    }
  }
  __device__ __forceinline__ void bring(int k, int block, unsigned char* lds) const {
    const uint8_t* from = base + int64_t(block) * kBlock8;
    unsigned char* to = lds + (N * uni(int(threadIdx.x >> 6)) + k) * (8 * kBlock8);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + at[k]),
                                     (__attribute__((address_space(3))) void*)to, 16, 0, 0);
  }
};
// A lane's 32 codes of a row of a block: pieces g and g + 4 of the eight, for both
// operands.  Where they are depends on the row's lowest bits alone, so other rows
// that a lane takes are at a distance that the instruction has in it.
struct Pieces {
  int a, b;
  template <bool PAIRS>
  static __device__ __forceinline__ Pieces of(int r, int g) {
    return {r * kBlock8 + 16 * (g ^ key<PAIRS>(r)), r * kBlock8 + 16 * ((g + 4) ^ key<PAIRS>(r))};
  }
};
__device__ __forceinline__ i8 take(const unsigned char* lds, Pieces p, int rows_on) {
  const u4v a = *reinterpret_cast<const u4v*>(lds + p.a + rows_on * kBlock8);
  const u4v b = *reinterpret_cast<const u4v*>(lds + p.b + rows_on * kBlock8);
  return i8{int(a[0]), int(a[1]), int(a[2]), int(a[3]), int(b[0]), int(b[1]), int(b[2]), int(b[3])};
}

// Tiles of rows of all experts: which tile is each expert's first, and its rows.
struct Tiles {
  int first[kMaxExperts + 1], from[kMaxExperts], to[kMaxExperts];
};
// Filled in by the first wavefront; the work-group waits for it.  Returns the
// number of tiles.
__device__ __forceinline__ int count_tiles(Tiles& t, const Product8Args& a, int rows) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    int before = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
      const int e = e0 + lane;
      int from = 0, to = 0;
      if (e < a.E) {
        from = a.offsets ? int(min(a.m, int64_t(max(0, a.offsets[e])))) : 0;
        to = a.offsets ? int(min(a.m, int64_t(max(from, a.offsets[e + 1])))) : int(a.m);
      }
      int sum = (to - from) / rows + ((to - from) % rows ? 1 : 0);
      const int mine = sum;
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const int up = __shfl_up(sum, o);
        if (lane >= o) sum += up;
      }
      if (e < a.E) {
        t.first[e] = before + sum - mine;
        t.from[e] = from;
        t.to[e] = to;
      }
      before += __shfl(sum, 63);
    }
    if (lane == 0) t.first[a.E] = before;
  }
  __syncthreads();
  return uni(t.first[a.E]);
}
__device__ __forceinline__ int expert_of(const Tiles& t, int E, int tile) {
  for (int e0 = 0;; e0 += 64) {
    const int e = min(E - 1, e0 + int(threadIdx.x & 63));
    const uint64_t mine = __ballot(t.first[e] <= tile && tile < t.first[e + 1]);
    if (mine || e0 + 64 >= E) return min(E - 1, e0 + int(__ffsll(static_cast<unsigned long long>(mine))) - 1);
  }
}

// STREAM: y is larger than the last cache and goes past it.
// A wavefront multiplies CF operands of W with RF of x: a tile of 256 x 256 has eight
// wavefronts of 128 rows x 64 outputs each (sixteen of 64 x 64, or four of 128 x 128, do
// not fit the registers), and its two buffers of codes take 128 KB of LDS; one of
// 128 x 128 four of 64 x 64, two work-groups a CU.
template <bool F32, int RF, int CF, int WR, int WC, bool STREAM = false>
__global__ __launch_bounds__(64 * WR * WC) void k_product(Product8Args a) {
  constexpr int kWaves = WR * WC, kRowTile = 16 * RF * WR, kColTile = 16 * CF * WC, kStage = (kRowTile + kColTile) * kBlock8;
  constexpr int kBringX = kRowTile / 8 / kWaves, kBringW = kColTile / 8 / kWaves;
  constexpr int kSide = F32 ? 1 : 2, kStores = RF * CF / kSide;
  // (two variables, not one with two halves: what is read from the one does not wait
  // for what is on its way to the other)
  __shared__ __attribute__((aligned(16))) unsigned char lds0[kStage], lds1[kStage];
  __shared__ __attribute__((aligned(16))) float col_bias[kColTile];
  __shared__ uint32_t row_exps[2 * kRowTile];                 // of four blocks, and of the four behind them
  __shared__ Tiles tiles;
  const int row_tiles = count_tiles(tiles, a, kRowTile), col_tiles = (a.N + kColTile - 1) / kColTile;
  // a work-group takes tiles of its XCD's share (work-groups go round the eight) in
  // turn with the others there: neighbours in time share rows or outputs in its cache
  const int64_t total = int64_t(row_tiles) * col_tiles;
  const int xcd = blockIdx.x & 7, slots = gridDim.x >> 3;
  const int last = uni(int(total * (xcd + 1) / 8));
  int id = uni(int(total * xcd / 8)) + int(blockIdx.x >> 3);
  if (id >= last) return;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, w = uni(int(threadIdx.x >> 6));
  const int rows0 = 16 * RF * (w % WR), cols0 = 16 * CF * (w / WR);   // of the wavefront, within the tile
  const int64_t kp = codes8(a.K);
  const uint32_t xp = uint32_t(exps8(a.K));
  const int blocks = (a.K + kBlock8 - 1) / kBlock8, blocks_n = (a.N + kBlock8 - 1) / kBlock8;
  // a wavefront's outputs are within one block of W
  static_assert(kBlock8 % (16 * CF) == 0);

  struct Tile {
    int expert, first, rows, n0;
  };
  const auto held = [](const Tile& t) { return Tile{uni(t.expert), uni(t.first), uni(t.rows), uni(t.n0)}; };
  const auto tile_of = [&](int t) {
    // eight tiles of rows beside each other for each tile of outputs
    const int band = t / (8 * col_tiles), in = t - band * 8 * col_tiles, deep = min(8, row_tiles - 8 * band);
    const int rt = 8 * band + in % deep;
    Tile v;
    v.expert = uni(expert_of(tiles, a.E, rt));
    v.first = uni(tiles.from[v.expert] + (rt - tiles.first[v.expert]) * kRowTile);
    v.rows = uni(min(kRowTile, tiles.to[v.expert] - v.first));
    v.n0 = uni(in / deep) * kColTile;
    return v;
  };
  const auto xstage_of = [&](const Tile& t) { return Stage<kBringX, false>(a.x + t.first * kp, kp, t.rows); };
  const auto wstage_of = [&](const Tile& t) {
    return Stage<kBringW, !F32>(a.w + (int64_t(t.expert) * a.N + t.n0) * kp, kp, min(kColTile, a.N - t.n0));
  };
  // On their way to LDS, for which a lane has one register: exponents of four blocks
  // of a row (the first wavefronts), the bias of one of the tile's outputs (the
  // others).  Those of the wavefront's outputs are in one block, and scalar.
  constexpr int kRowWaves = kRowTile / 64;
  constexpr int kColWaves = kColTile / 64;
  static_assert(kRowWaves + kColWaves <= kWaves);
  uint32_t we = 0, wnext, coming = 0;
  const auto exponents = [&](const Tile& t, int b) {
    wnext = *(const __attribute__((address_space(4))) uint32_t*)(a.w_exps + (int64_t(t.expert) * blocks_n + min(blocks_n - 1, (t.n0 + cols0) / kBlock8)) * xp + b);
    if (w < kRowWaves)
      coming = *reinterpret_cast<const uint32_t*>(a.x_exps + int64_t(t.first) * xp + b + uint32_t(min(t.rows - 1, 64 * w + anew(lane))) * xp);
  };
  const auto lay_exponents = [&](int half) {
    if (w < kRowWaves) row_exps[half * kRowTile + 64 * w + anew(lane)] = coming;
  };
  const auto bias = [&](const Tile& t) {
    if (a.bias && w >= kRowWaves && w < kRowWaves + kColWaves)
      coming = __float_as_uint(a.bias[int64_t(t.expert) * a.N + min(a.N - 1, t.n0 + 64 * (w - kRowWaves) + anew(lane))]);
  };
  const auto lay_bias = [&] {
    if (a.bias && w >= kRowWaves && w < kRowWaves + kColWaves) col_bias[64 * (w - kRowWaves) + anew(lane)] = __uint_as_float(coming);
  };

  Tile tile = tile_of(id);
  Stage<kBringX, false> xstage = xstage_of(tile);
  Stage<kBringW, !F32> wstage = wstage_of(tile);
  exponents(tile, 0);
#pragma unroll
  for (int k = 0; k < kBringX; ++k) xstage.bring(k, 0, lds0);
#pragma unroll
  for (int k = 0; k < kBringW; ++k) wstage.bring(k, 0, lds0 + kRowTile * kBlock8);
  lay_exponents(0);
  const Pieces xp0 = Pieces::of<false>(rows0 + r, g), wp0 = Pieces::of<!F32>(cols0 + output_of<F32>(0, r), g);
  int half = 1;                                               // of row_exps that has the block's
  bool more = id + slots < last;
  Tile then = tile_of(more ? id + slots : id);
  f4 sum[CF][RF];                                             // outputs, rows

  // Products of block b of the tile, in LDS at xs, and before the first of them requests
  // for block `after` of the tile that the stages are at (the last block once more,
  // unused, where there is none).
  const auto step = [&](int b, const unsigned char* xs, int after, unsigned char* next) {
    const unsigned char* const ws = xs + kRowTile * kBlock8;
    uint32_t xe[RF];
    {
      const uint8_t* const from = reinterpret_cast<const uint8_t*>(row_exps + half * kRowTile + rows0 + r) + (b & 3);
#pragma unroll
      for (int j = 0; j < RF; ++j) xe[j] = from[64 * j];
    }
    __builtin_amdgcn_sched_barrier(0);
    if (b % 4 == 0) {
      const bool on = b + 4 < blocks;
      exponents(on ? tile : then, on ? b + 4 : 0);
      if (b == 0) bias(tile);
    }
    const auto bring = [&] {
#pragma unroll
      for (int k = 0; k < kBringX; ++k) xstage.bring(k, after, next);
#pragma unroll
      for (int k = 0; k < kBringW; ++k) wstage.bring(k, after, next + kRowTile * kBlock8);
    };
    const auto of_x = [&](int j) { return take(xs, xp0, 16 * j); };
    const auto of_w = [&](int i) { return take(ws, wp0, output_of<F32>(i, 0)); };
    if constexpr (F32) {
      bf8 wv[CF][4];
#pragma unroll
      for (int i = 0; i < CF; ++i) widen(of_w(i), __uint_as_float((we & 255u) << 23), wv[i]);
#pragma unroll
      for (int j = 0; j < RF; ++j) {
        if (j == 0) bring();
        bf8 xv[4];
        widen(of_x(j), __uint_as_float(xe[j] << 23), xv);
#pragma unroll
        for (int i = 0; i < CF; ++i)
#pragma unroll
          for (int s = 0; s < 4; ++s) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[i][s], xv[s], sum[i][j], 0, 0, 0);
      }
    } else {
      i8 c[CF], x = of_x(0);
#pragma unroll
      for (int i = 0; i < CF; ++i) c[i] = of_w(i);
#pragma unroll
      for (int j = 0; j < RF; ++j) {
        i8 ahead = x;
        if (j + 1 < RF) ahead = of_x(j + 1);
        if (j == 0) bring();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < CF; ++i)
          sum[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(c[i], x, sum[i][j], 0, 0, 0, int(we), 0, int(xe[j]));
        __builtin_amdgcn_sched_barrier(0);
        x = ahead;
      }
    }
    we >>= 8;
  };
  // What was asked for is there, and what was read is used up, in all wavefronts.
  const auto meet = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  meet();
  for (;;) {
#pragma unroll
    for (int i = 0; i < CF; ++i)
#pragma unroll
      for (int j = 0; j < RF; ++j) sum[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    for (int b = 0; b < blocks; b += 2) {
      if (b % 4 == 0) {
        we = wnext;
        half ^= 1;
      }
      step(b, lds0, min(b + 1, blocks - 1), lds1);
      meet();
      if (b % 4 == 0) lay_exponents(half ^ 1);
      if (b == 0) lay_bias();
      // behind the last block the next tile's first one
      const bool on = b + 2 < blocks;
      if (!on) {
        xstage = xstage_of(then);
        wstage = wstage_of(then);
      }
      if (b + 1 < blocks) {
        step(b + 1, lds1, on ? b + 2 : 0, lds0);
      } else {
#pragma unroll
        for (int k = 0; k < kBringX; ++k) xstage.bring(k, 0, lds0);
#pragma unroll
        for (int k = 0; k < kBringW; ++k) wstage.bring(k, 0, lds0 + kRowTile * kBlock8);
      }
      if (on) meet();
    }

    // a lane has four neighbouring outputs of a row, with those of the next operand eight
    const int lane1 = anew(lane), r1 = rows0 + (lane1 & 15), g1 = lane1 >> 4;
    using Out = std::conditional_t<F32, float, uint16_t>;
    Out* const y = static_cast<Out*>(a.y) + int64_t(tile.first) * a.N;
    if (a.bias) {
      if (blocks <= 2) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
      for (int i = 0; i < CF; ++i) {
        const f4 c = *reinterpret_cast<const f4*>(col_bias + cols0 + output_of<F32>(i, 4 * g1));
#pragma unroll
        for (int j = 0; j < RF; ++j) sum[i][j] += c;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // 16 bytes at the alignment of one value, whatever the outputs' number.  Lanes of
    // neighbouring rows exchange halves, so that eight of them have 128 neighbouring
    // bytes of one row, a whole line, in one store.
    const auto put = [&](const u4v v, int p, int n, bool check) {
      Out* const to = y + int64_t(p) * a.N + n;
      if (!check || (p < tile.rows && n + 4 * kSide <= a.N)) {
        if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<U4*>(to));
        else *reinterpret_cast<U4*>(to) = v;
      } else if (p < tile.rows) {
#pragma unroll
        for (int q = 0; q < 4 * kSide - 1; ++q)
          if (n + q < a.N) {
            if constexpr (F32) to[q] = __uint_as_float(v[q]);
            else to[q] = uint16_t(v[q / 2] >> (16 * (q % 2)));
          }
      }
    };
    const auto store = [&](int j, bool check) {
      const bool odd = r1 & 1;
      constexpr int kEach = 4 * kSide, kHalf = 4 * kEach;     // outputs of a lane, of a row's half line
#pragma unroll
      for (int i = 0; i < CF; i += 2 * kSide) {
        u4v lo, hi, other;
        if constexpr (F32) {
          lo = __builtin_bit_cast(u4v, sum[i][j]);
          hi = __builtin_bit_cast(u4v, sum[i + 1][j]);
        } else {
          lo = bf16x8(sum[i][j], sum[i + 1][j]);
          hi = bf16x8(sum[i + 2][j], sum[i + 3][j]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
          other[q] = uint32_t(__builtin_amdgcn_update_dpp(0, int(odd ? lo[q] : hi[q]), 0xb1, 0xf, 0xf, true));
        const int n = tile.n0 + cols0 + 16 * i + kEach * g1 + (odd ? kHalf : 0);
        put(odd ? other : lo, (r1 & ~1) + 16 * j, n, check);
        put(odd ? hi : other, (r1 | 1) + 16 * j, n, check);
      }
    };
    const bool full = tile.rows == kRowTile && tile.n0 + kColTile <= a.N;
    if (full) {
#pragma unroll
      for (int j = 0; j < RF; ++j) {
        store(j, false);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < RF; ++j) {
        store(j, true);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (!more) break;
    id += slots;
    tile = held(then);
    more = id + slots < last;
    then = tile_of(more ? id + slots : id);
    // the next tile's first block is there; a full tile's stores, which were issued
    // after it and are counted in order, may be under way
    if (full) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(kStores) : "memory");
    else meet();
  }
}

// ---- few rows: 16 RF rows and 16 outputs, the blocks of inputs shared by wavefronts ----
//
// Bound by the weights, that is by memory or, for a row or two, by latency: they are
// read once for every 16 RF rows, straight to registers; a work-group has 16 outputs,
// and each of its wavefronts every fourth block of inputs, of which it asks for two
// at once.  One row, 1,024 inputs and outputs: 3.8 us.
template <bool F32, int RF>
__global__ __launch_bounds__(256) void k_product_few(Product8Args a, int col_tiles) {
  __shared__ f4 part_sum[3][RF][64];
  const int64_t id = blockIdx.x;
  const int64_t rt = id / col_tiles;
  const int n0 = int(id - rt * col_tiles) * 16;
  const Part part = find_part(a.offsets, a.E, a.m, 16 * RF, rt, false);
  if (part.expert < 0) return;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, w = uni(int(threadIdx.x >> 6));
  const int64_t kp = codes8(a.K), xp = exps8(a.K);
  const int blocks = (a.K + kBlock8 - 1) / kBlock8, blocks_n = (a.N + kBlock8 - 1) / kBlock8;
  const uint8_t* const wc = a.w + (int64_t(part.expert) * a.N + min(a.N - 1, n0 + r)) * kp + 16 * g;
  const uint8_t* const we = a.w_exps + (int64_t(part.expert) * blocks_n + n0 / kBlock8) * xp;
  const uint8_t* xc[RF];
  const uint8_t* xe[RF];
#pragma unroll
  for (int j = 0; j < RF; ++j) {
    const int64_t p = min(part.end - 1, part.first + 16 * j + r);
    xc[j] = a.x + p * kp + 16 * g;
    xe[j] = a.x_exps + p * xp;
  }
  f4 sum[RF];
#pragma unroll
  for (int j = 0; j < RF; ++j) sum[j] = f4{0.f, 0.f, 0.f, 0.f};
  const auto codes = [](const uint8_t* from) {
    const u4v u = *reinterpret_cast<const u4v*>(from), v = *reinterpret_cast<const u4v*>(from + 64);
    return i8{int(u[0]), int(u[1]), int(u[2]), int(u[3]), int(v[0]), int(v[1]), int(v[2]), int(v[3])};
  };
  for (int b0 = w; b0 < blocks; b0 += 8) {
    // (behind the last block the last one again, and not used)
    i8 c[2], x[2][RF];
    uint32_t ew[2], ex[2][RF];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = min(blocks - 1, b0 + 4 * h);
      c[h] = codes(wc + int64_t(b) * kBlock8);
      ew[h] = we[b];
#pragma unroll
      for (int j = 0; j < RF; ++j) {
        x[h][j] = codes(xc[j] + int64_t(b) * kBlock8);
        ex[h][j] = xe[j][b];
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (b0 + 4 * h >= blocks) break;
      if constexpr (F32) {
        bf8 cv[4];
        widen(c[h], __uint_as_float(ew[h] << 23), cv);
#pragma unroll
        for (int j = 0; j < RF; ++j) {
          bf8 xv[4];
          widen(x[h][j], __uint_as_float(ex[h][j] << 23), xv);
#pragma unroll
          for (int s = 0; s < 4; ++s) sum[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cv[s], xv[s], sum[j], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int j = 0; j < RF; ++j)
          sum[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(c[h], x[h][j], sum[j], 0, 0, 0, int(ew[h]), 0, int(ex[h][j]));
      }
    }
  }
  if (w > 0) {
#pragma unroll
    for (int j = 0; j < RF; ++j) part_sum[w - 1][j][lane] = sum[j];
  }
  __syncthreads();
  if (w > 0) return;
  const int n = n0 + 4 * g;
  f4 bias = {0.f, 0.f, 0.f, 0.f};
  if (a.bias) {
#pragma unroll
    for (int q = 0; q < 4; ++q) bias[q] = a.bias[int64_t(part.expert) * a.N + min(a.N - 1, n + q)];
  }
#pragma unroll
  for (int j = 0; j < RF; ++j) {
    const int64_t p = part.first + 16 * j + r;
    const f4 v = (sum[j] + part_sum[0][j][lane]) + (part_sum[1][j][lane] + part_sum[2][j][lane]) + bias;
    if (p < part.end) put4<F32>(a.y, p * a.N + n, a.N - n, v);
  }
}

// ---- gradients of the matrices ------------------------------------------------------
//
// The sum runs over rows, and an operand's values of one column are those of
// consecutive rows: rows go to LDS as they come, in bfloat16 (codes times their row's
// power of two, without rounding; a row's exponent differs from the next one's, so
// codes alone cannot be multiplied), and are read transposed by the instruction for
// that.  Every tile sums all rows of its expert; where tiles are too few for the CUs,
// slices of them, which k_add_slices adds up in order.
// 65,536 rows, 8 experts of 3,500 to 15,500 rows, 4,096 x 1,024: 550 to 615 us (890 to
// 1,000 TFLOP/s; a product of 8,192 x 8,192 x 8,192 of the library's bfloat16 1,072),
// 1.23 GB read past L2; 4,096 x 4,096 of one expert 1,220 TFLOP/s.  The matrix
// instructions are busy for 42% of the cycles, LDS for 37% (bank conflicts 10%).
// Columns laid transposed by the threads that write them were slower (851 us against
// 627), writes without conflicts too (645 against 636), sixteen wavefronts of 64 x 64
// as well (641 against 630).

constexpr int kRows = 32;                       // rows of a step

// One operand's rows of a step, on their way from memory to LDS: half of the
// work-group's threads have P pieces of 16 codes each, with their rows' powers of two.
template <int COLS, int THREADS>
struct Rows {
  static constexpr int kPieces = COLS / 16, P = kRows * kPieces / THREADS, kApart = THREADS / kPieces;
  static_assert(P >= 1 && P * THREADS == kRows * kPieces && kApart % 8 == 0);
  const uint8_t* codes;         // of the part's first row, the tile's first column
  const uint8_t* exps;
  uint32_t pitch, xpitch;
  int col;
  uint32_t at, xat;             // of a thread's first piece and its exponent
  u4v c[2][P];
  uint32_t e[2][P];

  __device__ __forceinline__ Rows(const uint8_t* all, const uint8_t* all_exps, int64_t width, int64_t first, int column) {
    col = column;
    pitch = uint32_t(codes8(width));
    xpitch = uint32_t(exps8(width));
    codes = all + first * pitch + col;
    exps = all_exps + first * xpitch + col / kBlock8;
    const int row = threadIdx.x % THREADS / kPieces, piece = threadIdx.x % kPieces;
    // (a block behind the last one of the row is the tile's first, and not used)
    const bool there = col + 16 * piece < int(pitch);
    at = row * pitch + (there ? 16 * piece : 0);
    xat = row * xpitch + (there ? piece / (kBlock8 / 16) : 0);
  }
  // Rows from step * kRows on into set s; zeros behind the part's `rows` (a buffer's
  // loads give those behind its end; all of the offset is in what is compared with it).
  __device__ __forceinline__ void fetch(int s, int64_t step, int64_t rows) {
    const int64_t p0 = step * kRows;
    const int left = int(max(int64_t(0), min(int64_t(kRows), rows - p0)));
    const auto from = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(codes + p0 * pitch), 0, max(0, left * int(pitch) - col), 0x27000);
    const auto efrom = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(exps + p0 * xpitch), 0, max(0, left * int(xpitch) - col / kBlock8), 0x27000);
#pragma unroll
    for (int q = 0; q < P; ++q) {
      c[s][q] = __builtin_bit_cast(u4v, __builtin_amdgcn_raw_buffer_load_b128(from, int(at) + q * kApart * int(pitch), 0, 0));
      e[s][q] = __builtin_amdgcn_raw_buffer_load_b8(efrom, int(xat) + q * kApart * int(xpitch), 0, 0);
    }
  }
  // To LDS in bfloat16, without rounding: rows of 2 COLS bytes, 16 values (32 bytes) c of row p at c ^ p % 8.
  __device__ __forceinline__ void lay(int s, int q, unsigned char* lds) const {
    const int row = threadIdx.x % THREADS / kPieces, piece = threadIdx.x % kPieces;
    const float unit = __uint_as_float(e[s][q] << 23);
    bf2 h[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      h[2 * k] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(c[s][q][k]), unit, false);
      h[2 * k + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(c[s][q][k]), unit, true);
    }
    u4v* to = reinterpret_cast<u4v*>(lds + row * (2 * COLS) + 32 * (piece ^ (row & 7)) + q * kApart * (2 * COLS));
#pragma unroll
    for (int k = 0; k < 2; ++k)
      to[k] = u4v{__builtin_bit_cast(uint32_t, h[4 * k]), __builtin_bit_cast(uint32_t, h[4 * k + 1]),
                  __builtin_bit_cast(uint32_t, h[4 * k + 2]), __builtin_bit_cast(uint32_t, h[4 * k + 3])};
  }
};
// Values of 16 columns (i: which 16, after the wavefront's first) and a step's rows
// as an operand: read transposed, 16 lanes have 4 rows of 16 values at a time.
template <int COLS>
__device__ __forceinline__ bf8 columns(const unsigned char* lds, int lane_at, int i) {
  typedef short s8 __attribute__((ext_vector_type(8)));
  s4 v[2];
#pragma unroll
  for (int s = 0; s < 2; ++s)
    v[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s4*)(lds + (lane_at ^ (32 * i)) + 16 * s * (2 * COLS)));
  return __builtin_bit_cast(bf8, s8{v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]});
}
// Where a lane's first four values of a wavefront's columns are.  `first` is a multiple
// of the wavefront's columns, a power of two of them, so that 16 i more of them is an
// exclusive or with 32 i bytes.
template <int COLS>
__device__ __forceinline__ int columns_at(int first) {
  const int lane = threadIdx.x & 63, p = 4 * (lane >> 4) + ((lane & 15) >> 2);
  return p * (2 * COLS) + 32 * ((first / 16) ^ (p & 7)) + 8 * (lane & 3);
}

// A wavefront has 16 NF outputs by 16 KF inputs, a work-group WN x WK of those.
// Three steps of rows are in LDS: one that is used, the next one, of which the first
// operands are read before the barrier that ends this one, and one that is laid.
// BIAS: the outputs' own sums too.
template <int NF, int KF, int WN, int WK, bool BIAS>
__device__ __forceinline__ void weights_tile(const Product8Args& a, const Part& part, int64_t item, int nt, int kt, unsigned char* lds) {
  constexpr int kThreads = 64 * WN * WK, kN = 16 * NF * WN, kK = 16 * KF * WK, kOne = kRows * (kN + kK) * 2;
  const int64_t first = uni64(part.first);
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, w = uni(int(threadIdx.x >> 6));
  const int wn = 16 * NF * (w % WN), wk = 16 * KF * (w / WN);         // of the wavefront, within the tile
  const int64_t rows = uni64(part.end - part.first), steps = (rows + kRows - 1) / kRows;
  // the first half of the wavefronts brings dy's rows, the other one x's
  static_assert(kN == kK);
  const bool front = w < WN * WK / 2;
  Rows<kN, kThreads / 2> mine(front ? a.w : a.x, front ? a.w_exps : a.x_exps, front ? a.N : a.K, first, front ? nt * kN : kt * kK);
  const int nat = columns_at<kN>(wn), kat = columns_at<kK>(wk);
  f4 sum[KF][NF];
  float own[NF];                                                 // inputs, outputs; the outputs' own, of a lane's rows
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    own[j] = 0.f;
#pragma unroll
    for (int i = 0; i < KF; ++i) sum[i][j] = f4{0.f, 0.f, 0.f, 0.f};
  }
  const auto lay = [&](int s, int q, unsigned char* to) { mine.lay(s, q, to + (front ? 0 : kRows * kN * 2)); };
  const auto fetch = [&](int s, int64_t step) { mine.fetch(s, step, rows); };
  bf8 dv[NF], xv;
  const auto of_n = [&](const unsigned char* from, int j) { return columns<kN>(from, nat, j); };
  const auto of_k = [&](const unsigned char* from, int i) { return columns<kK>(from + kRows * kN * 2, kat, i); };
  // Products of the step at `here`; the rows in set s go to `then` beside them.
  const auto step = [&](const unsigned char* here, const unsigned char* next, int s, unsigned char* then) {
    bf8 dnext[NF];
    if constexpr (BIAS) {
      // products with ones, and sums, two rows an instruction
#pragma unroll
      for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int q = 0; q < 8; q += 2)
          own[j] = __builtin_amdgcn_fdot2_f32_bf16(bf2{dv[j][q], dv[j][q + 1]}, bf2{__bf16(1.f), __bf16(1.f)}, own[j], false);
    }
#pragma unroll
    for (int i = 0; i < KF; ++i) {
      // (the order as it stands here: loads any earlier would be held in registers)
      __builtin_amdgcn_sched_barrier(0);
      const bf8 ahead = i + 1 < KF ? of_k(here, i + 1) : of_k(next, 0);
      if (i == KF - 2)
#pragma unroll
        for (int j = 0; j < NF; ++j) dnext[j] = of_n(next, j);
#pragma unroll
      for (int j = 0; j < NF; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv, dv[j], sum[i][j], 0, 0, 0);
#pragma unroll
      for (int q = 0; q < mine.P; ++q)
        if (q % KF == i) lay(s, q, then);
      xv = ahead;
    }
#pragma unroll
    for (int j = 0; j < NF; ++j) dv[j] = dnext[j];
  };
  const auto meet = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  // rows of a step are asked for two steps before they go to LDS, two steps before their use
  if (steps > 0) {
    fetch(0, 0);
    fetch(1, 1);
#pragma unroll
    for (int q = 0; q < mine.P; ++q) lay(0, q, lds);
    fetch(0, 2);
#pragma unroll
    for (int q = 0; q < mine.P; ++q) lay(1, q, lds + kOne);
    fetch(1, 3);
    meet();
#pragma unroll
    for (int j = 0; j < NF; ++j) dv[j] = of_n(lds, j);
    xv = of_k(lds, 0);
    unsigned char *here = lds, *next = lds + kOne, *then = lds + 2 * kOne;
    for (int64_t b = 0; b < steps; b += 2) {
      step(here, next, 0, then);
      fetch(0, b + 4);
      meet();
      step(next, then, 1, here);                              // (of zeros where there is none)
      fetch(1, b + 5);
      meet();
      unsigned char* const t = here;
      here = then;
      then = next;
      next = t;
    }
  }
  if constexpr (BIAS)
#pragma unroll
    for (int j = 0; j < NF; ++j) {
      own[j] += __shfl_xor(own[j], 16);
      own[j] += __shfl_xor(own[j], 32);
    }
  const int64_t to = a.slots ? item : part.expert;
  float* out = (a.slots ? a.slots : a.dweights) + to * a.N * a.K;
#pragma unroll
  for (int j = 0; j < NF; ++j) {
    const int n = nt * kN + wn + 16 * j + r;
    if (n >= a.N) continue;
#pragma unroll
    for (int i = 0; i < KF; ++i) {
      const int k = kt * kK + wk + 16 * i + 4 * g;
      put4<true>(out, int64_t(n) * a.K + k, a.K - k, sum[i][j]);
    }
    if (BIAS && w / WN == 0 && g == 0) (a.slots ? a.bias_slots : a.dbias)[to * a.N + n] = own[j];
  }
}

template <int NF, int KF, int WN, int WK>
__global__ __launch_bounds__(64 * WN * WK) void k_product_weights(Product8Args a, int tiles_n, int tiles_k) {
  __shared__ __attribute__((aligned(256))) unsigned char lds[3 * kRows * 2 * 16 * (NF * WN + KF * WK)];
  const int64_t id = blockIdx.x;
  const int tiles = tiles_n * tiles_k;
  const int64_t item = id / tiles;
  const int t = int(id - item * tiles), nt = uni(t / tiles_k), kt = uni(t - nt * tiles_k);
  const Part part = !a.slots && a.offsets && a.E <= 64 ? sized_part(a.offsets, a.E, a.m, uni(int(item)))
                                                        : find_part(a.offsets, a.E, a.m, a.slice, item, true);
  if (part.expert < 0) return;
  if (a.dbias && kt == 0) weights_tile<NF, KF, WN, WK, true>(a, part, item, nt, kt, lds);
  else weights_tile<NF, KF, WN, WK, false>(a, part, item, nt, kt, lds);
}

// The experts' sums of their slices, bound by memory.  SPLIT: four wavefronts have
// every fourth slice of 64 values, for matrices that would not fill the CUs with a
// thread a value (both kernels of a gradient, without and with: 262,144 rows, 64 x 64,
// 70 us and 35; 2,000 rows, 512 x 512, 15.3 and 17.4).
template <bool SPLIT>
__global__ __launch_bounds__(256) void k_add_slices(Product8Args a) {
  __shared__ float quarter[SPLIT ? 4 : 1][64];
  const int e = blockIdx.y, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  // slices of the experts before, and of this one
  int64_t before = 0, mine = 0;
  for (int f = lane; f <= e; f += 64) {
    int64_t from = 0, to = a.m;
    if (a.offsets) {
      from = min(a.m, max(int64_t(0), int64_t(a.offsets[f])));
      to = min(a.m, max(from, int64_t(a.offsets[f + 1])));
    }
    const int64_t parts = max(int64_t(1), (to - from + a.slice - 1) / a.slice);
    if (f < e) before += parts;
    else mine = parts;
  }
#pragma unroll
  for (int o = 32; o > 0; o /= 2) {
    before += __shfl_xor(static_cast<long long>(before), o);
    mine += __shfl_xor(static_cast<long long>(mine), o);
  }
  // (offsets that do not rise may ask for more than there are)
  mine = max(int64_t(0), min(mine, a.m / a.slice + a.E - before));
  const int64_t values = int64_t(a.N) * a.K, all = values + (a.dbias ? a.N : 0);
  constexpr int kEach = SPLIT ? 64 : 256, kBy = SPLIT ? 4 : 1;
  for (int64_t v0 = int64_t(blockIdx.x) * kEach; v0 < all; v0 += int64_t(gridDim.x) * kEach) {
    const int64_t v = v0 + (SPLIT ? lane : int(threadIdx.x));
    const bool weight = v < values;
    const int64_t stride = weight ? values : a.N, at = weight ? v : v - values;
    float sum = 0.f;
    if (v < all) {
      int64_t s = SPLIT ? w : 0;
      const float* from = (weight ? a.slots : a.bias_slots) + (before + s) * stride + at;
      for (; s + 3 * kBy < mine; s += 4 * kBy, from += 4 * kBy * stride) {
        const float t0 = from[0], t1 = from[kBy * stride], t2 = from[2 * kBy * stride], t3 = from[3 * kBy * stride];
        sum += (t0 + t1) + (t2 + t3);
      }
      for (; s < mine; s += kBy, from += kBy * stride) sum += *from;
    }
    if constexpr (SPLIT) {
      __syncthreads();
      quarter[w][lane] = sum;
      __syncthreads();
      sum = (quarter[0][lane] + quarter[1][lane]) + (quarter[2][lane] + quarter[3][lane]);
    }
    if ((!SPLIT || w == 0) && v < all) (weight ? a.dweights : a.dbias)[e * stride + at] = sum;
  }
}

}  // namespace

hipError_t launch_product8(const Product8Args& a, int n_cu, hipStream_t s) {
  // no more parts of T rows than this, whatever the experts' shares
  const auto parts = [&](int64_t t) { return a.offsets ? std::min(a.m, (a.m + int64_t(a.E) * (t - 1)) / t) : (a.m + t - 1) / t; };
  // Few rows: where there are not 16 for every expert, or tiles of 128 x 128 would
  // leave seven CUs of eight without one (1,024 inputs and outputs, bfloat16: 100 rows,
  // 8 tiles, 5.5 us against 10.2; 512 rows, 32 tiles, 8.3 against 10.3; 4,096 of both,
  // 64 rows, 32 tiles, 16.2 against 25.0; 1,000 rows of 4,096 inputs, 64 tiles, 53 against 30).
  // The experts' own sizes are not known here: 4,096 rows at one of 256 experts, 1,024 inputs
  // and outputs, take 93 us (101 with even shares), one expert's own 4,096 rows 11.
  const bool few = a.m <= int64_t(16) * a.E || parts(128) * ((a.N + 127) / 128) <= n_cu / 8;
  if (few) {
    const int cols = (a.N + 15) / 16;
    const auto run = [&](auto f32, auto rf) {
      k_product_few<f32.value, rf.value><<<unsigned(parts(16 * rf.value) * cols), 256, 0, s>>>(a, cols);
    };
    const auto with = [&](auto f32) {
      if (a.m <= int64_t(16) * a.E) run(f32, std::integral_constant<int, 1>());
      else if (a.m <= int64_t(32) * a.E) run(f32, std::integral_constant<int, 2>());
      else run(f32, std::integral_constant<int, 4>());
    };
    if (a.bf16) with(std::false_type());
    else with(std::true_type());
  } else {
    // `each` work-groups a CU, as many as there is LDS for
    const auto run = [&](auto kernel, int64_t row_tile, int col_tile, int threads, int each) {
      const int64_t tiles = parts(row_tile) * ((a.N + col_tile - 1) / col_tile);
      kernel<<<unsigned((std::min(tiles, int64_t(n_cu) * each) + 7) / 8 * 8), threads, 0, s>>>(a);
    };
    // Tiles of 256 x 256 read half as much for each product as tiles of 128 x 128, and a
    // CU has one of them at a time or two of those.  A round of the small ones takes
    // about 0.6 of a round of the large ones, and the last round is seldom full; an
    // expert's last tile is half full on average.  Small against large, in bfloat16 and
    // float32: 65,536 rows, 8 experts, 1,024 inputs to 4,096 outputs, 33 rounds to 17,
    // 381 us against 306 and 693 against 591; 8,192 rows, 1,024 to 2,048, 3 to 2, 35.2
    // against 40.3 and 43.4 against 58.7; 4,096 x 4,096 x 4,096, 2 to 1, 75 against 69.
    const auto rounds = [&](int64_t t, int at_once) {
      const int64_t tiles = ((a.m + t - 1) / t + (a.offsets ? a.E / 2 : 0)) * ((a.N + t - 1) / t);
      return (tiles + at_once - 1) / at_once;
    };
    const bool large = rounds(256, n_cu) * 5 <= rounds(128, 2 * n_cu) * 3;
    // Results that are larger than the last cache, of 256 MB, go past it (65,536 x 4,096:
    // 306 us against 334 and 591 against 632; results that fit are read by what comes next).
    // Those of 128 x 128 tiles do not: most are narrow, and parts of lines cost more past the
    // cache (float32, 4,300,000 x 33: 1,353 us through it, 1,432 past it; 300,000 x 257: 160 and
    // 197; 128 bfloat16 outputs, whole lines: 2,200,000 rows 238 and 232, 1,200,000 of 128 inputs 108 and 80).
    const bool stream = a.m * a.N * (a.bf16 ? 2 : 4) > int64_t(1) << 28;
    const auto with = [&](auto f32) {
      constexpr bool kF32 = f32.value;
      if (!large) run(k_product<kF32, 4, 4, 2, 2>, 128, 128, 256, 2);
      else if (stream) run(k_product<kF32, 8, 4, 2, 4, true>, 256, 256, 512, 1);
      else run(k_product<kF32, 8, 4, 2, 4>, 256, 256, 512, 1);
    };
    if (a.bf16) with(std::false_type());
    else with(std::true_type());
  }
  return hipGetLastError();
}

namespace {
int64_t items(const Product8Args& a) { return a.m / a.slice + a.E; }
}  // namespace

// Tiles of 256 x 256 where they fit the matrices about as well as tiles of 128 x 128,
// and there is work for all CUs: they read and convert half as much for each product
// (small against large: 65,536 rows, 8 experts, 4,096 x 1,024, 816 us against 613; 30,000
// rows, 4 experts, 1,000 x 1,000, 193 against 99; 8,000 rows, 500 x 500, 23.3 against 26.4;
// 262,144 rows, 64 x 64, 35 against 46).
static bool large_tiles(const Product8Args& a, int n_cu) {
  const auto tiles = [&](int t) { return int64_t((a.N + t - 1) / t) * ((a.K + t - 1) / t); };
  return tiles(256) * 4 * 5 <= tiles(128) * 6 && (a.m / 256) * tiles(256) >= n_cu;
}

size_t product8_weights_plan(Product8Args* a, int n_cu) {
  const bool large = large_tiles(*a, n_cu);
  const int tile = large ? 256 : 128;
  const int64_t tiles = int64_t((a->N + tile - 1) / tile) * ((a->K + tile - 1) / tile);
  a->slice = a->m;
  // slices of rows where the experts' tiles do not fill the CUs, one work-group each
  // or, of the small ones, two: as many as fit at once, each expert's last one shorter
  // (30,001 rows, 6 experts, 321 x 385: 41, 36 and 40 us with one, two and three, 131
  // without slices; 16,384 rows, 2,048 x 2,048: 152 with one, 169 with two, 444 without).
  // The experts' own sizes are not known here: with slices they hardly matter (262,144 rows, 64
  // experts, 256 x 256: 73 to 75 us), without them the largest one's tiles end late (512 x 512:
  // 159 us with even shares, 237, 348 and 634 where the largest has 2, 3 and 6 times the mean)
  const int64_t fit = int64_t(n_cu) * (large ? 1 : 2) / tiles, most = a->offsets ? fit - a->E : fit;
  if (tiles * a->E < n_cu) a->slice = std::max<int64_t>(256, most > 0 ? (a->m + most - 1) / most : a->m);
  a->slice = std::max<int64_t>(1, (a->slice + 63) / 64 * 64);
  if (a->slice >= a->m) return 0;
  return size_t(items(*a)) * size_t(int64_t(a->N) * a->K + a->N) * sizeof(float);
}

void product8_workspace(Product8Args* a, unsigned char* ws) {
  a->slots = nullptr;
  a->bias_slots = nullptr;
  if (a->slice >= a->m) return;
  a->slots = reinterpret_cast<float*>(ws);
  a->bias_slots = a->slots + items(*a) * a->N * a->K;
}

hipError_t launch_product8_weights(const Product8Args& a, int n_cu, hipStream_t s) {
  const int64_t count = a.slots ? items(a) : a.E;
  const auto run = [&](auto kernel, int tile, int threads) {
    const int tiles_n = (a.N + tile - 1) / tile, tiles_k = (a.K + tile - 1) / tile;
    kernel<<<unsigned(count * tiles_n * tiles_k), threads, 0, s>>>(a, tiles_n, tiles_k);
  };
  if (large_tiles(a, n_cu)) run(k_product_weights<4, 8, 4, 2>, 256, 512);
  else run(k_product_weights<4, 2, 2, 4>, 128, 512);
  if (a.slots) {
    const int64_t values = int64_t(a.N) * a.K + a.N;
    const auto blocks = [&](int64_t each) {
      const int64_t most = std::max<int64_t>(1, int64_t(n_cu) * 8 / a.E);
      return dim3{unsigned(std::min((values + each - 1) / each, most)), unsigned(a.E), 1};
    };
    if (values * a.E < int64_t(n_cu) * 1024) k_add_slices<true><<<blocks(64), 256, 0, s>>>(a);
    else k_add_slices<false><<<blocks(256), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace mlip
