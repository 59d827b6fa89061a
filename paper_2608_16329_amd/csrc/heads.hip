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
// of one head, each wavefront 16 of them as the columns of its matrix products;
// z and u never leave registers, y only for the weights' gradients: a layer's
// result is, register by register, the second operand of the next layer's product
// (which sums over the inputs in the order in which the lane groups hold them).
//
// Products: a float32 is three bfloat16 limbs, exactly (24 bits in 8 + 8 + 8,
// each the rest rounded to nearest, so the second and third are up to 2^-8 and
// 2^-17 of the value and of either sign), and the product of two is the six limb
// products without those of a second and a third, 2^-24 of it at most, which
// 16x16x32 bfloat16 matrix instructions add up in float32.  (Limbs cut off would
// leave out 2^-22 each, of the product's sign.)  The instruction rounds to nearest
// where its addend is not the smaller part, and otherwise down, by up to one unit
// in the last place, 0.17 on average.  Six products take 0.43 of the time of the
// float32 matrix instructions (2,100 against 150 TFLOP/s in a loop of nothing
// else).  Inputs in bfloat16 are one limb, and theirs are three products (all
// gradients of 131,071 such rows of 192 values, two heads each, took 0.88 of the
// time with six).  A first kernel splits the heads' matrices, in the order in which
// lanes take them, for products with the matrix and with its transpose; the main
// kernel brings them to LDS one 64x64 block at a time, the next block on its way
// while one is used.
//
// The weights' gradients are products over rows: the limbs of g and y change
// places through LDS, read transposed, each wavefront owns some of the 16
// result tiles of every block and keeps their sums over all of the work-group's
// tiles of a head, which are written once and added up in order by a third
// kernel.
//
// An infinity has no limbs, nor has a value that rounds to one (2^128 (1 - 2^-9) and
// more): in a row it gives NaN, in that row and in the weights' gradients, as a
// NaN does.  (The bias sums are products with ones and zeros, so a NaN in one
// layer's g is in the dc of all layers.)
#include <algorithm>
#include <type_traits>

#include "learn.h"
#include "learn_math.h"

namespace mlip {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kR = 64;                 // hidden width
constexpr int kFragBytes = 1024;       // an operand of one limb: 8 values a lane
constexpr int kBlockBytes = 24 * kFragBytes;   // a 64x64 block: 4 result tiles x 2 steps of 32 inputs x 3 limbs
constexpr int kRowBytes = 2 * kR;      // a row of one limb of g or y in LDS
constexpr int kChunksHeld = 2;         // 64-input chunks whose gradient sums stay in registers

__device__ __forceinline__ f4 mfma(u4 a, u4 b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

// The sum of products of two numbers of three limbs, but for those of a second
// and a third.
__device__ __forceinline__ f4 products(const u4 a[3], const u4 (&b)[3], f4 c) {
  c = mfma(a[2], b[0], c);
  c = mfma(a[0], b[2], c);
  c = mfma(a[1], b[1], c);
  c = mfma(a[1], b[0], c);
  c = mfma(a[0], b[1], c);
  return mfma(a[0], b[0], c);
}
// The same where the second has one limb, a bfloat16, and the products are all there are.
__device__ __forceinline__ f4 products(const u4 a[3], const u4 (&b)[1], f4 c) {
  c = mfma(a[2], b[0], c);
  c = mfma(a[1], b[0], c);
  return mfma(a[0], b[0], c);
}

// Limb k of four values, two to a register.
__device__ __forceinline__ void split4(const f4 v, u2 limb[3]) {
  f2 r[2] = {{v[0], v[1]}, {v[2], v[3]}};
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector(r[i], bf2));
      limb[k][i] = u;
      r[i][0] -= __uint_as_float(u << 16);
      r[i][1] -= __uint_as_float(u & 0xffff0000u);
    }
}

// Four bfloat16 are one limb as they are.
__device__ __forceinline__ void split4(const u2 v, u2 limb[1]) { limb[0] = v; }

// 64 values of a column as a product's second operand: step s, limb k.
template <int N>
struct Limbs {
  u4 v[2][N];
  template <typename T>
  __device__ __forceinline__ void step(int s, const T a, const T b) {
    u2 lo[N], hi[N];
    split4(a, lo);
    split4(b, hi);
#pragma unroll
    for (int k = 0; k < N; ++k) v[s][k] = u4{lo[k][0], lo[k][1], hi[k][0], hi[k][1]};
  }
  template <typename T>
  __device__ __forceinline__ void of(const T in[4]) {
    step(0, in[0], in[1]);
    step(1, in[2], in[3]);
  }
};
// Four inputs of a row, and how many limbs they have.
template <bool BF>
using Input = std::conditional_t<BF, u2, f4>;
template <bool BF>
constexpr int kInputLimbs = BF ? 1 : 3;

// Which of a block's 64 inputs value j of lane group g is in step s.
__device__ __forceinline__ int input_of(int s, int g, int j) { return 32 * s + 16 * (j >> 2) + 4 * g + (j & 3); }

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
      const int tiles = e <= a.E ? int((uint32_t(hi - lo) + uint32_t(rows - 1)) / uint32_t(rows)) : 0;
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

// First tile of work-group b of `groups` that share `tiles`, groups <= tiles.
__device__ __forceinline__ int share(int64_t tiles, int64_t b, int groups) { return int(tiles * b / groups); }

__device__ __forceinline__ f4 vec4(const float* p) {
  return *reinterpret_cast<const F4*>(p);
}
// The same value, not known to be: what is computed from it is computed where
// it is used and not kept in registers around the loop over tiles.
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}
// 64 values in LDS as the lanes hold a column: 16 t + 4 g + i in v[t][i].
__device__ __forceinline__ void column(const float* base, f4 v[4]) {
  const float* p = base + here((threadIdx.x & 48) / 4);
#pragma unroll
  for (int t = 0; t < 4; ++t) v[t] = *reinterpret_cast<const f4*>(p + 16 * t);
}
// The kernel's arguments read again: held in scalar registers across the loop
// over tiles, they do not fit beside the rest, and come and go through vector
// registers (50 to 70 of the weight gradients' still do).
__device__ __forceinline__ const HeadsArgs& again() {
  typedef const __attribute__((address_space(4))) HeadsArgs* Args;
  Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const HeadsArgs*)p;
}
// A value that all lanes hold, for the scalar registers.
__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A split block of weights from memory to LDS, 1 KB at a time, without passing
// registers; landed() waits for the wavefront's part.
template <int NW>
__device__ __forceinline__ void stage(const unsigned char* src, unsigned char* lds) {
  const int w = uni(threadIdx.x >> 6);
  const uint32_t lane16 = here(16 * (threadIdx.x & 63));
#pragma unroll
  for (int k = 0; k < kBlockBytes / kFragBytes / NW; ++k) {
    const int at = kFragBytes * (w + NW * k);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + at + lane16),
                                     (__attribute__((address_space(3))) void*)(lds + at), 16, 0, 0);
  }
}
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Between two matrix instructions, vector instructions of what stands beside
// them: 16 cycles of one take four of the other.
template <int N>
__device__ __forceinline__ void mixed() {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
  }
}

// out += block in, one tile of 16 results after another, the next tile's
// operands loaded before this one's products; beside(t) is work that goes with
// the products of tile t, such as what becomes of the results of the tiles before.
template <int N, typename F>
__device__ __forceinline__ void product(const unsigned char* block, const Limbs<N>& in, f4 out[4], F beside) {
  const unsigned char* p = block + here(16 * (threadIdx.x & 63));
  u4 a[2][3];   // of step 0, step 1
  auto fetch = [&](int t, int s) {
#pragma unroll
    for (int k = 0; k < 3; ++k) a[s][k] = *reinterpret_cast<const u4*>(p + kFragBytes * (3 * (4 * s + t) + k));
  };
  fetch(0, 0);
  fetch(0, 1);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    __builtin_amdgcn_sched_barrier(0);
    f4 sum = products(a[0], in.v[0], out[t]);
    if (t < 3) fetch(t + 1, 0);
    out[t] = products(a[1], in.v[1], sum);
    if (t < 3) fetch(t + 1, 1);
    beside(t);
    mixed<N == 3 ? 12 : 6>();
  }
  __builtin_amdgcn_sched_barrier(0);
}
template <int N>
__device__ __forceinline__ void product(const unsigned char* block, const Limbs<N>& in, f4 out[4]) {
  product(block, in, out, [](int) {});
}

// The heads' matrices in limbs: block b of head e (64 inputs of A_0 each, then
// A_1 ..) for products with it and, after it, with its transpose.  Heads
// without rows are left out.  Latency of a load and a store around LDS: 5.5 us
// for 6 heads of 128 inputs and 4 layers.  (Splitting in the main kernel would do
// the same work once a work-group.)
__global__ __launch_bounds__(256) void k_split(HeadsArgs a) {
  __shared__ float m[kR][kR + 1];
  const int b = blockIdx.x, e = blockIdx.y, chunks = (a.D + 63) / 64;
  if (a.offsets[e] == a.offsets[e + 1]) return;
  const float* w = a.weights + e * a.values;
  const float* src = b < chunks ? w + 64 * b : w + (kR * a.D + kR + (b - chunks) * (kR * kR + kR));
  const int ld = b < chunks ? a.D : kR, cols = b < chunks ? a.D - 64 * b : kR;
  // (the loads first, then what is stored of them)
  float v[kR * kR / 256];
#pragma unroll
  for (int k = 0; k < kR * kR / 256; ++k) {
    const int r = (256 * k + threadIdx.x) / kR, c = threadIdx.x % kR;
    v[k] = src[r * ld + (c < cols ? c : 0)];
  }
#pragma unroll
  for (int k = 0; k < kR * kR / 256; ++k) {
    const int r = (256 * k + threadIdx.x) / kR, c = threadIdx.x % kR;
    m[r][c] = c < cols ? v[k] : 0.f;
  }
  __syncthreads();
  unsigned char* dst = a.split + (e * int64_t(chunks + a.H - 1) + b) * a.split_block;
  const int turns = int(a.split_block / kBlockBytes);
  for (int at = threadIdx.x; at < turns * 512; at += 256) {
    const int turn = at >> 9, n = (at >> 6) & 7, lane = at & 63, g = lane >> 4, c = lane & 15;
    f4 v[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = 16 * (n & 3) + c, in = input_of(n >> 2, g, j);
      v[j >> 2][j & 3] = turn ? m[in][r] : m[r][in];
    }
    u2 lo[3], hi[3];
    split4(v[0], lo);
    split4(v[1], hi);
#pragma unroll
    for (int k = 0; k < 3; ++k)
      *reinterpret_cast<u4*>(dst + turn * kBlockBytes + kFragBytes * (3 * n + k) + 16 * lane) =
          u4{lo[k][0], lo[k][1], hi[k][0], hi[k][1]};
  }
}

// Sums over the 16 columns of a wavefront's rows: lane (g, c) gets that of value
// 16 (c / 4) + 4 g + c % 4.  Each step adds two lanes' halves of what is left.
template <int CTRL, int N>
__device__ __forceinline__ void fold_step(float* v, bool upper) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float send = upper ? v[k] : v[k + N], keep = upper ? v[k + N] : v[k];
    v[k] = keep + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(send), CTRL, 0xf, 0xf, true));
  }
}
__device__ __forceinline__ float fold16(const f4 in[4]) {
  const int c = threadIdx.x & 15;
  float v[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = in[k >> 2][k & 3];
  fold_step<0x140, 8>(v, c & 8);   // row mirror: lane 15 - c
  fold_step<0x141, 4>(v, c & 4);   // half row mirror
  fold_step<0x4e, 2>(v, c & 2);    // lane c ^ 2
  fold_step<0xb1, 1>(v, c & 1);    // lane c ^ 1
  return v[0];
}
__device__ __forceinline__ int fold_value() {
  const int lane = threadIdx.x & 63, c = lane & 15;
  return 16 * (c >> 2) + 4 * (lane >> 4) + (c & 3);
}

// The row of a lane's column in a tile.
struct Row {
  int32_t entry;   // -1: none
  int32_t i;
  float gate, up;  // gate and denergy
  const char* x;   // its inputs; of row 0 where there is none
  char* dx;        // where their gradient goes
};
__device__ __forceinline__ int32_t entry_of(const HeadsArgs& a, int64_t at, int64_t end) {
  return at < end ? a.order[at] : -1;
}
template <bool BF>
__device__ __forceinline__ Row row_of(const HeadsArgs& a, int32_t ent) {
  Row r{-1, 0, 0.f, 0.f, static_cast<const char*>(a.x), nullptr};
  if (ent >= 0 && ent < a.m) {
    r.entry = ent;
    r.i = a.K == 1 ? ent : ent / a.K;
    r.gate = a.gates ? a.gates[ent] : 1.f;
    r.up = a.denergy ? a.denergy[r.i] : 1.f;
    r.x += (BF ? 2 : 4) * (int64_t(r.i) * a.stride);
    r.dx = a.K == 1 ? static_cast<char*>(a.dx) + (BF ? 2 : 4) * (int64_t(r.i) * a.D)
                    : reinterpret_cast<char*>(a.entry_dx) + 4 * (int64_t(ent) * a.D);
  }
  return r;
}
// Inputs 64 ch .. 64 ch + 63 of the lane's row on their way: 16 T + 4 g + i in
// in[T][i].  Every lane loads four values that are there; ready() takes out those
// beyond the row's end and those of lanes without a row when they are used, so
// that loading does not wait.
template <bool BF>
__device__ __forceinline__ void load_x(const Row& r, int D, int ch, Input<BF> in[4]) {
  const int g = (threadIdx.x >> 4) & 3, last = max(D, 4) - 4;   // rows of fewer than four are copied to four (k_pad)
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    const int at = min(64 * ch + 16 * T + 4 * g, last);
    if constexpr (BF) in[T] = __builtin_bit_cast(u2, *reinterpret_cast<const H4*>(reinterpret_cast<const uint16_t*>(r.x) + at));
    else in[T] = vec4(reinterpret_cast<const float*>(r.x) + at);
  }
}
// (where fewer than four are left, what was loaded are the row's last four values)
__device__ __forceinline__ int inputs_left(const Row& r, int D, int ch, int T) {
  return r.entry >= 0 ? D - (64 * ch + 16 * T + 4 * int((threadIdx.x >> 4) & 3)) : 0;
}
__device__ __forceinline__ f4 ready(const Row& r, int D, int ch, int T, f4 f) {
  const int left = inputs_left(r, D, ch, T);
  if (D & 3) {
    const int shift = D < 4 ? 0 : (left < 4 ? 4 - left : 0);
    if (shift & 1) f = f4{f[1], f[2], f[3], 0.f};
    if (shift & 2) f = f4{f[2], f[3], 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = i < left ? f[i] : 0.f;
    return f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = left > 0 ? f[i] : 0.f;
  return f;
}
__device__ __forceinline__ u2 ready(const Row& r, int D, int ch, int T, u2 h) {
  const int left = inputs_left(r, D, ch, T);
  if (D & 3) {
    // (four values at D < 4: those beyond the row's end are zero)
    const int shift = D < 4 || left >= 4 || left <= 0 ? 0 : 4 - left;
    h = __builtin_bit_cast(u2, __builtin_bit_cast(uint64_t, h) >> (16 * shift));
  }
  return u2{left > 0 ? h[0] : 0u, left > 0 ? h[1] : 0u};
}

// d[T][i] to the gradient of the lane's row at inputs 64 ch + 16 T + 4 g + i.
__device__ __forceinline__ void store_dx(const Row& r, bool bf16, int D, int ch, const f4 d[4]) {
  const int g = (threadIdx.x >> 4) & 3;
  if (r.entry < 0) return;
#pragma unroll
  for (int T = 0; T < 4; ++T) {
    const int c = 64 * ch + 16 * T + 4 * g;
    if (c >= D) continue;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = d[T][i];
    store4(r.dx, bf16, c, D - c, v);
  }
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
  Row r = row_of<BF>(a, entry_of(a, at, end));
  r.gate = r.up = 0.f;   // the gate of such an entry may be anything
  store_value(a, r, 0.f);
  if (a.dx) {
    const f4 zero[4] = {};
    for (int ch = 0; 64 * ch < a.D; ++ch) store_dx(r, BF && a.K == 1, a.D, ch, zero);
  }
}

__device__ __forceinline__ const float* layer(const float* w, int D, int t) {
  return w + (kR * D + kR + (t - 1) * (kR * kR + kR));
}

// A head's vectors to LDS: c_0 .. c_{H-1}, a, c.  (Loaded where they are used they
// would wait for whatever loads and stores are under way.)
constexpr int vectors(int H) { return (H + 1) * kR + 4; }
__device__ __forceinline__ void load_vectors(const float* wt, int D, int H, float* to) {
  for (int at = threadIdx.x; at <= (H + 1) * kR; at += blockDim.x) {
    const int l = at / kR;
    const float* from = l == 0 ? wt + kR * D : (l < H ? layer(wt, D, l) + kR * kR : layer(wt, D, H));
    to[at] = from[l < H ? at % kR : at - H * kR];
  }
}

// Energies alone.  Two work-groups a CU (52 KB of LDS each), each with a share of
// the tiles, so that heads of all sizes fill the chip.  262,144 rows of 128 inputs,
// 4 layers: 92 us, 117 TFLOP/s of float32 products as the formulas count them.
// Bound by issue: limbs and activations beside the products.
template <int NW, bool BF>
__global__ __launch_bounds__(NW * 64) void k_energy(HeadsArgs a) {
  constexpr int kRows = 16 * NW;
  __shared__ int32_t s_first[kMaxExperts + 2], s_entry[kMaxExperts + 2];
  __shared__ __attribute__((aligned(16))) unsigned char s_w[2 * kBlockBytes];
  __shared__ __attribute__((aligned(16))) float s_vec[vectors(kMaxHeadLayers)];
  tile_table(a, kRows, s_first, s_entry);
  const int lane = threadIdx.x & 63, w = uni(threadIdx.x >> 6);
  const int tiles = uni(s_first[a.E + 1]), groups = min(a.blocks, tiles);
  if (int(blockIdx.x) >= groups) return;
  const int t_end = share(tiles, blockIdx.x + 1, groups);
  const int chunks = (a.D + 63) / 64, blocks = chunks + a.H - 1;
  int e = 0;
  for (int tile = share(tiles, blockIdx.x, groups); tile < t_end;) {
    while (tile >= uni(s_first[e + 1])) ++e;
    const int stop = min(t_end, uni(s_first[e + 1]));
    const int64_t begin = uni(s_entry[e]), end = uni(s_entry[e + 1]), t0 = uni(s_first[e]);
    if (e == a.E) {
      for (; tile < stop; ++tile) empty_tile<NW, BF>(a, begin + (tile - t0) * kRows, end);
      break;
    }
    const float* wt = a.weights + e * a.values;
    const unsigned char* split = a.split + e * int64_t(blocks) * a.split_block;
    int cur = 0;
    __syncthreads();
    load_vectors(wt, a.D, a.H, s_vec);
    stage<NW>(split, s_w);
    Row r = row_of<BF>(a, entry_of(a, begin + (tile - t0) * kRows + 16 * w + (lane & 15), end));
    Input<BF> in[4];
    load_x<BF>(r, a.D, 0, in);
    landed();
    __syncthreads();
    // block b is in use: the next one, or the next tile's first, on its way
    auto ahead = [&](int b) {
      if (b + 1 < blocks) stage<NW>(split + (b + 1) * a.split_block, s_w + (cur ^ 1) * kBlockBytes);
      else if (tile + 1 < stop) stage<NW>(split, s_w + (cur ^ 1) * kBlockBytes);
    };
    auto turn = [&]() {
      landed();
      __syncthreads();
      cur ^= 1;
    };
    for (; tile < stop; ++tile) {
      Limbs<kInputLimbs<BF>> x0;
      Limbs<3> x;
      f4 z[4], y[4] = {};
      // y += silu(z) of one tile, and the next product's operand from two
      auto activate = [&](int t, Limbs<3>& next) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[t][i] += z[t][i] * sigmoid(z[t][i]);
        if (t & 1) next.step(t >> 1, y[t - 1], y[t]);
      };
      column(s_vec, z);
      // the next tile's rows, in time for their inputs
      const int32_t entry = tile + 1 < stop ? entry_of(a, begin + (tile + 1 - t0) * kRows + 16 * w + (lane & 15), end) : -1;
      for (int ch = 0; ch < chunks; ++ch) {
        ahead(ch);
#pragma unroll
        for (int T = 0; T < 4; ++T) in[T] = ready(r, a.D, ch, T, in[T]);
        x0.of(in);
        if (ch + 1 < chunks) load_x<BF>(r, a.D, ch + 1, in);
        product(s_w + cur * kBlockBytes, x0, z);
        turn();
      }
      Row next = r;
      if (tile + 1 < stop) {
        next = row_of<BF>(a, entry);
        load_x<BF>(next, a.D, 0, in);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) activate(t, x);
      for (int l = 1; l < a.H; ++l) {
        ahead(chunks + l - 1);
        column(s_vec + l * kR, z);
        Limbs<3> after;
        product(s_w + cur * kBlockBytes, x, z, [&](int t) {
          if (t > 0) activate(t - 1, after);
        });
        activate(3, after);
        x = after;
        turn();
      }
      float v = 0.f;
      f4 o[4];
      column(s_vec + a.H * kR, o);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) v += o[t][i] * y[t][i];
      v += __shfl_xor(v, 16, 64);
      v += __shfl_xor(v, 32, 64);
      store_value(a, r, v + s_vec[(a.H + 1) * kR]);
      r = next;
    }
  }
}

// Values of a slot: result tiles in the order of the registers (256 a tile, 16
// tiles a 64x64 block: the chunks of A_0, then A_1 ..), then dc_0 .. dc_{H-1},
// da, dc.
__host__ __device__ __forceinline__ int64_t slot_block(int D, int b) { return int64_t(b) * kR * kR; }
__host__ __device__ __forceinline__ int64_t slot_values(int D, int H) {
  return int64_t((D + 63) / 64 + H - 1) * kR * kR + int64_t(H + 1) * kR + 64;
}

// The gradient of A_l needs y_{l-1} again (y_l - silu(z_l) would lose of it what
// silu(z_l) is larger by).  That of the last layer waits in LDS from the forward
// pass on; y_0 .. y_{kAgain - 1} are added up again from z; those between
// are left in memory, layers_kept() of them: registers for 16 values a layer there
// are none.  All gradients, 4 layers, 1,048,576 rows: 1,023 us so, 1,037 with y_0
// and y_1 in memory too; 8 layers, 131,072 rows: 354 us, with all of them added up
// again 388.
constexpr int kAgain = 2;
constexpr int layers_kept(int H) { return H > kAgain + 2 ? H - kAgain - 2 : 0; }

// Energies, gradients in the descriptors and (TRAIN) in the weights.
// 128 inputs, 4 layers, in a series of calls: without weight gradients 262,144 rows
// 163 us (132 TFLOP/s of float32 products as the formulas count them), with them
// 1,048,576 rows 997 us (130; the float32 matrix instructions reach 150 in a loop
// of nothing else); the first calls after a pause take 14 to 17% longer.  With them
// the matrix pipes are busy for 34% of the time, vector and matrix instructions are
// issued for 48%, a wavefront waits for 36% of its own, at barriers and between
// steps, with two wavefronts a SIMD, as many as the registers of z and the sums
// allow; without them 37, 52 and 31%.  A row alone takes 15 us: one wavefront's 5,600
// instructions, one after another.
template <int H, int NW, bool TRAIN, bool BF>
__global__ __launch_bounds__(NW * 64, TRAIN && NW == 4 ? 1 : 2) void k_gradient(HeadsArgs args) {
  // (what the loop over tiles uses all the time; the rest is read again where it
  // is used, away from LDS: scalar loads wait for what LDS has to do)
  const HeadsArgs& a = again();
  constexpr int kRows = 16 * NW;
  constexpr int kOwn = 16 / NW;          // result tiles of a wavefront in a 64x64 block
  constexpr int kPlane = kRows * kRowBytes;   // a limb of the tile's rows
  extern __shared__ __attribute__((aligned(16))) unsigned char s_mem[];
  unsigned char* const s_w = s_mem;                    // two blocks of weights
  unsigned char* const s_g = s_mem + 2 * kBlockBytes;  // limbs of g, then of y
  unsigned char* const s_y = s_g + 3 * kPlane;
  __shared__ int32_t s_first[kMaxExperts + 2], s_entry[kMaxExperts + 2];
  __shared__ __attribute__((aligned(16))) float s_vec[vectors(H)];
  tile_table(a, kRows, s_first, s_entry);
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int w = uni(tid >> 6);
  const int tiles = uni(s_first[a.E + 1]), groups = min(a.blocks, tiles);
  if (int(blockIdx.x) >= groups) return;
  const int t_begin = share(tiles, blockIdx.x, groups), t_end = share(tiles, blockIdx.x + 1, groups);
  const int D = a.D, chunks = (D + 63) / 64, blocks = chunks + H - 1;
  const bool one = a.K == 1, with_dx = a.dx != nullptr;
  // the wavefront's tiles of a block: outputs 16 ta .., inputs 16 (tb + k) ..
  const int ta = NW == 8 ? w >> 1 : w, tb = NW == 8 ? 2 * (w & 1) : 0;

  // values 16 t .. of y_l of the wavefront's rows in memory
  constexpr int kKept = layers_kept(H);
  float* const kept_here = a.kept + (int64_t(blockIdx.x) * kKept * NW + w) * (16 * kR);
  auto kept = [&](int l, int t) {
    float* from = kept_here + (l - kAgain) * (NW * 16 * kR);
    return reinterpret_cast<f4*>(reinterpret_cast<char*>(from) + uint32_t(kFragBytes * t + here(16 * lane)));
  };

  f4 sum_h[H > 1 ? H - 1 : 1][kOwn], sum_0[kChunksHeld][kOwn];
  f4 sum_b;                                   // of dc_t, column t: the sums of g_t are products with ones there
  float sum_a = 0.f, sum_c = 0.f;             // of da, value fold_value(); of dc

  // A limb's row is 128 bytes: four groups of 16 values, turned by the row's
  // bits 1 and 2, and the halves of a group by bit 3, so that the 32 lanes that
  // LDS serves at once meet all banks: writing (by column, four values a lane)
  // and reading.
  const int put_at = (16 * w + c) * kRowBytes + 8 * (g ^ (c >> 3 << 1)) + ((c << 4) & 96);
  const int get_at = (4 * g + (c >> 2)) * kRowBytes + 8 * ((c & 3) ^ (g & 2)) + (((4 * g + (c >> 2)) << 4) & 96);
  auto put = [&](unsigned char* to, int t, const auto& limb) {
    const int at = here(put_at) ^ (32 * t);
#pragma unroll
    for (int k = 0; k < int(sizeof(limb) / sizeof(u2)); ++k) *reinterpret_cast<u2*>(to + k * kPlane + at) = limb[k];
  };
  // group t of 16 values of rows 32 s .. 32 s + 31 as an operand: lane (g, c)
  // gets value c at rows 4 g + j and 16 + 4 g + j, j < 4
  auto get = [&](const unsigned char* from, int t, int s, auto& limb) {
    const int at = here(get_at) ^ (32 * t);
#pragma unroll
    for (int k = 0; k < int(sizeof(limb) / sizeof(u4)); ++k) {
      u2 half[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        half[h] = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s4*)(from + k * kPlane + (32 * s + 16 * h) * kRowBytes + at)));
      limb[k] = u4{half[0][0], half[0][1], half[1][0], half[1][1]};
    }
  };
  // sums of g y^T (y of `limbs` limbs) over the tile's rows into the wavefront's tiles, and (bias >=
  // 0) of g into column `bias` of sum_b, for which two wavefronts with the same
  // outputs take turns; beside(s) is work that goes with the products of the
  // s-th quarter of the rows (half, with four wavefronts: then it is called for
  // two quarters)
  auto outer = [&](auto limbs, f4 acc[kOwn], int bias, auto beside) {
#pragma unroll
    for (int s = 0; s < NW / 2; ++s) {
      u4 ga[3], yb[kOwn][limbs.value];
      __builtin_amdgcn_sched_barrier(0);
      get(s_g, ta, s, ga);
#pragma unroll
      for (int k = 0; k < kOwn; ++k) get(s_y, tb + k, s, yb[k]);
#pragma unroll
      for (int q = 0; q < 8 / NW; ++q) beside(8 / NW * s + q);
#pragma unroll
      for (int k = 0; k < kOwn; ++k) acc[k] = products(ga, yb[k], acc[k]);
      if (bias >= 0 && (NW == 4 || (w & 1) == (s & 1))) {
        const uint32_t one = c == bias ? 0x3f803f80u : 0u;
        const u4 ones = {one, one, one, one};
#pragma unroll
        for (int k = 2; k >= 0; --k) sum_b = mfma(ga[k], ones, sum_b);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto nothing = [](int) {};
  constexpr std::integral_constant<int, 3> limbs_y{};
  constexpr std::integral_constant<int, kInputLimbs<BF>> limbs_x{};
  auto put_limbs = [&](unsigned char* to, const Limbs<3>& l) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      u2 limb[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) limb[k] = u2{l.v[t >> 1][k][2 * (t & 1)], l.v[t >> 1][k][2 * (t & 1) + 1]};
      put(to, t, limb);
    }
  };
  auto put_value = [&](unsigned char* to, int t, const auto v) {
    u2 limb[sizeof(v) == sizeof(f4) ? 3 : 1];
    split4(v, limb);
    put(to, t, limb);
  };
  auto clear = [&]() {
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
#pragma unroll
      for (int t = 0; t < (H > 1 ? H - 1 : 1); ++t) sum_h[t][k] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < kChunksHeld; ++t) sum_0[t][k] = f4{0.f, 0.f, 0.f, 0.f};
    }
    sum_b = f4{0.f, 0.f, 0.f, 0.f};
    sum_a = 0.f;
    sum_c = 0.f;
  };
  auto place = [&](float* slot, int b, int k) {
    return reinterpret_cast<f4*>(reinterpret_cast<char*>(slot + slot_block(D, b) + (4 * ta + tb + k) * 256) + uint32_t(16 * lane));
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
    float* tail = slot + slot_block(D, blocks);
    // dc_t over the two wavefronts that have its value, da and dc over all
    float* const s_sum = reinterpret_cast<float*>(s_g);
    float* const s_all = s_sum + 2 * H * kR;
    __syncthreads();
    if (c < H)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_sum[((NW == 8 ? w & 1 : 0) * H + c) * kR + 16 * ta + 4 * g + i] = sum_b[i];
    s_all[w * 2 * kR + fold_value()] = sum_a;
    float v = sum_c;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) v += __shfl_xor(v, o, 64);
    if (lane == 0) s_all[w * 2 * kR + kR] = v;
    __syncthreads();
    for (int at = tid; at < H * kR; at += NW * 64) tail[at] = NW == 8 ? s_sum[at] + s_sum[H * kR + at] : s_sum[at];
    if (tid <= kR) {
      float v = 0.f;
#pragma unroll
      for (int u = 0; u < NW; ++u) v += s_all[u * 2 * kR + tid];
      tail[H * kR + tid] = v;
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
    const unsigned char* split = a.split + e * int64_t(blocks) * (2 * kBlockBytes);
    if (TRAIN) clear();
    // blocks of weights in LDS: one in use, the next on its way into the other
    int cur = 0;
    auto ahead = [&](int b, bool transposed) {
      stage<NW>(split + b * (2 * kBlockBytes) + (transposed ? kBlockBytes : 0), s_w + (cur ^ 1) * kBlockBytes);
    };
    auto turn = [&]() {
      landed();
      __syncthreads();
      cur ^= 1;
    };
    __syncthreads();
    load_vectors(a.weights + e * a.values, a.D, H, s_vec);
    cur = 1;
    ahead(0, false);
    Row r = row_of<BF>(a, entry_of(a, begin + (tile - t0) * kRows + 16 * w + c, end));
    Input<BF> in[4];
    load_x<BF>(r, D, 0, in);
    turn();
    for (bool first = true; tile < stop; ++tile, first = false) {
      // forward: z_t of every layer and the last y stay
      Limbs<kInputLimbs<BF>> x0;
      Limbs<3> x;
      f4 y[4] = {}, z[H][4];
      column(s_vec, z[0]);
      // the next tile's rows, in time for their inputs
      const bool follows = tile + 1 < stop;
      const int32_t entry = follows ? entry_of(again(), begin + (tile + 1 - t0) * kRows + 16 * w + c, end) : -1;
      for (int ch = 0; ch < chunks; ++ch) {
        const bool more = ch + 1 < chunks;
        if (more) ahead(ch + 1, false);
        else if (H > 1) ahead(chunks, false);
        else ahead(0, true);
#pragma unroll
        for (int T = 0; T < 4; ++T) in[T] = ready(r, D, ch, T, in[T]);
        x0.of(in);
        if (more) load_x<BF>(r, D, ch + 1, in);
        product(s_w + cur * kBlockBytes, x0, z[0]);
        turn();
      }
      // y += silu(z_l) of one tile, and the next product's operand from two
      auto activate = [&](int l, int t, Limbs<3>& next) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[t][i] += z[l][t][i] * sigmoid(z[l][t][i]);
        if (TRAIN && l >= kAgain && l < kAgain + kKept) *kept(l, t) = y[t];
        if (l + 1 < H && (t & 1)) next.step(t >> 1, y[t - 1], y[t]);
      };
#pragma unroll
      for (int t = 0; t < 4; ++t) activate(0, t, x);
#pragma unroll
      for (int l = 1; l < H; ++l) {
        column(s_vec + l * kR, z[l]);
        ahead(chunks + (l + 1 < H ? l : l - 1), l + 1 == H);
        if (TRAIN && l + 1 == H) put_limbs(s_y, x);   // for the first product over rows
        Limbs<3> after;
        product(s_w + cur * kBlockBytes, x, z[l], [&](int t) {
          if (t > 0) activate(l, t - 1, after);
        });
        activate(l, 3, after);
        if (l + 1 < H) x = after;
        turn();
      }
      f4 u[4];
      const float d = r.entry >= 0 ? r.up * r.gate : 0.f;
      {
        float v = 0.f;
        column(s_vec + H * kR, u);
        f4 dy[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v += u[t][i] * y[t][i];
            u[t][i] *= d;
            dy[t][i] = d * y[t][i];
          }
        if (TRAIN) {
          sum_c += d;
          sum_a += fold16(dy);
        }
        v += __shfl_xor(v, 16, 64);
        v += __shfl_xor(v, 32, 64);
        store_value(again(), r, v + s_vec[(H + 1) * kR]);
      }
      // (so that the compiler does not keep the forward pass's sigmoids)
      auto again_z = [](float v) {
        asm volatile("" : "+v"(v));
        return v;
      };
      auto silu_again = [&](float v) {
        v = again_z(v);
        return v * sigmoid(v);
      };
      // g_l = u silu'(z_l) of one tile, its limbs from two (the sigmoid again: for
      // silu' of every layer there are no registers either)
      f4 gz[4];
      auto back = [&](int l, int t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float zl = again_z(z[l][t][i]), s = sigmoid(zl);
          gz[t][i] = u[t][i] * (s * (1.f + zl * (1.f - s)));
        }
        if (t & 1) x.step(t >> 1, gz[t - 1], gz[t]);
      };
#pragma unroll
      for (int t = 0; t < 4; ++t) back(H - 1, t);
#pragma unroll
      for (int l = H - 1; l > 0; --l) {
        ahead(l > 1 ? chunks + l - 2 : 0, true);
        if (TRAIN && l == 1) load_x<BF>(r, D, 0, in);   // for the chunks below
        if (TRAIN) put_limbs(s_g, x);
        product(s_w + cur * kBlockBytes, x, u, [&](int t) {
          if (TRAIN && l <= kAgain && l + 1 < H) {
            y[t] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < l; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i) y[t][i] += silu_again(z[b][t][i]);
          }
          if (TRAIN && l + 1 < H) put_value(s_y, t, y[t]);
        });
        if (TRAIN) {
          if (l - 2 >= kAgain)   // for the next layer down
#pragma unroll
            for (int t = 0; t < 4; ++t) y[t] = *kept(l - 2, t);
          __syncthreads();
          outer(limbs_y, sum_h[l - 1], l, [&](int t) { back(l - 1, t); });
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t) back(l - 1, t);
        }
        turn();
      }
      if (TRAIN) {
        put_limbs(s_g, x);
        if (H == 1) load_x<BF>(r, D, 0, in);
      }
      const Row now = r;
      r = row_of<BF>(again(), entry);
      for (int ch = 0; ch < chunks; ++ch) {
        const bool more = ch + 1 < chunks;
        if (more) ahead(ch + 1, true);
        else if (follows) ahead(0, false);
        if (TRAIN) {
#pragma unroll
          for (int t = 0; t < 4; ++t) put_value(s_y, t, ready(now, D, ch, t, in[t]));
        }
        // the next chunk, or the next tile's first
        if (TRAIN && more) load_x<BF>(now, D, ch + 1, in);
        else if (!more && follows) load_x<BF>(r, D, 0, in);
        if (with_dx) {
          f4 dx[4] = {};
          product(s_w + cur * kBlockBytes, x, dx);
          store_dx(now, BF && one, D, ch, dx);
        }
        if (TRAIN) {
          __syncthreads();
          if (ch == 0) outer(limbs_x, sum_0[0], 0, nothing);
          else if (ch == 1) outer(limbs_x, sum_0[1], -1, nothing);
          else {
            float* slot = a.slots + (int64_t(blockIdx.x) + e) * a.slot;
            f4 acc[kOwn];
#pragma unroll
            for (int j = 0; j < kOwn; ++j) acc[j] = first ? f4{0.f, 0.f, 0.f, 0.f} : *place(slot, ch, j);
            outer(limbs_x, acc, -1, nothing);
#pragma unroll
            for (int j = 0; j < kOwn; ++j) *place(slot, ch, j) = acc[j];
          }
        }
        turn();
      }
    }
    if (TRAIN) flush(e);
  }
}

// A head's weight gradients: the slots of the work-groups that had tiles of
// it, added up in order (atomics would add them in any).  9 us for 262 slots of
// 21,000 values, 22 MB from the caches.
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
    const int groups = min(a.blocks, tiles);
    auto group_of = [&](int tile) {
      int b = int(int64_t(tile) * groups / tiles);
      while (b + 1 < groups && share(tiles, b + 1, groups) <= tile) ++b;
      while (share(tiles, b, groups) > tile) --b;
      return b;
    };
    const int b0 = group_of(lo), b1 = group_of(hi - 1);
    const float* slot = a.slots + (int64_t(b0) + e) * a.slot + at;
#pragma unroll 8
    for (int b = b0; b <= b1; ++b, slot += a.slot) v += *slot;
  }
  a.dweights[e * a.values + dst] = v;
}

// Rows of fewer than four values to rows of four, so that every load of four
// values is one that may be made.  Bound by memory: 1,048,576 rows of 3, 9 us.
template <typename T>
__global__ __launch_bounds__(256) void k_pad(const T* x, int64_t n, int64_t stride, int D, T* to) {
  const int c = threadIdx.x & 3;
  for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < 4 * n; at += int64_t(gridDim.x) * 256)
    to[at] = c < D ? x[(at >> 2) * stride + c] : T(0);
}

// Rows with several entries: their energies and gradients added up in order,
// in float32 (one rounding to the rows' type, at the end).  Bound by memory:
// 131,071 rows of 192, two entries each, 39 us (252 MB, 6.5 TB/s, part of it from
// the last-level cache).
__global__ __launch_bounds__(256) void k_sum_entries(HeadsArgs a) {
  const int64_t first = int64_t(blockIdx.x) * 256 + threadIdx.x, step = int64_t(gridDim.x) * 256;
  if (a.energy) {
    for (int64_t at = first; at < a.n; at += step) {
      float v = 0.f;
      for (int s = 0; s < a.K; ++s) v += a.entry_energy[at * a.K + s];
      a.energy[at] = v;
    }
  }
  if (!a.dx) return;
  const int groups = (a.D + 3) / 4;
  for (int64_t at = first; at < a.n * groups; at += step) {
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

// What the work-groups keep of a tile's layers.
size_t kept_values(const HeadsArgs& a) { return size_t(a.blocks) * size_t(layers_kept(a.H)) * size_t(16 * a.waves * kR); }

// Work-groups of 256 for that many values, fewer than 2^32 threads a launch.
unsigned blocks_for(int64_t values) { return unsigned(std::min<int64_t>((values + 255) / 256, 1 << 22)); }

template <int H, int NW, bool TRAIN, bool BF>
hipError_t gradient_of(const HeadsArgs& a, hipStream_t s) {
  constexpr size_t lds = 2 * kBlockBytes + (TRAIN ? 2 * 3 * 16 * NW * kRowBytes : 0);
  const hipError_t ready = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_gradient<H, NW, TRAIN, BF>),
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
  if (ready != hipSuccess) return ready;
  k_gradient<H, NW, TRAIN, BF><<<a.blocks, NW * 64, lds, s>>>(a);
  return hipGetLastError();
}

template <bool TRAIN, bool BF>
hipError_t gradient_by_layers(const HeadsArgs& a, hipStream_t s) {
  if (TRAIN && a.waves == 8) {
    switch (a.H) {
      case 1: return gradient_of<1, 8, true, BF>(a, s);
      case 2: return gradient_of<2, 8, true, BF>(a, s);
      case 3: return gradient_of<3, 8, true, BF>(a, s);
      default: return gradient_of<4, 8, true, BF>(a, s);
    }
  }
  switch (a.H) {
    case 1: return gradient_of<1, 4, TRAIN, BF>(a, s);
    case 2: return gradient_of<2, 4, TRAIN, BF>(a, s);
    case 3: return gradient_of<3, 4, TRAIN, BF>(a, s);
    case 4: return gradient_of<4, 4, TRAIN, BF>(a, s);
    case 5: return gradient_of<5, 4, TRAIN, BF>(a, s);
    case 6: return gradient_of<6, 4, TRAIN, BF>(a, s);
    case 7: return gradient_of<7, 4, TRAIN, BF>(a, s);
    default: return gradient_of<8, 4, TRAIN, BF>(a, s);
  }
}

}  // namespace

// Wavefronts of a work-group, 16 rows each.  For weight gradients eight, two a
// SIMD; four where each CU has at most one tile of 64 rows, which is sooner done
// than one of 128 (6 heads of 128 inputs and 3 layers, all gradients, with the
// grouping: 5,000 rows 42 us with four, 48 with eight, 10,000 rows 48 and 52;
// 20,000 rows 64 and 54, 100,000 rows 146 and 124), or where z of more than four
// layers and the sums of their gradients need all of a SIMD's registers.  Without
// weight gradients four, and two work-groups a CU that need not wait for each
// other.
size_t heads_plan(HeadsArgs* a, int n_cu) {
  a->waves = a->dweights && a->H <= 4 && a->m / 64 + a->E > n_cu ? 8 : 4;
  const int rows = 16 * a->waves;
  // at most one more tile than full ones for each head and for entries without
  const int64_t tiles = a->m / rows + a->E + 1;
  a->blocks = int(std::min<int64_t>(tiles, a->dweights ? n_cu : 2 * n_cu));
  a->slot = slot_values(a->D, a->H);
  a->split_block = (a->dx || a->dweights ? 2 : 1) * kBlockBytes;
  size_t b = size_t(a->E) * size_t((a->D + 63) / 64 + a->H - 1) * size_t(a->split_block);
  if (a->dweights) b += (size_t(a->blocks + a->E) * size_t(a->slot) + kept_values(*a)) * sizeof(float);
  if (a->K > 1 && a->energy) b += size_t(a->m) * sizeof(float);
  if (a->K > 1 && a->dx) b += size_t(a->m) * size_t(a->D) * sizeof(float);
  if (a->D < 4) b += size_t(a->n) * 4 * sizeof(float);
  return b;
}

void heads_workspace(HeadsArgs* a, unsigned char* ws) {
  a->split = ws;
  ws += size_t(a->E) * size_t((a->D + 63) / 64 + a->H - 1) * size_t(a->split_block);
  float* at = reinterpret_cast<float*>(ws);
  if (a->dweights) {
    a->slots = at, at += int64_t(a->blocks + a->E) * a->slot;
    a->kept = at, at += kept_values(*a);
  }
  if (a->K > 1 && a->dx) a->entry_dx = at, at += a->m * a->D;
  if (a->K > 1 && a->energy) a->entry_energy = at, at += a->m;
  if (a->D < 4) a->padded = at;
}

hipError_t launch_heads(const HeadsArgs& given, hipStream_t s) {
  hipError_t e = hipSuccess;
  HeadsArgs a = given;
  if (a.m > 0) {
    if (a.D < 4) {
      const unsigned blocks = blocks_for(4 * a.n);
      if (a.bf16) k_pad<<<blocks, 256, 0, s>>>(static_cast<const uint16_t*>(a.x), a.n, a.stride, a.D, static_cast<uint16_t*>(a.padded));
      else k_pad<<<blocks, 256, 0, s>>>(static_cast<const float*>(a.x), a.n, a.stride, a.D, static_cast<float*>(a.padded));
      if ((e = hipGetLastError()) != hipSuccess) return e;
      a.x = a.padded;
      a.stride = 4;
    }
    k_split<<<dim3((a.D + 63) / 64 + a.H - 1, a.E), 256, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (!a.dx && !a.dweights) {
      if (a.bf16) k_energy<4, true><<<a.blocks, 256, 0, s>>>(a);
      else k_energy<4, false><<<a.blocks, 256, 0, s>>>(a);
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
    if (a.waves == 8) k_sum_slots<8><<<g, 256, 0, s>>>(a);
    else k_sum_slots<4><<<g, 256, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.K > 1 && a.m > 0 && (a.energy || a.dx)) {
    const int64_t work = std::max<int64_t>(a.n, a.dx ? a.n * ((a.D + 3) / 4) : 0);
    k_sum_entries<<<blocks_for(work), 256, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace mlip
