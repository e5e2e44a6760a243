// Attention of a prompt's rows over the paged cache (oda_prompt_plan,
// oda_prompt_attn): causal behind the history that is there, of a native window,
// or without a mask over states of another length.
//
//   o = sum_j softmax_j(scale q k_j) v_j,   j in [lo, hi) of the row
//   causal: hi = place + 1, lo = max(0, hi - window) (window 0: 0); else [0, n)
//
// The G query heads of a KV head share its K/V, so a request's (token, head)
// pairs of one KV head are its columns f = token * G + head, and a tile is up to
// 256 of them.  A tile's work is its columns against the blocks that any of them
// attends; an item is a tile, or one range of blocks of it where tiles alone
// would leave CUs idle.  Scores are formed as S^T = K Q^T and outputs as
// O^T = V^T P^T, both by v_mfma_f32_32x32x16_bf16: a lane then holds 16 scores of
// one column (and what they are weighed against), which after rounding are the B
// operand of the second product without passing through LDS; a column's factor
// rescales the lane's own accumulators.
//
// The plan (tiles, ranges, their order) is made on the device from rows and
// lengths by one workgroup, once for all layers of a step.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>
#include <cmath>
#include <type_traits>

#include "oda.h"
#include "oda_device.h"
#include "oda_internal.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 16;            // positions per KV block
constexpr int kPair = 2 * kBlock;     // positions per score tile
constexpr int kCols = 32;             // columns of an MFMA tile, of a wavefront
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kTile = kWaves * kCols; // columns of an item
constexpr int kStageBlocks = 8;       // blocks staged together: one of K and one of V per wavefront
constexpr int kMaxBatch = 2048;
constexpr int kCus = 256;
constexpr int kPlanThreads = 1024;
constexpr uint32_t kMagic = 0x0da9f3u;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Plan buffer, int32 words: the header, the items, the merges.
struct PlanHeader {
  uint32_t magic;
  int32_t batch, rows, group, heads, max_blocks, max_len;   // what the plan was made for
  int32_t n_items, n_merges;
  int32_t causal, window;
  int32_t reserved[5];
};
struct Item {
  int32_t request;                   // whose block table
  int32_t row0;                      // the request's first row
  int32_t col0, ncols;               // columns token * G + head, counted from row0
  int32_t blk_lo, blk_hi;
  int32_t place0;                    // of the request's first row (causal)
  int32_t n;                         // positions that are there; -1: the rows become NaN
  int32_t part;                      // first partial column; -1: the item is its tile's only one
  int32_t reserved[3];
};
struct Merge {
  int32_t row0, col0, ncols;
  int32_t part, splits;              // column c of split s at part + s * ncols + c
  int32_t reserved[3];
};

__host__ __device__ constexpr int items_at() { return (int)(sizeof(PlanHeader) / 4); }
__host__ __device__ constexpr int merges_at(int max_items) { return items_at() + max_items * (int)(sizeof(Item) / 4); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// ---------------------------------------------------------------------------
// the plan
// ---------------------------------------------------------------------------

struct PlanArgs {
  const int32_t* row_start;
  const int32_t* seq_lens;
  int32_t* plan;
  int32_t B, R, G, Hkv, MB, max_len, causal, window;
  int32_t extra_items, max_items, max_merges;
};

// Cost of an item in blocks of 16 positions at the time in which one CU's share of
// HBM delivers them: up to that many columns a block's products and softmax take no
// longer.
constexpr float kColsFree = 96.f;
constexpr float kItemCost = 24.f;     // start-up, the join, the partial's share of the merge
constexpr float kLeastCost = 16.f;    // shortest range
constexpr int kClasses = 256;         // cost classes, eight to a factor of two

struct PlanRequest {
  int32_t row0, rows, n, tile;        // tile: the request's first
};

__device__ __forceinline__ int class_of(float cost) {
  return min(max((int)ceilf(8.f * __log2f(fmaxf(cost, 1.f))), 0), kClasses - 1);
}
// At or above every cost of the class (with a margin for the logarithm's rounding).
__device__ __forceinline__ float class_cost(int c) { return 1.001f * __builtin_amdgcn_exp2f((float)c * 0.125f); }
// Ranges of a tile of `blocks` blocks where an item may hold `cap` of them, even.
__device__ __forceinline__ int range_blocks(int blocks, int splits) { return ((blocks + splits - 1) / splits + 1) & ~1; }

__device__ __forceinline__ int2 block_scan(int2 x, int2* s_wave, int2& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int2 v = x;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int a = __shfl_up(v.x, s), b = __shfl_up(v.y, s);
    if (lane >= s) {
      v.x += a;
      v.y += b;
    }
  }
  __syncthreads();       // the sums of the call before have been read
  if (lane == 63) s_wave[wave] = v;
  __syncthreads();
  int2 base = make_int2(0, 0);
  total = make_int2(0, 0);
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const int2 t = s_wave[w];
    if (w < wave) {
      base.x += t.x;
      base.y += t.y;
    }
    total.x += t.x;
    total.y += t.y;
  }
  return make_int2(base.x + v.x - x.x, base.y + v.y - x.y);
}

// One workgroup.  Bound by latency: rows and lengths are asked for together, then
// everything goes through LDS.
__global__ __launch_bounds__(kPlanThreads) void prompt_plan_kernel(PlanArgs a) {
  __shared__ PlanRequest s_req[kMaxBatch];
  __shared__ int2 s_wave[kPlanThreads / 64];
  __shared__ int s_max[kPlanThreads / 64];
  __shared__ int s_class[kClasses], s_place[kClasses];
  __shared__ int s_count[kPlanThreads / 64][64];
  __shared__ float s_cost[kPlanThreads / 64][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  Item* items = reinterpret_cast<Item*>(a.plan + items_at());
  Merge* merges = reinterpret_cast<Merge*>(a.plan + merges_at(a.max_items));
  if (tid < kClasses) s_class[tid] = s_place[tid] = 0;

  // requests: row starts kept in [0, R] and ascending whatever the array holds
  int n_tiles = 0, carry = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int start = 0, end = 0, n = 0;
    if (b < a.B) {
      start = min(max(a.row_start[b], 0), a.R);
      end = min(max(a.row_start[b + 1], 0), a.R);
      n = a.seq_lens[b];
    }
    // running largest of all starts up to b, and of the ends up to b
    int top = max(start, carry);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int y = __shfl_up(top, s);
      if (lane >= s) top = max(top, y);
    }
    __syncthreads();
    if (lane == 63) s_max[wave] = top;
    __syncthreads();
    for (int w = 0; w < wave; ++w) top = max(top, s_max[w]);
    const int row0 = top, rows = max(end - row0, 0);
    for (int w = 0; w < kPlanThreads / 64; ++w) carry = max(carry, s_max[w]);
    const int tiles = (int)(((int64_t)rows * a.G + kTile - 1) / kTile);
    int2 total;
    const int2 at = block_scan(make_int2(tiles, 0), s_wave, total);
    if (b < a.B) {
      const bool bad = n < 0 || n > a.max_len || (a.causal && n < rows);
      s_req[b] = PlanRequest{row0, rows, bad ? -1 : n, n_tiles + at.x};
    }
    n_tiles += total.x;
  }
  __syncthreads();

  // a tile: its request, columns and blocks
  struct Tile {
    int b, col0, ncols, lo, hi;
  };
  auto tile_at = [&](int t) {
    int lo = 0, hi = a.B;            // the last request whose first tile is at or before t (one with rows)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_req[mid].tile <= t) lo = mid;
      else hi = mid;
    }
    const PlanRequest q = s_req[lo];
    Tile r;
    r.b = lo;
    r.col0 = (t - q.tile) * kTile;
    r.ncols = (int)min((int64_t)kTile, (int64_t)q.rows * a.G - r.col0);
    r.lo = r.hi = 0;
    if (q.n < 0) return r;
    const int first = q.n - q.rows + r.col0 / a.G, last = q.n - q.rows + (r.col0 + r.ncols - 1) / a.G;
    r.hi = (a.causal ? last + kBlock : q.n + kBlock - 1) / kBlock;
    r.lo = a.causal && a.window > 0 ? max(0, first - a.window + 1) / kBlock : 0;
    return r;
  };
  auto cost_of = [&](const Tile& t) { return (float)(t.hi - t.lo) * fmaxf(1.f, (float)((t.ncols + kCols - 1) / kCols * kCols) / kColsFree); };

  int most = 0;
  for (int t = tid; t < n_tiles; t += kPlanThreads) {
    const int c = class_of(cost_of(tile_at(t)));
    atomicAdd(&s_class[c], 1);
    most = max(most, c);
  }
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) most = max(most, __shfl_xor(most, s));
  __syncthreads();
  if (lane == 0) s_max[wave] = most;
  __syncthreads();
  for (int w = 0; w < kPlanThreads / 64; ++w) most = max(most, s_max[w]);

  // what an item may cost: every lane tries one value; the last splits nothing
  const float top = fmaxf(class_cost(most), kLeastCost);
  const float cap = lane == 63 ? top : kLeastCost * __builtin_amdgcn_exp2f(__log2f(top / kLeastCost) * (float)lane * (1.f / 63.f));
  int n = 0;
  float sum = 0.f;
  for (int c = wave; c < kClasses; c += kPlanThreads / 64) {
    const int count = s_class[c];
    if (count == 0) continue;
    const float cost = class_cost(c);
    const int splits = lane == 63 ? 1 : max(1, (int)ceilf(cost / cap));
    n += count * splits;
    sum += (float)count * (cost + kItemCost * (float)splits);
  }
  s_count[wave][lane] = n;
  s_cost[wave][lane] = sum;
  __syncthreads();
  n = 0;
  sum = 0.f;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    n += s_count[w][lane];
    sum += s_cost[w][lane];
  }
  float est = (float)a.Hkv * n <= (float)kCus ? cap + kItemCost : (float)a.Hkv * sum * (1.f / (float)kCus) + 0.5f * cap;
  if (n - n_tiles > a.extra_items) est = INFINITY;
  float best = est;
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) best = fminf(best, __shfl_xor(best, s));
  const uint64_t who = __ballot(est == best);
  const int pick = who ? 63 - __builtin_clzll(who) : 63;
  const float cap_best = __shfl(cap, pick);
  auto splits_of = [&](const Tile& t) {
    const int blocks = t.hi - t.lo;
    if (pick == 63 || blocks <= 0) return 1;
    const int splits = min(blocks, max(1, (int)ceilf(cost_of(t) / cap_best)));
    const int len = range_blocks(blocks, splits);
    return (blocks + len - 1) / len;
  };

  // items listed by their cost, the largest class first (within one in any order)
  __syncthreads();
  if (tid < kClasses) s_class[tid] = 0;
  __syncthreads();
  for (int t = tid; t < n_tiles; t += kPlanThreads) {
    const Tile r = tile_at(t);
    const int splits = splits_of(r);
    atomicAdd(&s_class[class_of(cost_of(r) / (float)splits)], splits);
  }
  __syncthreads();
  if (tid < 64) {
    // places from the largest class down, kClasses / 64 a lane
    constexpr int kPer = kClasses / 64;
    const int c0 = kClasses - 1 - kPer * lane;
    int own = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) own += s_class[c0 - i];
    int v = own;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int y = __shfl_up(v, s);
      if (lane >= s) v += y;
    }
    v -= own;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      s_place[c0 - i] = v;
      v += s_class[c0 - i];
    }
  }
  __syncthreads();
  int n_merges = 0, n_part = 0;
  for (int t0 = 0; t0 < n_tiles; t0 += kPlanThreads) {
    const int t = t0 + tid;
    Tile r{};
    int splits = 0;
    if (t < n_tiles) {
      r = tile_at(t);
      splits = splits_of(r);
    }
    const bool merged = splits > 1;
    int2 total;
    const int2 at = block_scan(make_int2(merged ? 1 : 0, merged ? splits * r.ncols : 0), s_wave, total);
    const int part = n_part + at.y, merge = n_merges + at.x;
    if (splits > 0) {
      const PlanRequest q = s_req[r.b];
      const int len = range_blocks(r.hi - r.lo, splits);
      const int place = atomicAdd(&s_place[class_of(cost_of(r) / (float)splits)], splits);
      for (int i = 0; i < splits; ++i) {
        Item it{};
        it.request = r.b;
        it.row0 = q.row0;
        it.col0 = r.col0;
        it.ncols = r.ncols;
        it.blk_lo = splits > 1 ? r.lo + i * len : r.lo;
        it.blk_hi = splits > 1 ? min(r.hi, it.blk_lo + len) : r.hi;
        it.place0 = q.n - q.rows;
        it.n = q.n;
        it.part = merged ? part + i * r.ncols : -1;
        if (place + i < a.max_items) items[place + i] = it;
      }
      if (merged && merge < a.max_merges) merges[merge] = Merge{q.row0, r.col0, r.ncols, part, splits, {}};
    }
    n_merges += total.x;
    n_part += total.y;
  }
  __syncthreads();
  if (tid == 0) {
    PlanHeader h{};
    h.magic = kMagic;
    h.batch = a.B;
    h.rows = a.R;
    h.group = a.G;
    h.heads = a.Hkv;
    h.max_blocks = a.MB;
    h.max_len = a.max_len;
    h.causal = a.causal;
    h.window = a.window;
    h.n_items = min(s_place[0], a.max_items);      // the end of the last class
    h.n_merges = min(n_merges, a.max_merges);
    *reinterpret_cast<PlanHeader*>(a.plan) = h;
  }
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------

struct PromptArgs {
  const uint16_t* q;         // [R][Hq][D]
  const uint16_t* k_cache;
  const uint16_t* v_cache;
  const int32_t* block_table;
  const int32_t* plan;
  void* out;                 // [R][Hq][D] fp32 or bf16
  float* lse;                // [R][Hq] or NULL
  float* part_o;             // [Hkv][part_cols][D]
  float* part_ml;            // [Hkv][part_cols][2]  (reference in exponents of 2, sum)
  int64_t num_blocks;
  int64_t part_cols;
  int32_t B, R, Hq, Hkv, G, MB, max_len;
  int32_t max_items, max_merges;
  float scale_log2;
};

__device__ __forceinline__ bool plan_fits(const PromptArgs& a, const PlanHeader& h) {
  return (h.magic == kMagic) & (h.batch == a.B) & (h.rows == a.R) & (h.group == a.G) & (h.heads == a.Hkv) &
         (h.max_blocks == a.MB) & (h.max_len == a.max_len);
}

__device__ __forceinline__ bf16x8 load16(const uint16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ float bf16_to_float(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }

// Two floats to bf16, and what the rounding leaves of them.
__device__ __forceinline__ uint32_t round_pair(float x, float y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
}

// The larger of the two lanes that share a column (l and l ^ 32).
__device__ __forceinline__ float column_max(float x) {
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Parts of a weight in the second product.  An output rounded to bf16 takes one: a
// weight's rounding (2^-9, of random sign) adds about as much as the output's own.
// An fp32 output takes three, which hold all 24 bits, as decode attention does.
template <typename Out>
constexpr int kPartsOf = std::is_same<Out, float>::value ? 3 : 1;

// A wavefront's columns (one per lane pair): o[n][4 i + j] is dimension 32 n + 8 i +
// 4 h + j of column lane % 32, h = lane / 32; c the reference of its weights in
// exponents of 2 (-infinity: none yet), l this lane's part of their sum; attended
// positions [lo, hi).
template <int D>
struct Columns {
  f32x16 o[D / 32];
  float c, l;
  int lo, hi;
};

// Scores of a pair of blocks (this lane: positions 8 h .. 8 h + 7 of either block)
// into the online softmax; the weights come back as bf16 parts, [0..3] of the first
// block and [4..7] of the second.
//
// Weights are taken against a reference kLag above the largest score at which it
// was set and below no later one: at most 1, and their sum 2^-kLag or more.  The
// largest score is looked for, and sums are rescaled, only where a lane's weights add
// up to more than 1 or there is no reference yet (its weights come out infinite or
// NaN).  The reference is kept as the exponent that is taken off, so that all weights
// of a column are against the same number, to the bit, whatever its size.
constexpr float kLag = 6.f;
template <int D, int P>
__device__ __forceinline__ void softmax_pair(float scale_log2, const f32x16& s, Columns<D>& w, bf16x8 (&part)[P][2]) {
  float p[16], sum;
  auto weights = [&](float ref) {
    float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale_log2, -ref));
      t[i & 3] += p[i];
    }
    sum = (t[0] + t[1]) + (t[2] + t[3]);
  };
  weights(w.c);
  if (__any(!(sum <= 1.f))) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    const float c_new = fmaxf(w.c, column_max(mx) * scale_log2 + kLag);
    const float ref = c_new == -INFINITY ? 0.f : c_new;
    const float alpha = __builtin_amdgcn_exp2f(w.c - ref);
    w.c = c_new;
    w.l *= alpha;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) w.o[n][i] *= alpha;
    weights(ref);
  }
  w.l += sum;
#pragma unroll
  for (int q = 0; q < P; ++q) {
    u32x4 r[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t x = round_pair(p[2 * e], p[2 * e + 1]);
      r[e >> 2][e & 3] = x;
      if (q + 1 < P) {
        p[2 * e] -= __uint_as_float(x << 16);
        p[2 * e + 1] -= __uint_as_float(x & 0xffff0000u);
      }
    }
    part[q][0] = __builtin_bit_cast(bf16x8, r[0]);
    part[q][1] = __builtin_bit_cast(bf16x8, r[1]);
  }
}

// Scores of positions that a column does not attend.  at: the first block's position
// of this lane's scores; bad: bit i = block i has no memory (its scores are NaN).
__device__ __forceinline__ void mask_scores(int at, int lo, int hi, int bad, f32x16& s) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int pos = at + (i & 7) + (i >> 3) * kBlock;
    const float x = (bad >> (i >> 3)) & 1 ? __builtin_nanf("") : s[i];
    s[i] = pos >= lo && pos < hi ? x : -INFINITY;
  }
}

// The first `room` of eight values, zeros behind them: slots that nobody attends may
// hold anything.
__device__ __forceinline__ bf16x8 first_values(int room, bf16x8 v) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] &= (room > 2 * i ? 0x0000FFFFu : 0u) | (room > 2 * i + 1 ? 0xFFFF0000u : 0u);
  return __builtin_bit_cast(bf16x8, w);
}

// The largest exponent fields' bits over values (0x7f80 or more: one is not finite).
__device__ __forceinline__ u16x2 most_of(u16x2 m, bf16x8 v) {
  const u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
  return m;
}
__device__ __forceinline__ bf16x8 finite_values(bf16x8 v) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
    if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0x0000ffffu;
  }
  return __builtin_bit_cast(bf16x8, w);
}

// One pair of blocks against a wavefront's columns.  k(kk), v(n, blk): this lane's
// operands; raw(d, pos): a value of the pair, for the masked form's rare case.
//
// K operand rows: row 16 b + r of the tile is position r of block b with bits 2 and 3
// of r exchanged, so that lane half h gets positions 8 h .. 8 h + 7 of both blocks,
// which is how it holds V's operand.
//
// Masked: a position that one column attends and another does not may hold a value
// that is not finite, which 0 * V would bring to both.  Such values are taken out of
// the product and added where they are attended (a weight is positive: it does not
// change an infinity or NaN).
template <int D, int P, bool kMasked, typename KOp, typename VOp, typename Raw>
__device__ __forceinline__ void attend_pair(float scale_log2, const bf16x8 (&qf)[D / 16], Columns<D>& w, int pos, int bad,
                                            KOp k, VOp v, Raw raw) {
  f32x16 s = {};
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k(kk), qf[kk], s, 0, 0, 0);
  const int h = (threadIdx.x & 63) >> 5;
  if (kMasked) mask_scores(pos + 8 * h, w.lo, w.hi, bad, s);
  bf16x8 part[P][2];
  softmax_pair<D, P>(scale_log2, s, w, part);
  bool finite = true;
  if (kMasked) {
    u16x2 m = {0, 0};
#pragma unroll
    for (int n = 0; n < D / 32; ++n) m = most_of(most_of(m, v(n, 0)), v(n, 1));
    finite = !__any(m[0] >= 0x7f80 || m[1] >= 0x7f80);
  }
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      bf16x8 x = v(n, b);
      if (kMasked && !finite) x = finite_values(x);
#pragma unroll
      for (int q = 0; q < P; ++q) w.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, part[q][b], w.o[n], 0, 0, 0);
    }
  if (kMasked && !finite) {
#pragma unroll 1
    for (int i = 0; i < kPair; ++i) {
      const bool in = pos + i >= w.lo && pos + i < w.hi;
#pragma unroll
      for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint16_t x = raw(32 * n + 8 * (r >> 2) + 4 * h + (r & 3), i);
          if (in && (x & 0x7f80u) == 0x7f80u) w.o[n][r] += bf16_to_float(x);
        }
    }
  }
}

// A wavefront's columns: queries as B operands, attended positions.
template <int D>
__device__ __forceinline__ void load_columns(const PromptArgs& a, const PlanHeader& h, const Item& it, int g, int first,
                                             Columns<D>& w, bf16x8 (&qf)[D / 16]) {
  const int lane = threadIdx.x & 63;
  const int col = first + (lane & 31);
  const bool in = col < it.ncols;
  const int at = it.col0 + (in ? col : 0);
  const int token = at / a.G, head = at - token * a.G;
  const uint16_t* q = a.q + ((int64_t)(it.row0 + token) * a.Hq + g * a.G + head) * D + 8 * (lane >> 5);
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) qf[kk] = load16(q + 16 * kk);
  w.hi = h.causal ? it.place0 + token + 1 : it.n;
  w.lo = h.causal && h.window > 0 ? max(0, w.hi - h.window) : 0;
  w.c = -INFINITY;
  w.l = 0.f;
#pragma unroll
  for (int n = 0; n < D / 32; ++n) w.o[n] = f32x16{};
}

// LDS: two stages of K and V blocks, or the wavefronts' O where ranges are joined.
// V's 16-byte groups (eight positions of a dimension) are kept by their half of the
// block, the halves 16 groups apart modulo the banks.
__host__ __device__ constexpr int v_half(int D) { return D * 8 + 64; }                 // elements
__host__ __device__ constexpr int k_elems(int D) { return kBlock * D; }
__host__ __device__ constexpr int v_elems(int D) { return 2 * v_half(D); }
__host__ __device__ constexpr int stage_elems(int D) { return kStageBlocks * (k_elems(D) + v_elems(D)); }
__host__ __device__ constexpr int o_stride(int D) { return D + 4; }                    // floats
__host__ __device__ constexpr int join_bytes(int D) { return kWaves * kCols * o_stride(D) * 4; }
__host__ __device__ constexpr int data_bytes(int D) {
  return 2 * stage_elems(D) * 2 > join_bytes(D) ? 2 * stage_elems(D) * 2 : join_bytes(D);
}
__host__ __device__ constexpr int lds_bytes(int D) { return data_bytes(D) + 2 * kWaves * kCols * 4; }
static_assert(lds_bytes(128) <= 160 * 1024, "an item fits LDS");
static_assert(kStageBlocks == kWaves, "a wavefront stages one block of K and one of V");

__device__ __forceinline__ void store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
__device__ __forceinline__ void store4(uint16_t* p, float4 x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(round_pair(x.x, x.y), round_pair(x.z, x.w));
}
__device__ __forceinline__ float lse_of(float c, float l) { return l == 0.f ? -INFINITY : (c + __log2f(l)) * kLn2; }
__device__ __forceinline__ float inverse_of(float l) { return l == 0.f ? 0.f : 1.f / l; }

// Columns to the partials, or, normalised, to the outputs.  put(col, f): f(d) gives
// four dimensions from d on.
template <int D, typename Out>
struct Target {
  Out* out;
  float* lse;
  float* part_o;
  float* part_ml;
};
template <int D, typename Out>
__device__ __forceinline__ Target<D, Out> target_of(const PromptArgs& a, const Item& it, int g, int col) {
  Target<D, Out> t{};
  if (it.part >= 0) {
    const int64_t at = (int64_t)g * a.part_cols + it.part + col;
    t.part_o = a.part_o + at * D;
    t.part_ml = a.part_ml + at * 2;
  } else {
    const int f = it.col0 + col, token = f / a.G;
    const int64_t row = (int64_t)(it.row0 + token) * a.Hq + g * a.G + (f - token * a.G);
    t.out = static_cast<Out*>(a.out) + row * D;
    t.lse = a.lse ? a.lse + row : nullptr;
  }
  return t;
}

// Joins the position ranges (wavefront = range * WC + column tile) and writes.
template <int D, typename Out>
__device__ __forceinline__ void join(const PromptArgs& a, const Item& it, int g, int wc_shift, Columns<D>& w, char* smem) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int WC = 1 << wc_shift, WP = kWaves >> wc_shift;
  float* sm_o = reinterpret_cast<float*>(smem);                      // [waves][32][D + 4]
  float* sm_c = reinterpret_cast<float*>(smem + data_bytes(D));      // [waves][32]
  float* sm_l = sm_c + kWaves * kCols;
  const int h = lane >> 5, c = lane & 31;
  if (h == 0) {
    sm_c[wave * kCols + c] = w.c;
    sm_l[wave * kCols + c] = w.l;
  }
  float* dst = sm_o + (wave * kCols + c) * o_stride(D) + 4 * h;
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4*>(dst + 32 * n + 8 * i) =
          make_float4(w.o[n][4 * i], w.o[n][4 * i + 1], w.o[n][4 * i + 2], w.o[n][4 * i + 3]);
  __syncthreads();
  for (int e = threadIdx.x; e < WC * kCols * (D / 4); e += kThreads) {
    const int d = e % (D / 4) * 4, col = e / (D / 4);
    if (col >= it.ncols) break;
    float top = -INFINITY;
    for (int p = 0; p < WP; ++p) top = fmaxf(top, sm_c[p * WC * kCols + col]);
    const float ref = top == -INFINITY ? 0.f : top;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
    for (int p = 0; p < WP; ++p) {
      const int at = p * WC * kCols + col;
      const float s = __builtin_amdgcn_exp2f(sm_c[at] - ref);
      const float4 x = *reinterpret_cast<const float4*>(sm_o + at * o_stride(D) + d);
      acc.x += s * x.x;
      acc.y += s * x.y;
      acc.z += s * x.z;
      acc.w += s * x.w;
      l += s * sm_l[at];
    }
    const Target<D, Out> t = target_of<D, Out>(a, it, g, col);
    if (it.part >= 0) {
      store4(t.part_o + d, acc);
      if (d == 0) *reinterpret_cast<float2*>(t.part_ml) = make_float2(ref, l);
    } else {
      const float inv = inverse_of(l);
      store4(t.out + d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
      if (d == 0 && t.lse) *t.lse = lse_of(ref, l);
    }
  }
}

// Columns straight from the registers, where a wavefront saw all of the item's blocks.
template <int D, typename Out>
__device__ __forceinline__ void write_columns(const PromptArgs& a, const Item& it, int g, int first, const Columns<D>& w) {
  const int lane = threadIdx.x & 63, h = lane >> 5, col = first + (lane & 31);
  if (col >= it.ncols) return;
  const Target<D, Out> t = target_of<D, Out>(a, it, g, col);
  const float ref = w.c == -INFINITY ? 0.f : w.c;
  const float inv = it.part >= 0 ? 1.f : inverse_of(w.l);
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 32 * n + 8 * i + 4 * h;
      const float4 x = make_float4(w.o[n][4 * i] * inv, w.o[n][4 * i + 1] * inv, w.o[n][4 * i + 2] * inv,
                                   w.o[n][4 * i + 3] * inv);
      if (it.part >= 0) store4(t.part_o + d, x);
      else store4(t.out + d, x);
    }
  if (h != 0) return;
  if (it.part >= 0) *reinterpret_cast<float2*>(t.part_ml) = make_float2(ref, w.l);
  else if (t.lse) *t.lse = lse_of(ref, w.l);
}

// One column tile: the wavefronts take contiguous ranges of pairs, K and V go
// straight to registers.
template <int D, typename Out>
__device__ __forceinline__ void run_narrow(const PromptArgs& a, const PlanHeader& head, const Item& it, int g, char* smem) {
  constexpr int P = kPartsOf<Out>;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int h = lane >> 5, m = lane & 31;
  const int pairs = (it.blk_hi - it.blk_lo + 1) >> 1;
  const int per = (pairs + kWaves - 1) / kWaves;
  const int lo = min(it.blk_hi, it.blk_lo + 2 * per * wave);
  const int hi = min(it.blk_hi, lo + 2 * per);
  const int32_t* table = a.block_table + (int64_t)it.request * a.MB;
  int entry = lo + lane < hi ? table[lo + lane] : 0;
  Columns<D> w;
  bf16x8 qf[D / 16];
  load_columns<D>(a, head, it, g, 0, w, qf);
  const int64_t blk_stride = (int64_t)a.Hkv * k_elems(D);
  const int pos16 = (m & 3) | ((m & 4) << 1) | ((m & 8) >> 1);
  const uint16_t* kbase = a.k_cache + (int64_t)g * k_elems(D) + (h * kBlock + pos16) * 8;
  const uint16_t* vbase = a.v_cache + (int64_t)g * k_elems(D) + m * kBlock + 8 * h;
  // positions that every column attends
  int all_lo = m < it.ncols ? w.lo : 0, all_hi = m < it.ncols ? w.hi : INT_MAX;
#pragma unroll
  for (int s = 16; s >= 1; s >>= 1) {
    all_lo = max(all_lo, __shfl_xor(all_lo, s));
    all_hi = min(all_hi, __shfl_xor(all_hi, s));
  }
  all_lo = uniform(all_lo);
  all_hi = uniform(all_hi);
  int tbl = 0;
  for (int v = lo; v < hi; v += 2) {
    const int i0 = (v - lo) & 63;
    if (i0 == 0) {
      if (v != lo) entry = v + lane < hi ? table[v + lane] : 0;
      tbl = entry >= 0 && entry < a.num_blocks ? entry : -1;
    }
    // (past an odd end the first block again, masked: no column attends it)
    const bool has1 = v + 1 < hi;
    const int e0 = __builtin_amdgcn_readlane(tbl, i0);
    const int e1 = has1 ? __builtin_amdgcn_readlane(tbl, i0 + 1) : e0;
    const int bad = (e0 < 0 ? 1 : 0) | (e1 < 0 ? 2 : 0);
    const int64_t b0 = (int64_t)max(e0, 0) * blk_stride, b1 = (int64_t)max(e1, 0) * blk_stride;
    const int64_t kb = m < kBlock ? b0 : b1;
    bf16x8 kr[D / 16], vr[D / 32][2];
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) kr[kk] = load16(kbase + kb + kk * 2 * kBlock * 8);
#pragma unroll
    for (int n = 0; n < D / 32; ++n) {
      vr[n][0] = load16(vbase + b0 + n * 32 * kBlock);
      vr[n][1] = load16(vbase + b1 + n * 32 * kBlock);
    }
    const int pos = v * kBlock;
    auto raw = [&](int d, int i) {
      const uint16_t* src = a.v_cache + (int64_t)g * k_elems(D) + (i < kBlock ? b0 : b1);
      return src[d * kBlock + (i & (kBlock - 1))];
    };
    auto k = [&](int kk) { return kr[kk]; };
    auto vv = [&](int n, int b) { return vr[n][b]; };
    if (has1 && bad == 0 && pos >= all_lo && pos + kPair <= all_hi) {
      attend_pair<D, P, false>(a.scale_log2, qf, w, pos, 0, k, vv, raw);
    } else {
#pragma unroll
      for (int n = 0; n < D / 32; ++n)     // slots behind the history may hold anything
#pragma unroll
        for (int b = 0; b < 2; ++b) vr[n][b] = first_values(it.n - pos - kBlock * b - 8 * h, vr[n][b]);
      const int hi_all = w.hi;
      w.hi = min(w.hi, hi * kBlock);       // the block beyond an odd end is another wavefront's
      attend_pair<D, P, true>(a.scale_log2, qf, w, pos, bad, k, vv, raw);
      w.hi = hi_all;
    }
  }
  w.l += __shfl_xor(w.l, 32);
  join<D, Out>(a, it, g, 0, w, smem);
}

// More column tiles: K and V are staged through LDS, eight blocks a stage (wavefront
// i brings block i while the stage before it is used).  Up to 64 and 128 columns the
// wavefronts are four and two position ranges, which share a stage's pairs
// alternately; more: every wavefront goes through all pairs with its 32 columns.
template <int D, typename Out>
__device__ __forceinline__ void run_wide(const PromptArgs& a, const PlanHeader& head, const Item& it, int g, int wc_shift,
                                         char* smem) {
  constexpr int P = kPartsOf<Out>;
  constexpr int kLoads = k_elems(D) / 512;           // 16-byte loads of a block per lane
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int h = lane >> 5, m = lane & 31;
  const int WP = kWaves >> wc_shift;
  const int wc = wave & ((1 << wc_shift) - 1), wp = wave >> wc_shift;
  const int blocks = it.blk_hi - it.blk_lo;
  const int stages = (blocks + kStageBlocks - 1) / kStageBlocks;
  const int32_t* table = a.block_table + (int64_t)it.request * a.MB + it.blk_lo;
  int entry = lane < blocks ? table[lane] : 0;       // 64 blocks, eight stages
  Columns<D> w;
  bf16x8 qf[D / 16];
  load_columns<D>(a, head, it, g, wc * kCols, w, qf);
  // positions that any, and that every, column of the wavefront attends
  const bool in = wc * kCols + m < it.ncols;
  int any_lo = in ? w.lo : INT_MAX, any_hi = in ? w.hi : 0, all_lo = in ? w.lo : 0, all_hi = in ? w.hi : INT_MAX;
#pragma unroll
  for (int s = 16; s >= 1; s >>= 1) {
    any_lo = min(any_lo, __shfl_xor(any_lo, s));
    any_hi = max(any_hi, __shfl_xor(any_hi, s));
    all_lo = max(all_lo, __shfl_xor(all_lo, s));
    all_hi = min(all_hi, __shfl_xor(all_hi, s));
  }
  any_lo = uniform(any_lo);
  any_hi = uniform(any_hi);
  all_lo = uniform(all_lo);
  all_hi = uniform(all_hi);

  const int64_t blk_stride = (int64_t)a.Hkv * k_elems(D);
  const int64_t base = (int64_t)g * k_elems(D);
  uint16_t* lds = reinterpret_cast<uint16_t*>(smem);
  bf16x8 kr[kLoads], vr[kLoads];
  int tbl_next = 0, bad_next = 0;    // of the stage that is fetched: valid entry of block i in lane 8 (st % 8) + i
  auto fetch = [&](int st) {
    if ((st & 7) == 0) {
      tbl_next = entry >= 0 && entry < a.num_blocks ? entry : -1;
      const int next = (st + 8) * kStageBlocks + lane;       // asked for eight stages ahead
      entry = next < blocks ? table[next] : 0;
    }
    const int i0 = (st & 7) * kStageBlocks;
    bad_next = (int)((__ballot(tbl_next < 0) >> i0) & 0xff);
    const int e = __builtin_amdgcn_readlane(tbl_next, i0 + wave);
    const int64_t at = (int64_t)max(e, 0) * blk_stride + base + lane * 8;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      kr[i] = load16(a.k_cache + at + i * 512);
      vr[i] = load16(a.v_cache + at + i * 512);
    }
  };
  // lane's group of V: dimension lane / 2 (+ 32 per load), half lane % 2
  uint16_t* k_put = lds + wave * k_elems(D) + lane * 8;
  uint16_t* v_put = lds + kStageBlocks * k_elems(D) + wave * v_elems(D) + (lane & 1) * v_half(D) + (lane >> 1) * 8;
  auto put = [&](int st) {
    const int off = (st & 1) * stage_elems(D);
    const int room = it.n - (it.blk_lo + st * kStageBlocks + wave) * kBlock;
    if (room < kBlock) {             // the history ends in or before this block: slots behind it may hold anything
#pragma unroll
      for (int i = 0; i < kLoads; ++i) vr[i] = first_values(room - 8 * (lane & 1), vr[i]);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      *reinterpret_cast<bf16x8*>(k_put + off + i * 512) = kr[i];
      *reinterpret_cast<bf16x8*>(v_put + off + i * 256) = vr[i];
    }
  };
  const int pos16 = (m & 3) | ((m & 4) << 1) | ((m & 8) >> 1);
  const uint16_t* k_get = lds + (m >> 4) * k_elems(D) + (h * kBlock + pos16) * 8;
  const uint16_t* v_get = lds + kStageBlocks * k_elems(D) + h * v_half(D) + m * 8;
  const uint16_t* v_raw = lds + kStageBlocks * k_elems(D);

  int bad = 0;
  if (stages > 0) {
    fetch(0);
    bad = bad_next;
    put(0);
    if (stages > 1) fetch(1);
  }
  __syncthreads();
  for (int st = 0; st < stages; ++st) {
    const int off = (st & 1) * stage_elems(D);
    for (int pr = wp; pr < kStageBlocks / 2; pr += WP) {
      const int pos = (it.blk_lo + st * kStageBlocks + 2 * pr) * kBlock;
      if (pos >= min(any_hi, it.blk_hi * kBlock)) break;
      if (pos + kPair <= any_lo) continue;
      const uint16_t* ks = k_get + off + 2 * pr * k_elems(D);
      const uint16_t* vs = v_get + off + 2 * pr * v_elems(D);
      const uint16_t* vraw = v_raw + off + 2 * pr * v_elems(D);
      auto k = [&](int kk) { return load16(ks + kk * 2 * kBlock * 8); };
      auto v = [&](int n, int b) { return load16(vs + b * v_elems(D) + n * 32 * 8); };
      auto raw = [&](int d, int i) {
        return vraw[(i >> 4) * v_elems(D) + ((i >> 3) & 1) * v_half(D) + d * 8 + (i & 7)];
      };
      const int b = (bad >> (2 * pr)) & 3;
      if (b == 0 && pos >= all_lo && pos + kPair <= min(all_hi, it.blk_hi * kBlock)) {
        attend_pair<D, P, false>(a.scale_log2, qf, w, pos, 0, k, v, raw);
      } else {
        const int hi_all = w.hi;
        w.hi = min(w.hi, it.blk_hi * kBlock);
        attend_pair<D, P, true>(a.scale_log2, qf, w, pos, b, k, v, raw);
        w.hi = hi_all;
      }
    }
    // the other buffer was last read before the barrier that ended the stage before
    if (st + 1 < stages) {
      bad = bad_next;
      put(st + 1);
      if (st + 2 < stages) fetch(st + 2);
    }
    __syncthreads();
  }
  w.l += __shfl_xor(w.l, 32);
  if (wc_shift != 3) join<D, Out>(a, it, g, wc_shift, w, smem);
  else write_columns<D, Out>(a, it, g, wc * kCols, w);
}

__device__ __forceinline__ void put_nan(float* p) { *p = __builtin_nanf(""); }
__device__ __forceinline__ void put_nan(uint16_t* p) { *p = 0x7fc0; }

template <int D, typename Out>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void prompt_attn_kernel(PromptArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const PlanHeader h = *reinterpret_cast<const PlanHeader*>(a.plan);
  const int i = blockIdx.x / a.Hkv, g = blockIdx.x - i * a.Hkv;
  // (asked for with the header: the grid has no more than the buffer's items)
  const Item it = reinterpret_cast<const Item*>(a.plan + items_at())[i];
  if (!plan_fits(a, h)) {            // a plan of other sizes, or none
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < (int64_t)a.R * a.Hq * D; e += (int64_t)gridDim.x * kThreads) {
      put_nan(static_cast<Out*>(a.out) + e);
      if (a.lse && e % D == 0) put_nan(a.lse + e / D);
    }
    return;
  }
  if (i >= min(h.n_items, a.max_items)) return;
  if (it.n < 0) {                    // a request whose length is out of range
    for (int e = threadIdx.x; e < it.ncols * D; e += kThreads) {
      const Target<D, Out> t = target_of<D, Out>(a, it, g, e / D);
      put_nan(t.out + e % D);
      if (t.lse && e % D == 0) put_nan(t.lse);
    }
    return;
  }
  const int tiles = (it.ncols + kCols - 1) / kCols;
  if (tiles == 1) run_narrow<D, Out>(a, h, it, g, smem);
  else run_wide<D, Out>(a, h, it, g, tiles <= 2 ? 1 : tiles <= 4 ? 2 : 3, smem);
}

// One workgroup per (split tile, KV head, kCols columns): the ranges in order.
template <int D, typename Out>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptArgs a) {
  const PlanHeader h = *reinterpret_cast<const PlanHeader*>(a.plan);
  const int parts = kTile / kCols;
  const int part = blockIdx.x % parts, u = blockIdx.x / parts;
  const int i = u / a.Hkv, g = u - i * a.Hkv;
  const Merge mg = reinterpret_cast<const Merge*>(a.plan + merges_at(a.max_items))[i];
  if (!plan_fits(a, h) || i >= min(h.n_merges, a.max_merges)) return;
  for (int e = threadIdx.x; e < kCols * (D / 4); e += 256) {
    const int d = e % (D / 4) * 4, col = part * kCols + e / (D / 4);
    if (col >= mg.ncols) return;
    const int64_t at = (int64_t)g * a.part_cols + mg.part + col;
    float top = -INFINITY;
#pragma unroll 8
    for (int s = 0; s < mg.splits; ++s) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (at + (int64_t)s * mg.ncols) * 2);
      if (ml.y != 0.f) top = fmaxf(top, ml.x);
    }
    const float ref = top == -INFINITY ? 0.f : top;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll 8
    for (int s = 0; s < mg.splits; ++s) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (at + (int64_t)s * mg.ncols) * 2);
      const float4 x = *reinterpret_cast<const float4*>(a.part_o + (at + (int64_t)s * mg.ncols) * D + d);
      // (a range of which the column attends nothing has a sum of 0 and any reference)
      const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - ref);
      acc.x += f * x.x;
      acc.y += f * x.y;
      acc.z += f * x.z;
      acc.w += f * x.w;
      l += f * ml.y;
    }
    const int fc = mg.col0 + col, token = fc / a.G;
    const int64_t row = (int64_t)(mg.row0 + token) * a.Hq + g * a.G + (fc - token * a.G);
    const float inv = inverse_of(l);
    store4(static_cast<Out*>(a.out) + row * D + d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (d == 0 && a.lse) a.lse[row] = lse_of(ref, l);
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

struct Sizes {
  int group, extra_items, max_items, max_merges;
  int64_t part_cols;
  size_t plan_bytes, off_ml, ws_bytes;
};

oda_status sizes_of(const oda_attn_shape* s, const oda_prompt_rows* r, Sizes* z) {
  if (s == nullptr) return oda::fail(ODA_ERR_NULL, "shape is NULL");
  if (r == nullptr) return oda::fail(ODA_ERR_NULL, "rows is NULL");
  size_t unused = 0;
  const oda_status st = oda_attn_workspace_size(s, 0, 0, &unused);   // the shape's own checks
  if (st != ODA_OK) return st;
  if (s->num_layers != 1) return oda::fail(ODA_ERR_SHAPE, "num_layers must be 1 (a layer's queries come from the one before)");
  if (s->split_blocks != 0) return oda::fail(ODA_ERR_SHAPE, "split_blocks must be 0 (the plan chooses)");
  if (s->batch > kMaxBatch) return oda::fail(ODA_ERR_UNSUPPORTED, "batch %d above %d", s->batch, kMaxBatch);
  if (r->num_rows < 1) return oda::fail(ODA_ERR_SHAPE, "num_rows must be >= 1");
  z->group = s->num_q_heads / s->num_kv_heads;
  const int64_t cols = (int64_t)r->num_rows * z->group;
  if ((int64_t)r->num_rows * s->num_q_heads > INT_MAX) return oda::fail(ODA_ERR_SHAPE, "num_rows * num_q_heads too large");
  z->extra_items = (int)oda::ceil_div(2 * kCus, s->num_kv_heads);
  const int64_t tiles = cols / kTile + s->batch;
  z->max_items = (int)(tiles + z->extra_items);
  z->max_merges = (int)std::min<int64_t>(tiles, z->extra_items);
  // a split tile has one item more than the extra ones that it takes
  z->part_cols = z->extra_items * std::min<int64_t>(kTile, cols) + std::min<int64_t>(cols, (int64_t)z->extra_items * kTile);
  z->plan_bytes = (size_t)oda::round_up(
      (merges_at(z->max_items) + (int64_t)z->max_merges * (int64_t)(sizeof(Merge) / 4)) * 4, 256);
  z->off_ml = (size_t)oda::round_up(z->part_cols * s->num_kv_heads * s->head_dim * 4, 256);
  z->ws_bytes = z->off_ml + (size_t)oda::round_up(z->part_cols * s->num_kv_heads * 8, 256);
  return ODA_OK;
}

oda_status check_buffer(const char* name, const void* p, size_t bytes, size_t need) {
  if (p == nullptr) return oda::fail(ODA_ERR_WORKSPACE, "%s is NULL (%zu bytes needed)", name, need);
  if (bytes < need) return oda::fail(ODA_ERR_WORKSPACE, "%s has %zu bytes, %zu needed", name, bytes, need);
  if (!oda::aligned(p, 256)) return oda::fail(ODA_ERR_WORKSPACE, "%s must be 256-byte aligned", name);
  return ODA_OK;
}

oda_status launch_status() {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return oda::fail(ODA_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return oda::ok();
}

// Raise a kernel's dynamic-LDS limit once per device (the attribute belongs to
// the device's copy of the kernel; host threads that race set the same value).
// A failure shows in the launch that needs the limit.
void raise_lds_limit(const void* kernel, std::atomic<uint64_t>* done, int bytes) {
  int dev = -1;
  (void)hipGetDevice(&dev);
  const uint64_t bit = (dev >= 0 && dev < 64) ? (1ull << dev) : 0ull;
  if (bit != 0 && (done->load(std::memory_order_acquire) & bit) != 0) return;
  if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess)
    done->fetch_or(bit, std::memory_order_acq_rel);
}

template <int D, typename Out>
oda_status launch_attention(const PromptArgs& a, hipStream_t stream) {
  const int64_t items = (int64_t)a.max_items * a.Hkv;
  const int64_t merges = (int64_t)a.max_merges * a.Hkv * (kTile / kCols);
  if (items > INT_MAX || merges > INT_MAX) return oda::fail(ODA_ERR_SHAPE, "grid too large");
  const int lds = lds_bytes(D);
  static std::atomic<uint64_t> raised{0};
  raise_lds_limit(reinterpret_cast<const void*>(prompt_attn_kernel<D, Out>), &raised, lds);
  (void)hipGetLastError();
  hipLaunchKernelGGL((prompt_attn_kernel<D, Out>), dim3((unsigned)items), dim3(kThreads), lds, stream, a);
  hipLaunchKernelGGL((prompt_merge_kernel<D, Out>), dim3((unsigned)merges), dim3(256), 0, stream, a);
  return launch_status();
}

}  // namespace

extern "C" oda_status oda_prompt_plan_size(const oda_attn_shape* shape, const oda_prompt_rows* rows, size_t* bytes) {
  Sizes z;
  const oda_status st = sizes_of(shape, rows, &z);
  if (st != ODA_OK) return st;
  if (bytes == nullptr) return oda::fail(ODA_ERR_NULL, "bytes is NULL");
  *bytes = z.plan_bytes;
  return oda::ok();
}

extern "C" oda_status oda_prompt_workspace_size(const oda_attn_shape* shape, const oda_prompt_rows* rows, size_t* bytes) {
  Sizes z;
  const oda_status st = sizes_of(shape, rows, &z);
  if (st != ODA_OK) return st;
  if (bytes == nullptr) return oda::fail(ODA_ERR_NULL, "bytes is NULL");
  *bytes = z.ws_bytes;
  return oda::ok();
}

extern "C" oda_status oda_prompt_plan(const oda_attn_shape* shape, const oda_prompt_rows* rows, const int32_t* seq_lens,
                                     int32_t causal, int32_t native_window, void* plan, size_t plan_bytes,
                                     hipStream_t stream) {
  Sizes z;
  oda_status st = sizes_of(shape, rows, &z);
  if (st != ODA_OK) return st;
  if (!seq_lens || !rows->row_start) return oda::fail(ODA_ERR_NULL, "seq_lens and row_start are required");
  if (causal != 0 && causal != 1) return oda::fail(ODA_ERR_SHAPE, "causal must be 0 or 1");
  if (native_window < 0 || (native_window > 0 && !causal))
    return oda::fail(ODA_ERR_SHAPE, "native_window must be >= 0, and 0 without the causal mask");
  st = check_buffer("plan", plan, plan_bytes, z.plan_bytes);
  if (st != ODA_OK) return st;
  PlanArgs a;
  a.row_start = rows->row_start;
  a.seq_lens = seq_lens;
  a.plan = static_cast<int32_t*>(plan);
  a.B = shape->batch;
  a.R = rows->num_rows;
  a.G = z.group;
  a.Hkv = shape->num_kv_heads;
  a.MB = shape->max_blocks_per_seq;
  a.max_len = shape->max_seq_len;
  a.causal = causal;
  a.window = native_window;
  a.extra_items = z.extra_items;
  a.max_items = z.max_items;
  a.max_merges = z.max_merges;
  (void)hipGetLastError();
  hipLaunchKernelGGL(prompt_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
  return launch_status();
}

extern "C" oda_status oda_prompt_attn(const oda_attn_shape* shape, const oda_attn_inputs* in, const oda_prompt_rows* rows,
                                     const void* plan, size_t plan_bytes, void* out, int32_t out_type, float* lse,
                                     void* workspace, size_t workspace_bytes, hipStream_t stream) {
  Sizes z;
  oda_status st = sizes_of(shape, rows, &z);
  if (st != ODA_OK) return st;
  if (in == nullptr) return oda::fail(ODA_ERR_NULL, "inputs is NULL");
  if (!in->q || !in->k_cache || !in->v_cache || !in->block_table || !out)
    return oda::fail(ODA_ERR_NULL, "q, k_cache, v_cache, block_table and out are required");
  if (in->k_cur || in->v_cur) return oda::fail(ODA_ERR_SHAPE, "k_cur and v_cur must be NULL: the rows' K/V is in the cache");
  if (out_type != ODA_F32 && out_type != ODA_BF16) return oda::fail(ODA_ERR_SHAPE, "unknown out_type %d", out_type);
  if (!oda::aligned(in->q, 16) || !oda::aligned(in->k_cache, 16) || !oda::aligned(in->v_cache, 16) || !oda::aligned(out, 16))
    return oda::fail(ODA_ERR_SHAPE, "q, caches and out must be 16-byte aligned");
  if (!(in->scale > 0.f) || !std::isfinite(in->scale)) return oda::fail(ODA_ERR_SHAPE, "scale must be finite and > 0");
  st = check_buffer("plan", plan, plan_bytes, z.plan_bytes);
  if (st != ODA_OK) return st;
  st = check_buffer("workspace", workspace, workspace_bytes, z.ws_bytes);
  if (st != ODA_OK) return st;
  PromptArgs a;
  a.q = in->q;
  a.k_cache = in->k_cache;
  a.v_cache = in->v_cache;
  a.block_table = in->block_table;
  a.plan = static_cast<const int32_t*>(plan);
  a.out = out;
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + z.off_ml);
  a.num_blocks = shape->num_blocks;
  a.part_cols = z.part_cols;
  a.B = shape->batch;
  a.R = rows->num_rows;
  a.Hq = shape->num_q_heads;
  a.Hkv = shape->num_kv_heads;
  a.G = z.group;
  a.MB = shape->max_blocks_per_seq;
  a.max_len = shape->max_seq_len;
  a.max_items = z.max_items;
  a.max_merges = z.max_merges;
  a.scale_log2 = in->scale * kLog2e;
  if (out_type == ODA_F32)
    return shape->head_dim == 128 ? launch_attention<128, float>(a, stream) : launch_attention<64, float>(a, stream);
  return shape->head_dim == 128 ? launch_attention<128, uint16_t>(a, stream) : launch_attention<64, uint16_t>(a, stream);
}
