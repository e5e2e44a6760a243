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
//
// Bound by the matrix cores and the vector operations beside them: 8,192 tokens of 32
// heads over 8 KV heads in 518 us with bf16 outputs, 1.06 PFLOP/s (a large library product
// of this card: 1.26), 512 behind 65,001 in 482 (1.14).  Of 128 dimensions a pair of blocks
// takes a wavefront 16 products (8 of scores, 8 of values) and, of its 16 scores a lane, 16
// exponentials and about 100 other vector operations; two wavefronts a SIMD take turns.
// With fp32 outputs, whose weights have three parts, it is 32 products: 887 and 849 us with
// the plan, 1.24 and 1.29 PFLOP/s of the products that are made.  Single rows against states
// are bound by HBM: 32 requests, 123 MB, in 23 us (5.3 TB/s) behind the plan.
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

constexpr int kBlock = 16;            // positions per KV block
constexpr int kPair = 2 * kBlock;     // positions per score tile
constexpr int kCols = 32;             // columns of an MFMA tile, of a wavefront
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kTile = kWaves * kCols; // columns of an item
constexpr int kStageBlocks = 4;       // blocks staged together: one of K or V per wavefront
constexpr int kMaxBatch = 2048;
constexpr int kLongest = INT_MAX - 64;   // positions up to a stage behind the last are counted in 32 bits
constexpr int kCus = 256;
constexpr int kPlanThreads = 256;
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

// Costs in the time in which one CU's share of HBM delivers a block of 16 positions: a
// block's products and softmax take no longer up to half a tile's columns.
constexpr float kWideCost = 1.3f;      // a block's for more columns
constexpr float kItemCost = 24.f;      // start and end of an item
constexpr float kPartCost = 8.f;       // an item's partial, written and merged
constexpr float kWidePartCost = 36.f;  // of more than half a tile's columns
constexpr float kLeastCost = 16.f;     // shortest range
constexpr int kClasses = 256;          // cost classes, eight to a factor of two

// Where there is little work, the length of an item counts: there tiles are one
// wavefront's 32 columns, whose positions all eight wavefronts share, although K and V
// are then read once for each (four requests of 100 rows behind 100: 20 us against 31;
// 64 behind 3,900 of 16 heads 27 : 34, behind 15,900 35 : 50; 256 behind 3,000 of 32 heads
// 35 : 43.  Beyond the limits: four of 60 behind 8,000 of 32 heads 73 : 65, 128 behind 16,000
// 67 : 63, 256 behind 16,000 104 : 90).
constexpr int kNarrowItems = 2 * kCus;     // narrow tiles of all KV heads together
constexpr float kNarrowWork = 288.f * kCus; // their blocks, all together

struct PlanRequest {
  int32_t row0, rows, n, tile, narrow_tile;        // tile: the request's first
};

__device__ __forceinline__ int class_of(float cost) {
  return min(max((int)ceilf(8.f * __log2f(fmaxf(cost, 1.f))), 0), kClasses - 1);
}
// At or above every cost of the class (with a margin for the logarithm's rounding).
__device__ __forceinline__ float class_cost(int c) { return 1.001f * __builtin_amdgcn_exp2f((float)c * 0.125f); }
// Ranges of a tile of `blocks` blocks where an item may hold `cap` of them, even.
__device__ __forceinline__ int range_blocks(int blocks, int splits) { return ((blocks + splits - 1) / splits + 1) & ~1; }

// Running sum, and running largest of values >= 0, over the wavefront's lanes: row shifts
// by 1, 2, 4, 8, then each row's last lane into the next row, then the lower half's into
// the upper (the lanes that nothing is shifted into get 0).
template <int kCtrl, int kRows>
__device__ __forceinline__ int shifted(int x) {
  return __builtin_amdgcn_update_dpp(0, x, kCtrl, kRows, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int x) {
  x += shifted<0x111, 0xf>(x);
  x += shifted<0x112, 0xf>(x);
  x += shifted<0x114, 0xf>(x);
  x += shifted<0x118, 0xf>(x);
  x += shifted<0x142, 0xa>(x);
  x += shifted<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ int wave_scan_max(int x) {
  x = max(x, shifted<0x111, 0xf>(x));
  x = max(x, shifted<0x112, 0xf>(x));
  x = max(x, shifted<0x114, 0xf>(x));
  x = max(x, shifted<0x118, 0xf>(x));
  x = max(x, shifted<0x142, 0xa>(x));
  x = max(x, shifted<0x143, 0xc>(x));
  return x;
}
__device__ __forceinline__ int2 block_scan(int2 x, int2* s_wave, int2& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int2 v = make_int2(wave_scan(x.x), wave_scan(x.y));
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
// everything goes through LDS (5.4 us for a request of 33 rows, 6.7 for one of 8,192, 7.3
// for sixteen mixed ones; with scans by shuffles and the cost classes to a wavefront each
// about one more).
__global__ __launch_bounds__(kPlanThreads) void prompt_plan_kernel(PlanArgs a) {
  __shared__ PlanRequest s_req[kMaxBatch];
  __shared__ int2 s_wave[kPlanThreads / 64];
  __shared__ int s_max[kPlanThreads / 64];
  __shared__ int s_class[2 * kClasses], s_place[kClasses];      // [wide][class]; places by the class alone
  __shared__ int s_count[kPlanThreads / 64][64];
  __shared__ float s_cost[kPlanThreads / 64][64], s_big[kPlanThreads / 64][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  Item* items = reinterpret_cast<Item*>(a.plan + items_at());
  Merge* merges = reinterpret_cast<Merge*>(a.plan + merges_at(a.max_items));
  for (int i = tid; i < 2 * kClasses; i += kPlanThreads) s_class[i] = 0;

  // requests: row starts kept in [0, R] and ascending whatever the array holds
  int n_tiles = 0, n_narrow = 0, carry = 0;
  float work = 0.f;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int start = 0, end = 0, n = 0;
    if (b < a.B) {
      start = min(max(a.row_start[b], 0), a.R);
      end = min(max(a.row_start[b + 1], 0), a.R);
      n = a.seq_lens[b];
    }
    // running largest of all starts up to b, and of the ends up to b
    int top = wave_scan_max(max(start, carry));
    __syncthreads();
    if (lane == 63) s_max[wave] = top;
    __syncthreads();
    for (int w = 0; w < wave; ++w) top = max(top, s_max[w]);
    const int row0 = top, rows = max(end - row0, 0);
    for (int w = 0; w < kPlanThreads / 64; ++w) carry = max(carry, s_max[w]);
    // (narrow tiles are counted up to more than may be)
    const int tiles = (int)(((int64_t)rows * a.G + kTile - 1) / kTile);
    const int narrow = (int)min(((int64_t)rows * a.G + kCols - 1) / kCols, (int64_t)kNarrowItems + 1);
    int2 total;
    const int2 at = block_scan(make_int2(tiles, narrow), s_wave, total);
    if (b < a.B) {
      const bool bad = n < 0 || n > min(a.max_len, kLongest) || (a.causal && n < rows);
      s_req[b] = PlanRequest{row0, rows, bad ? -1 : n, n_tiles + at.x, n_narrow + at.y};
      if (!bad) {
        const int reach = a.causal && a.window > 0 && a.window < n - rows ? a.window + rows : n;
        work += (float)narrow * (float)(reach / kBlock + 1);
      }
    }
    n_tiles += total.x;
    n_narrow += total.y;
  }
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) work += __shfl_xor(work, s);
  __syncthreads();
  if (lane == 0) s_big[wave][0] = work;
  __syncthreads();
  work = 0.f;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) work += s_big[w][0];
  const bool narrow = n_narrow <= kNarrowItems / a.Hkv && work * (float)a.Hkv <= kNarrowWork;
  const int width = narrow ? kCols : kTile;
  if (narrow) n_tiles = n_narrow;
  __syncthreads();

  // a tile: its request, columns and blocks
  struct Tile {
    int b, col0, ncols, lo, hi;
  };
  auto tile_at = [&](int t) {
    int lo = 0, hi = a.B;            // the last request whose first tile is at or before t (one with rows)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if ((narrow ? s_req[mid].narrow_tile : s_req[mid].tile) <= t) lo = mid;
      else hi = mid;
    }
    const PlanRequest q = s_req[lo];
    Tile r;
    r.b = lo;
    r.col0 = (t - (narrow ? q.narrow_tile : q.tile)) * width;
    r.ncols = (int)min((int64_t)width, (int64_t)q.rows * a.G - r.col0);
    r.lo = r.hi = 0;
    if (q.n < 0) return r;
    const int first = q.n - q.rows + r.col0 / a.G, last = q.n - q.rows + (r.col0 + r.ncols - 1) / a.G;
    r.hi = (a.causal ? last + kBlock : q.n + kBlock - 1) / kBlock;
    r.lo = a.causal && a.window > 0 ? max(0, first - a.window + 1) / kBlock : 0;
    return r;
  };
  const Tile own = tid < n_tiles ? tile_at(tid) : Tile{};
  auto is_wide = [&](const Tile& t) { return t.ncols > kTile / 2; };
  auto cost_of = [&](const Tile& t) { return (float)(t.hi - t.lo) * (is_wide(t) ? kWideCost : 1.f); };

  int most = 0;
  for (int t = tid; t < n_tiles; t += kPlanThreads) {
    const Tile r = t == tid ? own : tile_at(t);
    const int c = class_of(cost_of(r));
    atomicAdd(&s_class[(is_wide(r) ? kClasses : 0) + c], 1);
    most = max(most, c);
  }
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) most = max(most, __shfl_xor(most, s));
  if (lane == 0) s_max[wave] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) most = max(most, s_max[w]);

  // what an item may cost: every lane tries one value; the last splits nothing
  const float top = fmaxf(class_cost(most), kLeastCost);
  const float cap = lane == 63 ? top : kLeastCost * __builtin_amdgcn_exp2f(__log2f(top / kLeastCost) * (float)lane * (1.f / 63.f));
  const float inv = 1.f / cap;
  // (items beyond the tiles are counted up to more than may be: what is above is refused below)
  const int limit = a.extra_items + 1;
  int more = 0;
  float sum = 0.f, big = 0.f;
  // (classes that are there lie side by side: the wavefronts take them in turn)
  for (int c0 = 0; c0 < 2 * kClasses; c0 += 64) {
    if ((c0 & (kClasses - 1)) > most) continue;
    const int here = s_class[c0 + lane];
    const float part = c0 >= kClasses ? kWidePartCost : kPartCost;
    for (uint64_t todo = __ballot(here != 0 && (lane & (kPlanThreads / 64 - 1)) == wave); todo != 0; todo &= todo - 1) {
      const int i = __builtin_ctzll(todo);
      const int count = __builtin_amdgcn_readlane(here, i);
      const float cost = class_cost((c0 + i) & (kClasses - 1));
      const int splits = lane == 63 ? 1 : max(1, (int)ceilf(cost * inv));
      more += min(count, limit) * min(splits - 1, limit);
      big = fmaxf(big, cost * __builtin_amdgcn_rcpf((float)splits));
      sum += (float)count * (cost + (float)splits * (kItemCost + (splits > 1 ? part : 0.f)));
    }
  }
  s_count[wave][lane] = more;
  s_cost[wave][lane] = sum;
  s_big[wave][lane] = big;
  __syncthreads();
  more = 0;
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    more += s_count[w][lane];
    sum += s_cost[w][lane];
    big = fmaxf(big, s_big[w][lane]);
  }
  // rounds of items of mean cost, the last one whole where they are alike; at least the largest item
  const int n = n_tiles + more;
  const float rounds = (float)a.Hkv * (float)n * (1.f / (float)kCus);
  const float mean = sum / (float)max(n, 1);
  const float alike = fminf(1.f, mean / (big + kItemCost));
  float est = fmaxf(big + kItemCost, mean * (rounds + alike * (ceilf(rounds) - rounds)));
  if (more > a.extra_items) est = INFINITY;
  float best = est;
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) best = fminf(best, __shfl_xor(best, s));
  const uint64_t who = __ballot(est == best);
  // (of equal ones the smallest: a class's cost is above its tiles', which a larger value would split less)
  const int pick = who ? __builtin_ctzll(who) : 63;
  const float inv_best = __shfl(inv, pick);
  auto splits_of = [&](const Tile& t) {
    const int blocks = t.hi - t.lo;
    if (pick == 63 || blocks <= 0) return 1;
    const int splits = min(blocks, max(1, (int)ceilf(cost_of(t) * inv_best)));
    const int len = range_blocks(blocks, splits);
    return (blocks + len - 1) / len;
  };

  // items listed by their cost, the largest class first (within one in any order)
  __syncthreads();
  for (int i = tid; i < kClasses; i += kPlanThreads) s_class[i] = 0;
  __syncthreads();
  for (int t = tid; t < n_tiles; t += kPlanThreads) {
    const Tile r = t == tid ? own : tile_at(t);
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
      r = t == tid ? own : tile_at(t);
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
  float* part_ml;            // [Hkv][part_cols][2]  (reference in score units, sum)
  int64_t num_blocks;
  int64_t part_cols;
  int32_t B, R, Hq, Hkv, G, MB, max_len;
  int32_t max_items, max_merges;
  int32_t merge_parts;       // of kCols columns that a tile may have
  float scale_log2;          // of a score, for exponents of 2
  float lag;                 // kLag in score units
};

__device__ __forceinline__ bool plan_fits(const PromptArgs& a, const PlanHeader& h) {
  return (h.magic == kMagic) & (h.batch == a.B) & (h.rows == a.R) & (h.group == a.G) & (h.heads == a.Hkv) &
         (h.max_blocks == a.MB) & (h.max_len == a.max_len);
}

__device__ __forceinline__ bf16x8 load16(const uint16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }

// Two floats to bf16.
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
// weight's rounding (up to 2^-8 of it, of random sign) adds about as much as the output's own.
// An fp32 output takes three, which hold all 24 bits, as decode attention does.
template <typename Out>
constexpr int kPartsOf = std::is_same<Out, float>::value ? 3 : 1;

// A wavefront's columns: o[n][4 i + j] is dimension 32 n + 8 i + 4 h + j of column
// lane % 32, h = lane / 32; ref the reference of its weights in score units
// (-infinity: none yet), sum this lane's part of their sum; attended positions [lo, hi).
template <int D>
struct Columns {
  f32x16 o[D / 32];
  float ref, sum;
  int lo, hi;
};
// A pair's weights as bf16 parts, by the block.
template <int P>
struct Parts {
  bf16x8 x[P][2];
};

// S^T = K Q^T of a pair of blocks: [8 b + e] is position 8 h + e of block b.  k(kk): the
// lane's operand.  Operand row 16 b + r is position r of block b with bits 2 and 3 of r
// exchanged, so that lane half h gets positions 8 h .. 8 h + 7 of both blocks, which is
// how it holds V's operand.
template <int D, typename KOp>
__device__ __forceinline__ f32x16 score_pair(const bf16x8 (&qf)[D / 16], KOp k) {
  f32x16 s = {};
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k(kk), qf[kk], s, 0, 0, 0);
  return s;
}

template <int P>
__device__ __forceinline__ Parts<P> parts_of(f32x16 p) {
  Parts<P> r;
#pragma unroll
  for (int q = 0; q < P; ++q) {
    u32x4 t[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t x = round_pair(p[2 * e], p[2 * e + 1]);
      t[e >> 2][e & 3] = x;
      if (q + 1 < P) {                 // what the rounding leaves
        p[2 * e] -= __uint_as_float(x << 16);
        p[2 * e + 1] -= __uint_as_float(x & 0xffff0000u);
      }
    }
    r.x[q][0] = __builtin_bit_cast(bf16x8, t[0]);
    r.x[q][1] = __builtin_bit_cast(bf16x8, t[1]);
  }
  return r;
}

// O^T += V^T P^T.  v(n, b): the lane's operand.
template <int D, int P, typename VOp>
__device__ __forceinline__ void weigh_pair(const Parts<P>& part, Columns<D>& w, VOp v) {
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const bf16x8 x = v(n, b);
#pragma unroll
      for (int q = 0; q < P; ++q) w.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, part.x[q][b], w.o[n], 0, 0, 0);
    }
}

// The weight of a score against a reference.  (The difference first: it is exact where
// it matters, also for scores whose product with the scale would be off by more than
// the exponents' range.)
__device__ __forceinline__ float weight_of(float s, float ref, float scale_log2) {
  return __builtin_amdgcn_exp2f((s - ref) * scale_log2);
}
// Weights of a pair's scores against the column's reference, and the lane's sum.
//
// Weights are taken against a reference kLag (in exponents of 2) above the largest score
// at which it was set and below no later one: at most 1, and their sum 2^-kLag or more.
// The largest score is looked for, and sums are rescaled, only where a lane's weights add
// up to more than 1 or there is no reference yet (its weights come out infinite or NaN).
constexpr float kLag = 6.f;
constexpr float kMaxLag = 1e37f;     // (scores of a scale that small all weigh the same)
template <int P>
__device__ __forceinline__ float weights_of(float scale_log2, const f32x16& s, float ref, Parts<P>& part) {
  f32x16 p;
  float t[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    p[i] = weight_of(s[i], ref, scale_log2);
    t[i & 1] += p[i];
  }
  part = parts_of<P>(p);
  return t[0] + t[1];
}
// The sum's check, after all products of earlier pairs: raises the reference where it fails.
template <int D, int P>
__device__ __forceinline__ void settle(float scale_log2, float lag, const f32x16& s, Columns<D>& w, Parts<P>& part, float sum) {
  if (__any(!(sum <= 1.f))) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    const float top = fmaxf(w.ref, fminf(column_max(mx) + lag, FLT_MAX));
    const float ref = top == -INFINITY ? 0.f : top;
    const float alpha = weight_of(w.ref, ref, scale_log2);
    w.ref = top;
    w.sum *= alpha;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) w.o[n][i] *= alpha;
    sum = weights_of<P>(scale_log2, s, ref, part);
  }
  w.sum += sum;
}

// Scores of positions that a column does not attend.  at: the first block's position
// of this lane's scores; end: of the item; bad: bit b = block b has no memory (its
// scores are NaN).
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
// Values that are not finite become 0, and are told.
__device__ __forceinline__ bf16x8 finite_values(bf16x8 v, bool& odd) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (w[i] & 0x7f80u) == 0x7f80u, hi = (w[i] & 0x7f800000u) == 0x7f800000u;
    odd |= lo | hi;
    w[i] &= (lo ? 0u : 0x0000ffffu) | (hi ? 0u : 0xffff0000u);
  }
  return __builtin_bit_cast(bf16x8, w);
}
// Positions that one column attends and another does not may hold values that are not
// finite, which 0 * V would bring to both.  There such values are taken out of the
// product (finite_values) and added to the columns that attend them (a weight is
// positive: it does not change an infinity or NaN).  v0, v1: the pair's blocks.
template <int D>
__device__ __forceinline__ void add_odd_values(const uint16_t* v0, const uint16_t* v1, int pos, int end, Columns<D>& w) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll 1
  for (int i = 0; i < kPair; ++i) {
    const uint16_t* src = (i < kBlock ? v0 : v1) + 4 * h * kBlock + (i & (kBlock - 1));
    const bool in = pos + i >= w.lo && pos + i < min(w.hi, end);
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t x = src[(32 * n + 8 * (r >> 2) + (r & 3)) * kBlock];
        if (in && (x & 0x7f80u) == 0x7f80u) w.o[n][r] += __uint_as_float(x << 16);
        __builtin_amdgcn_sched_barrier(0);     // one load at a time: no registers for a rare case
      }
  }
}

// A wavefront's columns: queries as B operands, attended positions.
template <int D>
__device__ __forceinline__ void load_columns(const PromptArgs& a, const PlanHeader& h, const Item& it, int g, int first,
                                             Columns<D>& w, bf16x8 (&qf)[D / 16]) {
  const int lane = threadIdx.x & 63;
  const int col = first + (lane & 31);
  const int at = it.col0 + (col < it.ncols ? col : 0);       // (past the last column the first again, not written)
  const int token = at / a.G, head = at - token * a.G;
  const uint16_t* q = a.q + ((int64_t)(it.row0 + token) * a.Hq + g * a.G + head) * D + 8 * (lane >> 5);
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) qf[kk] = load16(q + 16 * kk);
  w.hi = h.causal ? it.place0 + token + 1 : it.n;
  w.lo = h.causal && h.window > 0 ? max(0, w.hi - h.window) : 0;
  w.ref = -INFINITY;
  w.sum = 0.f;
#pragma unroll
  for (int n = 0; n < D / 32; ++n) w.o[n] = f32x16{};
}
// Positions that any, and that every, one of `count` columns from `first` on attends.
struct Reach {
  int any_lo, any_hi, all_lo, all_hi;
};
__device__ __forceinline__ Reach reach_of(const PromptArgs& a, const PlanHeader& h, const Item& it, int first, int count) {
  const int end = min(first + count, it.ncols) - 1;
  if (!h.causal) return Reach{0, first <= end ? it.n : 0, 0, it.n};
  // columns are in the order of their tokens
  const int lo = it.place0 + (it.col0 + first) / a.G + 1, hi = it.place0 + (it.col0 + max(first, end)) / a.G + 1;
  Reach r;
  r.any_lo = h.window > 0 ? max(0, lo - h.window) : 0;
  r.all_lo = h.window > 0 ? max(0, hi - h.window) : 0;
  r.any_hi = first <= end ? hi : 0;
  r.all_hi = lo;
  return r;
}

// LDS: a ring of four stages of K blocks and one of V blocks, or the wavefronts' O where
// ranges are joined.  Blocks lie as in the cache, but for V's 16-byte groups (eight
// positions of a dimension), whose halves are exchanged in every other eight dimensions:
// sixteen lanes' operand reads then meet all banks.
constexpr int kStages = 4;
__host__ __device__ constexpr int block_elems(int D) { return kBlock * D; }
__host__ __device__ constexpr int stage_elems(int D) { return kStageBlocks * block_elems(D); }
__host__ __device__ constexpr int o_stride(int D) { return D + 4; }                    // floats
__host__ __device__ constexpr int join_bytes(int D) { return kWaves * kCols * o_stride(D) * 4; }
__host__ __device__ constexpr int data_bytes(int D) {
  return 2 * kStages * stage_elems(D) * 2 > join_bytes(D) ? 2 * kStages * stage_elems(D) * 2 : join_bytes(D);
}
__host__ __device__ constexpr int lds_bytes(int D) { return data_bytes(D) + 2 * kWaves * kCols * 4 + kStages * kStageBlocks * 4; }
static_assert(lds_bytes(128) <= 160 * 1024, "an item fits LDS");
static_assert(2 * kStageBlocks == kWaves, "a wavefront brings one block of K or V");

// A block from memory straight to LDS: 1 KiB per load, lane i's 16 bytes to place i.
// (In assembly, as the compiler would wait for all of them before any read of LDS.  No
// registers are written; the address is read when the load is issued; the caller waits
// with wait_loads and a barrier before the block is read.  A load to LDS needs a wait
// state behind a scalar write of M0, which nobody puts into an asm block but its author.)
constexpr int kLoadBytes = 64 * 16;
template <int D>
__device__ __forceinline__ void load_to_lds(const uint16_t* src, uint32_t dst) {
  if constexpr (D == 128)
    asm volatile(
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %0, off\n\t"
        "global_load_lds_dwordx4 %0, off offset:%2\n\t"
        "global_load_lds_dwordx4 %0, off offset:2*%2\n\t"
        "global_load_lds_dwordx4 %0, off offset:3*%2"
        :
        : "v"(src), "s"(dst), "n"(kLoadBytes)
        : "memory", "m0");
  else
    asm volatile(
        "s_mov_b32 m0, %1\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %0, off\n\t"
        "global_load_lds_dwordx4 %0, off offset:%2"
        :
        : "v"(src), "s"(dst), "n"(kLoadBytes)
        : "memory", "m0");
}
// Waits for all of this wavefront's loads but one block's (the one issued last), or all.
template <int D>
__device__ __forceinline__ void wait_loads(bool but_one) {
  if (!but_one) __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0)
  else __builtin_amdgcn_s_waitcnt(D == 128 ? 0x0f74 : 0x0f72);   // vmcnt(4), vmcnt(2)
}

__device__ __forceinline__ void store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
__device__ __forceinline__ void store4(uint16_t* p, float4 x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(round_pair(x.x, x.y), round_pair(x.z, x.w));
}
__device__ __forceinline__ float lse_of(float ref, float l, float scale_log2) {
  return l == 0.f ? -INFINITY : (ref * scale_log2 + __log2f(l)) * kLn2;
}
__device__ __forceinline__ float inverse_of(float l) { return l == 0.f ? 0.f : 1.f / l; }

// Where a column goes: a partial, or the outputs.
template <typename Out>
struct Target {
  Out* out;
  float* lse;
  float* part_o;
  float* part_ml;
};
template <int D, typename Out>
__device__ __forceinline__ Target<Out> target_of(const PromptArgs& a, const Item& it, int g, int col) {
  Target<Out> t{};
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

// Joins the wavefronts' position ranges and writes.
template <int D, typename Out>
__device__ __forceinline__ void join(const PromptArgs& a, const Item& it, int g, Columns<D>& w, char* smem) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  float* sm_o = reinterpret_cast<float*>(smem);                      // [waves][32][D + 4]
  float* sm_c = reinterpret_cast<float*>(smem + data_bytes(D));      // [waves][32]
  float* sm_l = sm_c + kWaves * kCols;
  const int h = lane >> 5, at = wave * kCols + (lane & 31);
  if (h == 0) {
    sm_c[at] = w.ref;
    sm_l[at] = w.sum;
  }
  float* dst = sm_o + at * o_stride(D) + 4 * h;
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4*>(dst + 32 * n + 8 * i) =
          make_float4(w.o[n][4 * i], w.o[n][4 * i + 1], w.o[n][4 * i + 2], w.o[n][4 * i + 3]);
  __syncthreads();
  for (int e = threadIdx.x; e < kCols * (D / 4); e += kThreads) {
    const int d = e % (D / 4) * 4, col = e / (D / 4);
    if (col >= it.ncols) break;
    float top = -INFINITY;
#pragma unroll
    for (int p = 0; p < kWaves; ++p) top = fmaxf(top, sm_c[p * kCols + col]);
    const float ref = top == -INFINITY ? 0.f : top;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll
    for (int p = 0; p < kWaves; ++p) {
      const int from = p * kCols + col;
      const float s = weight_of(sm_c[from], ref, a.scale_log2);
      const float4 x = *reinterpret_cast<const float4*>(sm_o + from * o_stride(D) + d);
      acc.x += s * x.x;
      acc.y += s * x.y;
      acc.z += s * x.z;
      acc.w += s * x.w;
      l += s * sm_l[from];
    }
    const Target<Out> t = target_of<D, Out>(a, it, g, col);
    if (it.part >= 0) {
      store4(t.part_o + d, acc);
      if (d == 0) *reinterpret_cast<float2*>(t.part_ml) = make_float2(ref, l);
    } else {
      const float inv = inverse_of(l);
      store4(t.out + d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
      if (d == 0 && t.lse) *t.lse = lse_of(ref, l, a.scale_log2);
    }
  }
}

// Columns straight from the registers, where a wavefront saw all of the item's blocks.
template <int D, typename Out>
__device__ __forceinline__ void write_columns(const PromptArgs& a, const Item& it, int g, int first, const Columns<D>& w) {
  const int lane = threadIdx.x & 63, h = lane >> 5, col = first + (lane & 31);
  if (col >= it.ncols) return;
  const Target<Out> t = target_of<D, Out>(a, it, g, col);
  const float ref = w.ref == -INFINITY ? 0.f : w.ref;
  const float inv = it.part >= 0 ? 1.f : inverse_of(w.sum);
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
  if (it.part >= 0) *reinterpret_cast<float2*>(t.part_ml) = make_float2(ref, w.sum);
  else if (t.lse) *t.lse = lse_of(ref, w.sum, a.scale_log2);
}

// One column tile: the wavefronts take contiguous ranges of pairs, K and V go straight
// to registers.
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
  const Reach reach = reach_of(a, head, it, 0, kCols);
  const int64_t blk_stride = (int64_t)a.Hkv * block_elems(D);
  const int pos16 = (m & 3) | ((m & 4) << 1) | ((m & 8) >> 1);
  const uint16_t* kbase = a.k_cache + (int64_t)g * block_elems(D) + (h * kBlock + pos16) * 8;
  const uint16_t* vbase = a.v_cache + (int64_t)g * block_elems(D) + m * kBlock + 8 * h;
  const int end = hi * kBlock;
  int tbl = 0;
  for (int v = lo; v < hi; v += 2) {
    const int i0 = (v - lo) & 63;
    if (i0 == 0) {
      tbl = entry >= 0 && entry < a.num_blocks ? entry : -1;
      entry = v + 64 + lane < hi ? table[v + 64 + lane] : 0;
    }
    // (past an odd end the first block again: no column attends it)
    const int e0 = __builtin_amdgcn_readlane(tbl, i0);
    const int e1 = v + 1 < hi ? __builtin_amdgcn_readlane(tbl, i0 + 1) : e0;
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
    f32x16 s = score_pair<D>(qf, [&](int kk) { return kr[kk]; });
    bool odd = false;
    if (v + 1 >= hi || bad != 0 || pos < reach.all_lo || pos + kPair > reach.all_hi) {
      mask_scores(pos + 8 * h, w.lo, min(w.hi, end), bad, s);
#pragma unroll
      for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int b = 0; b < 2; ++b) vr[n][b] = finite_values(first_values(it.n - pos - kBlock * b - 8 * h, vr[n][b]), odd);
    }
    Parts<P> part;
    const float sum = weights_of<P>(a.scale_log2, s, w.ref, part);
    settle<D, P>(a.scale_log2, a.lag, s, w, part, sum);
    weigh_pair<D, P>(part, w, [&](int n, int b) { return vr[n][b]; });
    if (__any(odd)) {
      const uint16_t* v0 = a.v_cache + (int64_t)g * block_elems(D);
      add_odd_values<D>(v0 + b0, v0 + b1, pos, end, w);
    }
  }
  w.sum += __shfl_xor(w.sum, 32);
  join<D, Out>(a, it, g, w, smem);
}

// More columns: K and V are staged through LDS, four blocks a stage, a wavefront
// bringing one of them, and every wavefront that has columns goes through all pairs with
// its 32.  (Two position ranges where there are up to 128 columns: 64 requests of 64 columns
// behind 2,000 120 us against 116.)
//
// While the weights of pair i are formed (vector operations), the matrix cores form the
// scores of the wavefront's next pair and add the products of the one before: round st
// reads K of stages st and st + 1 and V of st - 1 and st, one barrier a round.  K of
// st + 3 and V of st + 2 are asked for in round st, so that a load has two rounds.
template <int D, typename Out>
__device__ __forceinline__ void run_wide(const PromptArgs& a, const PlanHeader& head, const Item& it, int g, char* smem) {
  constexpr int P = kPartsOf<Out>;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int h = lane >> 5, m = lane & 31;
  const int blocks = it.blk_hi - it.blk_lo;
  const int stages = (blocks + kStageBlocks - 1) / kStageBlocks;
  const int32_t* table = a.block_table + (int64_t)it.request * a.MB + it.blk_lo;
  int entry = lane < blocks ? table[lane] : 0;       // 64 blocks, sixteen stages
  Columns<D> w;
  bf16x8 qf[D / 16];
  load_columns<D>(a, head, it, g, wave * kCols, w, qf);
  const Reach own = reach_of(a, head, it, wave * kCols, kCols), all = reach_of(a, head, it, 0, it.ncols);
  const int base_pos = it.blk_lo * kBlock, end = it.blk_hi * kBlock;
  // the column tile's pairs
  const int own_end = min(own.any_hi, end) - base_pos;
  const int first = max(0, own.any_lo - base_pos) / kPair, last = own_end > 0 ? (own_end + kPair - 1) / kPair : 0;

  const int64_t blk_stride = (int64_t)a.Hkv * block_elems(D);
  const int64_t base = (int64_t)g * block_elems(D);
  uint16_t* lds = reinterpret_cast<uint16_t*>(smem);
  uint16_t* lds_v = lds + kStages * stage_elems(D);
  int* sm_odd = reinterpret_cast<int*>(smem + lds_bytes(D) - kStages * kStageBlocks * 4);     // [stage][block]
  const bool brings_v = wave >= kStageBlocks;
  const int lead = brings_v ? 2 : 3;                 // stages from the round's to the one asked for
  const int mine = wave & (kStageBlocks - 1);
  const int v_swap = (lane >> 4) & 1;                // whether the lane's group of V is its dimension's other half
  const uint16_t* cache = brings_v ? a.v_cache + base + (lane ^ v_swap) * 8 : a.k_cache + base + lane * 8;
  const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem +
                          ((brings_v ? kStages * stage_elems(D) : 0) + mine * block_elems(D)) * 2;
  int tbl = 0;
  uint32_t bad_ring = 0;             // of the stages, four bits each, the one asked for last in the low ones
  auto fetch = [&](int st) {
    bad_ring <<= 4;
    if (st >= stages) return;
    if ((st & 15) == 0) {
      tbl = entry >= 0 && entry < a.num_blocks ? entry : -1;
      const int next = (st + 16) * kStageBlocks + lane;       // asked for sixteen stages ahead
      entry = next < blocks ? table[next] : 0;
    }
    const int i0 = (st & 15) * kStageBlocks;
    bad_ring |= (uint32_t)((__ballot(tbl < 0) >> i0) & 0xf);
    const uint16_t* src = cache + (int64_t)max(__builtin_amdgcn_readlane(tbl, i0 + mine), 0) * blk_stride;
    load_to_lds<D>(src, uniform((int)(lds_at + (st & (kStages - 1)) * stage_elems(D) * 2)));
  };
  // Stages that not every column attends in full, or without memory: values that nobody
  // attends and, told in sm_odd, those that are not finite become 0.
  auto unclean = [&](int st, int bad) {
    const int pos = base_pos + st * kStageBlocks * kBlock;
    return bad != 0 || pos < all.all_lo || pos + kStageBlocks * kBlock > all.all_hi;
  };
  auto clean = [&](int st, int bad) {
    if (brings_v) {
      uint16_t* v = lds_v + (st & (kStages - 1)) * stage_elems(D) + mine * block_elems(D) + lane * 8;
      const int room = (bad >> mine) & 1 ? 0 : it.n - base_pos - (st * kStageBlocks + mine) * kBlock - 8 * ((lane & 1) ^ v_swap);
      bool odd = false;
#pragma unroll
      for (int i = 0; i < block_elems(D) / 512; ++i) {
        const bf16x8 x = finite_values(first_values(room, load16(v + i * 512)), odd);
        *reinterpret_cast<bf16x8*>(v + i * 512) = x;
      }
      const int told = __any(odd) ? 1 : 0;
      if (lane == 0) sm_odd[(st & (kStages - 1)) * kStageBlocks + mine] = told;
    }
    __syncthreads();
  };
  const int pos16 = (m & 3) | ((m & 4) << 1) | ((m & 8) >> 1);
  const uint16_t* k_get = lds + (m >> 4) * block_elems(D) + (h * kBlock + pos16) * 8;
  const uint16_t* v_get = lds_v + (2 * m + (h ^ ((m >> 3) & 1))) * 8;
  auto stage_of = [&](int i) { return ((i >> 1) & (kStages - 1)) * stage_elems(D) + (i & 1) * 2 * block_elems(D); };

  Parts<P> part;         // weights of the wavefront's pair before
  bf16x8 kf[D / 16];     // K of its next pair
  auto load_keys = [&](int i) {
    const uint16_t* ks = k_get + stage_of(i);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) kf[kk] = load16(ks + kk * 2 * kBlock * 8);
  };
  auto add_odd = [&](int i) {
    const int blk = 2 * i;
    int64_t at[2];
    for (int b = 0; b < 2; ++b) {
      const int e = blk + b < blocks ? table[blk + b] : -1;
      at[b] = (int64_t)(e >= 0 && e < a.num_blocks ? e : 0) * blk_stride + base;
    }
    add_odd_values<D>(a.v_cache + at[0], a.v_cache + at[1], base_pos + i * kPair, end, w);
  };
  // Where nothing is masked and the pair is neither the wavefront's first nor its last:
  auto full_step = [&](int i, f32x16& s_now, f32x16& s_next) {
    const uint16_t* vs = v_get + stage_of(i - 1);
    bf16x8 vf[D / 32][2];
    Parts<P> now;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int b = 0; b < 2; ++b) vf[n][b] = load16(vs + b * block_elems(D) + n * 32 * kBlock);
    __builtin_amdgcn_s_setprio(1);     // products before the other wavefront's (sixteen mixed requests, fp32: 387 us against 410)
    s_next = score_pair<D>(qf, [&](int kk) { return kf[kk]; });
    load_keys(i + 2);
    const float sum = weights_of<P>(a.scale_log2, s_now, w.ref, now);
    weigh_pair<D, P>(part, w, [&](int n, int b) { return vf[n][b]; });
    __builtin_amdgcn_s_setprio(0);
    settle<D, P>(a.scale_log2, a.lag, s_now, w, now, sum);
    part = now;
  };
  const int full_lo = max(first + 1, (own.all_lo - base_pos + kPair - 1) / kPair);
  const int full_hi = min(last - 1, (min(own.all_hi, end) - base_pos) / kPair);
  // Any pair i, its scores in s_now: its weights beside the next pair's scores (behind the
  // last one of what lies in LDS, not used) and the products of the one before (of the
  // first one's values with weights of 0).  bad: its blocks; odd: whether values were
  // taken out of its stage (bit 0) and of that of the pair before (bit 1).
  auto step = [&](int i, int bad, int odd, f32x16& s_now) {
    if (i < first || i >= last) return;
    const bool fills = i - 1 < first, drains = i + 1 >= last;
    if (fills) {
      const uint16_t* ks = k_get + stage_of(i);
      s_now = score_pair<D>(qf, [&](int kk) { return load16(ks + kk * 2 * kBlock * 8); });
      load_keys(i + 1);
#pragma unroll
      for (int q = 0; q < P; ++q) part.x[q][0] = part.x[q][1] = bf16x8{};
    }
    const int pos = base_pos + i * kPair;
    if (bad != 0 || pos < own.all_lo || pos + kPair > min(own.all_hi, end))
      mask_scores(pos + 8 * h, w.lo, min(w.hi, end), bad, s_now);
    const uint16_t* vs = v_get + stage_of(fills ? i : i - 1);
    bf16x8 vf[D / 32][2];
    Parts<P> now;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int b = 0; b < 2; ++b) vf[n][b] = load16(vs + b * block_elems(D) + n * 32 * kBlock);
    __builtin_amdgcn_s_setprio(1);
    const f32x16 s_next = score_pair<D>(qf, [&](int kk) { return kf[kk]; });
    load_keys(i + 2);
    const float sum = weights_of<P>(a.scale_log2, s_now, w.ref, now);
    weigh_pair<D, P>(part, w, [&](int n, int b) { return vf[n][b]; });
    __builtin_amdgcn_s_setprio(0);
    settle<D, P>(a.scale_log2, a.lag, s_now, w, now, sum);
    part = now;
    s_now = s_next;
    if ((odd & 2) != 0 && !fills) add_odd(i - 1);
    if (drains) {
      vs = v_get + stage_of(i);
      weigh_pair<D, P>(part, w, [&](int n, int b) { return load16(vs + b * block_elems(D) + n * 32 * kBlock); });
      if ((odd & 1) != 0) add_odd(i);
    }
  };

  if (stages > 0) {
    for (int st = 0; st < lead; ++st) fetch(st);
    wait_loads<D>(false);
    __syncthreads();
    f32x16 s = {};
    // A round asks for later blocks, then sees to its own; whether its steps are full.
    int bad = 0, odd = 0;              // odd: of the stage and the one before
    auto begin_round = [&](int st) {
      fetch(st + lead);
      bad = (int)(bad_ring >> (4 * lead)) & 0xf;
      odd = odd << 1 & 2;
      if (st < stages && unclean(st, bad)) {
        clean(st, bad);
        const int* f = sm_odd + (st & (kStages - 1)) * kStageBlocks;
        odd |= uniform(f[0] | f[1] | f[2] | f[3]) != 0 ? 1 : 0;
      }
      return uniform(bad == 0 && odd == 0 && 2 * st >= full_lo && 2 * st + 1 < full_hi ? 1 : 0) != 0;
    };
    auto end_round = [&](int st) {     // what the round asked for may still be on its way
      wait_loads<D>(st + lead < stages);
      __syncthreads();
    };
    // (loops of their own, so that a path's registers need not be the other's)
    int st = 0;
    bool full = begin_round(0);
    while (st < stages) {
      while (full) {
        f32x16 t;
        full_step(2 * st, s, t);
        full_step(2 * st + 1, t, s);
        end_round(st);
        full = begin_round(++st);
      }
      while (!full && st < stages) {
#pragma unroll 1
        for (int e = 0; e < 2; ++e) step(2 * st + e, (bad >> (2 * e)) & 3, e == 1 ? odd << 1 | (odd & 1) : odd, s);
        end_round(st);
        full = begin_round(++st);
      }
    }
  }
  w.sum += __shfl_xor(w.sum, 32);
  write_columns<D, Out>(a, it, g, wave * kCols, w);
}

__device__ __forceinline__ void put_nan(float* p) { *p = __builtin_nanf(""); }
__device__ __forceinline__ void put_nan(uint16_t* p) { *p = 0x7fc0; }

template <int D, typename Out>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
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
      const Target<Out> t = target_of<D, Out>(a, it, g, e / D);
      put_nan(t.out + e % D);
      if (t.lse && e % D == 0) put_nan(t.lse);
    }
    return;
  }
  if (it.ncols <= kCols) run_narrow<D, Out>(a, h, it, g, smem);
  else run_wide<D, Out>(a, h, it, g, smem);
}

// One workgroup per (split tile, KV head, kCols columns): the ranges in order, two at a
// time, kCols / 8 columns side by side in a thread so that its loads are in flight
// together.
template <int D, typename Out>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptArgs a) {
  constexpr int kSide = kCols * (D / 4) / 256;       // columns of a thread
  const PlanHeader h = *reinterpret_cast<const PlanHeader*>(a.plan);
  const int parts = a.merge_parts;
  const int part = blockIdx.x % parts, u = blockIdx.x / parts;
  const int i = u / a.Hkv, g = u - i * a.Hkv;
  const Merge mg = reinterpret_cast<const Merge*>(a.plan + merges_at(a.max_items))[i];
  if (!plan_fits(a, h) || i >= min(h.n_merges, a.max_merges) || part * kCols >= mg.ncols) return;
  const int d = threadIdx.x % (D / 4) * 4, c0 = part * kCols + threadIdx.x / (D / 4);
  const int64_t at = (int64_t)g * a.part_cols + mg.part;
  int col[kSide];
  float top[kSide], l[kSide] = {};
  float4 acc[kSide];
#pragma unroll
  for (int k = 0; k < kSide; ++k) {
    col[k] = min(c0 + k * (1024 / D), mg.ncols - 1);      // (past the last column it again, not written)
    top[k] = -INFINITY;
    acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  auto range = [&](int s, float2 (&ml)[kSide], float4 (&x)[kSide]) {
#pragma unroll
    for (int k = 0; k < kSide; ++k) {
      const int64_t from = at + (int64_t)s * mg.ncols + col[k];
      ml[k] = *reinterpret_cast<const float2*>(a.part_ml + from * 2);
      x[k] = *reinterpret_cast<const float4*>(a.part_o + from * D + d);
    }
  };
  // (a range of which a column attends nothing has a sum of 0 and any reference)
  auto add = [&](const float2 (&ml)[kSide], const float4 (&x)[kSide]) {
#pragma unroll
    for (int k = 0; k < kSide; ++k) {
      const float to = ml[k].y == 0.f ? top[k] : fmaxf(top[k], ml[k].x);
      const float ref = to == -INFINITY ? 0.f : to;
      const float f0 = weight_of(top[k], ref, a.scale_log2), f1 = ml[k].y == 0.f ? 0.f : weight_of(ml[k].x, ref, a.scale_log2);
      top[k] = to;
      acc[k].x = f0 * acc[k].x + f1 * x[k].x;
      acc[k].y = f0 * acc[k].y + f1 * x[k].y;
      acc[k].z = f0 * acc[k].z + f1 * x[k].z;
      acc[k].w = f0 * acc[k].w + f1 * x[k].w;
      l[k] = f0 * l[k] + f1 * ml[k].y;
    }
  };
  float2 ml0[kSide], ml1[kSide];
  float4 x0[kSide], x1[kSide];
  range(0, ml0, x0);
  for (int s = 0; s < mg.splits; s += 2) {
    if (s + 1 < mg.splits) range(s + 1, ml1, x1);
    add(ml0, x0);
    if (s + 2 < mg.splits) range(s + 2, ml0, x0);
    if (s + 1 < mg.splits) add(ml1, x1);
  }
#pragma unroll
  for (int k = 0; k < kSide; ++k) {
    if (c0 + k * (1024 / D) >= mg.ncols) continue;
    const int fc = mg.col0 + col[k], token = fc / a.G;
    const int64_t row = (int64_t)(mg.row0 + token) * a.Hq + g * a.G + (fc - token * a.G);
    const float inv = inverse_of(l[k]);
    store4(static_cast<Out*>(a.out) + row * D + d, make_float4(acc[k].x * inv, acc[k].y * inv, acc[k].z * inv, acc[k].w * inv));
    if (d == 0 && a.lse) a.lse[row] = lse_of(top[k] == -INFINITY ? 0.f : top[k], l[k], a.scale_log2);
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
  // (narrow tiles are no more than kNarrowItems / Hkv, which is no more than the extra items)
  z->max_items = (int)(std::max<int64_t>(tiles, z->extra_items) + z->extra_items);
  z->max_merges = (int)std::min<int64_t>(cols / kCols + s->batch, z->extra_items);
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
  const int64_t merges = (int64_t)a.max_merges * a.Hkv * a.merge_parts;
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
  a.merge_parts = (int)oda::ceil_div(std::min<int64_t>(kTile, (int64_t)a.R * a.G), kCols);
  a.scale_log2 = in->scale * kLog2e;
  a.lag = std::min(kLag / a.scale_log2, kMaxLag);
  if (out_type == ODA_F32)
    return shape->head_dim == 128 ? launch_attention<128, float>(a, stream) : launch_attention<64, float>(a, stream);
  return shape->head_dim == 128 ? launch_attention<128, uint16_t>(a, stream) : launch_attention<64, uint16_t>(a, stream);
}
