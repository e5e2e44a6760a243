// Decode attention of requests that share a prefix (oda_prefix_plan,
// oda_prefix_decode_attn): the K/V of a group's common blocks is read once for
// all of the group's rows, each request's own blocks once for its rows.
//
// A row is (request, current token); its G query heads of a KV head are G
// columns of a score tile S^T = K Q^T.  Work of one (layer, KV head) unit comes
// in items: a range of blocks against up to 256 columns, either a group's
// (prefix) or one request's (the rest of its history).  An item's eight
// wavefronts form a grid of position ranges times column pairs of tiles; each
// keeps a running maximum and sum per column (one pass over the data) and its
// share of O = P V in registers, and the position ranges are joined in LDS.  An
// item writes an unnormalised partial (m, l, o) per column; the merge joins a
// row's partials of both parts in order and adds the positions that only this
// row or later ones see (the current tokens), one at a time.
//
// The plan (which rows, items and splits) is made on the device from lengths,
// members and flags, by one workgroup, once for all layers of a step.
//
// Bound by HBM where columns are few, by the products and the softmax beside them
// where they are many.  Measured, plan, split and merge together: eight requests
// of two tenants, up to five tokens each, four layers (424 MB) 88 us, the split at
// 6 TB/s; 32 requests behind 16,384 positions, one layer (207 MB) 56 us; 64
// requests of 64 heads behind 65,536 positions, two layers, 485 to 515 us on three
// cards, the split at 1.1 to 1.2 PFLOP/s of products, what a large library product
// reaches.
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
#include "oda_internal.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 16;            // positions per KV block, columns per MFMA tile
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kWaveTiles = 2;         // column tiles a wavefront holds
constexpr int kMaxCols = kWaves * kWaveTiles * kBlock;   // columns of an item
constexpr int kParts = 3;             // bf16 parts of a weight
constexpr int kMaxTokens = 16;
constexpr int kMaxBatch = 2048;       // members and groups that the plan's workgroup holds in LDS
constexpr int kCus = 256;
constexpr int kPlanThreads = 256;
constexpr uint32_t kMagic = 0x0da9f1u;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Plan buffer, int32 words: the header, then a Row per current token of the
// batch, then the items.
struct PlanHeader {
  uint32_t magic;
  int32_t batch, tokens, group, max_blocks, cached, part_cols;   // what the plan was made for
  int32_t n_items, n_rows, n_bad;    // items; rows with work; rows after them that become NaN
  int32_t groups;                    // num_groups, on which the launch's items depend
  int32_t reserved[5];
};
struct Row {
  int32_t id;                        // request * tokens + token
  int32_t len;                       // positions before the row's own: below len for all rows of the request
  int32_t pre_part, pre_splits, pre_stride;   // partial columns of the prefix: head h of split s at part + s * stride + h
  int32_t own_part, own_splits, own_stride;   // of the request's own blocks
};
struct Item {
  int32_t row0;                      // first row of the columns' rows
  int32_t col0, ncols;               // columns: col = row * G + head, counted from row0
  int32_t request;                   // whose block table
  int32_t blk_lo, blk_hi;
  int32_t limit;                     // positions from here on are not attended
  int32_t part;                      // first partial column
};

__host__ __device__ constexpr int rows_at() { return (int)(sizeof(PlanHeader) / 4); }
__host__ __device__ constexpr int items_at(int rows) { return rows_at() + rows * (int)(sizeof(Row) / 4); }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// ---------------------------------------------------------------------------
// the plan
// ---------------------------------------------------------------------------

struct PlanArgs {
  const int32_t* seq_lens;
  const int32_t* group_start;
  const int32_t* members;
  const int32_t* prefix_blocks;
  const int32_t* n_tokens;
  const int32_t* flags;
  int32_t* plan;
  int32_t B, NG, T, G, MB, max_len, cached;   // cached: the current tokens are in the cache
  int32_t units;                              // (layer, KV head) pairs
  int32_t extra_items;                        // items beyond one per piece
  int32_t chunk_cols;                         // columns of a whole prefix item: a multiple of G
  int32_t part_cols;
};

// Cost of an item: blocks times what a block takes, in eighths of the time in
// which one CU's share of HBM delivers it: a tile's products and softmax take
// about an eighth of that, so up to eight tiles are free.
constexpr float kBlockCost = 8.f;
// Start-up, the join and the partial's share of the merge.  The counts of splits that
// it leads to matter more than the figure: over 18 sizes of one to 64 requests the
// mean time at 60, 110, 160, 220, 320 is 41.0, 41.1, 40.7, 41.1, 40.8 us, 32 requests
// behind 16,384 positions 66, 61, 57, 57, 65.
constexpr float kItemCost = 160.f;
constexpr float kLeastCost = 16 * kBlockCost;   // shortest split: two blocks per wavefront

constexpr int kBuckets = 32;

// What the plan holds in LDS per slot (place in `members`), per group and per
// piece of work (the groups' prefixes, then the slots' own blocks).
struct PlanSlot {
  int32_t request;      // -1: not attended
  int32_t tokens;       // rows (0: none)
  int32_t len;          // positions common to the request's rows
  int32_t row;          // first row
  int32_t group;
};
struct PlanGroup {
  int32_t start;        // first slot
  int32_t blocks;       // of the prefix; -1: outside the table
  int32_t leader;       // first slot with rows, whose table is read (INT_MAX: none)
  int32_t row, rows;
  int32_t chunks;       // items side by side that hold its columns
};
struct PlanPiece {
  float cost;           // of one chunk of columns over all blocks (0: no work)
  int32_t splits, item, part;
};
static_assert(kMaxBatch * (sizeof(PlanSlot) + sizeof(PlanGroup) + 2 * sizeof(PlanPiece)) < 158 * 1024, "the plan fits LDS");
__host__ __device__ constexpr size_t plan_lds(int B, int NG) {
  return (size_t)B * sizeof(PlanSlot) + (size_t)(NG + 1) * sizeof(PlanGroup) + (size_t)(B + NG) * sizeof(PlanPiece);
}

__device__ __forceinline__ float piece_cost(int blocks, int cols) {
  return blocks <= 0 ? 0.f : (float)blocks * fmaxf(kBlockCost, (float)((cols + kBlock - 1) / kBlock));
}
// Splits of a piece where an item may cost 1 / inv.
__device__ __forceinline__ int split_count(float cost, float inv) { return cost > 0.f ? max(1, (int)ceilf(cost * inv)) : 0; }
// Blocks per split: even, as blocks are taken in pairs.
__device__ __forceinline__ int split_length(int blocks, int splits) { return ((blocks + splits - 1) / splits + 1) & ~1; }

// Exclusive sums of (x, y) over the workgroup's threads, and the totals.
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

// One workgroup.  Bound by latency: the arrays are asked for together, then the
// phases go through LDS.
__global__ __launch_bounds__(kPlanThreads) void prefix_plan_kernel(PlanArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  PlanSlot* slots = reinterpret_cast<PlanSlot*>(lds);
  PlanGroup* groups = reinterpret_cast<PlanGroup*>(slots + a.B);
  PlanPiece* pieces = reinterpret_cast<PlanPiece*>(groups + a.NG + 1);
  __shared__ int2 s_wave[kPlanThreads / 64];
  __shared__ float s_sum[kPlanThreads / 64], s_most[kPlanThreads / 64];
  __shared__ int s_count[kPlanThreads / 64][64];
  __shared__ int s_bucket[kBuckets];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  PlanHeader* head = reinterpret_cast<PlanHeader*>(a.plan);
  Row* rows = reinterpret_cast<Row*>(a.plan + rows_at());
  Item* items = reinterpret_cast<Item*>(a.plan + items_at(a.B * a.T));

  if (tid < kBuckets) s_bucket[tid] = 0;
  // the first round of members comes with the group arrays
  int member = tid < a.B ? a.members[tid] : -1;
  // group starts, kept in [0, B] and ascending whatever the array holds
  int carry = 0;
  for (int j0 = 0; j0 <= a.NG; j0 += 64) {
    const int j = j0 + lane;
    int start = j <= a.NG ? min(max(a.group_start[j], 0), a.B) : 0;
    const int blocks = j < a.NG ? a.prefix_blocks[j] : 0;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int y = __shfl_up(start, s);
      if (lane >= s) start = max(start, y);
    }
    start = max(start, carry);
    carry = __shfl(start, 63);
    if (wave == 0 && j <= a.NG) {
      groups[j].start = start;
      groups[j].leader = INT_MAX;
      groups[j].blocks = blocks <= a.MB ? blocks : -1;
    }
  }
  __syncthreads();
  const int first = groups[0].start, count = groups[a.NG].start;

  // slots: who attends what; rows in slot order, those that become NaN from the
  // table's end
  int n_rows = 0, n_bad = 0;
  for (int s0 = 0; s0 < count; s0 += kPlanThreads) {
    const int s = s0 + tid;
    PlanSlot p{};
    p.request = -1;
    bool bad = false;
    if (s < count) {
      const int b = s0 == 0 ? member : a.members[s];
      if (s >= first && b >= 0 && b < a.B) {
        const int n = a.seq_lens[b], tokens = a.n_tokens ? a.n_tokens[b] : a.T, flag = a.flags ? a.flags[b] : 1;
        int lo = 0, hi = a.NG;        // the last group that starts at or before s
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (groups[mid].start <= s) lo = mid;
          else hi = mid;
        }
        const int pre = groups[lo].blocks;
        p.group = lo;
        p.request = b;
        p.tokens = flag != 0 ? min(max(tokens, 0), a.T) : 0;
        p.len = a.cached ? n : n - 1;
        bad = p.tokens > 0 && (n < 1 || n > a.max_len || pre < 0 || p.len / kBlock < pre ||
                               (a.cached && n > a.max_len - (p.tokens - 1)));
        if (!bad && p.tokens > 0) atomicMin(&groups[lo].leader, s);
      }
    }
    int2 total;
    const int2 at = block_scan(bad ? make_int2(0, p.tokens) : make_int2(p.tokens, 0), s_wave, total);
    if (bad) {
      for (int t = 0; t < p.tokens; ++t) {
        Row r{};
        r.id = p.request * a.T + t;
        rows[a.B * a.T - 1 - (n_bad + at.y + t)] = r;
      }
      p.tokens = 0;
    }
    p.row = n_rows + at.x;
    n_rows += total.x;
    n_bad += total.y;
    if (s < count) slots[s] = p;
  }
  __syncthreads();

  // pieces and their costs
  const auto own_blocks = [&](const PlanSlot& p) { return (p.len + kBlock - 1) / kBlock - groups[p.group].blocks; };
  float sum = 0.f, most = kLeastCost;
  const int n_pieces = a.NG + count;
  for (int i = tid; i < n_pieces; i += kPlanThreads) {
    PlanPiece p{};
    int chunks = 1;
    if (i < a.NG) {
      const int s0 = groups[i].start, s1 = groups[i + 1].start;
      const int row = s0 < count ? slots[s0].row : n_rows;
      const int n = (s1 < count ? slots[s1].row : n_rows) - row;
      groups[i].row = row;
      groups[i].rows = n;
      groups[i].chunks = chunks = (n * a.G + a.chunk_cols - 1) / a.chunk_cols;
      p.cost = n > 0 ? piece_cost(groups[i].blocks, min(n * a.G, a.chunk_cols)) : 0.f;
    } else if (slots[i - a.NG].tokens > 0) {
      p.cost = piece_cost(own_blocks(slots[i - a.NG]), slots[i - a.NG].tokens * a.G);
    }
    most = fmaxf(most, p.cost);
    sum += p.cost * (float)chunks;
    pieces[i] = p;
  }
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) {
    sum += __shfl_xor(sum, s);
    most = fmaxf(most, __shfl_xor(most, s));
  }
  if (lane == 0) {
    s_sum[wave] = sum;
    s_most[wave] = most;
  }
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    sum += s_sum[w];
    most = fmaxf(most, s_most[w]);
  }

  // what an item may cost: every lane tries one value; the last, with a margin for
  // rounding, splits nothing
  const float t = lane == 63 ? most : kLeastCost * __builtin_amdgcn_exp2f(__log2f(most / kLeastCost) * (float)lane * (1.f / 63.f));
  const float inv = 0.999f / t;
  int n = 0;
#pragma unroll 4
  for (int i = wave; i < n_pieces; i += kPlanThreads / 64) {
    n += split_count(pieces[i].cost, inv) * (i < a.NG ? groups[i].chunks : 1);
  }
  s_count[wave][lane] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) n += s_count[w][lane];
  const int least = __shfl(n, 63);
  float est = (float)a.units * n <= (float)kCus
                  ? t + kItemCost
                  : (float)a.units * (sum + (float)n * kItemCost) * (1.f / (float)kCus) + 0.5f * t;
  if (n - least > a.extra_items) est = INFINITY;
  float best = est;
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) best = fminf(best, __shfl_xor(best, s));
  const uint64_t who = __ballot(est == best);
  const float inv_best = __shfl(inv, who ? 63 - __builtin_clzll(who) : 63);

  // splits, items and partial columns
  int n_items = 0, n_part = 0;
  for (int i0 = 0; i0 < n_pieces; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int splits = 0, cols = 0, chunks = 0, bucket = 0;
    if (i < n_pieces) {
      chunks = i < a.NG ? groups[i].chunks : 1;
      splits = split_count(pieces[i].cost, inv_best);
      cols = (i < a.NG ? groups[i].rows : slots[i - a.NG].tokens) * a.G;
      if (splits > 0) {
        const int blocks = i < a.NG ? groups[i].blocks : own_blocks(slots[i - a.NG]);
        const int length = split_length(blocks, splits);
        splits = (blocks + length - 1) / length;
        const float cost = pieces[i].cost * (float)min(length, blocks) / (float)blocks;
        bucket = min(max((int)((1.f - cost * inv_best) * (float)kBuckets), 0), kBuckets - 1);
        atomicAdd(&s_bucket[bucket], chunks * splits);
      }
    }
    int2 total;
    const int2 at = block_scan(make_int2(chunks * splits, cols * splits), s_wave, total);
    if (i < n_pieces) {
      pieces[i].splits = splits;
      pieces[i].item = n_items + at.x;
      pieces[i].cost = (float)bucket;
      pieces[i].part = n_part + at.y;
    }
    n_items += total.x;
    n_part += total.y;
  }
  // More than one round of items: listed by their cost, the largest first (in
  // kBuckets steps, within one in any order), so that the launch ends evenly (32
  // requests behind 16,384 positions 56.7 us against 60.1; the places cost 0.35).
  if ((int64_t)a.units * n_items > kCus) {
    __syncthreads();
    if (tid < 64) {
      int v = lane < kBuckets ? s_bucket[lane] : 0;
      const int own = v;
#pragma unroll
      for (int s = 1; s < kBuckets; s <<= 1) {
        const int y = __shfl_up(v, s);
        if (lane >= s) v += y;
      }
      if (lane < kBuckets) s_bucket[lane] = v - own;
    }
    __syncthreads();
    for (int i = tid; i < n_pieces; i += kPlanThreads) {
      const PlanPiece p = pieces[i];
      if (p.splits > 0) pieces[i].item = atomicAdd(&s_bucket[(int)p.cost], p.splits * (i < a.NG ? groups[i].chunks : 1));
    }
  }
  __syncthreads();
  for (int j = 0; j < a.NG; ++j) {
    const PlanPiece p = pieces[j];
    if (p.splits == 0) continue;
    const PlanGroup g = groups[j];
    const int cols = g.rows * a.G, length = split_length(g.blocks, p.splits);
    for (int i = tid; i < g.chunks * p.splits; i += kPlanThreads) {
      const int split = i / g.chunks, c = i - split * g.chunks;     // the chunks of a range next to each other
      Item it;
      it.row0 = g.row;
      it.col0 = c * a.chunk_cols;
      it.ncols = min(a.chunk_cols, cols - it.col0);
      it.request = slots[g.leader].request;
      it.blk_lo = split * length;
      it.blk_hi = min(g.blocks, it.blk_lo + length);
      it.limit = g.blocks * kBlock;
      it.part = p.part + it.col0 * p.splits + split * it.ncols;
      items[p.item + i] = it;
    }
  }
  for (int s = first + tid; s < count; s += kPlanThreads) {
    const PlanSlot p = slots[s];
    if (p.tokens <= 0) continue;
    const PlanGroup g = groups[p.group];
    const PlanPiece pre = pieces[p.group], own = pieces[a.NG + s];
    const int cols = p.tokens * a.G;
    const int blocks = own_blocks(p), length = own.splits > 0 ? split_length(blocks, own.splits) : 0;
    for (int i = 0; i < own.splits; ++i) {
      Item it;
      it.row0 = p.row;
      it.col0 = 0;
      it.ncols = cols;
      it.request = p.request;
      it.blk_lo = g.blocks + i * length;
      it.blk_hi = min(g.blocks + blocks, it.blk_lo + length);
      it.limit = p.len;
      it.part = own.part + i * cols;
      items[own.item + i] = it;
    }
    for (int k = 0; k < p.tokens; ++k) {
      Row r;
      r.id = p.request * a.T + k;
      r.len = p.len;
      const int col = (p.row + k - g.row) * a.G, chunk = col / a.chunk_cols * a.chunk_cols;
      r.pre_splits = pre.splits;
      r.pre_stride = min(a.chunk_cols, g.rows * a.G - chunk);
      r.pre_part = pre.part + chunk * pre.splits + (col - chunk);
      r.own_splits = own.splits;
      r.own_stride = cols;
      r.own_part = own.part + k * a.G;
      rows[p.row + k] = r;
    }
  }
  if (tid == 0) {
    PlanHeader h{};
    h.magic = kMagic;
    h.batch = a.B;
    h.tokens = a.T;
    h.group = a.G;
    h.max_blocks = a.MB;
    h.cached = a.cached;
    h.part_cols = a.part_cols;
    h.n_items = n_part <= a.part_cols ? n_items : 0;
    h.n_rows = n_rows;
    h.n_bad = n_bad;
    h.groups = a.NG;
    *head = h;
  }
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------

struct PrefixArgs {
  const uint16_t* q;
  const uint16_t* k_cache;
  const uint16_t* v_cache;
  const int32_t* block_table;
  const uint16_t* k_cur;
  const uint16_t* v_cur;
  const int32_t* plan;
  float* out;
  float* lse;
  float* part_o;      // [units][part_cols][D]
  float* part_ml;     // [units][part_cols][2]  (m: a reference in score units, l)
  int64_t kv_layer_stride;
  int64_t num_blocks;
  int32_t L, B, T, Hq, Hkv, G, MB, NG;
  int32_t part_cols, max_items;
  float scale_log2;   // of a score, for exponents of 2
  float lag;          // kLag in score units
};

__device__ __forceinline__ bool plan_fits(const PrefixArgs& a, const PlanHeader& h) {
  // (no short cuts: each would be a wait of its own)
  return (h.magic == kMagic) & (h.batch == a.B) & (h.tokens == a.T) & (h.group == a.G) & (h.max_blocks == a.MB) &
         (h.cached == (a.k_cur == nullptr ? 1 : 0)) & (h.part_cols == a.part_cols) & (h.groups == a.NG);
}

__device__ __forceinline__ bf16x8 load16(const uint16_t* p) { return *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ u32x2 load8(const uint16_t* p) { return *reinterpret_cast<const u32x2*>(p); }
// blocks of one request's own: read once per call
__device__ __forceinline__ bf16x8 stream16(const uint16_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(p));
}
__device__ __forceinline__ u32x2 stream8(const uint16_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
}
__device__ __forceinline__ bf16x8 cat(u32x2 lo, u32x2 hi) {
  u32x4 t = {lo.x, lo.y, hi.x, hi.y};
  return __builtin_bit_cast(bf16x8, t);
}
// The weight of a score against a reference.  (The difference first: it is exact
// where it matters, also for scores whose product with the scale would be off by
// more than the exponents' range; one fused step instead of two saves 1%.)
__device__ __forceinline__ float weight_of(float s, float ref, float scale_log2) {
  return __builtin_amdgcn_exp2f((s - ref) * scale_log2);
}
__device__ __forceinline__ float bf16_to_float(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
// Register layouts of v_mfma_f32_16x16x32_bf16 and the cache layouts' fit with
// them are those of the decode attention (attention.hip): a K block's 16-byte
// groups are A operands of S^T, the scores come out as the A operand of P V, two
// V blocks are its B.

// A wavefront's share of N column tiles: O = P V (rows: columns 4j..4j+3 of the
// tile, 16 n + h16 the dimension), the reference of column h16's weights (at or
// above its scores; -infinity: none yet) and this lane's part of their
// sum.
template <int D, int N>
struct WaveState {
  f32x4 o[N][D / 16];
  float m[N], l[N];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int c = 0; c < N; ++c) {
      m[c] = -INFINITY;
      l[c] = 0.f;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) o[c][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// The largest over the four lanes that share a column (h16 + 16 j).
__device__ __forceinline__ float column_max(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Two floats to bf16, and what the rounding leaves of them.
__device__ __forceinline__ uint32_t round_pair(float& x, float& y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
  x -= __uint_as_float(w << 16);
  y -= __uint_as_float(w & 0xffff0000u);
  return w;
}

// Scores of 32 positions of column h16 (this lane: 4j.. of either block) into the
// online softmax; p comes back as kParts bf16 parts, which together hold all of a
// weight's 24 bits: two would be off by 2.4e-6 (rms, of a sum of random values),
// three leave the 3e-7 of the exponent's rounding and the sums, for a third more
// products per value.
//
// Weights are taken against the column's reference, kLag above the largest score
// at which it was set and below no later one: weights are at most 1, so that sums
// of weights times values stay where the values do (as with the largest score
// itself), and the sum at 2^-kLag or more.  So the largest score is looked for, and
// sums are rescaled, only where a lane's weights add up to more than 1 or a column
// has no reference yet (its weights come out infinite or NaN): a third fewer vector
// operations per score than with the largest score of every step.  A small lag
// raises references more often, a large one costs the exponents' low bits (two
// layers of 64 requests behind 65,536 positions at 2, 4, 6, 8, 16: 532, 518, 516,
// 517, 515 us on one card; 32 behind 16,384, rms error: 4.0e-7, 4.1e-7, 4.2e-7,
// 4.5e-7, 5.9e-7).
constexpr float kLag = 6.f;
constexpr float kMaxLag = 1e37f;     // (scores of a scale that small all weigh the same)
template <int D>
__device__ __forceinline__ void softmax_tile(const PrefixArgs& a, const f32x4& s0, const f32x4& s1, f32x4 (&o)[D / 16],
                                             float& m, float& l, bf16x8 (&part)[kParts]) {
  float p[8], sum;
  auto weights = [&](float ref) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = weight_of(i < 4 ? s0[i] : s1[i - 4], ref, a.scale_log2);
      sum += p[i];
    }
  };
  weights(m);
  if (__any(!(sum <= 1.f))) {
    float mx = s0[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, i < 4 ? s0[i] : s1[i - 4]);
    const float m_new = fmaxf(m, fminf(column_max(mx) + a.lag, FLT_MAX));
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = weight_of(m, ref, a.scale_log2);
    m = m_new;
    l *= alpha;
    const int j = (threadIdx.x & 63) >> 4;
    float al[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) al[i] = __shfl(alpha, 4 * j + i);
#pragma unroll
    for (int n = 0; n < D / 16; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] *= al[i];
    weights(ref);
  }
  l += sum;
#pragma unroll
  for (int q = 0; q < kParts; ++q) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = round_pair(p[2 * e], p[2 * e + 1]);
    part[q] = __builtin_bit_cast(bf16x8, w);
  }
}

// The last pair of an item may end early: positions from the limit on are not
// attended, nor is the second block of an odd end.  Attended positions of the
// pair whose first block is v:
__device__ __forceinline__ int pair_positions(int v, bool has1, int limit) {
  return (has1 ? limit : min(limit, (v + 1) * kBlock)) - v * kBlock;
}
// room: attended positions from the scores' first on.
__device__ __forceinline__ void mask_scores(int room, f32x4& s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = i < room ? s[i] : -INFINITY;
}
// Unattended slots may hold anything (even NaN): zeroed so that 0 * V stays 0.
__device__ __forceinline__ u32x2 mask_values(int room, u32x2 v) {
  const uint32_t w0 = (room > 0 ? 0x0000FFFFu : 0u) | (room > 1 ? 0xFFFF0000u : 0u);
  const uint32_t w1 = (room > 2 ? 0x0000FFFFu : 0u) | (room > 3 ? 0xFFFF0000u : 0u);
  return u32x2{v.x & w0, v.y & w1};
}

// The queries of a wavefront's column tiles as B operands, in two steps, so that
// the rows' ids and the first table entries come in one trip to memory.
template <int N>
struct QueryRows {
  int id[N], head[N];
  bool in[N];
};
template <int N>
__device__ __forceinline__ void find_rows(const PrefixArgs& a, const Item& it, const Row* rows, int tile0, QueryRows<N>& q) {
  const int h16 = threadIdx.x & 15;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const int col = (tile0 + c) * kBlock + h16;
    q.in[c] = col < it.ncols;
    const int at = q.in[c] ? it.col0 + col : it.col0;
    const int row = at / a.G;
    q.head[c] = at - row * a.G;
    q.id[c] = rows[it.row0 + row].id;
  }
}
template <int D, int N>
__device__ __forceinline__ void load_queries(const PrefixArgs& a, const QueryRows<N>& r, int l, int g,
                                             bf16x8 (&qf)[N][D / 32]) {
  const int j = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const uint16_t* q = a.q + (((int64_t)l * a.B * a.T + r.id[c]) * a.Hq + g * a.G + r.head[c]) * D;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) qf[c][kk] = load16(q + 32 * kk + 8 * j);
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk)
      if (!r.in[c]) qf[c][kk] = bf16x8{};
  }
}

// LDS: the staged blocks of wide items (two stages), or one O tile per wavefront
// where position ranges are joined; then m and l per wavefront and column.
constexpr int kStagePairs = 4;
__host__ __device__ constexpr int block_bytes(int D) { return kBlock * D * 2; }      // of K, of V
__host__ __device__ constexpr int stage_bytes(int D) { return 2 * kStagePairs * 2 * block_bytes(D); }
__host__ __device__ constexpr int lds_bytes(int D) { return 2 * stage_bytes(D) + 2 * kWaves * kWaveTiles * kBlock * 4 + 16; }
static_assert(2 * 2 * kStagePairs * 2 * kBlock * 2 >= kWaves * kBlock * 4, "a tile of O per wavefront fits the stages");
static_assert(2 * kStagePairs == kWaves, "a wavefront stages one block of K and one of V");

// Joins the position ranges (WP of them; wavefront = range * WC + column position)
// of N tiles per column position and writes the partials.
template <int D, int N>
__device__ __forceinline__ void join(const PrefixArgs& a, const Item& it, int l, int g, int wc_shift, WaveState<D, N>& w,
                                     char* smem) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int h16 = lane & 15, j = lane >> 4;
  const int WC = 1 << wc_shift, WP = kWaves >> wc_shift;
  float* sm_o = reinterpret_cast<float*>(smem);                          // [waves][16][D]
  float* sm_m = reinterpret_cast<float*>(smem + 2 * stage_bytes(D));     // [waves][N][16]
  float* sm_l = sm_m + kWaves * kWaveTiles * kBlock;
  if (j == 0) {
#pragma unroll
    for (int c = 0; c < N; ++c) {
      sm_m[(wave * N + c) * kBlock + h16] = w.m[c];
      sm_l[(wave * N + c) * kBlock + h16] = w.l[c];
    }
  }
  const int64_t part0 = ((int64_t)(l * a.Hkv + g)) * a.part_cols + it.part;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    if (c > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* dst = sm_o + (wave * kBlock + 4 * j + i) * D + h16;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) dst[16 * n] = w.o[c][n][i];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < WC * kBlock * D / 2; e += kThreads) {
      const int d = e % (D / 2) * 2, col16 = e / (D / 2) % kBlock, q = e / (D / 2) / kBlock;
      const int col = (q * N + c) * kBlock + col16;
      if (col >= it.ncols) continue;
      float M = -INFINITY;
      for (int p = 0; p < WP; ++p) M = fmaxf(M, sm_m[((p * WC + q) * N + c) * kBlock + col16]);
      const float Mu = M == -INFINITY ? 0.f : M;
      float acc0 = 0.f, acc1 = 0.f, lam = 0.f;
      for (int p = 0; p < WP; ++p) {
        const int wv = p * WC + q;
        const float s = weight_of(sm_m[(wv * N + c) * kBlock + col16], Mu, a.scale_log2);
        const float2 ow = *reinterpret_cast<const float2*>(sm_o + (wv * kBlock + col16) * D + d);
        acc0 += s * ow.x;
        acc1 += s * ow.y;
        lam += s * sm_l[(wv * N + c) * kBlock + col16];
      }
      *reinterpret_cast<float2*>(a.part_o + (part0 + col) * D + d) = make_float2(acc0, acc1);
      if (d == 0) *reinterpret_cast<float2*>(a.part_ml + (part0 + col) * 2) = make_float2(M, lam);
    }
  }
}

// The sums of a column's four lanes; NaN where a table entry was out of range.
template <int D, int N>
__device__ __forceinline__ void finish(WaveState<D, N>& w, bool bad) {
#pragma unroll
  for (int c = 0; c < N; ++c) {
    w.l[c] += __shfl_xor(w.l[c], 16);
    w.l[c] += __shfl_xor(w.l[c], 32);
    if (bad) w.m[c] = w.l[c] = __builtin_nanf("");
  }
}

// Narrow items (one or two column tiles): the wavefronts take contiguous position
// ranges, K and V go straight to registers.
template <int D, int N>
__device__ __forceinline__ void run_narrow(const PrefixArgs& a, const Item& it, const Row* rows, int l, int g, char* smem) {
  constexpr int KK = D / 32, NT = D / 16;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int h16 = lane & 15, j = lane >> 4;
  const int pairs = (it.blk_hi - it.blk_lo + 1) >> 1;
  const int per = (pairs + kWaves - 1) / kWaves;
  const int lo = min(it.blk_hi, it.blk_lo + 2 * per * wave);
  const int hi = min(it.blk_hi, lo + 2 * per);
  WaveState<D, N> w;
  w.clear();
  if (lo < hi) {
    const int64_t base = (int64_t)l * a.kv_layer_stride + (int64_t)g * kBlock * D;
    const uint16_t* kbase = a.k_cache + base + lane * 8;
    const uint16_t* vbase = a.v_cache + base + h16 * kBlock + 4 * j;
    const int32_t* table = a.block_table + (int64_t)it.request * a.MB;
    const int64_t blk_stride = (int64_t)a.Hkv * kBlock * D;
    int tbl = 0, bad = 0, entry = lo + lane < hi ? table[lo + lane] : 0;
    QueryRows<N> qr;
    find_rows<N>(a, it, rows, 0, qr);
    bf16x8 qf[N][KK];
    load_queries<D, N>(a, qr, l, g, qf);
    auto pair = [&](int v, auto masked) {
      constexpr bool kMasked = decltype(masked)::value;
      const int i0 = (v - lo) & 63;
      if (i0 == 0) {
        if (v != lo) entry = v + lane < hi ? table[v + lane] : 0;
        const int e = entry;
        const bool ok = e >= 0 && e < a.num_blocks;
        bad |= ok ? 0 : 1;
        tbl = ok ? e : 0;
      }
      const bool has1 = !kMasked || v + 1 < hi;
      const int64_t pb0 = (int64_t)__builtin_amdgcn_readlane(tbl, i0) * blk_stride;
      const int64_t pb1 = has1 ? (int64_t)__builtin_amdgcn_readlane(tbl, i0 + 1) * blk_stride : pb0;
      bf16x8 ka[KK], kb[KK];
      u32x2 va[NT], vb[NT];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        ka[kk] = stream16(kbase + pb0 + kk * 512);
        kb[kk] = stream16(kbase + pb1 + kk * 512);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        va[n] = stream8(vbase + pb0 + n * kBlock * kBlock);
        vb[n] = stream8(vbase + pb1 + n * kBlock * kBlock);
      }
      const int room = kMasked ? pair_positions(v, has1, it.limit) - 4 * j : 0;
      if (kMasked) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          va[n] = mask_values(room, va[n]);
          vb[n] = mask_values(room - kBlock, vb[n]);
        }
      }
#pragma unroll
      for (int c = 0; c < N; ++c) {
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[kk], qf[c][kk], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb[kk], qf[c][kk], s1, 0, 0, 0);
        }
        if (kMasked) {
          mask_scores(room, s0);
          mask_scores(room - kBlock, s1);
        }
        bf16x8 part[kParts];
        softmax_tile<D>(a, s0, s1, w.o[c], w.m[c], w.l[c], part);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const bf16x8 vf = cat(va[n], vb[n]);
#pragma unroll
          for (int q = 0; q < kParts; ++q)
            w.o[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[q], vf, w.o[c][n], 0, 0, 0);
        }
      }
    };
    int v = lo;
    for (; v + 2 <= hi && (v + 2) * kBlock <= it.limit; v += 2) pair(v, std::false_type{});
    if (v < hi) pair(v, std::true_type{});
    finish<D, N>(w, __any(bad));
  }
  join<D, N>(a, it, l, g, 0, w, smem);
}

// Wide items: K and V are staged through LDS once for all column tiles, eight
// blocks a stage (wavefront i brings block i while the stage before it is used),
// with the positions of K ordered so that operand reads are free of bank
// conflicts.  Up to four tiles: two position ranges, which share a stage's pairs alternately;
// more: every wavefront goes through all pairs with its N tiles.
template <int D, int N>
__device__ __forceinline__ void run_wide(const PrefixArgs& a, const Item& it, const Row* rows, int l, int g, int wc_shift,
                                         char* smem) {
  constexpr int KK = D / 32, NT = D / 16;
  constexpr int kLoads = block_bytes(D) / 1024;      // 16-byte loads of a block per lane
  constexpr int kElems = kBlock * D;                 // of a block
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int h16 = lane & 15, j = lane >> 4;
  const int WP = kWaves >> wc_shift;
  const int wc = wave & ((1 << wc_shift) - 1), wp = wave >> wc_shift;
  int& s_bad = *reinterpret_cast<int*>(smem + lds_bytes(D) - 16);
  if (threadIdx.x == 0) s_bad = 0;
  const bool active = wc * N * kBlock < it.ncols;
  WaveState<D, N> w;
  w.clear();

  const int64_t base = (int64_t)l * a.kv_layer_stride + (int64_t)g * kElems;
  // staged slot lane % 16 of a 16-position row of K holds position (bits 0, 1, 3, 2 of the slot)
  const int k_lane = ((lane & 48) | (lane & 3) | ((lane & 4) << 1) | ((lane & 8) >> 1)) * 8;
  const int32_t* table = a.block_table + (int64_t)it.request * a.MB + it.blk_lo + wave;
  const int64_t blk_stride = (int64_t)a.Hkv * kElems;
  const int blocks = it.blk_hi - it.blk_lo;
  const int stages = (blocks + kWaves - 1) / kWaves;
  int tbl = 0, bad = 0, entry = lane * kWaves + wave < blocks ? table[lane * kWaves] : 0;
  QueryRows<N> qr;
  find_rows<N>(a, it, rows, wc * N, qr);
  bf16x8 qf[N][KK];
  load_queries<D, N>(a, qr, l, g, qf);
  bf16x8 kr[kLoads], vr[kLoads];
  // a stage's block of this wavefront; past the end the cache's first (masked, and zeroed where V is used)
  auto fetch = [&](int st) {
    if ((st & 63) == 0) {
      if (st > 0) entry = (st + lane) * kWaves + wave < blocks ? table[(st + lane) * kWaves] : 0;
      const int e = entry;
      const bool ok = e >= 0 && e < a.num_blocks;
      bad |= ok ? 0 : 1;
      tbl = ok ? e : 0;
    }
    const int64_t pb = (int64_t)__builtin_amdgcn_readlane(tbl, st & 63) * blk_stride + base;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      kr[i] = load16(a.k_cache + pb + k_lane + i * 512);
      vr[i] = load16(a.v_cache + pb + lane * 8 + i * 512);
    }
  };
  uint16_t* lds = reinterpret_cast<uint16_t*>(smem);
  auto put = [&](int st) {      // stage: K blocks, then V blocks
    uint16_t* dst = lds + (st & 1) * (stage_bytes(D) / 2) + wave * kElems + lane * 8;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      *reinterpret_cast<bf16x8*>(dst + i * 512) = kr[i];
      *reinterpret_cast<bf16x8*>(dst + kWaves * kElems + i * 512) = vr[i];
    }
  };
  // One pair of staged blocks against the N tiles.  Row 4a + i of the first score
  // tile is position 8a + i of the pair's 32, of the second 8a + 4 + i, so that lane
  // j's scores are eight neighbours and V comes in one 16-byte read; the staged
  // slots put the first tile's rows of a block in front of the second's.
  const int k_at = (h16 >> 3) * kElems + (j * kBlock + (h16 & 7)) * 8;
  const int v_at = (kWaves + (j >> 1)) * kElems + h16 * kBlock + 8 * (j & 1);
  auto pair = [&](const uint16_t* k0, const uint16_t* v0, int room, auto masked) {
    constexpr bool kMasked = decltype(masked)::value;
    f32x4 s0[N], s1[N];
#pragma unroll
    for (int c = 0; c < N; ++c) s0[c] = s1[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const bf16x8 ka = load16(k0 + kk * 512), kb = load16(k0 + kk * 512 + 8 * 8);
#pragma unroll
      for (int c = 0; c < N; ++c) {
        s0[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[c][kk], s0[c], 0, 0, 0);
        s1[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qf[c][kk], s1[c], 0, 0, 0);
      }
    }
    bf16x8 part[N][kParts];
#pragma unroll
    for (int c = 0; c < N; ++c) {
      if (kMasked) {
        mask_scores(room, s0[c]);
        mask_scores(room - 4, s1[c]);
      }
      softmax_tile<D>(a, s0[c], s1[c], w.o[c], w.m[c], w.l[c], part[c]);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      bf16x8 vf = load16(v0 + n * kBlock * kBlock);
      if (kMasked) {
        const u32x4 q = __builtin_bit_cast(u32x4, vf);
        vf = cat(mask_values(room, u32x2{q.x, q.y}), mask_values(room - 4, u32x2{q.z, q.w}));
      }
#pragma unroll
      for (int c = 0; c < N; ++c)
#pragma unroll
        for (int q = 0; q < kParts; ++q)
          w.o[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[c][q], vf, w.o[c][n], 0, 0, 0);
    }
  };
  fetch(0);
  put(0);
  if (stages > 1) fetch(1);
  __syncthreads();
  for (int st = 0; st < stages; ++st) {
    if (active) {
      const uint16_t* stage = lds + (st & 1) * (stage_bytes(D) / 2);
      for (int pr = wp; pr < kStagePairs; pr += WP) {
        const int v = it.blk_lo + st * kWaves + 2 * pr;
        if (v >= it.blk_hi) break;
        if (v + 2 > it.blk_hi || (v + 2) * kBlock > it.limit) break;   // the last pair, below
        pair(stage + k_at + 2 * pr * kElems, stage + v_at + 2 * pr * kElems, 0, std::false_type{});
      }
    }
    // the other buffer was last read before the barrier that ended the stage before
    if (st + 1 < stages) {
      put(st + 1);
      if (st + 2 < stages) fetch(st + 2);
    }
    __syncthreads();
  }
  // a last pair that ends early, still staged: its range's wavefronts
  const int v_last = it.blk_lo + (blocks - 1) / 2 * 2, pr_last = (blocks - 1) / 2 % kStagePairs;
  if (active && (pr_last & (WP - 1)) == wp && (v_last + 2 > it.blk_hi || (v_last + 2) * kBlock > it.limit)) {
    const uint16_t* stage = lds + ((stages - 1) & 1) * (stage_bytes(D) / 2);
    pair(stage + k_at + 2 * pr_last * kElems, stage + v_at + 2 * pr_last * kElems,
         pair_positions(v_last, v_last + 1 < it.blk_hi, it.limit) - 8 * j, std::true_type{});
  }
  if (bad) s_bad = 1;
  __syncthreads();
  finish<D, N>(w, s_bad != 0);
  if (wc_shift != 3) {
    join<D, N>(a, it, l, g, wc_shift, w, smem);
    return;
  }
  // one position range: the partials straight from the registers
  const int64_t part0 = ((int64_t)(l * a.Hkv + g)) * a.part_cols + it.part;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const int col0 = (wc * N + c) * kBlock;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (col0 + 4 * j + i >= it.ncols) continue;
      float* dst = a.part_o + (part0 + col0 + 4 * j + i) * D + h16;
#pragma unroll
      for (int n = 0; n < NT; ++n) dst[16 * n] = w.o[c][n][i];
    }
    if (j == 0 && col0 + h16 < it.ncols)
      *reinterpret_cast<float2*>(a.part_ml + (part0 + col0 + h16) * 2) =
          make_float2(w.m[c], w.l[c]);
  }
}

template <int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void prefix_split_kernel(PrefixArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const PlanHeader h = *reinterpret_cast<const PlanHeader*>(a.plan);
  const int units = a.L * a.Hkv;
  const int i = blockIdx.x / units, u = blockIdx.x - i * units;
  const Row* rows = reinterpret_cast<const Row*>(a.plan + rows_at());
  // (asked for with the header: the grid has no more than the buffer's items; none
  // has no columns, so the item is read before the branch)
  const Item it = reinterpret_cast<const Item*>(a.plan + items_at(a.B * a.T))[i];
  if (!plan_fits(a, h) | (i >= min(h.n_items, a.max_items)) | (it.ncols <= 0)) return;
  const int l = u / a.Hkv, g = u - l * a.Hkv;
  const int tiles = (it.ncols + kBlock - 1) / kBlock;
  if (tiles == 1) run_narrow<D, 1>(a, it, rows, l, g, smem);
  else if (tiles == 2) run_narrow<D, 2>(a, it, rows, l, g, smem);
  else if (tiles <= kWaves) run_wide<D, 1>(a, it, rows, l, g, tiles <= 4 ? 2 : 3, smem);
  else run_wide<D, 2>(a, it, rows, l, g, 3, smem);
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) x = fmaxf(x, __shfl_xor(x, s));
  return x;
}

// One wavefront per (layer, row, query head): the prefix's partials, the own
// blocks' partials, then the current tokens up to the row's own.  The weights of
// up to 64 partials are formed side by side, one per lane, and the partials read
// kMergeLoads at a time.
constexpr int kMergeLoads = 8;
template <int D>
__global__ __launch_bounds__(256) void prefix_merge_kernel(PrefixArgs a) {
  constexpr int PD = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6);
  const int64_t per_layer = (int64_t)a.B * a.T * a.Hq;
  const int l = (int)(wave / per_layer);
  if (l >= a.L) return;
  const int rest = (int)(wave - l * per_layer);
  const int r = rest / a.Hq, head = rest - r * a.Hq;
  const PlanHeader h = *reinterpret_cast<const PlanHeader*>(a.plan);
  const Row* rows = reinterpret_cast<const Row*>(a.plan + rows_at());
  const int all = a.B * a.T;
  const Row row = rows[r];
  const bool fits = plan_fits(a, h);        // (else a plan of other sizes, or none)
  const bool has = r < h.n_rows, spoiled = r >= all - h.n_bad;
  // (a planned row's id is never negative: read before the branch)
  if (fits & ((!has & !spoiled) | (row.id < 0))) return;
  const int64_t id = fits ? row.id : r;
  const bool nan = !fits | !has;
  float* out = a.out + (((int64_t)l * all + id) * a.Hq + head) * D + lane * PD;
  float* lse = a.lse ? a.lse + ((int64_t)l * all + id) * a.Hq + head : nullptr;
  if (nan) {
#pragma unroll
    for (int e = 0; e < PD; ++e) out[e] = __builtin_nanf("");
    if (lse && lane == 0) *lse = __builtin_nanf("");
    return;
  }
  const int g = head / a.G, hh = head - g * a.G;
  const int64_t part0 = (int64_t)(l * a.Hkv + g) * a.part_cols + hh;
  const int b = (int)(id / a.T), t = (int)(id - (int64_t)b * a.T);
  float q[PD];
#pragma unroll
  for (int e = 0; e < PD; ++e) q[e] = bf16_to_float(a.q[(((int64_t)l * all + id) * a.Hq + head) * D + lane * PD + e]);

  // the current tokens this row attends: candidates, or the cache's last positions;
  // the first one's values are asked for before the partials, each next one's
  // before one is used
  const int more = a.k_cur ? t + 1 : t;
  float k_next[PD] = {}, v_next[PD] = {};
  bool bad = false;
  auto fetch = [&](int i) {
    if (a.k_cur) {
      const int64_t at = ((((int64_t)l * a.B + b) * a.T + i) * a.Hkv + g) * D + lane * PD;
#pragma unroll
      for (int e = 0; e < PD; ++e) {
        k_next[e] = bf16_to_float(a.k_cur[at + e]);
        v_next[e] = bf16_to_float(a.v_cur[at + e]);
      }
    } else {
      const int pos = row.len + i;          // below the table's end: the plan checked the length
      const int blk = a.block_table[(int64_t)b * a.MB + pos / kBlock];
      if (blk < 0 || blk >= a.num_blocks) {
        bad = true;
        return;
      }
      const int64_t at = (int64_t)l * a.kv_layer_stride + ((int64_t)blk * a.Hkv + g) * kBlock * D;
#pragma unroll
      for (int e = 0; e < PD; ++e) {
        const int d = lane * PD + e;
        k_next[e] = bf16_to_float(a.k_cache[at + ((d / 8) * kBlock + pos % kBlock) * 8 + d % 8]);
        v_next[e] = bf16_to_float(a.v_cache[at + d * kBlock + pos % kBlock]);
      }
    }
  };
  if (more > 0) fetch(0);

  float M = -INFINITY, sum = 0.f, o[PD] = {};
  // weights against a new largest logit
  auto rescale = [&](float m) {
    const float top = fmaxf(M, m);
    const float s = M == -INFINITY ? 0.f : weight_of(M, top, a.scale_log2);
    sum *= s;
#pragma unroll
    for (int e = 0; e < PD; ++e) o[e] *= s;
    M = top;
  };
  const int splits = row.pre_splits + row.own_splits;
  auto column = [&](int s) {
    return part0 + (s < row.pre_splits ? row.pre_part + (int64_t)s * row.pre_stride
                                       : row.own_part + (int64_t)(s - row.pre_splits) * row.own_stride);
  };
  for (int s0 = 0; s0 < splits; s0 += 64) {
    const int n = min(64, splits - s0);
    float m = -INFINITY, part = 0.f;
    if (lane < n) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + column(s0 + lane) * 2);
      m = ml.x;
      part = ml.y;
    }
    float po[kMergeLoads][PD];
    auto load = [&](int k0) {
#pragma unroll
      for (int k = 0; k < kMergeLoads; ++k) {
        const float* p = a.part_o + column(s0 + min(k0 + k, n - 1)) * D + lane * PD;
#pragma unroll
        for (int e = 0; e < PD; ++e) po[k][e] = p[e];
      }
    };
    load(0);
    rescale(wave_max(m));
    const float w = weight_of(m, M == -INFINITY ? 0.f : M, a.scale_log2);    // NaN of a bad entry stays
    sum += wave_sum(lane < n ? w * part : 0.f);
    for (int k0 = 0; k0 < n; k0 += kMergeLoads) {
      if (k0 > 0) load(k0);
#pragma unroll
      for (int k = 0; k < kMergeLoads; ++k) {
        const float wk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), (k0 + k) & 63));
        if (k0 + k < n)
#pragma unroll
          for (int e = 0; e < PD; ++e) o[e] += wk * po[k][e];
      }
    }
  }
  for (int i = 0; i < more; ++i) {
    float kd[PD], vd[PD], dot = 0.f;
#pragma unroll
    for (int e = 0; e < PD; ++e) {
      kd[e] = k_next[e];
      vd[e] = v_next[e];
    }
    if (i + 1 < more) fetch(i + 1);
#pragma unroll
    for (int e = 0; e < PD; ++e) dot += q[e] * kd[e];
    dot = wave_sum(dot);
    rescale(dot);
    const float w = weight_of(dot, M == -INFINITY ? 0.f : M, a.scale_log2);
    sum += w;
#pragma unroll
    for (int e = 0; e < PD; ++e) o[e] += w * vd[e];
  }
  if (bad) sum = __builtin_nanf("");
#pragma unroll
  for (int e = 0; e < PD; ++e) out[e] = o[e] / sum;
  if (lse && lane == 0) *lse = (M * a.scale_log2 + __log2f(sum)) * kLn2;
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

// Sizes that host and plan agree on.  Items beyond one per piece fill the CUs
// twice; each of them has at most kMaxCols partial columns, and no more than the
// batch has.
struct Sizes {
  int group, chunk_cols, extra_items, part_cols, max_items;
  size_t plan_bytes, off_ml, ws_bytes;
};

oda_status sizes_of(const oda_attn_shape* s, const oda_prefix_groups* p, Sizes* z) {
  if (s == nullptr) return oda::fail(ODA_ERR_NULL, "shape is NULL");
  if (p == nullptr) return oda::fail(ODA_ERR_NULL, "groups is NULL");
  size_t unused = 0;
  const oda_status st = oda_attn_workspace_size(s, 0, 0, &unused);   // the shape's own checks
  if (st != ODA_OK) return st;
  if (s->split_blocks != 0) return oda::fail(ODA_ERR_SHAPE, "split_blocks must be 0 (the plan chooses)");
  if (p->tokens < 1 || p->tokens > kMaxTokens) return oda::fail(ODA_ERR_SHAPE, "tokens %d not in 1..%d", p->tokens, kMaxTokens);
  if (p->num_groups < 1 || p->num_groups > kMaxBatch)
    return oda::fail(ODA_ERR_SHAPE, "num_groups %d not in 1..%d", p->num_groups, kMaxBatch);
  if (s->batch > kMaxBatch) return oda::fail(ODA_ERR_UNSUPPORTED, "batch %d above %d", s->batch, kMaxBatch);
  const int64_t units = (int64_t)s->num_layers * s->num_kv_heads;
  z->group = s->num_q_heads / s->num_kv_heads;
  z->chunk_cols = kMaxCols / z->group * z->group;
  const int64_t cols = (int64_t)s->batch * p->tokens * z->group;
  z->extra_items = (int)oda::ceil_div(2 * kCus, units);
  z->part_cols = (int)(2 * cols + (int64_t)z->extra_items * std::min<int64_t>(kMaxCols, cols));
  z->max_items = (int)(s->batch + std::min<int64_t>(p->num_groups, s->batch) + cols / z->chunk_cols + z->extra_items);
  z->plan_bytes = (size_t)oda::round_up(
      (items_at(s->batch * p->tokens) + (int64_t)z->max_items * (int64_t)(sizeof(Item) / 4)) * 4, 256);
  z->off_ml = (size_t)oda::round_up(units * z->part_cols * s->head_dim * 4, 256);
  z->ws_bytes = z->off_ml + (size_t)oda::round_up(units * z->part_cols * 8, 256);
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

template <int D>
oda_status launch_attention(const PrefixArgs& a, hipStream_t stream) {
  const int64_t items = (int64_t)a.max_items * a.L * a.Hkv;
  const int64_t merges = oda::ceil_div((int64_t)a.L * a.B * a.T * a.Hq, 4);
  if (items > INT_MAX || merges > INT_MAX) return oda::fail(ODA_ERR_SHAPE, "grid too large");
  const int lds = lds_bytes(D);
  static std::atomic<uint64_t> raised{0};
  raise_lds_limit(reinterpret_cast<const void*>(prefix_split_kernel<D>), &raised, lds);
  (void)hipGetLastError();
  hipLaunchKernelGGL(prefix_split_kernel<D>, dim3((unsigned)items), dim3(kThreads), lds, stream, a);
  hipLaunchKernelGGL(prefix_merge_kernel<D>, dim3((unsigned)merges), dim3(256), 0, stream, a);
  return launch_status();
}

}  // namespace

extern "C" oda_status oda_prefix_plan_size(const oda_attn_shape* shape, const oda_prefix_groups* groups, size_t* bytes) {
  Sizes z;
  const oda_status st = sizes_of(shape, groups, &z);
  if (st != ODA_OK) return st;
  if (bytes == nullptr) return oda::fail(ODA_ERR_NULL, "bytes is NULL");
  *bytes = z.plan_bytes;
  return oda::ok();
}

extern "C" oda_status oda_prefix_workspace_size(const oda_attn_shape* shape, const oda_prefix_groups* groups,
                                               size_t* bytes) {
  Sizes z;
  const oda_status st = sizes_of(shape, groups, &z);
  if (st != ODA_OK) return st;
  if (bytes == nullptr) return oda::fail(ODA_ERR_NULL, "bytes is NULL");
  *bytes = z.ws_bytes;
  return oda::ok();
}

extern "C" oda_status oda_prefix_plan(const oda_attn_shape* shape, const oda_attn_inputs* in,
                                     const oda_prefix_groups* groups, void* plan, size_t plan_bytes, hipStream_t stream) {
  Sizes z;
  oda_status st = sizes_of(shape, groups, &z);
  if (st != ODA_OK) return st;
  if (in == nullptr) return oda::fail(ODA_ERR_NULL, "inputs is NULL");
  if (!in->seq_lens || !groups->group_start || !groups->members || !groups->prefix_blocks)
    return oda::fail(ODA_ERR_NULL, "seq_lens, group_start, members and prefix_blocks are required");
  if ((in->k_cur == nullptr) != (in->v_cur == nullptr))
    return oda::fail(ODA_ERR_NULL, "k_cur and v_cur must both be NULL or both be set");
  st = check_buffer("plan", plan, plan_bytes, z.plan_bytes);
  if (st != ODA_OK) return st;
  PlanArgs a;
  a.seq_lens = in->seq_lens;
  a.group_start = groups->group_start;
  a.members = groups->members;
  a.prefix_blocks = groups->prefix_blocks;
  a.n_tokens = groups->n_tokens;
  a.flags = groups->flags;
  a.plan = static_cast<int32_t*>(plan);
  a.B = shape->batch;
  a.NG = groups->num_groups;
  a.T = groups->tokens;
  a.G = z.group;
  a.MB = shape->max_blocks_per_seq;
  a.max_len = shape->max_seq_len;
  a.cached = in->k_cur == nullptr ? 1 : 0;
  a.units = shape->num_layers * shape->num_kv_heads;
  a.extra_items = z.extra_items;
  a.chunk_cols = z.chunk_cols;
  a.part_cols = z.part_cols;
  const int lds = (int)plan_lds(a.B, a.NG);
  static std::atomic<uint64_t> raised{0};
  raise_lds_limit(reinterpret_cast<const void*>(prefix_plan_kernel), &raised, (int)plan_lds(kMaxBatch, kMaxBatch));
  (void)hipGetLastError();
  hipLaunchKernelGGL(prefix_plan_kernel, dim3(1), dim3(kPlanThreads), lds, stream, a);
  return launch_status();
}

extern "C" oda_status oda_prefix_decode_attn(const oda_attn_shape* shape, const oda_attn_inputs* in,
                                            const oda_prefix_groups* groups, const void* plan, size_t plan_bytes,
                                            float* out, float* lse, void* workspace, size_t workspace_bytes,
                                            hipStream_t stream) {
  Sizes z;
  oda_status st = sizes_of(shape, groups, &z);
  if (st != ODA_OK) return st;
  if (in == nullptr) return oda::fail(ODA_ERR_NULL, "inputs is NULL");
  if (!in->q || !in->k_cache || !in->v_cache || !in->block_table || !out)
    return oda::fail(ODA_ERR_NULL, "q, k_cache, v_cache, block_table and out are required");
  if ((in->k_cur == nullptr) != (in->v_cur == nullptr))
    return oda::fail(ODA_ERR_NULL, "k_cur and v_cur must both be NULL or both be set");
  if (!oda::aligned(in->q, 16) || !oda::aligned(in->k_cache, 16) || !oda::aligned(in->v_cache, 16) ||
      !oda::aligned(out, 16) || (in->k_cur && (!oda::aligned(in->k_cur, 16) || !oda::aligned(in->v_cur, 16))))
    return oda::fail(ODA_ERR_SHAPE, "q, caches, k_cur, v_cur and out must be 16-byte aligned");
  if (!(in->scale > 0.f) || !std::isfinite(in->scale)) return oda::fail(ODA_ERR_SHAPE, "scale must be finite and > 0");
  st = check_buffer("plan", plan, plan_bytes, z.plan_bytes);
  if (st != ODA_OK) return st;
  st = check_buffer("workspace", workspace, workspace_bytes, z.ws_bytes);
  if (st != ODA_OK) return st;
  PrefixArgs a;
  a.q = in->q;
  a.k_cache = in->k_cache;
  a.v_cache = in->v_cache;
  a.block_table = in->block_table;
  a.k_cur = in->k_cur;
  a.v_cur = in->v_cur;
  a.plan = static_cast<const int32_t*>(plan);
  a.out = out;
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + z.off_ml);
  a.kv_layer_stride = shape->layer_stride_kv != 0
                          ? shape->layer_stride_kv
                          : shape->num_blocks * shape->num_kv_heads * kBlock * shape->head_dim;
  a.num_blocks = shape->num_blocks;
  a.L = shape->num_layers;
  a.B = shape->batch;
  a.T = groups->tokens;
  a.Hq = shape->num_q_heads;
  a.Hkv = shape->num_kv_heads;
  a.G = z.group;
  a.MB = shape->max_blocks_per_seq;
  a.NG = groups->num_groups;
  a.part_cols = z.part_cols;
  a.max_items = z.max_items;
  a.scale_log2 = in->scale * kLog2e;
  a.lag = std::min(kLag / a.scale_log2, kMaxLag);
  return shape->head_dim == 128 ? launch_attention<128>(a, stream) : launch_attention<64>(a, stream);
}
