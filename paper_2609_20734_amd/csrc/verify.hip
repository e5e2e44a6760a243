// Verification of drafted tokens (oda_verify_drafts): rejection sampling of a
// draft's tokens against the target's probabilities, by given random numbers.
//
//   p_i = softmax(z_i / T) (T > 0), all mass on the first largest logit else
//   x_i accepted iff u_i q_i(x_i) < p_i(x_i); j = the first refusal, or n
//   next token: inverse CDF of max(p_j - q_j, 0), or of p_n, at u_K
//
// Two launches.  The first reads every row in use once, in splits: the largest
// logit and the sum of exp((z - max) / T) of each.  The second joins a request's
// splits, decides, and, after a refusal, reads the refused row (from cache) and
// its draft row for the weights' sums per split; the last of its workgroups
// finds the split, and then the token, where the cumulative weight passes
// u_K times the whole.  Without a refusal the first launch's sums already are
// the weights' sums, and one workgroup reads one split.
//
// Weights and sums are fp64: the next token has to be the one whose interval
// holds u_K, and a vocabulary of 150,000 tokens has so many borders that fp32
// sums (2^-24 of the whole per border) would put about one draw in a hundred on
// the other side of one.  That makes 30 vector instructions a logit, 20 of them the
// exponential's, which is most of what bounds many rows: 32 requests with four
// drafts, 151,936 tokens, take 42 us, the first launch 25 for 88 MB, 17 of them
// vector work by its counters (at 2.4 GHz), the rest the start and end of workgroups
// of three tiles.  Few rows are bound by the second launch's chain of trips to memory
// (one request: 13.4 us).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <cfloat>
#include <climits>

#include "oda.h"
#include "oda_internal.h"

namespace {

constexpr int kThreads = 512;
constexpr int kPer = 8;                      // logits a thread holds at a time
constexpr int kTile = kThreads * kPer;
constexpr int kMaxSplits = 64;               // splits of a row: one per lane where they are joined
constexpr int kMaxDrafts = 63;
constexpr int kStatGroups = 2048;            // workgroups the launches aim for
constexpr int kDrawGroups = 768;
constexpr double kLog2e = 1.4426950408889634074;

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));   // rows start anywhere

// Largest logit of a split (the first index that holds it) and the sum of its
// weights against that logit.
struct SplitStat {
  double sum;
  float top;
  int32_t first;
};

struct VerifyArgs {
  const float* logits;
  const float* draft_probs;
  const int32_t* draft_tokens;
  const int32_t* n_drafts;
  const float* temperature;
  const float* uniform;
  int32_t* n_accepted;
  int32_t* tokens;
  const int32_t* work_list;
  const int32_t* n_work;
  SplitStat* stats;       // [B][K + 1][splits]
  double* sums;           // [slot][kMaxSplits]: weights of the row that the next token is drawn from
  uint32_t* tickets;      // [slot], zero between calls (slots, as a request may be listed twice)
  int32_t B, K, V;
  int32_t splits, chunk;            // of a row in the first launch
  int32_t draw_splits, draw_chunk;  // of a refused row in the second
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int selected_count(const VerifyArgs& a) {
  return a.n_work ? min(max(a.n_work[0], 0), a.B) : a.B;
}
__device__ __forceinline__ bool selected_request(const VerifyArgs& a, int slot, int& b) {
  if (slot >= selected_count(a)) return false;
  b = uniform(a.work_list ? a.work_list[slot] : slot);
  return b >= 0 && b < a.B;
}
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int b) {
  return a.n_drafts ? min(max(a.n_drafts[b], 0), a.K) : a.K;
}
// log2(e) / temperature, 0 for greedy.  Temperatures count as at most 2^100 and at
// least 2^-100, where logits a step of fp32 apart no longer or fully differ.
__device__ __forceinline__ float temperature_of(const VerifyArgs& a, int b) { return a.temperature ? a.temperature[b] : 1.f; }
__device__ __forceinline__ double slope_of(float t) {
  return t > 0.f ? kLog2e / (double)fminf(fmaxf(t, 0x1p-100f), 0x1p100f) : 0.0;
}

// 2^(x slope) for x <= 0, by 2^k 2^f with |f| <= 1/2: the polynomial through 2^f at
// the eleven Chebyshev nodes of the interval is off by 3.2e-16 of the value at most,
// as much as fp64's own steps (with two terms fewer, off by 1.1e-12, 32 requests took
// 41.0 us instead of 42.2, but a draw's borders moved by as much).  k comes out of
// the low bits of x slope + 1.5 2^52, f keeps all of the product's.  0 below about
// 2^-1000, and for NaN.
__device__ __forceinline__ double exp2_neg(double x, double slope) {
  constexpr double kShift = 6755399441055744.0;
  const double t = fma(x, slope, kShift);
  const double f = fma(x, slope, kShift - t);
  double p = 7.072585949269223e-09;
  p = fma(p, f, 1.0208690299958306e-07);
  p = fma(p, f, 1.321544258792169e-06);
  p = fma(p, f, 1.5252657260200837e-05);
  p = fma(p, f, 0.0001540353044173605);
  p = fma(p, f, 0.0013333558230164974);
  p = fma(p, f, 0.009618129107606888);
  p = fma(p, f, 0.05550410866444772);
  p = fma(p, f, 0.24022650695910097);
  p = fma(p, f, 0.69314718055995);
  p = fma(p, f, 1.0);
  const double e = ldexp(p, (int)(uint32_t)__builtin_bit_cast(uint64_t, t));
  return t >= kShift - 1000.0 ? e : 0.0;
}

// Weights of a row's logits against `top`, its largest (above -infinity): slope =
// log2(e) / temperature.  (The difference first: a logit may be the type's lowest
// value, whose product is off by more than the whole range.)  Weights below about
// 2^-1000 are 0, and so is NaN's.  Where the largest is +infinity it alone weighs.
struct Weights {
  double slope, top;
};
__device__ __forceinline__ Weights weights_against(float top, double slope) { return Weights{slope, (double)top}; }
__device__ __forceinline__ double finite_weight(const Weights& w, float z) {
  return exp2_neg((double)z - w.top, w.slope);
}
__device__ __forceinline__ double weight(const Weights& w, float z) {
  return w.top == (double)INFINITY ? (z == INFINITY ? 1.0 : 0.0) : finite_weight(w, z);
}
// The same for a split's or thread's largest logit against a row's, 0 where it
// holds nothing.
__device__ __forceinline__ double rescale(float m, float top, double slope) {
  return m == top && m != -INFINITY ? 1.0 : weight(weights_against(top, slope), m);
}

// kPer logits of a split from v on, -infinity past its end.
__device__ __forceinline__ void load_tile(const float* row, int v0, int end, int at, float (&z)[kPer]) {
#pragma unroll
  for (int q = 0; q < kPer / 4; ++q) {
    const int v = v0 + (q * kThreads + at) * 4;
    if (v + 4 <= end) {
      const f32x4u w = *reinterpret_cast<const f32x4u*>(row + v);
#pragma unroll
      for (int e = 0; e < 4; ++e) z[4 * q + e] = w[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) z[4 * q + e] = v + e < end ? row[v + e] : -INFINITY;
    }
  }
}

// Reductions over the wavefront in six DPP steps (row shifts by 1, 2, 4, 8, then
// each row's last lane into the next row, then the lower half's into the upper):
// inclusive scans, whose last lane holds the whole.
template <int kCtrl, int kRows>
__device__ __forceinline__ double shifted(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, kCtrl, kRows, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), kCtrl, kRows, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_scan(double x) {
  x += shifted<0x111, 0xf>(x);
  x += shifted<0x112, 0xf>(x);
  x += shifted<0x114, 0xf>(x);
  x += shifted<0x118, 0xf>(x);
  x += shifted<0x142, 0xa>(x);
  x += shifted<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ double lane_value(double x, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x) { return lane_value(wave_scan(x), 63); }
template <int kCtrl, int kRows>
__device__ __forceinline__ float shifted_max(float x) {
  const int none = __builtin_bit_cast(int, -INFINITY);
  return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(none, __builtin_bit_cast(int, x), kCtrl, kRows, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float x) {
  x = shifted_max<0x111, 0xf>(x);
  x = shifted_max<0x112, 0xf>(x);
  x = shifted_max<0x114, 0xf>(x);
  x = shifted_max<0x118, 0xf>(x);
  x = shifted_max<0x142, 0xa>(x);
  x = shifted_max<0x143, 0xc>(x);
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) x = min(x, __shfl_xor(x, s));
  return x;
}

// Launch 1: one workgroup per (split, row of a request).
__global__ __launch_bounds__(kThreads) void verify_stats_kernel(VerifyArgs a) {
  __shared__ float s_top[kThreads / 64];
  __shared__ double s_sum[kThreads / 64];
  __shared__ int s_first[kThreads / 64];
  const int split = blockIdx.x, i = blockIdx.y;
  int b;
  if (!selected_request(a, blockIdx.z, b)) return;
  const int n = drafts_of(a, b);
  const float t = temperature_of(a, b);
  if (i > n) return;
  const double slope = slope_of(t);
  const bool greedy = slope == 0.0;
  const float* row = a.logits + ((int64_t)b * (a.K + 1) + i) * a.V;
  const int begin = min(a.V, split * a.chunk), end = min(a.V, begin + a.chunk);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  float top = -INFINITY;
  double sum = 0.0;
  int first = INT_MAX;
  float next[kPer];
  load_tile(row, begin, end, tid, next);
  for (int v0 = begin; v0 < end; v0 += kTile) {
    float z[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) z[e] = next[e];
    if (v0 + kTile < end) load_tile(row, v0 + kTile, end, tid, next);
    float m = top;
#pragma unroll
    for (int e = 0; e < kPer; ++e) m = fmaxf(m, z[e]);     // passes NaN over
    if (m == -INFINITY) continue;
    if (greedy) {
      if (m > top)
#pragma unroll
        for (int e = kPer - 1; e >= 0; --e)
          if (z[e] == m) first = v0 + ((e / 4) * kThreads + tid) * 4 + e % 4;
    } else {
      if (m > top) sum *= rescale(top, m, slope);
      if (m == INFINITY) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) sum += z[e] == INFINITY ? 1.0 : 0.0;
      } else {
        const Weights w = weights_against(m, slope);
#pragma unroll
        for (int e = 0; e < kPer; ++e) sum += finite_weight(w, z[e]);
      }
    }
    top = m;
  }
  const float wave_top = wave_max(top);
  if (lane == 0) s_top[wave] = wave_top;
  __syncthreads();
  float all = s_top[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) all = fmaxf(all, s_top[w]);
  if (greedy) {
    const int f = wave_min(top == all && all != -INFINITY ? first : INT_MAX);
    if (lane == 0) s_first[wave] = f;
  } else {
    const double s = wave_sum(all == -INFINITY ? 0.0 : sum * rescale(top, all, slope));
    if (lane == 0) s_sum[wave] = s;
  }
  __syncthreads();
  if (tid != 0) return;
  SplitStat out;
  out.top = all;
  out.first = INT_MAX;
  out.sum = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (greedy) out.first = min(out.first, s_first[w]);
    else out.sum += s_sum[w];
  }
  a.stats[((int64_t)b * (a.K + 1) + i) * a.splits + split] = out;
}

// A row's splits joined: lane s holds split s.
struct RowStat {
  float top;        // -infinity: nothing to choose
  double sum;       // of all weights against top
  double part;      // of this lane's split
  int first;        // greedy: the first index of the largest
};
__device__ __forceinline__ SplitStat split_of(const VerifyArgs& a, int b, int i, int lane) {
  SplitStat s;
  s.top = -INFINITY;
  s.sum = 0.0;
  s.first = INT_MAX;
  if (lane < a.splits) s = a.stats[((int64_t)b * (a.K + 1) + i) * a.splits + lane];
  return s;
}
__device__ __forceinline__ RowStat join_row(const SplitStat& s, bool greedy, double slope) {
  RowStat r;
  r.top = wave_max(s.top);
  r.part = r.top == -INFINITY || greedy ? 0.0 : s.sum * rescale(s.top, r.top, slope);
  r.sum = wave_sum(r.part);
  r.first = greedy ? wave_min(s.top == r.top ? s.first : INT_MAX) : INT_MAX;
  return r;
}

// How the next token's weights come from a row: p, or what p has over q.
struct Draw {
  const float* row;
  const float* q;       // the draft's probabilities, or NULL
  int skip;             // a draft that was not drawn: its own weight is 0 (-1: none)
  bool residual;
  Weights w;
  double scale;         // 1 / the row's sum
};

// The weights of N neighbouring tokens from v on (0 past the end).
template <int N>
__device__ __forceinline__ void draw_run(const Draw& d, int v, int end, double (&w)[N]) {
  float z[N], q[N];
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    if (v + e + 4 <= end) {
      const f32x4u t = *reinterpret_cast<const f32x4u*>(d.row + v + e);
      z[e] = t[0], z[e + 1] = t[1], z[e + 2] = t[2], z[e + 3] = t[3];
    } else {
#pragma unroll
      for (int k = e; k < e + 4; ++k) z[k] = v + k < end ? d.row[v + k] : -INFINITY;
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) q[e] = 0.f;
  if (d.residual && d.q != nullptr) {
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      if (v + e + 4 <= end) {
        const f32x4u t = *reinterpret_cast<const f32x4u*>(d.q + v + e);
        q[e] = t[0], q[e + 1] = t[1], q[e + 2] = t[2], q[e + 3] = t[3];
      } else {
#pragma unroll
        for (int k = e; k < e + 4; ++k) q[k] = v + k < end ? d.q[v + k] : 0.f;
      }
    }
  }
  if (d.w.top == (double)INFINITY) {
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = z[e] == INFINITY ? 1.0 : 0.0;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = finite_weight(d.w, z[e]);
  }
  if (d.residual) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      w[e] *= d.scale;
      if (d.q != nullptr) w[e] = fmax(w[e] - (double)fmaxf(q[e], 0.f), 0.0);
      else w[e] = v + e == d.skip ? 0.0 : w[e];
    }
  }
}

// The first token of the split whose cumulative weight, with `below` in front of
// the split, exceeds `goal`; else its last token with a weight (-1: none).  Threads
// take kFind neighbours each, so their sums are in the tokens' order.
constexpr int kFind = 16;
struct FindScratch {
  double sum[kThreads / 64];
  int hit[kThreads / 64], last[kThreads / 64];
};
__device__ __forceinline__ int find_token(const Draw& d, int begin, int end, double below, double goal, FindScratch& sm) {
  constexpr int kWaves = kThreads / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  int last_token = -1;
  for (int v0 = begin; v0 < end; v0 += kThreads * kFind) {
    const int v = v0 + tid * kFind;
    double w[kFind], sum = 0.0;
    draw_run(d, v, end, w);
    int last = -1;
#pragma unroll
    for (int e = 0; e < kFind; ++e) {
      sum += w[e];
      if (w[e] > 0.0) last = v + e;
    }
    const double upto = wave_scan(sum);
    __syncthreads();          // the round before has been read
    if (lane == 63) sm.sum[wave] = upto;
    __syncthreads();
    double base = below, all = below;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const double x = sm.sum[k];
      if (k < wave) base += x;
      all += x;
    }
    below = all;
    // the first lane whose sum passes the goal looks where (by rounding alone: its last)
    const uint64_t past = __ballot(last >= 0 && base + upto > goal), some = __ballot(last >= 0);
    int hit = -1;
    if (past != 0 && lane == __builtin_ctzll(past)) {
      double c = base + (upto - sum);
#pragma unroll
      for (int e = 0; e < kFind; ++e) {
        c += w[e];
        if (hit < 0 && w[e] > 0.0 && c > goal) hit = v + e;
      }
      if (hit < 0) hit = last;
    }
    const int wave_hit = past ? __builtin_amdgcn_readlane(hit, __builtin_ctzll(past)) : -1;
    const int wave_last = some ? __builtin_amdgcn_readlane(last, 63 - __builtin_clzll(some)) : -1;
    if (lane == 0) {
      sm.hit[wave] = wave_hit;
      sm.last[wave] = wave_last;
    }
    __syncthreads();
    int found = -1;
#pragma unroll
    for (int k = kWaves - 1; k >= 0; --k) found = sm.hit[k] >= 0 ? sm.hit[k] : found;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) last_token = max(last_token, sm.last[k]);
    if (found >= 0) return found;
  }
  return last_token;
}

// Split sums pass between workgroups of different XCDs: write-through stores
// and loads past the caches (relaxed, device scope), as the attention's partials.
__device__ __forceinline__ void publish(double* p, double x) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ double published(const double* p) {
  return __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED,
                                                      __HIP_MEMORY_SCOPE_AGENT));
}

// Launch 2: one workgroup per (split of a refused row, request).
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(VerifyArgs a) {
  constexpr int kWaves = kThreads / 64;
  __shared__ double s_sum[kMaxDrafts + 1];
  __shared__ float s_top[kMaxDrafts + 1];
  __shared__ int s_first[kMaxDrafts + 1];
  __shared__ int s_ok[kMaxDrafts + 1], s_token[kMaxDrafts + 1];
  __shared__ double s_scan[kWaves];
  __shared__ FindScratch s_find;
  __shared__ int s_from_p, s_split, s_last;
  __shared__ double s_below, s_goal;
  const int split = blockIdx.x, slot = blockIdx.y;
  int b;
  if (!selected_request(a, slot, b)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int n = drafts_of(a, b);
  const float temperature = temperature_of(a, b);
  const float* u = a.uniform + (int64_t)b * (a.K + 1);
  const float u_next = u[a.K];
  // (the token and number of a wavefront's first row come with the counts)
  const int first = min(wave, a.K);
  int x_i = first < a.K ? a.draft_tokens[(int64_t)b * a.K + first] : -1;
  float u_i = u[first];
  const double slope = slope_of(temperature);
  const bool greedy = slope == 0.0;

  // every row's splits joined, every draft decided (by each workgroup alike)
  for (int i = wave; i <= n; i += kWaves) {
    // the draft's own logit and probability come beside the splits
    const SplitStat s = split_of(a, b, i, lane);
    if (i > wave && i < n) {
      x_i = a.draft_tokens[(int64_t)b * a.K + i];
      u_i = u[i];
    }
    const int x = i < n ? uniform(x_i) : -1;
    const bool known = x >= 0 && x < a.V;
    const float z = known ? a.logits[((int64_t)b * (a.K + 1) + i) * a.V + x] : 0.f;
    const float qx = known && a.draft_probs ? a.draft_probs[((int64_t)b * a.K + i) * a.V + x] : 1.f;
    const RowStat r = join_row(s, greedy, slope);
    if (lane != 0) continue;
    int ok = 0;
    if (known && r.top != -INFINITY) {
      const double p = greedy ? (x == r.first ? 1.0 : 0.0) : weight(weights_against(r.top, slope), z) / r.sum;
      ok = (double)u_i * (double)fmaxf(qx, 0.f) < p ? 1 : 0;
    }
    s_ok[i] = ok;
    s_token[i] = x;
    s_top[i] = r.top;
    s_sum[i] = r.sum;
    s_first[i] = r.first;
  }
  __syncthreads();
  int j = 0;
  while (j < n && s_ok[j] != 0) ++j;
  const bool refused = j < n;
  const float top = s_top[j];
  Draw d;
  d.row = a.logits + ((int64_t)b * (a.K + 1) + j) * a.V;
  d.residual = refused && !greedy;
  d.q = d.residual && a.draft_probs ? a.draft_probs + ((int64_t)b * a.K + j) * a.V : nullptr;
  d.skip = d.residual && !a.draft_probs ? s_token[j] : -1;
  d.w = weights_against(top, slope);
  d.scale = 1.0 / s_sum[j];
  const int begin = min(a.V, split * a.draw_chunk), end = min(a.V, begin + a.draw_chunk);

  const bool summed = d.residual && top != -INFINITY;   // this call sums the weights itself
  if (summed) {
    double sum = 0.0;
    for (int v0 = begin; v0 < end; v0 += kTile) {
      double w[kPer];
      draw_run(d, v0 + tid * kPer, end, w);
#pragma unroll
      for (int e = 0; e < kPer; ++e) sum += w[e];
    }
    sum = wave_sum(sum);
    if (lane == 0) s_scan[wave] = sum;
    __syncthreads();
    if (tid == 0) {
      double all = 0.0;
      for (int w = 0; w < kWaves; ++w) all += s_scan[w];
      publish(a.sums + (int64_t)slot * kMaxSplits + split, all);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (tid == 0) {
      const uint32_t k =
          __builtin_amdgcn_atomic_inc32(a.tickets + slot, (uint32_t)(a.draw_splits - 1), __ATOMIC_RELAXED, "agent");
      s_last = k == (uint32_t)(a.draw_splits - 1) ? 1 : 0;
    }
    __syncthreads();
    if (!s_last) return;
  } else if (split != 0) {
    return;
  }

  int token = -1;
  if (top != -INFINITY && greedy) {
    token = s_first[j];
  } else if (top != -INFINITY) {
    // the split whose interval holds the goal; a residual of nothing draws from p
    if (wave == 0) {
      double part = 0.0, all = 0.0;
      bool from_p = !summed;
      if (summed) {
        if (lane < a.draw_splits) part = published(a.sums + (int64_t)slot * kMaxSplits + lane);
        all = wave_sum(part);
        from_p = !(all > 0.0);
      }
      if (from_p) part = join_row(split_of(a, b, j, lane), false, slope).part;
      const double upto = wave_scan(part);
      const double goal = (double)u_next * lane_value(upto, 63);
      const uint64_t past = __ballot(upto > goal && part > 0.0);
      const uint64_t some = __ballot(part > 0.0);
      const int at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
      if (lane == at) {
        s_split = at;
        s_below = upto - part;
        s_goal = past ? goal : INFINITY;
        s_from_p = from_p ? 1 : 0;
      }
    }
    __syncthreads();
    if (s_from_p) d.residual = false;
    // (a residual's splits are this launch's, p's the first one's)
    const int chunk = d.residual ? a.draw_chunk : a.chunk;
    const int from = s_split * chunk;
    token = find_token(d, min(a.V, from), min(a.V, from + chunk), s_below, s_goal, s_find);
  }
  int32_t* out = a.tokens + (int64_t)b * (a.K + 1);
  for (int i = tid; i <= a.K; i += kThreads)
    out[i] = i < j ? s_token[i] : i == j ? token : -1;
  if (tid == 0) a.n_accepted[b] = j;
}

struct Layout {
  int splits, chunk, draw_splits, draw_chunk;
  size_t off_sums, off_stats, bytes;
};

// Splits of a row into at most kMaxSplits: about `groups` workgroups over `rows`
// rows, of at least a tile (50,257 logits of 64 rows in 13 splits 18 us, in 25 of
// 2,012 logits 21); a split past one takes whole ones.
void split_row(int64_t vocab, int64_t rows, int64_t groups, int* splits, int* chunk) {
  const int64_t most = std::min<int64_t>(kMaxSplits, oda::ceil_div(vocab, kTile));
  const int64_t n = std::min(most, std::max<int64_t>(1, oda::ceil_div(groups, rows)));
  const int64_t c = oda::ceil_div(vocab, n);
  *chunk = (int)oda::round_up(c, c > kTile ? kTile : 4);
  *splits = (int)oda::ceil_div(vocab, *chunk);
}

Layout layout(int64_t batch, int64_t vocab, int64_t max_drafts) {
  Layout l;
  const int64_t rows = batch * (max_drafts + 1);
  split_row(vocab, rows, kStatGroups, &l.splits, &l.chunk);
  split_row(vocab, batch, kDrawGroups, &l.draw_splits, &l.draw_chunk);
  l.off_sums = (size_t)oda::round_up(batch * 4, 256);                     // tickets first
  l.off_stats = l.off_sums + (size_t)oda::round_up(batch * kMaxSplits * 8, 256);
  l.bytes = l.off_stats + (size_t)oda::round_up(rows * kMaxSplits * (int64_t)sizeof(SplitStat), 256);
  return l;
}

oda_status check_sizes(int32_t batch, int32_t vocab, int32_t max_drafts) {
  if (batch < 1 || vocab < 1) return oda::fail(ODA_ERR_SHAPE, "batch and vocab must be >= 1");
  if (vocab > (1 << 30)) return oda::fail(ODA_ERR_SHAPE, "vocab %d too large", vocab);
  if (max_drafts < 0 || max_drafts > kMaxDrafts)
    return oda::fail(ODA_ERR_SHAPE, "max_drafts %d not in 0..%d", max_drafts, kMaxDrafts);
  if (batch > 65535) return oda::fail(ODA_ERR_SHAPE, "batch %d above 65535", batch);
  return ODA_OK;
}

}  // namespace

extern "C" oda_status oda_verify_workspace_size(int32_t batch, int32_t vocab, int32_t max_drafts, size_t* bytes) {
  oda_status st = check_sizes(batch, vocab, max_drafts);
  if (st != ODA_OK) return st;
  if (bytes == nullptr) return oda::fail(ODA_ERR_NULL, "bytes is NULL");
  *bytes = layout(batch, vocab, max_drafts).bytes;
  return oda::ok();
}

extern "C" oda_status oda_verify_drafts(const oda_verify_desc* desc, int32_t batch, int32_t* n_accepted,
                                       int32_t* tokens, const int32_t* work_list, const int32_t* n_work,
                                       void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (desc == nullptr) return oda::fail(ODA_ERR_NULL, "desc is NULL");
  if (!desc->logits || !desc->uniform || !n_accepted || !tokens)
    return oda::fail(ODA_ERR_NULL, "logits, uniform, n_accepted and tokens are required");
  if ((work_list == nullptr) != (n_work == nullptr))
    return oda::fail(ODA_ERR_NULL, "work_list and n_work must both be NULL or both be set");
  oda_status st = check_sizes(batch, desc->vocab, desc->max_drafts);
  if (st != ODA_OK) return st;
  if (desc->max_drafts > 0 && !desc->draft_tokens) return oda::fail(ODA_ERR_NULL, "draft_tokens is required");
  const Layout l = layout(batch, desc->vocab, desc->max_drafts);
  if (workspace == nullptr) return oda::fail(ODA_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", l.bytes);
  if (workspace_bytes < l.bytes)
    return oda::fail(ODA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, l.bytes);
  if (!oda::aligned(workspace, 256)) return oda::fail(ODA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  VerifyArgs a;
  a.logits = desc->logits;
  a.draft_probs = desc->max_drafts > 0 ? desc->draft_probs : nullptr;
  a.draft_tokens = desc->draft_tokens;
  a.n_drafts = desc->n_drafts;
  a.temperature = desc->temperature;
  a.uniform = desc->uniform;
  a.n_accepted = n_accepted;
  a.tokens = tokens;
  a.work_list = work_list;
  a.n_work = n_work;
  a.tickets = static_cast<uint32_t*>(workspace);
  a.sums = reinterpret_cast<double*>(static_cast<char*>(workspace) + l.off_sums);
  a.stats = reinterpret_cast<SplitStat*>(static_cast<char*>(workspace) + l.off_stats);
  a.B = batch;
  a.K = desc->max_drafts;
  a.V = desc->vocab;
  a.splits = l.splits;
  a.chunk = l.chunk;
  a.draw_splits = l.draw_splits;
  a.draw_chunk = l.draw_chunk;
  (void)hipGetLastError();
  hipLaunchKernelGGL(verify_stats_kernel, dim3((unsigned)l.splits, (unsigned)(a.K + 1), (unsigned)batch),
                     dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(verify_draw_kernel, dim3((unsigned)l.draw_splits, (unsigned)batch), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return oda::fail(ODA_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return oda::ok();
}
