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
// the other side of one.  The exponential costs 18 fp64 operations a logit.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <climits>

#include "oda.h"
#include "oda_internal.h"

namespace {

constexpr int kThreads = 512;
constexpr int kPer = 8;                      // logits a thread holds at a time
constexpr int kTile = kThreads * kPer;
constexpr int kMaxSplits = 64;               // splits of a row: one per lane where they are joined
constexpr int kMaxDrafts = 63;
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
  double* sums;           // [B][splits]: weights of the row that the next token is drawn from
  uint32_t* tickets;      // [B], zero between calls
  int32_t B, K, V, splits, chunk;
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
__device__ __forceinline__ double temperature_of(const VerifyArgs& a, int b) {
  return a.temperature ? (double)a.temperature[b] : 1.0;
}

// 2^y for y <= 0 (NaN: 0), by 2^k 2^f with |f| <= 1/2 and the Taylor series of
// e^(f ln 2) to the eleventh power (the next term is below 2^-47 of the value).
// Below 2^-1022 it runs out into subnormals and 0.
__device__ __forceinline__ double exp2_neg(double y) {
  y = fmax(y, -1100.0);
  const double k = rint(y), f = y - k;
  constexpr double c = 0.69314718055994530942;
  constexpr double c2 = c * c, c3 = c2 * c, c4 = c2 * c2, c5 = c4 * c, c6 = c4 * c2, c7 = c4 * c3, c8 = c4 * c4, c9 = c8 * c,
                   c10 = c8 * c2, c11 = c8 * c3;
  double p = c11 / 39916800.0;
  p = fma(p, f, c10 / 3628800.0);
  p = fma(p, f, c9 / 362880.0);
  p = fma(p, f, c8 / 40320.0);
  p = fma(p, f, c7 / 5040.0);
  p = fma(p, f, c6 / 720.0);
  p = fma(p, f, c5 / 120.0);
  p = fma(p, f, c4 / 24.0);
  p = fma(p, f, c3 / 6.0);
  p = fma(p, f, c2 / 2.0);
  p = fma(p, f, c);
  p = fma(p, f, 1.0);
  return ldexp(p, (int)k);
}

// Weights of a row's logits against `top`, its largest (above -infinity): slope =
// log2(e) / temperature.  (The difference first: a logit may be the type's lowest
// value, whose product is off by more than the whole range.)  Where the largest is
// +infinity it alone weighs.
struct Weights {
  double slope, top;
};
__device__ __forceinline__ Weights weights_against(float top, double slope) { return Weights{slope, (double)top}; }
__device__ __forceinline__ double finite_weight(const Weights& w, float z) {
  return exp2_neg(((double)z - w.top) * w.slope);
}
__device__ __forceinline__ double weight(const Weights& w, float z) {
  return w.top == (double)INFINITY ? (z == INFINITY ? 1.0 : 0.0) : finite_weight(w, z);
}
// The same for a split's or thread's largest logit against a row's, 0 where it
// holds nothing.
__device__ __forceinline__ double rescale(float m, float top, double slope) {
  return m == -INFINITY ? 0.0 : m == top ? 1.0 : exp2_neg(((double)m - (double)top) * slope);
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

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) x = fmaxf(x, __shfl_xor(x, s));
  return x;
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
  if (!selected_request(a, blockIdx.z, b) || i > drafts_of(a, b)) return;
  const double t = temperature_of(a, b);
  const bool greedy = !(t > 0.0);
  const double slope = greedy ? 0.0 : kLog2e / t;
  const float* row = a.logits + ((int64_t)b * (a.K + 1) + i) * a.V;
  const int begin = min(a.V, split * a.chunk), end = min(a.V, begin + a.chunk);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  float top = -INFINITY;
  double sum = 0.0;
  int first = INT_MAX;
  for (int v0 = begin; v0 < end; v0 += kTile) {
    float z[kPer];
    load_tile(row, v0, end, tid, z);
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
__device__ __forceinline__ RowStat join_row(const VerifyArgs& a, int b, int i, int lane, bool greedy, double slope) {
  SplitStat s;
  s.top = -INFINITY;
  s.sum = 0.0;
  s.first = INT_MAX;
  if (lane < a.splits) s = a.stats[((int64_t)b * (a.K + 1) + i) * a.splits + lane];
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

// Inclusive sums over the lanes.
__device__ __forceinline__ double wave_scan(double x, int lane) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const double y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  return x;
}

// The weights of kPer neighbouring tokens from v on (0 past the end).
__device__ __forceinline__ void draw_run(const Draw& d, int v, int end, double (&w)[kPer]) {
  float z[kPer], q[kPer];
#pragma unroll
  for (int e = 0; e < kPer; e += 4) {
    if (v + e + 4 <= end) {
      const f32x4u t = *reinterpret_cast<const f32x4u*>(d.row + v + e);
      z[e] = t[0], z[e + 1] = t[1], z[e + 2] = t[2], z[e + 3] = t[3];
    } else {
#pragma unroll
      for (int k = e; k < e + 4; ++k) z[k] = v + k < end ? d.row[v + k] : -INFINITY;
    }
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) q[e] = 0.f;
  if (d.residual && d.q != nullptr) {
#pragma unroll
    for (int e = 0; e < kPer; e += 4) {
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
    for (int e = 0; e < kPer; ++e) w[e] = z[e] == INFINITY ? 1.0 : 0.0;
  } else {
#pragma unroll
    for (int e = 0; e < kPer; ++e) w[e] = finite_weight(d.w, z[e]);
  }
  if (d.residual) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      w[e] *= d.scale;
      if (d.q != nullptr) w[e] = fmax(w[e] - (double)fmaxf(q[e], 0.f), 0.0);
      else w[e] = v + e == d.skip ? 0.0 : w[e];
    }
  }
}

// The first token of the split whose cumulative weight, with `below` in front of
// the split, exceeds `goal`; else its last token with a weight (INT_MAX: none).
// Threads take kPer neighbours each, so their sums are in the tokens' order.
__device__ __forceinline__ int find_token(const Draw& d, int begin, int end, double below, double goal, double* s_scan,
                                          int* s_hit) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) {
    s_hit[0] = INT_MAX;
    s_hit[1] = -1;
  }
  for (int v0 = begin; v0 < end; v0 += kTile) {
    const int v = v0 + tid * kPer;
    double w[kPer], sum = 0.0;
    draw_run(d, v, end, w);
    int last = -1;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      sum += w[e];
      if (w[e] > 0.0) last = v + e;
    }
    const double upto = wave_scan(sum, lane);
    __syncthreads();          // the tile before has been summed up; s_hit is set
    if (lane == 63) s_scan[wave] = upto;
    __syncthreads();
    double base = below;
    for (int k = 0; k < wave; ++k) base += s_scan[k];
    for (int k = 0; k < kThreads / 64; ++k) below += s_scan[k];
    if (last >= 0) {
      atomicMax(&s_hit[1], last);
      if (base + upto > goal) {
        double c = base + (upto - sum);
        int hit = INT_MAX;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          c += w[e];
          if (hit == INT_MAX && w[e] > 0.0 && c > goal) hit = v + e;
        }
        // a thread whose sum passes the goal only by rounding takes its last
        atomicMin(&s_hit[0], hit == INT_MAX ? last : hit);
      }
    }
  }
  __syncthreads();
  return s_hit[0] != INT_MAX ? s_hit[0] : s_hit[1] >= 0 ? s_hit[1] : INT_MAX;
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

// Launch 2: one workgroup per (split, request).
__global__ __launch_bounds__(kThreads) void verify_draw_kernel(VerifyArgs a) {
  constexpr int kWaves = kThreads / 64;
  __shared__ double s_sum[kMaxDrafts + 1];
  __shared__ float s_top[kMaxDrafts + 1];
  __shared__ int s_first[kMaxDrafts + 1];
  __shared__ int s_ok[kMaxDrafts + 1];
  __shared__ double s_scan[kWaves];
  __shared__ int s_hit[2], s_split, s_last;
  __shared__ double s_below, s_goal;
  const int split = blockIdx.x;
  int b;
  if (!selected_request(a, blockIdx.y, b)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const double t = temperature_of(a, b);
  const bool greedy = !(t > 0.0);
  const double slope = greedy ? 0.0 : kLog2e / t;
  const int n = drafts_of(a, b);
  const float* u = a.uniform + (int64_t)b * (a.K + 1);

  // every row's splits joined, every draft decided (by each workgroup alike)
  for (int i = wave; i <= n; i += kWaves) {
    // the draft's own logit and probability come beside the splits
    const int x = i < n ? uniform(a.draft_tokens[(int64_t)b * a.K + i]) : -1;
    const bool known = x >= 0 && x < a.V;
    const float z = known ? a.logits[((int64_t)b * (a.K + 1) + i) * a.V + x] : 0.f;
    const float qx = known && a.draft_probs ? a.draft_probs[((int64_t)b * a.K + i) * a.V + x] : 1.f;
    const RowStat r = join_row(a, b, i, lane, greedy, slope);
    if (lane != 0) continue;
    int ok = 0;
    if (known && r.top != -INFINITY) {
      const double p = greedy ? (x == r.first ? 1.0 : 0.0) : weight(weights_against(r.top, slope), z) / r.sum;
      ok = (double)u[i] * (double)fmaxf(qx, 0.f) < p ? 1 : 0;
    }
    s_ok[i] = ok;
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
  d.skip = d.residual && !a.draft_probs ? a.draft_tokens[(int64_t)b * a.K + j] : -1;
  d.w = weights_against(top, slope);
  d.scale = 1.0 / s_sum[j];
  const int begin = min(a.V, split * a.chunk), end = min(a.V, begin + a.chunk);

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
      publish(a.sums + (int64_t)b * a.splits + split, all);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (tid == 0) {
      const uint32_t k =
          __builtin_amdgcn_atomic_inc32(a.tickets + b, (uint32_t)(a.splits - 1), __ATOMIC_RELAXED, "agent");
      s_last = k == (uint32_t)(a.splits - 1) ? 1 : 0;
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
        if (lane < a.splits) part = published(a.sums + (int64_t)b * a.splits + lane);
        all = wave_sum(part);
        from_p = !(all > 0.0);
      }
      if (from_p) part = join_row(a, b, j, lane, false, slope).part;
      const double upto = wave_scan(part, lane);
      const double goal = (double)u[a.K] * __shfl(upto, 63);
      const uint64_t past = __ballot(upto > goal && part > 0.0);
      const uint64_t some = __ballot(part > 0.0);
      const int at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
      if (lane == at) {
        s_split = at;
        s_below = upto - part;
        s_goal = past ? goal : INFINITY;
        s_hit[0] = from_p ? 1 : 0;
      }
    }
    __syncthreads();
    if (s_hit[0]) d.residual = false;
    const int at = s_split;
    const double below = s_below, goal = s_goal;
    __syncthreads();
    const int v = find_token(d, min(a.V, at * a.chunk), min(a.V, (at + 1) * a.chunk), below, goal, s_scan, s_hit);
    token = v == INT_MAX ? -1 : v;
  }
  int32_t* out = a.tokens + (int64_t)b * (a.K + 1);
  for (int i = tid; i <= a.K; i += kThreads)
    out[i] = i < j ? a.draft_tokens[(int64_t)b * a.K + i] : i == j ? token : -1;
  if (tid == 0) a.n_accepted[b] = j;
}

struct Layout {
  int splits, chunk;
  size_t off_sums, off_stats, bytes;
};

// Splits of a row: enough that the rows' splits cover the chip a few times over,
// of at least 2,048 logits, whole groups of four, at most kMaxSplits.
Layout layout(int64_t batch, int64_t vocab, int64_t max_drafts) {
  Layout l;
  const int64_t rows = batch * (max_drafts + 1);
  const int64_t want = std::max<int64_t>(1, oda::ceil_div(2048, rows));
  const int64_t most = std::min<int64_t>(kMaxSplits, oda::ceil_div(vocab, 2048));
  const int64_t least = std::min<int64_t>(most, oda::ceil_div(vocab, kTile));
  const int64_t n = std::min(most, std::max(want, least));
  l.chunk = (int)std::min<int64_t>(INT_MAX / 2, oda::round_up(oda::ceil_div(vocab, n), 4));
  l.splits = (int)oda::ceil_div(vocab, l.chunk);
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
  (void)hipGetLastError();
  hipLaunchKernelGGL(verify_stats_kernel, dim3((unsigned)l.splits, (unsigned)(a.K + 1), (unsigned)batch),
                     dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(verify_draw_kernel, dim3((unsigned)l.splits, (unsigned)batch), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return oda::fail(ODA_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return oda::ok();
}
