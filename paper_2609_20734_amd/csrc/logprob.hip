// Log probabilities of given tokens, entropy and the most probable alternatives
// (oda_token_logprobs).  With m the row's largest logit:
//
//   S = sum e^(z - m), T = sum e^(z - m) (m - z)
//   log p(v) = z_v - m - log S,   H = log S + T / S   (every term >= 0: nothing cancels)
//
// One pass over the logits with a running m, S and T per lane; the place of the given
// token is counted and the first k tokens are kept on the way.  A row is split over
// workgroups where rows are few; the last of a row's workgroups joins them.
//
// Many rows are bound by HBM and, close behind, the vector operations (four bytes and
// about a dozen instructions a logit): 1,024 rows of 50,257 with five alternatives in
// 48.8 us, 4.2 TB/s.  Few rows are bound by one chain: four of 151,936 with twenty take
// 12.4 us, of which a wavefront's logits and first places take 5, the joins 3, the trips
// between workgroups 2.5, start and end 2 (without alternatives 6.6).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <climits>

#include "oda.h"
#include "oda_device.h"
#include "oda_internal.h"

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kLoads = 4;                     // 16-byte loads of a lane's batch
constexpr int kBatch = 64 * 4 * kLoads;       // logits of a wavefront's batch
constexpr int kMaxTop = ODA_MAX_TOP;
constexpr int kMaxSplits = 64;                // of a row: one per lane where they are joined
constexpr int kTickets = 1024;                // rows that may be split
constexpr int kTicketStride = 32;             // words: a cache line each (side by side: sixteen rows of 151,936 12.2 us against 8.6)
constexpr int kGroups = 1024;                 // workgroups that split rows make at most
constexpr int kLeastSplit = kWaves * kBatch / 2;  // (half and twice of it: 10% slower for four rows of 151,936)
constexpr int kRun = 64;                      // runs of wavefronts are multiples of it
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFar = 1e30f;                 // stands for an infinite distance (its weight is 0)

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));   // rows start anywhere

struct LogprobArgs {
  const float* logits;
  const int32_t* tokens;
  float* logprob;
  int32_t* rank;
  float* entropy;
  float* top_logprobs;
  int32_t* top_tokens;
  const int32_t* work_list;
  const int32_t* n_work;
  uint32_t* tickets;       // [kTickets][kTicketStride], zero between calls
  uint64_t* parts;         // [slot][splits][2 + top]: (m, S), (T, ahead), then (logit, token)
  int64_t stride;
  int32_t R, V, top, splits, chunk;
  uint32_t top_inv;        // i * top_inv >> 16 is i / top for i < kMaxSplits * kMaxTop
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float lane_value(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}
__device__ __forceinline__ uint64_t pack(float x, uint32_t y) { return (uint64_t)__float_as_uint(x) << 32 | y; }
__device__ __forceinline__ float first_of(uint64_t w) { return __uint_as_float((uint32_t)(w >> 32)); }
// Parts pass between workgroups of different XCDs: write-through stores, loads that
// bypass the caches.
__device__ __forceinline__ void publish(uint64_t* p, uint64_t x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t published(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Reductions over the wavefront in six DPP steps (row shifts by 1, 2, 4, 8, then each
// row's last lane into the next row, then the lower half's into the upper).
template <int kCtrl, int kRows>
__device__ __forceinline__ float shifted(float none, float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(x), kCtrl, kRows, 0xf, false));
}
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, shifted<0x111, 0xf>(-INFINITY, x));
  x = fmaxf(x, shifted<0x112, 0xf>(-INFINITY, x));
  x = fmaxf(x, shifted<0x114, 0xf>(-INFINITY, x));
  x = fmaxf(x, shifted<0x118, 0xf>(-INFINITY, x));
  x = fmaxf(x, shifted<0x142, 0xa>(-INFINITY, x));
  x = fmaxf(x, shifted<0x143, 0xc>(-INFINITY, x));
  return lane_value(x, 63);
}
__device__ __forceinline__ float wave_sum(float x) {
  x += shifted<0x111, 0xf>(0.f, x);
  x += shifted<0x112, 0xf>(0.f, x);
  x += shifted<0x114, 0xf>(0.f, x);
  x += shifted<0x118, 0xf>(0.f, x);
  x += shifted<0x142, 0xa>(0.f, x);
  x += shifted<0x143, 0xc>(0.f, x);
  return lane_value(x, 63);
}

// A running largest logit with the sums of weights against it.
struct Stat {
  float m, s, t;
};
// The factor of sums against m where they are taken against top >= m (infinite
// logits weigh 1 against an infinite largest one, everything else 0).
__device__ __forceinline__ float factor(float m, float top) {
  return m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * kLog2e);
}
__device__ __forceinline__ Stat against(Stat x, float top) {
  if (x.s == 0.f) return Stat{top, 0.f, 0.f};
  const float f = factor(x.m, top);
  const float d = x.m == top ? 0.f : fminf(top - x.m, kFar);
  return Stat{top, f * x.s, f * (x.t + d * x.s)};
}
__device__ __forceinline__ Stat wave_join(Stat x) {
  x = against(x, wave_max(x.m));
  x.s = wave_sum(x.s);
  x.t = wave_sum(x.t);
  return x;
}

// The first tokens of the order: lane i holds place i (-infinity, -1: none).
struct Best {
  float z;
  int id;
};
// Larger the earlier a (logit, token) comes, above 0.  (-0 as 0.)
__device__ __forceinline__ uint64_t key_of(float z, int id) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return (uint64_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32 | (uint32_t)~id;
}
// A number that at least k lanes' values reach (-infinity where fewer are above it), near
// the k-th of them: the upper half of its bits, in the order of floats, found bit by bit.
__device__ __forceinline__ float kth_bound(float x, int k) {
  const uint32_t u = __float_as_uint(x);
  const uint32_t key = (u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) >> 16;
  uint32_t found = 0;
#pragma unroll
  for (int b = 15; b >= 0; --b) {
    const uint32_t t = found | 1u << b;
    if (__builtin_popcountll(__ballot(key >= t)) >= k) found = t;
  }
  found <<= 16;
  const float y = __uint_as_float(found & 0x80000000u ? found ^ 0x80000000u : ~found);
  return y > -INFINITY ? y : -INFINITY;                                // (below it the bits of NaN)
}

// A logit above the last place's, behind those that are equal to it.
__device__ __forceinline__ void insert(Best& best, float z, int id) {
  const int lane = threadIdx.x & 63;
  const int at = __builtin_popcountll(__ballot(best.z >= z));
  const float zs = shifted<0x138, 0xf>(-INFINITY, best.z);            // from the lane before
  const int is = __builtin_amdgcn_update_dpp(-1, best.id, 0x138, 0xf, 0xf, false);
  best.z = lane > at ? zs : lane == at ? z : best.z;
  best.id = lane > at ? is : lane == at ? id : best.id;
}
// The places of n <= 64 candidates, one a lane (ids differ): by counting those ahead.
__device__ __forceinline__ Best in_order(float z, int id, int n) {
  const int lane = threadIdx.x & 63;
  z = lane < n ? z : -INFINITY;
  const uint64_t key = lane < n ? key_of(z, id) : 0;
  int ahead = 0;
  for (int j0 = 0; j0 < n; j0 += 4) {                 // (past the last candidate none is ahead of one)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t kj = (uint64_t)__builtin_amdgcn_readlane((uint32_t)(key >> 32), j0 + j) << 32 |
                          (uint32_t)__builtin_amdgcn_readlane((uint32_t)key, j0 + j);
      ahead += kj > key ? 1 : 0;
    }
  }
  const int to = 4 * (lane < n ? ahead : lane);
  Best b;
  b.z = __uint_as_float(__builtin_amdgcn_ds_permute(to, __float_as_uint(z)));
  b.id = __builtin_amdgcn_ds_permute(to, lane < n ? id : -1);
  return b;
}
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

__device__ __forceinline__ float log_prob(float z, float m, double log_s) {
  if (m == -INFINITY) return __builtin_nanf("");
  if (z == m) return (float)-log_s;
  return (float)((double)z - (double)m - log_s);
}

struct Scratch {
  float m[kWaves], s[kWaves], t[kWaves];
  int ahead[kWaves];
  float deep[kWaves];                          // a place of each wavefront's, below
  float z[kMaxSplits * kMaxTop];               // lists to join: [list][place]
  int id[kMaxSplits * kMaxTop];
  float pz[kWaves][64];                        // candidates
  int pi[kWaves][64];
  uint64_t cand[kMaxSplits * kMaxTop];         // keys of a join's candidates
  float best_z[kMaxTop];                       // the joined list
  int best_id[kMaxTop];
  int n, last;
  Stat all;                                    // of the workgroup or the row
  double log_s;
  int all_ahead;
};

// Before a join (and a barrier): the joined list empty, no candidates.
__device__ __forceinline__ void clear_join(Scratch& sm) {
  if (threadIdx.x < kMaxTop) {
    sm.best_z[threadIdx.x] = -INFINITY;
    sm.best_id[threadIdx.x] = -1;
  }
  if (threadIdx.x == 0) sm.n = 0;
}
// Joins sm.z / sm.id, `lists` of k places in order, a list's tokens before the later lists',
// by the whole workgroup.  Where the c-th places of ceil(k / c) lists reach a bound, k
// logits do: those that reach it are placed by counting the ones ahead.  (With c about
// 2 k / lists half of the lists decide; where fewer have that many places, a larger one.)
// The last wavefront, which seldom has a candidate, does `beside` meanwhile.
template <typename F>
__device__ __forceinline__ void join_lists(Scratch& sm, int lists, int k, F beside) {
  const int tid = threadIdx.x, lane = tid & 63;
  float bound = -INFINITY;
  for (int c = min(k, (2 * k + lists - 1) / lists);; c = min(k, 2 * c)) {
    bound = kth_bound(lane < lists ? sm.z[lane * k + c - 1] : -INFINITY, (k + c - 1) / c);
    if (bound > -INFINITY || c == k) break;
  }
  for (int i0 = 0; i0 < lists * k; i0 += kThreads) {
    const int i = i0 + tid;
    const float y = i < lists * k ? sm.z[i] : -INFINITY;
    const bool in = y >= bound && y > -INFINITY;
    const uint64_t mask = __ballot(in);
    if (mask == 0) continue;
    int at = 0;
    if (lane == 0) at = atomicAdd(&sm.n, __builtin_popcountll(mask));
    at = uniform(at) + lanes_before(mask);
    if (in) sm.cand[at] = key_of(y, sm.id[i]);
  }
  __syncthreads();
  const int n = sm.n;
  if (uniform(tid >> 6) == kWaves - 1) beside();
  for (int i0 = uniform(tid >> 6) * 32; i0 < n; i0 += kThreads / 2) {              // two lanes a candidate
    const int i = i0 + (lane >> 1);
    const uint64_t own = sm.cand[min(i, n - 1)];
    int ahead = 0;
#pragma unroll 8
    for (int j = tid & 1; j < n; j += 2) ahead += sm.cand[j] > own ? 1 : 0;
    ahead += __builtin_amdgcn_update_dpp(0, ahead, 0xb1, 0xf, 0xf, false);      // the other lane's
    if ((tid & 1) == 0 && i < n && ahead < k) {
      const uint32_t u = (uint32_t)(own >> 32);
      sm.best_z[ahead] = __uint_as_float(u ^ (~(uint32_t)((int32_t)u >> 31) | 0x80000000u));
      sm.best_id[ahead] = (int)~(uint32_t)own;
    }
  }
  __syncthreads();
}

// Outputs of a row, by one wavefront.
__device__ __forceinline__ void write_row(const LogprobArgs& a, int row, const Scratch& sm, float zt, bool known) {
  const int lane = threadIdx.x & 63;
  const Stat x = sm.all;
  const double log_s = sm.log_s;
  if (lane < a.top) {
    const float z = sm.best_z[lane];
    a.top_logprobs[(int64_t)row * a.top + lane] = z > -INFINITY ? log_prob(z, x.m, log_s) : -INFINITY;
    a.top_tokens[(int64_t)row * a.top + lane] = sm.best_id[lane];
  }
  if (lane != 0) return;
  if (a.entropy) a.entropy[row] = x.m == -INFINITY ? __builtin_nanf("") : (float)(log_s + (double)x.t / (double)x.s);
  if (a.logprob) a.logprob[row] = known ? log_prob(zt, x.m, log_s) : __builtin_nanf("");
  if (a.rank) a.rank[row] = known ? sm.all_ahead + 1 : 0;
}

// (Every workgroup runs most of the code once, so its size counts: one path for
// every value, loops over registers kept few.)
__global__ __launch_bounds__(kThreads) void logprob_kernel(LogprobArgs a) {
  __shared__ Scratch sm;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int slot = blockIdx.x, split = blockIdx.y;
  const int count = a.n_work ? min(max(a.n_work[0], 0), a.R) : a.R;
  if (slot >= count) return;
  const int row = uniform(a.work_list ? a.work_list[slot] : slot);
  if (row < 0 || row >= a.R) return;
  const float* z_row = a.logits + (int64_t)row * a.stride;

  // the wavefront's logits: one run of the split's, in ascending order
  const int begin = min(a.V, split * a.chunk), end = min(a.V, begin + a.chunk);
  const int run = ((end - begin + kWaves - 1) / kWaves + kRun - 1) & ~(kRun - 1);
  const int from = min(end, begin + wave * run), to = min(end, from + run);
  float z[4 * kLoads], next[4 * kLoads];
  auto load = [&](int v0, float (&x)[4 * kLoads]) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int v = v0 + (u * 64 + lane) * 4;
      if (v + 4 <= to) {
        const f32x4u w = *reinterpret_cast<const f32x4u*>(z_row + v);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * u + e] = w[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * u + e] = v + e < to ? z_row[v + e] : -INFINITY;
      }
    }
  };
  load(from, next);
  const int token = a.tokens ? uniform(a.tokens[row]) : -1;
  const bool known = token >= 0 && token < a.V;
  if (tid < kWaves) sm.deep[tid] = -INFINITY;
  __syncthreads();
  const float zt = known ? fmaxf(z_row[token], -INFINITY) + 0.f : 0.f;       // (NaN counts as -infinity, -0 as 0)
  // above this is at or above zt: the float before it (nothing at all before -infinity: NaN)
  const float zt_below = zt == -INFINITY ? __builtin_nanf("")
                         : zt > 0.f      ? __uint_as_float(__float_as_uint(zt) - 1)
                         : zt < 0.f      ? __uint_as_float(__float_as_uint(zt) + 1)
                                         : __uint_as_float(0x80000001u);

  Stat x{-INFINITY, 0.f, 0.f};
  Best best{-INFINITY, -1};
  float least = -INFINITY;          // the last place
  int least_id = -1;
  int ahead = 0;
  for (int v0 = from; v0 < to; v0 += kBatch) {
#pragma unroll
    for (int i = 0; i < 4 * kLoads; ++i) z[i] = fmaxf(next[i], -INFINITY);
    if (v0 + kBatch < to) load(v0 + kBatch, next);
    float top = z[0];
#pragma unroll
    for (int i = 1; i < 4 * kLoads; ++i) top = fmaxf(top, z[i]);
    if (top > x.m) x = against(x, top);
    if (x.m != -INFINITY) {
#pragma unroll
      for (int i = 0; i < 4 * kLoads; ++i) {
        const float d = z[i] == x.m ? 0.f : fminf(x.m - z[i], kFar), w = __builtin_amdgcn_exp2f(d * -kLog2e);
        x.s += w;
        x.t += w * d;
      }
    }
    if (a.rank) {
      // (past the run's end -infinity stands, which is no place before the token's)
      const int before = min(token, to) - v0 - 4 * lane;
#pragma unroll
      for (int i = 0; i < 4 * kLoads; ++i)
        ahead += __builtin_popcountll(__ballot(!(z[i] <= (256 * (i >> 2) + (i & 3) < before ? zt_below : zt))));
    }
    if (a.top > 0 && __any(top > least)) {
      if (v0 == from) {
        // What k lanes' largest reach, the k-th place does: those that reach it and what comes
        // before the last place so far, up to 64 at a time.
        const float bound = kth_bound(top, a.top);
        for (bool more = true; more;) {
          int n = __builtin_popcountll(__ballot(best.z > -INFINITY));
          if (lane < n) {
            sm.pz[wave][lane] = best.z;
            sm.pi[wave][lane] = best.id;
          }
#pragma unroll
          for (int i = 0; i < 4 * kLoads; ++i) {
            const int id = v0 + ((i >> 2) * 64 + lane) * 4 + (i & 3);
            const bool in = (z[i] >= bound) & ((z[i] > least) | ((z[i] == least) & (id < least_id)));
            const uint64_t mask = __ballot(in);
            const int at = n + lanes_before(mask);
            if (in && at < 64) {
              sm.pz[wave][at] = z[i];
              sm.pi[wave][at] = id;
              z[i] = -INFINITY;
            }
            n += __builtin_popcountll(mask);
          }
          more = n > 64;
          oda::wave_lds_fence();
          best = in_order(sm.pz[wave][lane], sm.pi[wave][lane], min(n, 64));
          if (lane >= a.top) best = Best{-INFINITY, -1};
          least = lane_value(best.z, a.top - 1);
          least_id = __builtin_amdgcn_readlane(best.id, a.top - 1);
          oda::wave_lds_fence();
        }
      } else {
        // Later, what every wavefront has ceil(k / kWaves) logits at or above; the few that
        // come before the last place one by one, in ascending order.
        float bound = lane < kWaves ? __hip_atomic_load(&sm.deep[lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) : INFINITY;
        bound = -wave_max(-bound);
        if (__any(top > least && top >= bound)) {
#pragma unroll
          for (int u = 0; u < kLoads; ++u) {
            const float most = fmaxf(fmaxf(z[4 * u], z[4 * u + 1]), fmaxf(z[4 * u + 2], z[4 * u + 3]));
            for (uint64_t todo = __ballot(most > least && most >= bound); todo != 0; todo &= todo - 1) {
              const int l = __builtin_ctzll(todo);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float y = lane_value(z[4 * u + e], l);
                if (y > least && y >= bound) {
                  insert(best, y, v0 + (u * 64 + l) * 4 + e);
                  least = lane_value(best.z, a.top - 1);
                }
              }
            }
          }
        }
      }
      const float mine = lane_value(best.z, (a.top + kWaves - 1) / kWaves - 1);
      if (lane == 0) __hip_atomic_store(&sm.deep[wave], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
  }
  x = wave_join(x);
  if (lane == 0) {
    sm.m[wave] = x.m;
    sm.s[wave] = x.s;
    sm.t[wave] = x.t;
    sm.ahead[wave] = ahead;
  }
  if (lane < a.top) {
    sm.z[wave * a.top + lane] = best.z;
    sm.id[wave * a.top + lane] = best.id;
  }
  clear_join(sm);
  __syncthreads();

  // The workgroup's wavefronts joined, then, by the last of a row's workgroups, its splits.
  // Lane l's part of the statistics, joined; of all of the row with the sum's logarithm.
  auto join_stats = [&](Stat part, int part_ahead, bool whole) {
    part = wave_join(part);
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) part_ahead += __shfl_xor(part_ahead, s);
    if (lane == 0) {
      sm.all = part;
      sm.all_ahead = part_ahead;
      if (whole) sm.log_s = log((double)part.s);
    }
  };
  auto join_waves = [&] {
    join_stats(lane < kWaves ? Stat{sm.m[lane], sm.s[lane], sm.t[lane]} : Stat{-INFINITY, 0.f, 0.f},
               lane < kWaves ? sm.ahead[lane] : 0, a.splits == 1);
  };
  // (Without alternatives the first wavefront is alone from here on: four rows 7.6 us
  // against 7.8 where all stay.)
  const bool alone = a.top == 0;
  if (alone && wave != 0) return;
  auto sync = [&] {
    if (alone) oda::wave_lds_fence();
    else __syncthreads();
  };
  auto join = [&](int lists, auto beside) {
    if (!alone) {
      join_lists(sm, lists, a.top, beside);
    } else {
      beside();
      oda::wave_lds_fence();
    }
  };
  join(kWaves, join_waves);
  if (a.splits > 1) {
    const int words = 2 + a.top;
    const uint64_t* parts = a.parts + (int64_t)slot * a.splits * words;
    if (wave == 0) {
      uint64_t* part = a.parts + ((int64_t)slot * a.splits + split) * words;
      if (lane == 0) publish(part, pack(sm.all.m, __float_as_uint(sm.all.s)));
      if (lane == 1) publish(part + 1, pack(sm.all.t, (uint32_t)sm.all_ahead));
      if (lane < a.top) publish(part + 2 + lane, pack(sm.best_z[lane], (uint32_t)sm.best_id[lane]));
      __builtin_amdgcn_s_waitcnt(0);
      __builtin_amdgcn_wave_barrier();
      if (lane == 0)
        sm.last = __builtin_amdgcn_atomic_inc32(a.tickets + slot * kTicketStride, (uint32_t)(a.splits - 1), __ATOMIC_RELAXED, "agent") ==
                          (uint32_t)(a.splits - 1)
                      ? 1
                      : 0;
    }
    sync();
    if (sm.last == 0) return;
    const uint64_t* list = parts + (int64_t)min(lane, a.splits - 1) * words;
    const uint64_t p0 = published(list), p1 = published(list + 1);
    constexpr int kEach = kMaxSplits * kMaxTop / kThreads;
    const int all = a.splits * a.top;
    uint64_t p[kEach];
    if (a.top > 0) {
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int i = min(j * kThreads + tid, all - 1), l = (int)((uint32_t)i * a.top_inv >> 16);
        p[j] = published(parts + (int64_t)l * words + 2 + (i - l * a.top));
      }
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int i = j * kThreads + tid;
      if (i >= all) continue;
      sm.z[i] = first_of(p[j]);
      sm.id[i] = (int)(uint32_t)p[j];
    }
    clear_join(sm);
    sync();
    join(a.splits, [&] {
      join_stats(lane < a.splits ? Stat{first_of(p0), __uint_as_float((uint32_t)p0), first_of(p1)} : Stat{-INFINITY, 0.f, 0.f},
                 lane < a.splits ? (int)(uint32_t)p1 : 0, true);
    });
  }
  if (wave == 0) write_row(a, row, sm, zt, known);
}

// Workgroups of a row: at most kGroups in all, each of at least kLeastSplit logits.
void split_row(int64_t rows, int64_t vocab, int* splits, int* chunk) {
  int64_t n = 1;
  if (rows <= kTickets)
    n = std::max<int64_t>(1, std::min<int64_t>({kMaxSplits, kGroups / rows, vocab / kLeastSplit}));
  *chunk = (int)oda::round_up(oda::ceil_div(vocab, n), n > 1 ? kWaves * kRun : 4);
  *splits = (int)oda::ceil_div(vocab, *chunk);
}

oda_status check(const oda_logprob_desc* desc, int32_t rows, size_t* bytes, int* splits, int* chunk) {
  if (desc == nullptr) return oda::fail(ODA_ERR_NULL, "desc is NULL");
  if (rows < 1) return oda::fail(ODA_ERR_SHAPE, "rows must be >= 1");
  if (desc->vocab < 1 || desc->vocab > (1 << 30)) return oda::fail(ODA_ERR_SHAPE, "vocab %d not in 1..2^30", desc->vocab);
  if (desc->top < 0 || desc->top > ODA_MAX_TOP) return oda::fail(ODA_ERR_SHAPE, "top %d not in 0..%d", desc->top, ODA_MAX_TOP);
  if (desc->row_stride != 0 && desc->row_stride < desc->vocab)
    return oda::fail(ODA_ERR_SHAPE, "row_stride must be 0 or at least vocab");
  split_row(rows, desc->vocab, splits, chunk);
  // (rows that are split have kGroups parts at most, whatever the call's sizes)
  *bytes = kTickets * kTicketStride * 4 + (size_t)kGroups * (2 + ODA_MAX_TOP) * 8;
  return ODA_OK;
}

}  // namespace

extern "C" oda_status oda_logprob_workspace_size(const oda_logprob_desc* desc, int32_t rows, size_t* bytes) {
  int splits, chunk;
  size_t need;
  const oda_status st = check(desc, rows, &need, &splits, &chunk);
  if (st != ODA_OK) return st;
  if (bytes == nullptr) return oda::fail(ODA_ERR_NULL, "bytes is NULL");
  *bytes = need;
  return oda::ok();
}

extern "C" oda_status oda_token_logprobs(const oda_logprob_desc* desc, int32_t rows, float* logprob, int32_t* rank,
                                        float* entropy, float* top_logprobs, int32_t* top_tokens,
                                        const int32_t* work_list, const int32_t* n_work, void* workspace,
                                        size_t workspace_bytes, hipStream_t stream) {
  LogprobArgs a;
  size_t need;
  const oda_status st = check(desc, rows, &need, &a.splits, &a.chunk);
  if (st != ODA_OK) return st;
  if (!desc->logits) return oda::fail(ODA_ERR_NULL, "logits is required");
  if ((logprob || rank) && !desc->tokens) return oda::fail(ODA_ERR_NULL, "logprob and rank need tokens");
  if ((top_logprobs == nullptr) != (desc->top == 0) || (top_tokens == nullptr) != (desc->top == 0))
    return oda::fail(ODA_ERR_NULL, "top_logprobs and top_tokens must be set iff top > 0");
  if (!logprob && !rank && !entropy && desc->top == 0) return oda::fail(ODA_ERR_NULL, "no output");
  if ((work_list == nullptr) != (n_work == nullptr))
    return oda::fail(ODA_ERR_NULL, "work_list and n_work must both be NULL or both be set");
  if (workspace == nullptr) return oda::fail(ODA_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", need);
  if (workspace_bytes < need) return oda::fail(ODA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  if (!oda::aligned(workspace, 256)) return oda::fail(ODA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  a.logits = desc->logits;
  a.tokens = desc->tokens;
  a.logprob = logprob;
  a.rank = rank;
  a.entropy = entropy;
  a.top_logprobs = top_logprobs;
  a.top_tokens = top_tokens;
  a.work_list = work_list;
  a.n_work = n_work;
  a.tickets = static_cast<uint32_t*>(workspace);
  a.parts = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + kTickets * kTicketStride * 4);
  a.stride = desc->row_stride != 0 ? desc->row_stride : desc->vocab;
  a.R = rows;
  a.V = desc->vocab;
  a.top = desc->top;
  a.top_inv = (uint32_t)oda::ceil_div(65536, std::max(a.top, 1));
  (void)hipGetLastError();
  hipLaunchKernelGGL(logprob_kernel, dim3((unsigned)rows, (unsigned)a.splits), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return oda::fail(ODA_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return oda::ok();
}
