// Rows of prompts appended to the paged cache (oda_append_qkv): per-head RMSNorm of
// q and k, rotary embedding of one or several axes, bf16 rounding; q to its buffer,
// K and V to the cache's blocks and the rings.
//
//   x' = x / sqrt(mean x^2 + eps) * gain
//   (x'_i, x'_{i + D/2}) turned by p[axis(i)] theta^(-2i/D)
//
// Bound by HBM: a projection's element is read once and written once.  Sixteen prompts of
// 201 to 1,900 rows of 32 + 2 x 8 heads with positions of three axes, 414 MB: 102 us, 4.1
// TB/s (a large copy of this card: 5.0).  Few rows are bound by one chain of trips (starts and lengths, rows,
// stores): eight single tokens 4.9 us.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "oda.h"
#include "oda_device.h"
#include "oda_internal.h"

namespace {

constexpr int kBlock = 16;       // positions per KV block, rows of a workgroup
constexpr int kWaves = 8;        // share the heads
constexpr int kThreads = kWaves * 64;

struct AppendArgs {
  const void* qkv;
  const float* q_gain;
  const float* k_gain;
  const int32_t* positions;
  const int32_t* row_start;
  const int32_t* seq_lens;
  const int32_t* block_table;
  uint16_t* q_out;
  uint16_t* k_cache;
  uint16_t* v_cache;
  uint16_t* k_ring;
  uint16_t* v_ring;
  int64_t num_blocks;
  double log2_theta;             // 0: no rotation
  float eps;
  int32_t B, R, Hq, Hkv, MB, max_len;     // Hq or Hkv may be 0 (rows without them)
  int32_t axes, axis_end[ODA_MAX_AXES];   // pairs of the axes up to each
  int32_t sink_blocks, ring_blocks;
  int32_t slots, chunk;          // head slots, and of one workgroup
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The request and block of tile `tile`: tiles are the blocks that the requests' rows
// touch, request by request.  Starts are taken into [0, R] and as ascending.
struct Tile {
  int request, row0, rows, place0, block;   // request -1: none
  bool bad;                                 // of a length out of range: blocks count from the rows' first
};
__device__ __forceinline__ Tile find_tile(const AppendArgs& a, int tile) {
  const int lane = threadIdx.x & 63;
  int carry = 0, before = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int b = b0 + lane;
    int start = 0, end = 0, n = 0;
    if (b < a.B) {
      start = min(max(a.row_start[b], 0), a.R);
      end = min(max(a.row_start[b + 1], 0), a.R);
      n = a.seq_lens[b];
    }
    int row0 = max(start, carry);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int y = __shfl_up(row0, s);
      if (lane >= s) row0 = max(row0, y);
    }
    carry = __shfl(row0, 63);
    const int rows = max(end - row0, 0);
    const bool bad = n < rows || n > a.max_len;
    const int place0 = bad ? 0 : n - rows;
    const int tiles = rows > 0 ? (place0 + rows - 1) / kBlock - place0 / kBlock + 1 : 0;
    int upto = tiles;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int y = __shfl_up(upto, s);
      if (lane >= s) upto += y;
    }
    const uint64_t past = __ballot(before + upto > tile);
    if (past != 0) {
      const int who = __builtin_ctzll(past);
      Tile t;
      t.request = b0 + who;
      t.row0 = __builtin_amdgcn_readlane(row0, who);
      t.rows = __builtin_amdgcn_readlane(rows, who);
      t.place0 = __builtin_amdgcn_readlane(place0, who);
      t.bad = __builtin_amdgcn_readlane(bad ? 1 : 0, who) != 0;
      const int first = __builtin_amdgcn_readlane(before + upto - tiles, who);
      t.block = t.place0 / kBlock + (tile - first);
      return t;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  Tile t{};
  t.request = -1;
  return t;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
// Four neighbouring values as they lie in memory, and widened.
template <typename In>
struct Four;
template <>
struct Four<float> {
  typedef f32x4 raw;
  static __device__ __forceinline__ f32x4 wide(f32x4 x) { return x; }
};
template <>
struct Four<uint16_t> {
  typedef uint2 raw;
  static __device__ __forceinline__ f32x4 wide(uint2 w) {
    return f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                 __uint_as_float(w.y & 0xffff0000u)};
  }
};
__device__ __forceinline__ uint2 round4(f32x4 x) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint2, __builtin_convertvector(x, bf16x4));
}

// Four rows (one per 16 lanes) of four dimensions each to one dimension (the lane's
// sixteenth's number) of four rows.
__device__ __forceinline__ uint2 transpose4(uint2 x, int r) {
  const uint32_t odd = (uint32_t)(r & 1), high = (uint32_t)(r >> 1);
  // dimensions 0, 1 in x.x and 2, 3 in x.y: the neighbour's value of the own parity's dimension
  const uint32_t a = __shfl_xor(odd ? (x.x & 0xffffu) : (x.x >> 16), 16);
  const uint32_t b = __shfl_xor(odd ? (x.y & 0xffffu) : (x.y >> 16), 16);
  const uint32_t lo = odd ? (a & 0xffffu) | (x.x & 0xffff0000u) : (x.x & 0xffffu) | a << 16;   // dimension odd
  const uint32_t hi = odd ? (b & 0xffffu) | (x.y & 0xffff0000u) : (x.y & 0xffffu) | b << 16;   // 2 + odd
  const uint32_t other = __shfl_xor(high ? lo : hi, 32);
  return high ? make_uint2(other, hi) : make_uint2(lo, other);
}

// One workgroup per (block of a request's rows, chunk of head slots).  A wavefront
// takes every kWaves-th slot and goes through its rows four at a time, sixteen lanes a
// row: a lane has four dimensions and those half a head behind them (the pairs that the
// rotation mixes) of one head, or of one of two heads of 64.  The rows' angles are formed
// once for all heads, side by side, and lie in LDS.
// (In flight together per wavefront: loads of four rows and a slot.  Six or eight of them,
// and workgroups of four or sixteen wavefronts, were slower or equal.)
constexpr int kInFlight = 4;
template <int D, typename In>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  constexpr int HS = 128 / D;    // heads of a slot
  constexpr int kLanes = D / 8;  // lanes of a head
  __shared__ __attribute__((aligned(16))) float s_cos[kBlock][D / 2], s_sin[kBlock][D / 2];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const Tile t = find_tile(a, blockIdx.x);
  if (t.request < 0) return;
  const int r = lane >> 4, sub = lane & (kLanes - 1), which = (lane >> 3) & (HS - 1);
  const int first = max(t.place0 - t.block * kBlock, 0);                         // rows of the block
  const int last = min(t.place0 + t.rows - t.block * kBlock, kBlock) - 1;
  const int row0 = t.row0 + t.block * kBlock - t.place0;                          // of the block's first place
  const int heads = a.Hq + 2 * a.Hkv;

  // slots: of q, then k, then v heads
  const int q_slots = (a.Hq + HS - 1) / HS, k_slots = (a.Hkv + HS - 1) / HS;
  const int s0 = blockIdx.y * a.chunk, s1 = min(a.slots, s0 + a.chunk);
  struct Head {
    int kind, head;              // 0 q, 1 k, 2 v
    bool in;
  };
  auto head_of = [&](int s) {
    Head h;
    h.kind = s < q_slots ? 0 : s < q_slots + k_slots ? 1 : 2;
    h.head = (s - (h.kind == 0 ? 0 : h.kind == 1 ? q_slots : q_slots + k_slots)) * HS + which;
    h.in = h.head < (h.kind == 0 ? a.Hq : a.Hkv);
    return h;
  };
  // items of the wavefront: its slots, of each the groups of four rows
  const int g0 = first >> 2, groups = (last >> 2) - g0 + 1;
  const int items = s0 + wave < s1 ? ((s1 - s0 - wave + kWaves - 1) / kWaves) * groups : 0;
  typename Four<In>::raw x[kInFlight][2];
  int load_s = s0 + wave, load_g = 0;
  auto load = [&](int u) {       // the next item's; past the last one it again
    const Head h = head_of(load_s);
    const int at = h.in ? (h.kind == 0 ? h.head : h.kind == 1 ? a.Hq + h.head : a.Hq + a.Hkv + h.head) : 0;
    const int row = row0 + min(max(4 * (g0 + load_g) + r, first), last);
    const In* src = static_cast<const In*>(a.qkv) + ((int64_t)row * heads + at) * D + 4 * sub;
    x[u][0] = *reinterpret_cast<const typename Four<In>::raw*>(src);
    x[u][1] = *reinterpret_cast<const typename Four<In>::raw*>(src + D / 2);
    if (load_g + 1 < groups) {
      ++load_g;
    } else if (load_s + kWaves < s1) {
      load_g = 0;
      load_s += kWaves;
    }
  };
  if (items > 0) {
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) load(u);
  }

  // block and ring block of the rows (places without a block are in the ring neither)
  int64_t blk = -1, ring = -1;
  if (a.Hkv > 0 && !t.bad && s1 > q_slots) {
    const int e = a.block_table[(int64_t)t.request * a.MB + t.block];
    blk = e >= 0 && e < a.num_blocks ? e : -1;
    const int end = (t.place0 + t.rows - 1) / kBlock;
    if (blk >= 0 && a.k_ring != nullptr && (t.block < a.sink_blocks || t.block > end - a.ring_blocks))
      ring = (int64_t)t.request * (a.sink_blocks + a.ring_blocks) +
             (t.block < a.sink_blocks ? t.block : a.sink_blocks + t.block % a.ring_blocks);
  }
  const bool turns = a.log2_theta != 0.0 && s0 < q_slots + k_slots;
  if (turns) {
    const int pair = threadIdx.x % (D / 2);
    const double frequency = oda::rope_frequency(pair, D, a.log2_theta);
    int axis = 0;
    for (int k = 0; k + 1 < a.axes; ++k) axis += pair >= a.axis_end[k] ? 1 : 0;
    for (int i = first + threadIdx.x / (D / 2); i <= last; i += kThreads / (D / 2)) {
      const int p = a.positions != nullptr ? a.positions[(int64_t)(row0 + i) * a.axes + axis] : t.block * kBlock + i;
      double sd, cd;
      oda::sincos_angle((double)p * frequency, sd, cd);
      s_cos[i][pair] = (float)cd;
      s_sin[i][pair] = (float)sd;
    }
    __syncthreads();
  }

  int s = s0 + wave, g = 0;
  for (int i0 = 0; i0 < items; i0 += kInFlight) {
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (i0 + u >= items) break;
      f32x4 lo = Four<In>::wide(x[u][0]), hi = Four<In>::wide(x[u][1]);
      load(u);
      const Head h = head_of(s);
      const int slot0 = 4 * (g0 + g), slot = slot0 + r;          // places of the block
      const bool valid = slot >= first && slot <= last;
      const int row = row0 + min(max(slot, first), last);
      if (g + 1 < groups) {
        ++g;
      } else {
        g = 0;
        s += kWaves;
      }
      if (h.kind < 2) {
        const float* gain = h.kind == 0 ? a.q_gain : a.k_gain;
        if (gain != nullptr) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) ss += lo[e] * lo[e] + hi[e] * hi[e];
#pragma unroll
          for (int k = kLanes / 2; k >= 1; k >>= 1) ss += __shfl_xor(ss, k);
          const float inv = rsqrtf(ss / (float)D + a.eps);
          const f32x4 a0 = *reinterpret_cast<const f32x4*>(gain + 4 * sub), a1 = *reinterpret_cast<const f32x4*>(gain + 4 * sub + D / 2);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            lo[e] = lo[e] * inv * a0[e];
            hi[e] = hi[e] * inv * a1[e];
          }
        }
        if (turns) {
          const int at = min(max(slot, first), last);
          const f32x4 cs = *reinterpret_cast<const f32x4*>(&s_cos[at][4 * sub]), sn = *reinterpret_cast<const f32x4*>(&s_sin[at][4 * sub]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float r1 = lo[e] * cs[e] - hi[e] * sn[e], r2 = hi[e] * cs[e] + lo[e] * sn[e];
            lo[e] = r1;
            hi[e] = r2;
          }
        }
      }
      uint2 lo4 = round4(lo), hi4 = round4(hi);
      const int64_t head = (int64_t)h.head * kBlock * D, head_stride = (int64_t)a.Hkv * kBlock * D;
      if (h.kind == 0) {
        if (t.bad) lo4 = hi4 = make_uint2(0x7fc07fc0u, 0x7fc07fc0u);
        if (valid && h.in) {
          uint16_t* dst = a.q_out + ((int64_t)row * a.Hq + h.head) * D + 4 * sub;
          *reinterpret_cast<uint2*>(dst) = lo4;
          *reinterpret_cast<uint2*>(dst + D / 2) = hi4;
        }
      } else if (h.kind == 1) {
        // a block of one KV head: [D/8][16][8]
        const int64_t at = head + ((sub >> 1) * kBlock + slot) * 8 + 4 * (sub & 1), half = (D / 16) * kBlock * 8;
        if (valid && h.in && blk >= 0) {
          *reinterpret_cast<uint2*>(a.k_cache + blk * head_stride + at) = lo4;
          *reinterpret_cast<uint2*>(a.k_cache + blk * head_stride + at + half) = hi4;
        }
        if (valid && h.in && ring >= 0) {
          *reinterpret_cast<uint2*>(a.k_ring + ring * head_stride + at) = lo4;
          *reinterpret_cast<uint2*>(a.k_ring + ring * head_stride + at + half) = hi4;
        }
      } else {
        // [D][16]: the lane's dimension 4 sub + r of four rows
        lo4 = transpose4(lo4, r);
        hi4 = transpose4(hi4, r);
        auto put = [&](uint16_t* p) {
          p += head + (4 * sub + r) * kBlock + slot0;
          if (slot0 >= first && slot0 + 3 <= last) {
            *reinterpret_cast<uint2*>(p) = lo4;
            *reinterpret_cast<uint2*>(p + (D / 2) * kBlock) = hi4;
            return;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (slot0 + e < first || slot0 + e > last) continue;
            p[e] = (uint16_t)((e < 2 ? lo4.x : lo4.y) >> (16 * (e & 1)));
            p[(D / 2) * kBlock + e] = (uint16_t)((e < 2 ? hi4.x : hi4.y) >> (16 * (e & 1)));
          }
        };
        if (h.in && blk >= 0) put(a.v_cache + blk * head_stride);
        if (h.in && ring >= 0) put(a.v_ring + ring * head_stride);
      }
    }
  }
}

template <typename In>
oda_status launch(const AppendArgs& a, int head_dim, dim3 grid, hipStream_t stream) {
  (void)hipGetLastError();
  if (head_dim == 128) hipLaunchKernelGGL((append_kernel<128, In>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((append_kernel<64, In>), grid, dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return oda::fail(ODA_ERR_HIP, "kernel launch failed: %s", hipGetErrorString(e));
  return oda::ok();
}

}  // namespace

extern "C" oda_status oda_append_qkv(const oda_attn_shape* shape, const oda_prompt_rows* rows, const oda_append_desc* desc,
                                    uint16_t* k_cache, uint16_t* v_cache, const int32_t* block_table,
                                    const int32_t* seq_lens, uint16_t* q_out, uint16_t* k_ring, uint16_t* v_ring,
                                    int32_t n_sink, int32_t window, hipStream_t stream) {
  if (shape == nullptr) return oda::fail(ODA_ERR_NULL, "shape is NULL");
  if (rows == nullptr) return oda::fail(ODA_ERR_NULL, "rows is NULL");
  if (desc == nullptr) return oda::fail(ODA_ERR_NULL, "desc is NULL");
  size_t unused = 0;
  const oda_status st = oda_attn_workspace_size(shape, 0, 0, &unused);   // the shape's own checks
  if (st != ODA_OK) return st;
  if (shape->num_layers != 1) return oda::fail(ODA_ERR_SHAPE, "num_layers must be 1 (the projection is one layer's)");
  if (rows->num_rows < 1) return oda::fail(ODA_ERR_SHAPE, "num_rows must be >= 1");
  if (!rows->row_start || !seq_lens || !desc->qkv) return oda::fail(ODA_ERR_NULL, "row_start, seq_lens and qkv are required");
  if ((k_cache == nullptr) != (v_cache == nullptr))
    return oda::fail(ODA_ERR_NULL, "k_cache and v_cache must both be NULL or both be set");
  if (!k_cache && !q_out) return oda::fail(ODA_ERR_NULL, "q_out or the caches are required");
  if (k_cache && !block_table) return oda::fail(ODA_ERR_NULL, "block_table is required with the caches");
  if ((k_ring == nullptr) != (v_ring == nullptr))
    return oda::fail(ODA_ERR_NULL, "k_ring and v_ring must both be NULL or both be set");
  if (k_ring && !k_cache) return oda::fail(ODA_ERR_NULL, "rings need the caches");
  if (k_ring && (n_sink < 0 || window < 1)) return oda::fail(ODA_ERR_SHAPE, "rings need n_sink >= 0 and window >= 1");
  if (desc->qkv_type != ODA_F32 && desc->qkv_type != ODA_BF16) return oda::fail(ODA_ERR_SHAPE, "unknown qkv_type %d", desc->qkv_type);
  if (!(desc->rope_theta == 0.0 || desc->rope_theta > 1.0) || !std::isfinite(desc->rope_theta))
    return oda::fail(ODA_ERR_SHAPE, "rope_theta must be > 1, or 0 for no rotation");
  if (!(desc->rms_eps >= 0.f) || !std::isfinite(desc->rms_eps)) return oda::fail(ODA_ERR_SHAPE, "rms_eps must be >= 0");
  if (desc->num_axes < 1 || desc->num_axes > ODA_MAX_AXES)
    return oda::fail(ODA_ERR_SHAPE, "num_axes %d not in 1..%d", desc->num_axes, ODA_MAX_AXES);
  if (desc->num_axes > 1 && !desc->positions) return oda::fail(ODA_ERR_NULL, "several axes need positions");
  AppendArgs a{};
  a.axes = desc->num_axes;
  if (a.axes > 1) {
    int64_t sum = 0;
    for (int i = 0; i < a.axes; ++i) {
      if (desc->axis_pairs[i] < 0) return oda::fail(ODA_ERR_SHAPE, "axis_pairs must be >= 0");
      sum += desc->axis_pairs[i];
      a.axis_end[i] = (int32_t)std::min<int64_t>(sum, INT_MAX);
    }
    if (sum != shape->head_dim / 2) return oda::fail(ODA_ERR_SHAPE, "axis_pairs must add up to head_dim / 2");
  }
  if (!oda::aligned(desc->qkv, 16) || (k_cache && (!oda::aligned(k_cache, 16) || !oda::aligned(v_cache, 16))) ||
      (q_out && !oda::aligned(q_out, 16)) || (k_ring && (!oda::aligned(k_ring, 16) || !oda::aligned(v_ring, 16))) ||
      (desc->q_gain && !oda::aligned(desc->q_gain, 16)) || (desc->k_gain && !oda::aligned(desc->k_gain, 16)))
    return oda::fail(ODA_ERR_SHAPE, "qkv, gains, q_out, caches and rings must be 16-byte aligned");
  a.qkv = desc->qkv;
  a.q_gain = desc->q_gain;
  a.k_gain = desc->k_gain;
  a.positions = desc->positions;
  a.row_start = rows->row_start;
  a.seq_lens = seq_lens;
  a.block_table = block_table;
  a.q_out = q_out;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.k_ring = k_ring;
  a.v_ring = v_ring;
  a.num_blocks = shape->num_blocks;
  a.log2_theta = desc->rope_theta == 0.0 ? 0.0 : std::log2(desc->rope_theta);
  a.eps = desc->rms_eps;
  a.B = shape->batch;
  a.R = rows->num_rows;
  a.Hq = q_out ? shape->num_q_heads : 0;
  a.Hkv = k_cache ? shape->num_kv_heads : 0;
  a.MB = shape->max_blocks_per_seq;
  a.max_len = shape->max_seq_len;
  if (k_ring) {
    const oda::RingGeometry ring = oda::ring_geometry(n_sink, window);
    a.sink_blocks = ring.sink_blocks;
    a.ring_blocks = ring.ring_blocks;
  }
  const int per = 128 / shape->head_dim;
  a.slots = (int)(oda::ceil_div(a.Hq, per) + 2 * oda::ceil_div(a.Hkv, per));
  // a request's m rows touch at most m / 16 + 2 blocks, and at most m
  const int64_t tiles = std::min<int64_t>(a.R, (int64_t)a.R / kBlock + 2 * (int64_t)a.B);
  // heads shared out while there are fewer than 512 workgroups (one workgroup a block: 2,048
  // rows 21.8 us against 18.1, eight 7.4 against 5.2; 256 or 1,024 within 2%)
  const int64_t chunks = std::min<int64_t>(oda::ceil_div(a.slots, kWaves), std::max<int64_t>(1, oda::ceil_div(512, tiles)));
  a.chunk = (int)oda::ceil_div(a.slots, chunks);
  const dim3 grid((unsigned)tiles, (unsigned)oda::ceil_div(a.slots, a.chunk));
  return desc->qkv_type == ODA_F32 ? launch<float>(a, shape->head_dim, grid, stream)
                                   : launch<uint16_t>(a, shape->head_dim, grid, stream);
}
