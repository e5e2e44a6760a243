/*
 * oda.h -- C ABI of the On-Demand Attention (ODA) decode-step hot path on
 * AMD Instinct MI355X (gfx950).
 *
 * One decode step of ODA (Alg. 1) runs, in stream order:
 *   1. oda_local_decode_attn  -- attention over the Local access set S^L
 *                                (s initial positions + a recent window of w
 *                                positions that includes the current token;
 *                                §2.1, access-set equation);
 *   2. oda_recall_gate        -- the recall score q_t = R(h_{t-1}, E(x_t), h_t^L)
 *                                (§2.1, recall-head equation; head of App. A.2,
 *                                or a two-layer MLP stand-in) and the device
 *                                predicate "Full iff q_t > theta or q_t is
 *                                nonfinite" (§2.1, Alg. 1, App. A.5), written
 *                                as per-request flags plus a compacted list;
 *   3. oda_full_decode_attn   -- attention over the native access set, from the
 *                                same pre-step history, for flagged requests
 *                                only; it overwrites their rows of the output,
 *                                so the output buffer ends up holding the
 *                                selected branch (App. A.5, commit equation).
 *
 * Conventions (all entry points):
 *   - Pointers are DEVICE pointers unless marked (host).  The caller owns every
 *     buffer; the library never allocates, never synchronises and never copies
 *     device memory to the host.
 *   - Host-visible arguments are validated synchronously; on any error the call
 *     returns a negative status and enqueues nothing.  oda_last_error() then
 *     holds a thread-local description.
 *   - All work is enqueued on `stream` (NULL = the default stream).
 *   - Device-data contract: seq_lens[b] in [1, max_seq_len]; every block-table
 *     entry a request uses in [0, num_blocks); listed requests in [0, batch).
 *     The kernels check it and never address memory with a value outside it:
 *     attention writes NaN rows (out and lse) for a request whose length or
 *     used table entry is out of range, the commit writes nothing for it, and
 *     listed requests outside the batch are skipped.
 *   - The library keeps no state between calls other than what a caller's
 *     workspace holds: attention workspaces carry merge-ticket words that
 *     every call leaves zero (see oda_attn_workspace_size).  Workspaces may be
 *     reused by later calls on the same stream; calls that share a workspace
 *     must not overlap in time.
 *   - Results are deterministic: a fixed split order, no floating-point
 *     atomics; reruns are bit-identical.
 *
 * Data layouts (bf16 = IEEE bfloat16 stored as uint16_t):
 *   q        bf16 [L][B][Hq][D]   post-RoPE queries of the current token
 *   k_cache  bf16 [L][num_blocks][Hkv][D/8][16][8]
 *            paged keys, 16 positions per block; within a block and KV head,
 *            16-byte groups of 8 consecutive dims, position-minor:
 *            K(pos, d) = k_cache[l][blk][g][d/8][pos%16][d%8]
 *   v_cache  bf16 [L][num_blocks][Hkv][D][16]
 *            paged values, dims-major:  V(pos, d) = v_cache[l][blk][g][d][pos%16]
 *            where blk = block_table[b][pos/16]; layer l starts layer_stride_kv
 *            elements after layer l-1 (dense by default)
 *   (Every 16-byte lane load of K is one matrix-core operand fragment and a
 *   wavefront's load instruction reads 1 KiB contiguous; V needs no transpose.
 *   Blocks stored position-major, [16][D] for both K and V as many paged
 *   caches keep them, measured 55% slower on this hardware -- Full over the
 *   32-layer 32,768-position stack 626 -> 970..990 us, Local 28 -> 41..44 us --
 *   because each K load instruction then touches 16 separate half lines and V
 *   must be transposed (through LDS or 2-byte gathers); the library does not
 *   take that layout.)
 *   k_cur, v_cur  bf16 [L][B][Hkv][D]  (optional) the current token's candidate
 *            K/V, not yet committed to the cache (App. A.5)
 *   out      fp32 [L][B][Hq][D];  lse fp32 [L][B][Hq]  (natural log)
 *   GQA: query head h reads KV head h / (Hq/Hkv)  (contiguous groups).
 */
#ifndef ODA_H_
#define ODA_H_

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ODA_OK = 0,
  ODA_ERR_NULL = -1,        /* a required pointer is NULL                      */
  ODA_ERR_SHAPE = -2,       /* inconsistent or out-of-range sizes              */
  ODA_ERR_UNSUPPORTED = -3, /* valid but not implemented (e.g. D not 64/128)   */
  ODA_ERR_WORKSPACE = -4,   /* workspace NULL or smaller than required         */
  ODA_ERR_HIP = -5          /* a kernel launch failed (hipGetLastError)        */
} oda_status;

/* Shape of one attention call (host struct).  Every layer of the stack
 * shares B, heads, D, the block table and seq_lens. */
typedef struct {
  int32_t num_layers;         /* L >= 1: layers in this call's stack              */
  int32_t batch;              /* B >= 1                                           */
  int32_t num_q_heads;        /* Hq                                               */
  int32_t num_kv_heads;       /* Hkv; Hq % Hkv == 0 and 1 <= Hq/Hkv <= 16         */
  int32_t head_dim;           /* D: 64 or 128                                     */
  int32_t block_size;         /* must be 16                                       */
  int32_t max_blocks_per_seq; /* row stride of block_table (>= ceil(max_seq_len/16)) */
  int32_t max_seq_len;        /* host-known upper bound of seq_lens[]             */
  int64_t num_blocks;         /* physical blocks per layer in k_cache / v_cache   */
  int32_t split_blocks;       /* KV blocks per split-K work item (one workgroup
                                 each): 0 = automatic, otherwise an even number >= 2 */
  int32_t reserved;           /* must be 0                                        */
  int64_t layer_stride_kv;    /* elements between layers in k_cache / v_cache:
                                 0 = num_blocks * Hkv * 16 * D (dense); else at
                                 least that and a multiple of 8 (e.g. one
                                 allocation holding several layer groups)       */
} oda_attn_shape;

/* Inputs of one attention call (host struct holding device pointers). */
typedef struct {
  const uint16_t *q;            /* bf16 [L][B][Hq][D]                             */
  const uint16_t *k_cache;      /* bf16, layout above                             */
  const uint16_t *v_cache;      /* bf16, layout above                             */
  const int32_t *block_table;   /* int32 [B][max_blocks_per_seq]: logical block i
                                   of request b -> physical block id              */
  const int32_t *seq_lens;      /* int32 [B]: n_b >= 1 attended positions
                                   0..n_b-1; position n_b-1 is the current token  */
  const uint16_t *k_cur;        /* NULL: the current token is already in the cache.
                                   Else bf16 [L][B][Hkv][D]: position n_b-1 is taken
                                   from here and the cache holds 0..n_b-2          */
  const uint16_t *v_cur;        /* NULL iff k_cur is NULL                         */
  float scale;                  /* softmax scale (> 0), usually 1/sqrt(D)         */
} oda_attn_inputs;

/* Bytes of workspace an attention call with this shape and access set needs
 * (one merge-ticket word per (layer, request, KV head), then the split-K
 * partials), whatever number of requests a Full call selects: the split
 * count depends on that number and the size covers the largest.  It is 0 when
 * every request fits one work item; the workspace pointer may then be NULL.  window == 0 means "no window" (the whole
 * history); window > 0 limits the recent part to `window` positions.
 * n_sink >= 0.  (host out)
 * A workspace must be zero-filled before its first use (e.g. allocated
 * zeroed).  Every call leaves its ticket words zero again, so later calls on
 * the same stream with the same num_layers * batch * num_kv_heads (any sinks,
 * window or branch) reuse it as it is, graph replays included; zero it again
 * before using it with a larger product.  Calls that may run concurrently
 * need separate workspaces. */
oda_status oda_attn_workspace_size(const oda_attn_shape *shape, int32_t n_sink, int32_t window,
                                   size_t *bytes);

/* Local decode attention (§2.1 access-set equation; App. A.5 Local path).
 * For every (layer, request, query head) attends to
 *     S^L = {j : j < min(n_sink, n)}  U  {j : max(0, n - window) <= j < n}
 * (0-based, each position once).  window >= 1, n_sink >= 0.  When
 * n_sink + window >= n the set is the whole history (Local == Full).
 * Writes out[L][B][Hq][D] and, if lse != NULL, lse[L][B][Hq] for all rows.
 * workspace: >= oda_attn_workspace_size(shape, n_sink, window) bytes,
 * 256-byte aligned. */
oda_status oda_local_decode_attn(const oda_attn_shape *shape, const oda_attn_inputs *in,
                                 int32_t n_sink, int32_t window, float *out, float *lse,
                                 void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Recall-head kinds. */
typedef enum {
  ODA_HEAD_PAPER = 0, /* App. A.2: RMSNorm->Linear->SiLU towers on h_prev, emb,
                         h_local; interaction vector; fusion; two pre-RMSNorm
                         residual SwiGLU blocks; RMSNorm; scalar projection.
                         d_hidden = tower width dt (SwiGLU hidden 2*dt).       */
  ODA_HEAD_MLP = 1    /* stand-in: logit = w2 . GELU(W1 h_local + b1) + b2
                         (exact-erf GELU; sigmoid(logit) is the probability).
                         d_hidden = h.                                         */
} oda_head_kind;

/* Recall-gate description (host struct).  params: fp32, packed in this order
 *   PAPER: for t in (h_prev, emb, h_local): rms_t[d], W_t[dt][d], b_t[dt];
 *          W_f[dt][9dt], b_f[dt];
 *          for k in (1,2): rms_k[dt], W_gate_k[2dt][dt], W_up_k[2dt][dt], W_down_k[dt][2dt];
 *          rms_o[dt], w_o[dt], b_o[1]
 *   MLP:   W1[h][d], b1[h], w2[h], b2[1]
 * RMSNorm(x) = x / sqrt(mean(x^2) + rms_eps) * gain. */
typedef struct {
  int32_t kind;       /* oda_head_kind                                         */
  int32_t d_model;    /* d: width of h_prev / emb / h_local, multiple of 4     */
  int32_t d_hidden;   /* dt (PAPER) or h (MLP), multiple of 4                  */
  float rms_eps;      /* >= 0; ignored by the MLP                              */
  const float *params;/* device, oda_gate_param_count() floats                 */
} oda_gate_desc;

/* Number of fp32 parameters of a head (host out).  For PAPER with d = 2048,
 * dt = 1024 this is 28,325,889 (App. A.2). */
oda_status oda_gate_param_count(int32_t kind, int32_t d_model, int32_t d_hidden, int64_t *count);

/* Bytes of workspace oda_recall_gate needs for `batch` requests (host out). */
oda_status oda_gate_workspace_size(const oda_gate_desc *gate, int32_t batch, size_t *bytes);

/* Recall score and device predicate (§2.1, Alg. 1; App. A.5; App. B.7).
 *   h_prev, emb, h_local: fp32 [B][d_model] (PAPER reads all three; MLP only
 *                         h_local; the others may be NULL for MLP)
 *   tau:      threshold on the raw score (PAPER q_t; MLP pre-sigmoid logit);
 *             +-INFINITY allowed
 *   forced:   NULL, or int32 [B] prescribed flags (device-side schedule)
 *   score:    fp32 [B] out
 *   flags:    int32 [B] out; 1 iff score > tau or score is nonfinite
 *             (with `forced`: 1 iff forced[b] != 0 or score is nonfinite)
 *   work_list, n_work: NULL, or int32 [B] / int32 [1] out: the flagged request
 *             ids in ascending order and their count
 *   recall_counter: NULL, or int64 [1]; incremented by the number flagged
 *             (realised Full-call rate = counter / routed request-steps)
 * Everything stays on the device; no score is read by the host. */
oda_status oda_recall_gate(const oda_gate_desc *gate, int32_t batch, const float *h_prev,
                           const float *emb, const float *h_local, float tau, const int32_t *forced,
                           float *score, int32_t *flags, int32_t *work_list, int32_t *n_work,
                           int64_t *recall_counter, void *workspace, size_t workspace_bytes,
                           hipStream_t stream);

/* oda_recall_gate for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same computation and results, with the intermediate activations in a
 * workspace the library holds itself -- a 16 MiB device array per GPU, set
 * up on the first call on that GPU and kept until the process ends -- so the
 * call takes no workspace argument and allocates nothing.  Returns
 * ODA_ERR_WORKSPACE when oda_gate_workspace_size(gate, batch) exceeds 16 MiB
 * (the App. A.2 head takes 28 * batch * dt bytes for three or more requests:
 * up to 2,340 requests at dt = 256, 585 at dt = 1,024).  Every call on a GPU uses that GPU's one array: calls that may
 * overlap in time on one GPU (other streams, other host threads) race and
 * must be serialised by the caller.  The array's contents between calls do
 * not matter (each call writes what it reads). */
oda_status oda_recall_gate_static(const oda_gate_desc *gate, int32_t batch, const float *h_prev, const float *emb,
                                  const float *h_local, float tau, const int32_t *forced, float *score,
                                  int32_t *flags, int32_t *work_list, int32_t *n_work, int64_t *recall_counter,
                                  hipStream_t stream);

/* Full decode attention in the layers' native configuration (§2.1; App. A.5).
 * native_window == 0: S^F = all positions 0..n-1 (full-history layers);
 * native_window  > 0: the last native_window positions (natively
 * sliding-window layers, which ODA leaves unrestricted).
 * Request selection:
 *   work_list != NULL (with n_work != NULL): exactly the listed requests
 *                       (work_list[0 .. *n_work-1], distinct, as
 *                       oda_recall_gate writes them; a request listed twice
 *                       gets unspecified rows, but the workspace and every
 *                       other request are unaffected);
 *   else flags != NULL: the requests with flags[b] != 0;
 *   else              : every request.
 * Only selected requests read KV; only their rows of out (and lse, if not
 * NULL) are written, so after oda_local_decode_attn + oda_recall_gate the
 * buffer holds the selected branch per request.
 * workspace: >= oda_attn_workspace_size(shape, 0, native_window) bytes. */
oda_status oda_full_decode_attn(const oda_attn_shape *shape, const oda_attn_inputs *in,
                                int32_t native_window, const int32_t *flags,
                                const int32_t *work_list, const int32_t *n_work, float *out,
                                float *lse, void *workspace, size_t workspace_bytes,
                                hipStream_t stream);

/* Current-token preparation fused into a one-layer attention call (host
 * struct holding device pointers), for the decoder around the path (below):
 * the call builds the query and the current candidate K/V itself from the
 * fp32 QKV projection output, exactly as oda_qk_norm_rope would (per-head
 * RMSNorm of q and k, rotary embedding at position seq_lens[b] - 1, bf16
 * rounding; the same device code), instead of reading q / k_cur / v_cur, and
 * saves that launch.  Results are bit-identical to oda_qk_norm_rope followed
 * by the plain call.
 *   qkv     fp32 [B][(Hq + 2 Hkv) D]: q heads, then k heads, then v heads
 *   q_gain, k_gain  fp32 [D] per-head RMSNorm gains, or NULL (no norm)
 *   k_out, v_out    bf16 [B][Hkv][D]: the candidate K/V of the requests the
 *                   call attends (for the commit), or both NULL */
typedef struct {
  const float *qkv;
  const float *q_gain;
  const float *k_gain;
  float rms_eps;                /* >= 0                                          */
  double rope_theta;            /* > 1                                           */
  uint16_t *k_out;
  uint16_t *v_out;
} oda_qkv_prep;

/* oda_local_decode_attn / oda_full_decode_attn of one layer (num_layers == 1)
 * with the current token prepared in the call (oda_qkv_prep): in->q, k_cur and
 * v_cur must be NULL; the cache holds positions 0..n_b-2 and position n_b-1 is
 * the prepared candidate.  Everything else (sets, selection, workspace, the
 * rows written) is as in the plain calls. */
oda_status oda_local_decode_attn_qkv(const oda_attn_shape *shape, const oda_attn_inputs *in,
                                     const oda_qkv_prep *prep, int32_t n_sink, int32_t window, float *out,
                                     float *lse, void *workspace, size_t workspace_bytes, hipStream_t stream);
oda_status oda_full_decode_attn_qkv(const oda_attn_shape *shape, const oda_attn_inputs *in,
                                    const oda_qkv_prep *prep, int32_t native_window, const int32_t *flags,
                                    const int32_t *work_list, const int32_t *n_work, float *out, float *lse,
                                    void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace oda_commit_kv needs when it advances the lengths: one
 * ticket word per request, rounded up to 256 bytes (host out).  Zero-fill it
 * before its first use; every call leaves it zero again. */
oda_status oda_commit_workspace_size(const oda_attn_shape *shape, size_t *bytes);

/* Selected-state commit (App. A.5, commit equation C_t = C_{t-1} || dC_t^{b_t},
 * and its single fused cross-layer commit): in one launch, for every layer l,
 * request b and KV head g, copies the selected branch's current-position K/V
 * -- the Full candidate (k_full, v_full) if flags[b] != 0, else the Local
 * candidate (k_local, v_local) -- into position n_b - 1 of the paged cache
 * (block block_table[b][(n_b-1)/16], slot (n_b-1)%16, layouts above), where
 * n_b = seq_lens[b] is the step's attended count (the candidate was supplied
 * to the attention calls as k_cur/v_cur).  Then, if advance != 0,
 * seq_lens[b] += 1, ready for the next step's candidate.
 *   k_local, v_local: bf16 [L][B][Hkv][D] (required)
 *   k_full, v_full:   NULL (both) = same as the Local candidate
 *   flags:            NULL = every request keeps Local
 *   workspace:        required when advance != 0: >= oda_commit_workspace_size
 *                     bytes, 256-byte aligned, zero-filled before first use
 *                     (every call leaves it zero); ignored otherwise.  Calls
 *                     that may overlap in time need separate workspaces.
 * Only shape->num_layers, batch, num_kv_heads, head_dim, block_size,
 * max_blocks_per_seq and num_blocks are used.  The caller guarantees that the
 * block holding position n_b - 1 is allocated in block_table. */
oda_status oda_commit_kv(const oda_attn_shape *shape, uint16_t *k_cache, uint16_t *v_cache,
                         const int32_t *block_table, int32_t *seq_lens, const uint16_t *k_local,
                         const uint16_t *v_local, const uint16_t *k_full, const uint16_t *v_full,
                         const int32_t *flags, int32_t advance, void *workspace, size_t workspace_bytes,
                         hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Direct-ring Local (App. A.5: the Local path reads a contiguous workspace
 * holding the attention sinks and the recent window, with the current token
 * supplied separately, instead of the paged cache).  Per (layer, request, KV
 * head) unit, a ring of whole 16-position blocks in the cache's block
 * layouts.  For sinks s and window w:
 *   SB = ceil(s / 16) sink blocks, then RB = ceil(w / 16) + 2 ring blocks;
 *   logical block j of a request is held in ring block j if j < SB, else in
 *   ring block SB + (j mod RB)
 *   k_ring  bf16 [L][B][SB + RB][Hkv][D/8][16][8]
 *   v_ring  bf16 [L][B][SB + RB][Hkv][D][16]
 * RB blocks keep every block a Local call reads until the window has moved
 * past it, so a ring filled once (oda_ring_fill) and then kept current by the
 * commit (oda_commit_kv_ring) serves every later step.  A Local call through
 * the ring reads no block table and the same positions, in the same order,
 * as oda_local_decode_attn: the results are bit-identical.  Ring slots of
 * positions not yet committed may hold anything; no call reads them.  n_sink
 * and window must be the same in every call on a ring.
 * ------------------------------------------------------------------------- */

/* bf16 elements of each of k_ring and v_ring (host out). */
oda_status oda_ring_elements(const oda_attn_shape *shape, int32_t n_sink, int32_t window, int64_t *elements);

/* Fill the rings from the paged cache (one launch): every sink block, and in
 * every ring block the latest logical block j <= (seq_lens[b] - 1) / 16 that
 * maps to it, copied whole.  A request whose length is outside
 * [1, max_seq_len], or a table entry outside [0, num_blocks), leaves the ring
 * blocks concerned as they are.  Uses the same shape fields as
 * oda_local_decode_attn (layer_stride_kv included). */
oda_status oda_ring_fill(const oda_attn_shape *shape, const uint16_t *k_cache, const uint16_t *v_cache,
                         const int32_t *block_table, const int32_t *seq_lens, int32_t n_sink, int32_t window,
                         uint16_t *k_ring, uint16_t *v_ring, hipStream_t stream);

/* oda_local_decode_attn reading the rings: in->q, seq_lens, k_cur / v_cur
 * (the uncommitted candidate, or NULL when position n_b - 1 is in the ring)
 * and scale as there; in->k_cache, v_cache and block_table are not read (may
 * be NULL).  Same workspace (oda_attn_workspace_size(shape, n_sink, window)),
 * same outputs, bit for bit. */
oda_status oda_local_decode_attn_ring(const oda_attn_shape *shape, const oda_attn_inputs *in,
                                      const uint16_t *k_ring, const uint16_t *v_ring, int32_t n_sink,
                                      int32_t window, float *out, float *lse, void *workspace,
                                      size_t workspace_bytes, hipStream_t stream);

/* oda_commit_kv that also writes each committed position into the rings
 * (ring block of logical block (n_b - 1) / 16, slot (n_b - 1) % 16), in the
 * same launch.  The rings' shape is the commit's (L, B, Hkv, D). */
oda_status oda_commit_kv_ring(const oda_attn_shape *shape, uint16_t *k_cache, uint16_t *v_cache,
                              const int32_t *block_table, int32_t *seq_lens, const uint16_t *k_local,
                              const uint16_t *v_local, const uint16_t *k_full, const uint16_t *v_full,
                              const int32_t *flags, int32_t advance, void *workspace, size_t workspace_bytes,
                              uint16_t *k_ring, uint16_t *v_ring, int32_t n_sink, int32_t window,
                              hipStream_t stream);

/* ---------------------------------------------------------------------------
 * The decoder around the hot path (the backbone f_theta of §2.1 that Local and
 * Full share; App. A.6's cost model).  A pre-norm decoder layer is, per request:
 *   qkv = W_qkv . RMSNorm(h)              oda_dense_bf16 (gain = input norm)
 *   q, k, v = split(qkv); q, k per-head RMSNorm and rotary embedding at the
 *   current position, cast to bf16       oda_qk_norm_rope
 *   a = attention(q, cache, k, v)         oda_local_decode_attn / oda_full_decode_attn
 *   (the last two in one launch: oda_local_decode_attn_qkv / oda_full_decode_attn_qkv)
 *   h = h + W_o . a                       oda_dense_bf16 (residual = h)
 *   m = SiLU(W_g . RMSNorm(h)) * (W_u . RMSNorm(h))   oda_dense_bf16 (SWIGLU)
 *   h = h + W_d . m                       oda_dense_bf16 (residual = h)
 * then logits = W_vocab . RMSNorm(h) and the greedy token (oda_argmax).
 * Weights bf16, activations fp32.  Every call below can be restricted to the
 * recall gate's list (work_list, n_work: both NULL = every request; entries
 * must be in [0, batch)): only those requests are read and written.
 * ------------------------------------------------------------------------- */

typedef enum { ODA_DENSE_PLAIN = 0, ODA_DENSE_SWIGLU = 1 } oda_dense_mode;

typedef struct {
  int32_t in_features;     /* K, a multiple of 8                                  */
  int32_t out_features;    /* N                                                   */
  int32_t mode;            /* oda_dense_mode                                      */
  float rms_eps;           /* RMSNorm epsilon (used when norm_gain != NULL)       */
  const uint16_t *weight;  /* device bf16, PLAIN: [N][K]; SWIGLU: [2N][K], the N
                              gate rows then the N up rows; 16-byte aligned       */
  const float *norm_gain;  /* device fp32 [K]: x' = x / sqrt(mean(x^2) + eps) * gain;
                              NULL: x' = x                                        */
} oda_dense_desc;

/* Dense layer for `batch` requests, fp32 accumulation:
 *   PLAIN:  y[b][r] = sum_k W[r][k] x'[b][k]  (+ residual[b][r] if residual != NULL)
 *   SWIGLU: y[b][r] = SiLU(sum_k W[r][k] x'[b][k]) * sum_k W[N + r][k] x'[b][k]
 *           (no residual)
 * x fp32 [batch][K] (16-byte aligned); residual, y fp32 [batch][N].  y may be
 * the residual buffer (in-place residual add); x must not overlap y. */
oda_status oda_dense_bf16(const oda_dense_desc *desc, int32_t batch, const float *x, const float *residual,
                          float *y, const int32_t *work_list, const int32_t *n_work, hipStream_t stream);

/* Query/key preparation for the current token.  qkv fp32 [batch][(Hq + 2 Hkv) D]
 * holds the q heads, then the k heads, then the v heads.  q and k heads get a
 * per-head RMSNorm (gains q_gain / k_gain fp32 [D], or NULL for none) and then
 * the rotary embedding at position p = seq_lens[b] - 1 (rotate-half pairing:
 * dims i and i + D/2 rotate by angle p * theta^(-2i/D), angles in double);
 * results are rounded to bf16 (nearest-even):
 *   q_out bf16 [batch][Hq][D] (the attention query; as q of a one-layer call),
 *   k_out, v_out bf16 [batch][Hkv][D] (the current candidate, k_cur / v_cur).
 * D even, at most 128. */
oda_status oda_qk_norm_rope(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                            const float *qkv, const float *q_gain, const float *k_gain, float rms_eps,
                            double rope_theta, const int32_t *seq_lens, uint16_t *q_out, uint16_t *k_out,
                            uint16_t *v_out, const int32_t *work_list, const int32_t *n_work,
                            hipStream_t stream);

/* x[b] = table[tokens[b]] widened to fp32; table bf16 [vocab][d_model] (d_model a
 * multiple of 8); a token outside [0, vocab) gives a NaN row (and so a nonfinite
 * recall score, i.e. Full). */
oda_status oda_embed_bf16(const uint16_t *table, int32_t vocab, int32_t d_model, int32_t batch,
                          const int32_t *tokens, float *x, hipStream_t stream);

/* dst[b] = src[b] (fp32 rows of row_len, a multiple of 4) for the listed
 * requests (all if the list is NULL): moves the Full retry's results into the
 * selected state. */
oda_status oda_copy_rows(int32_t batch, int32_t row_len, const float *src, float *dst,
                         const int32_t *work_list, const int32_t *n_work, hipStream_t stream);

/* y[b] = x[b] / sqrt(mean(x[b]^2) + rms_eps) * gain for the listed requests
 * (all if the list is NULL): the final normalised hidden state, which §2.1
 * names as the recall head's Local input h_t^L and App. A.5 as the selected
 * state h_{t-1} the head reads at the next step.  x, y fp32 [batch][row_len]
 * (row_len a multiple of 4, 16-byte aligned; y may be x), gain fp32 [row_len]. */
oda_status oda_rms_norm_rows(int32_t batch, int32_t row_len, const float *x, const float *gain, float rms_eps,
                             float *y, const int32_t *work_list, const int32_t *n_work, hipStream_t stream);

/* index[b] = the first position of the largest non-NaN value of x[b][0..n)
 * (-1 if all are NaN); x fp32 [batch][n], n a multiple of 4. */
oda_status oda_argmax(int32_t batch, int32_t n, const float *x, int32_t *index, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Many tenants, drafted tokens.  A step in which each request brings T current
 * tokens (its last sampled token and up to T - 1 drafts of what follows), rows
 * of one tenant use that tenant's low-rank adapters, and the tokens that the
 * target's probabilities refuse are drawn anew.  Rows (b, t) of every buffer
 * are row b * T + t of the calls above (batch * T rows).
 * ------------------------------------------------------------------------- */

/* Requests whose histories begin with the same blocks (host struct holding
 * device pointers).  Group j holds the requests members[group_start[j] ..
 * group_start[j + 1] - 1]; the first prefix_blocks[j] entries of all their block
 * table rows name the same blocks (the call reads the first attended member's).
 * prefix_blocks[j] == 0: a group that shares nothing, such as a single request.
 * A request belongs to one group and is listed once; requests in none are left
 * alone. */
typedef struct {
  int32_t num_groups;           /* 1..2048                                          */
  int32_t tokens;               /* T: current tokens per request, 1..16             */
  const int32_t *group_start;   /* int32 [num_groups + 1], ascending, within [0, B] */
  const int32_t *members;       /* int32 [B]: request ids in group order            */
  const int32_t *prefix_blocks; /* int32 [num_groups]                               */
  const int32_t *n_tokens;      /* int32 [B]: current tokens of each request, clamped
                                   to [0, T]; NULL: T each                          */
  const int32_t *flags;         /* int32 [B]: members with flags[b] == 0 are left alone
                                   (oda_recall_gate's flags); NULL: all             */
} oda_prefix_groups;

/* Bytes of the plan buffer and of the workspace of calls with these sizes (the
 * shape, num_groups and tokens) (host out).  Neither needs to be cleared. */
oda_status oda_prefix_plan_size(const oda_attn_shape *shape, const oda_prefix_groups *groups, size_t *bytes);
oda_status oda_prefix_workspace_size(const oda_attn_shape *shape, const oda_prefix_groups *groups, size_t *bytes);

/* Plans oda_prefix_decode_attn on the device: which rows are attended, and how
 * their histories are split over the chip.  One plan serves every call of a step
 * whose shape, groups, lengths and kind of candidate are the plan's (all layers
 * of a stack or one call per layer: num_layers counts, so plan with the shape
 * that is called).  Of `in`, seq_lens and whether k_cur is NULL are used.  When
 * lengths, members, token counts or flags change, plan again: the attention reads
 * them from the plan.  shape->split_blocks must be 0; batch at most 2048.
 *   plan: >= oda_prefix_plan_size bytes, 256-byte aligned */
oda_status oda_prefix_plan(const oda_attn_shape *shape, const oda_attn_inputs *in, const oda_prefix_groups *groups,
                           void *plan, size_t plan_bytes, hipStream_t stream);

/* Full decode attention (whole histories) of T current tokens per request, with
 * the K/V of a group's prefix read once for all its members.  Row (b, t) attends
 * positions 0 .. seq_lens[b] - 1 + t:
 *   q        bf16 [L][B][T][Hq][D];  out fp32 [L][B][T][Hq][D];  lse fp32 [L][B][T][Hq]
 *   k_cur, v_cur  bf16 [L][B][T][Hkv][D]: the current tokens' candidates; the cache
 *            holds positions 0 .. seq_lens[b] - 2, row t attends candidates 0..t.
 *            NULL: the cache holds the current tokens too, positions up to
 *            seq_lens[b] - 2 + n_tokens[b]
 * The result of each row is that of oda_full_decode_attn for a request of length
 * seq_lens[b] + t, up to rounding.  Only rows of the groups' flagged members with
 * t < n_tokens[b] are written.
 * A request whose length (with its current tokens in the cache, their last
 * position) is outside [1, max_seq_len] or shorter than its group's prefix, or
 * that uses a table entry outside [0, num_blocks), gets NaN rows; an entry of the
 * prefix does that to the whole group.  A plan made for another batch, num_groups,
 * tokens, table width, number of query heads per KV head or kind of candidate
 * gives NaN throughout.  workspace: >= oda_prefix_workspace_size bytes, 256-byte aligned;
 * calls that may overlap in time need separate ones (a plan may be shared). */
oda_status oda_prefix_decode_attn(const oda_attn_shape *shape, const oda_attn_inputs *in,
                                  const oda_prefix_groups *groups, const void *plan, size_t plan_bytes, float *out,
                                  float *lse, void *workspace, size_t workspace_bytes, hipStream_t stream);

#define ODA_LORA_MAX_PARTS 4

/* Low-rank adapters of a dense layer (host struct holding device pointers).  A
 * fused projection has parts (query, key and value; gate and up), each with
 * rank rows of A of its own: output row r of part p of a request with adapter
 * a gets  scale[a] * sum_i B[a][r][i] (A[a] x')[p * rank + i].
 * Adapters of lower rank are padded with zero rows of A or columns of B. */
typedef struct {
  int32_t num_adapters;      /* >= 1                                                */
  int32_t rank;              /* a multiple of 8, at most 128                         */
  int32_t num_parts;         /* 1..ODA_LORA_MAX_PARTS                                */
  int32_t part_rows[ODA_LORA_MAX_PARTS]; /* rows of each part (>= 1); their sum is the
                                weight's rows: N, or 2N for SWIGLU                   */
  const uint16_t *a;         /* device bf16 [num_adapters][num_parts * rank][K]      */
  const uint16_t *b;         /* device bf16 [num_adapters][rows][rank]               */
  const float *scale;        /* device fp32 [num_adapters] (alpha / rank)            */
} oda_lora_desc;

/* Bytes of workspace oda_dense_lora_bf16 needs for `batch` requests (host out).
 * Its contents between calls do not matter. */
oda_status oda_lora_workspace_size(const oda_lora_desc *lora, int32_t batch, size_t *bytes);

/* oda_dense_bf16 with a low-rank adapter beside the weight, per request:
 *   PLAIN:  y[b] = (W + s_a B_a A_a) x'[b]  (+ residual[b])
 *   SWIGLU: the same sum before SiLU and the product
 * where a = adapter_ids[b] and x' is the (normalised) input.
 *   adapter_ids: int32 [batch]; -1: no adapter (the shared layer alone); an id
 *                outside [-1, num_adapters) gives a row of NaN
 *   workspace:   >= oda_lora_workspace_size bytes, 256-byte aligned; calls that
 *                may overlap in time need separate workspaces
 * Everything else (modes, residual, list, alignment) as in oda_dense_bf16; a and
 * b 16-byte aligned.  Sums are fp32. */
oda_status oda_dense_lora_bf16(const oda_dense_desc *desc, const oda_lora_desc *lora, int32_t batch,
                               const float *x, const float *residual, float *y, const int32_t *adapter_ids,
                               const int32_t *work_list, const int32_t *n_work, void *workspace,
                               size_t workspace_bytes, hipStream_t stream);

/* Drafts to verify (host struct holding device pointers).  Row i of a request's
 * logits is the target's distribution of the token at draft i's place (the last
 * one in use: of the token after the drafts). */
typedef struct {
  int32_t vocab;               /* V >= 1                                            */
  int32_t max_drafts;          /* K, 0..63 (0: draws one token from one row)        */
  const float *logits;         /* fp32 [batch][K + 1][V]; NaN counts as -infinity    */
  const float *draft_probs;    /* fp32 [batch][K][V]: the probabilities each draft was
                                  drawn from (negative or NaN counts as 0); NULL:
                                  drafts that were not drawn (probability 1 each)   */
  const int32_t *draft_tokens; /* int32 [batch][K]; NULL iff K == 0                  */
  const int32_t *n_drafts;     /* int32 [batch], clamped to [0, K]; NULL: K each     */
  const float *temperature;    /* fp32 [batch]; NULL: 1.  Above 0: softmax of logits /
                                  temperature, clamped to [2^-100, 2^100]; else (0,
                                  negative, NaN) greedy                             */
  const float *uniform;        /* fp32 [batch][K + 1] in [0, 1): u_0..u_{K-1} for the
                                  drafts, u_K for the next token                    */
} oda_verify_desc;

/* Bytes of workspace oda_verify_drafts needs (host out).  Zero-fill it before
 * its first use (ticket words; every call leaves them zero); it serves any later
 * call on the stream with the same batch and at most the same V and K. */
oda_status oda_verify_workspace_size(int32_t batch, int32_t vocab, int32_t max_drafts, size_t *bytes);

/* Verification of drafted tokens by rejection sampling, which keeps the target's
 * distribution.  With p_i = softmax(logits_i / temperature) (greedy: all on the
 * first largest logit) and q_i the draft's probabilities, draft x_i is accepted
 * iff u_i q_i(x_i) < p_i(x_i), up to the first refusal, at j.  The next token is
 * then the smallest v whose cumulative weight exceeds u_K times the sum of all,
 * with the weights max(p_j - q_j, 0) after a refusal (p_j where these are all
 * zero), p_n when all n drafts were accepted.
 *   n_accepted: int32 [batch] out
 *   tokens:     int32 [batch][K + 1] out: the accepted drafts, the next token,
 *               then -1
 * A draft outside [0, V) is refused.  A row with no logit above -infinity
 * refuses its draft and gives the next token -1; logits of +infinity share the
 * row's probability evenly.  Weights and sums are fp64 (weights below about
 * 2^-1000 of the row's largest are 0).  Rows past n_drafts are not read.  work_list / n_work as in oda_dense_bf16. */
oda_status oda_verify_drafts(const oda_verify_desc *desc, int32_t batch, int32_t *n_accepted, int32_t *tokens,
                             const int32_t *work_list, const int32_t *n_work, void *workspace,
                             size_t workspace_bytes, hipStream_t stream);

/* oda_commit_kv of several tokens per request: the first n_accepted[b] + 1
 * (clamped to [0, tokens]) current tokens' candidates of every layer go to
 * positions n_b - 1, n_b, ... of the paged cache, and to the rings if given;
 * then, if advance != 0, seq_lens[b] grows by that number.
 *   tokens:       T, 1..64
 *   k_cand, v_cand: bf16 [L][B][T][Hkv][D]
 *   n_accepted:   int32 [B], as oda_verify_drafts writes it (-1: nothing is
 *                 committed for the request), or NULL: all T tokens
 *   row_lens:     NULL, or int32 [B][T] out (advance != 0): the new seq_lens[b]
 *                 + t, the lengths of the next step's rows (oda_qk_norm_rope)
 *   k_ring, v_ring, n_sink, window: as in oda_commit_kv_ring, or NULL, 0, 0
 * Workspace, shape fields and the rest as in oda_commit_kv.  A table entry
 * outside [0, num_blocks), or a position outside the table, drops that token's
 * candidates (the length still grows). */
oda_status oda_commit_drafts(const oda_attn_shape *shape, int32_t tokens, uint16_t *k_cache, uint16_t *v_cache,
                             const int32_t *block_table, int32_t *seq_lens, const uint16_t *k_cand,
                             const uint16_t *v_cand, const int32_t *n_accepted, int32_t advance, int32_t *row_lens,
                             void *workspace, size_t workspace_bytes, uint16_t *k_ring, uint16_t *v_ring,
                             int32_t n_sink, int32_t window, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Prompts.  A chunk of new tokens per request, from single tokens to whole
 * prompts, side by side in the rows of every buffer (no padding between requests):
 * their K/V is appended to the paged cache, their attention runs over it, and the
 * log probabilities of their tokens are formed.  decoder.PromptDecoder composes the
 * forward of a chunk from these and the dense layers above.
 * ------------------------------------------------------------------------- */

typedef enum { ODA_F32 = 0, ODA_BF16 = 1 } oda_type;

/* Rows of a batch (host struct holding device pointers): request b has the rows
 * row_start[b] .. row_start[b + 1] - 1, possibly none.  Starts are taken into
 * [0, num_rows] and as ascending, whatever the array holds; rows in front of the
 * first or behind the last request's are neither read nor written. */
typedef struct {
  int32_t num_rows;           /* rows of the buffers, >= 1                          */
  const int32_t *row_start;   /* int32 [B + 1]                                      */
} oda_prompt_rows;

/* What oda_append_qkv does to the rows on their way (host struct holding device
 * pointers).
 *   qkv        fp32 or bf16 [num_rows][(Hq + 2 Hkv) D]: q heads, then k heads, then
 *              v heads (k and v heads alone where q_out is NULL, q heads alone where
 *              the caches are); 16-byte aligned
 *   q_gain, k_gain  fp32 [D] per-head RMSNorm gains, or NULL (no norm)
 *   rope_theta > 1: dims i and i + D/2 of q and k heads turn by p theta^(-2i/D),
 *              angles in double; 0: no rotation
 *   positions  int32 [num_rows][num_axes]: p of a pair is its axis's position; NULL
 *              (one axis): the row's place in the history
 *   axis_pairs pairs of each axis (time, height, width ...): the first axis_pairs[0]
 *              pairs take the first, and so on; their sum is D/2.  Ignored for one axis
 * All of D turns, by these frequencies as they are: axes that alternate from pair to
 * pair, rotations of a part of D and rescaled frequencies are the caller's (theta 0). */
#define ODA_MAX_AXES 4
typedef struct {
  const void *qkv;
  int32_t qkv_type;             /* oda_type                                          */
  float rms_eps;                /* >= 0                                              */
  const float *q_gain;
  const float *k_gain;
  double rope_theta;
  const int32_t *positions;
  int32_t num_axes;             /* 1..ODA_MAX_AXES                                   */
  int32_t axis_pairs[ODA_MAX_AXES];
} oda_append_desc;

/* Appends a chunk of one layer (num_layers == 1): row i of a request's m rows is
 * place seq_lens[b] - m + i of its history, seq_lens[b] counting the chunk.  Heads
 * are normed, turned and rounded to bf16 (nearest-even) as by oda_qk_norm_rope; q
 * goes to q_out, K and V to the paged cache and, if given, to the rings (what they
 * still hold after the chunk), in one launch.
 *   q_out    bf16 [num_rows][Hq][D], or NULL: the rows have no q heads
 *   k_cache, v_cache  both NULL: the rows have q heads alone (the queries of an
 *            attention over other states); block_table is then not read
 *   k_ring, v_ring, n_sink, window: as in oda_commit_kv_ring, or NULL, 0, 0
 * A request whose length is outside [0, max_seq_len] or shorter than its rows gets
 * NaN queries and appends nothing; a table entry outside [0, num_blocks) drops the
 * K/V of its places, from the rings too.  Places are written once: requests must not
 * share the blocks that they append to. */
oda_status oda_append_qkv(const oda_attn_shape *shape, const oda_prompt_rows *rows, const oda_append_desc *desc,
                          uint16_t *k_cache, uint16_t *v_cache, const int32_t *block_table, const int32_t *seq_lens,
                          uint16_t *q_out, uint16_t *k_ring, uint16_t *v_ring, int32_t n_sink, int32_t window,
                          hipStream_t stream);

/* Bytes of the plan buffer and of the workspace of calls with these sizes (the
 * shape and num_rows) (host out).  Neither needs to be cleared. */
oda_status oda_prompt_plan_size(const oda_attn_shape *shape, const oda_prompt_rows *rows, size_t *bytes);
oda_status oda_prompt_workspace_size(const oda_attn_shape *shape, const oda_prompt_rows *rows, size_t *bytes);

/* Plans oda_prompt_attn on the device: the rows' tiles, and how their histories are
 * split over the chip.  One plan serves every call whose shape, rows, lengths and
 * mask are the plan's (all layers of a step).  When lengths or row starts change,
 * plan again: the attention reads them from the plan.
 *   causal:        1: row i of a request's m rows attends places 0 .. seq_lens[b] - m + i;
 *                  0: every row attends all of 0 .. seq_lens[b] - 1 (states of another
 *                  length, such as an encoder's; seq_lens[b] may be 0: the rows are then
 *                  zeros, their lse -infinity)
 *   native_window: > 0 (causal): only the last native_window of them (natively
 *                  windowed layers)
 *   plan:          >= oda_prompt_plan_size bytes, 256-byte aligned
 * shape->num_layers must be 1 and split_blocks 0; batch at most 2048. */
oda_status oda_prompt_plan(const oda_attn_shape *shape, const oda_prompt_rows *rows, const int32_t *seq_lens,
                           int32_t causal, int32_t native_window, void *plan, size_t plan_bytes, hipStream_t stream);

/* Attention of the planned rows over the paged cache, which holds all they attend
 * (the chunk's own K/V too: oda_append_qkv).  in->seq_lens is not read (the plan has
 * the lengths); in->k_cur and v_cur must be NULL.
 *   q    bf16 [num_rows][Hq][D]
 *   out  fp32 or bf16 (out_type) [num_rows][Hq][D], 16-byte aligned: the weights of an
 *        fp32 output hold all of their 24 bits, as in decode attention; those of a bf16
 *        output are rounded to bf16, which takes half the matrix operations
 *   lse  fp32 [num_rows][Hq] (natural log), or NULL
 * A request whose length is outside [0, max_seq_len] (or above 2^31 - 65) or
 * (causal) shorter than its rows gets NaN rows, and so does a row that attends a
 * block whose table entry is outside [0, num_blocks); other rows do not see it.
 * Slots that no row attends may hold anything; a value that is not finite reaches
 * the rows that attend it alone.  A plan made for another batch, num_rows, head
 * counts, table width or max_seq_len gives NaN throughout.
 * workspace: >= oda_prompt_workspace_size bytes, 256-byte
 * aligned; calls that may overlap in time need separate ones (a plan may be shared). */
oda_status oda_prompt_attn(const oda_attn_shape *shape, const oda_attn_inputs *in, const oda_prompt_rows *rows,
                           const void *plan, size_t plan_bytes, void *out, int32_t out_type, float *lse,
                           void *workspace, size_t workspace_bytes, hipStream_t stream);

#define ODA_MAX_TOP 32

/* Rows of logits to score (host struct holding device pointers). */
typedef struct {
  int32_t vocab;                /* V >= 1                                            */
  int32_t top;                  /* k: alternatives per row, 0..ODA_MAX_TOP            */
  int64_t row_stride;           /* floats from one row to the next; 0: V, else >= V   */
  const float *logits;          /* fp32; NaN counts as -infinity                      */
  const int32_t *tokens;        /* int32 [rows]: the given tokens, or NULL            */
} oda_logprob_desc;

/* Bytes of workspace oda_token_logprobs needs (host out).  Zero-fill it before its
 * first use (ticket words; every call leaves them zero); it serves any later call on
 * the stream. */
oda_status oda_logprob_workspace_size(const oda_logprob_desc *desc, int32_t rows, size_t *bytes);

/* With p = softmax(logits of the row) and tokens in the order of their logits (equal
 * ones by their index):
 *   logprob      fp32 [rows]: log p(tokens[r]); rank int32 [rows]: its place in the
 *                order, from 1.  A token outside [0, V): NaN and 0.  Both NULL where
 *                tokens is NULL; either may be NULL
 *   entropy      fp32 [rows]: -sum p log p, or NULL
 *   top_logprobs fp32 [rows][k], top_tokens int32 [rows][k]: the first k of the order;
 *                where fewer logits are above -infinity, -infinity and -1 behind
 *                them.  Both NULL iff k == 0
 * Logits of +infinity share the row's probability evenly.  A row with no logit above
 * -infinity has no distribution: logprob and entropy are NaN.  work_list / n_work as
 * in oda_dense_bf16 (the listed rows alone are read and written). */
oda_status oda_token_logprobs(const oda_logprob_desc *desc, int32_t rows, float *logprob, int32_t *rank, float *entropy,
                              float *top_logprobs, int32_t *top_tokens, const int32_t *work_list, const int32_t *n_work,
                              void *workspace, size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Measurement aid (not a step of the method): the streaming-read ceiling that
 * the attention kernels' bandwidth is quoted against.
 * ------------------------------------------------------------------------- */

/* Reads `bytes` of device memory at src once (16-byte nontemporal loads, the
 * attention kernels' KV loads) and discards them.  src 16-byte aligned, bytes a
 * multiple of 16; sink: device uint32[1], left unchanged in practice (written
 * only if the XOR of everything read hits one fixed value); groups: workgroups
 * of 256 threads, 0 for the default (256). */
oda_status oda_stream_read(const void *src, size_t bytes, uint32_t *sink, int32_t groups, hipStream_t stream);

/* Static description of a status code. */
const char *oda_status_string(oda_status status);

/* Thread-local detail of the last non-OK return on this thread ("" if none). */
const char *oda_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* ODA_H_ */
