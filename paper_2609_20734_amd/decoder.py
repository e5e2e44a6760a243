"""A whole ODA decode step on a synthetic decoder, composed from the C-ABI
entry points (every operation runs in liboda's HIP kernels; this module only
prepares the calls).

Per step (Alg. 1 with the commit of App. A.5):

  local stage   embed the step's tokens; the Local forward (every layer:
                QKV, q/k norm + rotary, Local attention with the Local
                candidate, output projection, SwiGLU MLP); the final RMSNorm
                of the Local hidden state (h^L_t, §2.1); the recall gate on
                (h_{t-1}, E(x_t), h^L_t), writing flags and the compacted list
  retry stage   the Full forward from the same pre-step history for the listed
                requests only, then their final hidden rows replace the Local
                ones (App. A.5: only the selected state is kept)
  output stage  the final RMSNorm of the selected state (this is h_{t-1} of
                the next step's gate, App. A.5) and the vocabulary projection
                of it, greedy token, the fused commit of the selected
                candidates of every layer

Native Full (always Full, no gate) and standalone Local (no gate, no retry)
use the same pieces.  DraftDecoder composes the step of many tenants with drafted
tokens: shared-prefix attention, adapters beside the dense layers, verification
and the commit of what was accepted.  PromptDecoder takes prompts in: chunks of many
tokens per request through the same layers into the paged cache, from which the
others go on.  Stages are lists of pre-marshalled calls, so they can be
launched eagerly or captured as HIP graphs.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

from . import _lib as P


@dataclass(frozen=True)
class DecoderShape:
    num_layers: int
    d_model: int
    num_q_heads: int
    num_kv_heads: int
    head_dim: int
    d_ffn: int
    vocab: int
    rms_eps: float = 1e-6
    rope_theta: float = 1e6

    @property
    def qkv_dim(self) -> int:
        return (self.num_q_heads + 2 * self.num_kv_heads) * self.head_dim

    def weight_bytes(self) -> int:
        """bf16 weight bytes one forward streams (vocabulary projection included)."""
        d, L = self.d_model, self.num_layers
        per_layer = (self.qkv_dim * d + d * self.num_q_heads * self.head_dim + 3 * self.d_ffn * d) * 2
        return L * per_layer + self.vocab * d * 2


# Qwen3-1.7B-shaped backbone (the model of the paper's throughput table):
# 28 layers, d = 2048, 16 query / 8 KV heads of 128, SwiGLU 6144, 151,936 tokens.
QWEN3_1_7B = DecoderShape(28, 2048, 16, 8, 128, 6144, 151936)


class Decoder:
    """Device buffers and prepared calls of one decoder over a paged cache.

    weights: dict of device tensors named as oda_synth.decoder_tensor_specs
    (bf16 weights, fp32 gains); cache, table and lengths as the attention ABI
    takes them; gate: a GateDesc for the recall head (None: no gate);
    prescribed: the gate takes its flags from `self.forced` (int32 [B], written
    before each step) instead of comparing the score with tau (App. B.7);
    fused_prep: each attention call builds its query and candidate K/V from the
    QKV projection itself (oda_*_decode_attn_qkv, bit-identical), else
    oda_qk_norm_rope runs as a launch of its own before it."""

    def __init__(self, shape: DecoderShape, weights: dict, batch: int, k_cache, v_cache, block_table, seq_lens,
                 max_blocks_per_seq: int, max_seq_len: int, num_blocks: int, n_sink: int, window: int,
                 gate=None, tau: float = 0.0, prescribed: bool = False, split_blocks: int = 0,
                 fused_prep: bool = True):
        import torch
        s, B = shape, batch
        dev = k_cache.device
        self.shape, self.B, self.w = s, B, weights
        self.k_cache, self.v_cache, self.table, self.seq_lens = k_cache, v_cache, block_table, seq_lens
        self.n_sink, self.window = n_sink, window
        self.fused_prep = fused_prep
        f32 = dict(dtype=torch.float32, device=dev)
        bf = dict(dtype=torch.bfloat16, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        L, d, Hq, Hkv, D = s.num_layers, s.d_model, s.num_q_heads, s.num_kv_heads, s.head_dim
        self.tokens = torch.zeros(B, **i32)            # the step's tokens (written before each step)
        self.emb = torch.zeros(B, d, **f32)
        self.h = torch.zeros(B, d, **f32)               # selected state (Local stream, then selected)
        self.h_full = torch.zeros(B, d, **f32)          # Full retry stream
        self.h_prev = torch.zeros(B, d, **f32)         # final-normalised selected state of the last step
        self.h_local = torch.zeros(B, d, **f32)        # final-normalised Local state (the gate's h^L_t)
        self.qkv = torch.zeros(B, s.qkv_dim, **f32)
        self.q = torch.zeros(B, Hq, D, **bf)
        self.attn = torch.zeros(B, Hq * D, **f32)
        self.lse = torch.zeros(B, Hq, **f32)
        self.mlp = torch.zeros(B, s.d_ffn, **f32)
        self.logits = torch.zeros(B, s.vocab, **f32)
        self.next_token = torch.zeros(B, **i32)
        self.k_loc = torch.zeros(L, B, Hkv, D, **bf)
        self.v_loc = torch.zeros(L, B, Hkv, D, **bf)
        self.k_full = torch.zeros(L, B, Hkv, D, **bf)
        self.v_full = torch.zeros(L, B, Hkv, D, **bf)
        self.score = torch.zeros(B, **f32)
        self.flags = torch.zeros(B, **i32)
        self.work = torch.zeros(B, **i32)
        self.n_work = torch.zeros(1, **i32)
        self.counter = torch.zeros(1, dtype=torch.int64, device=dev)
        self.gate, self.tau = gate, tau
        self.forced = torch.zeros(B, **i32) if prescribed else None
        self.ws_gate = None if gate is None else torch.zeros(P.gate_workspace_size(gate, B), dtype=torch.uint8,
                                                             device=dev)
        # one-layer attention calls: the layer's slices of the caches and candidates
        self.attn_shape = P.Shape(1, B, Hq, Hkv, D, max_blocks_per_seq, max_seq_len, num_blocks, split_blocks)
        self.ws_local = torch.zeros(max(256, P.attn_workspace_size(self.attn_shape, n_sink, window)),
                                    dtype=torch.uint8, device=dev)
        self.ws_full = torch.zeros(max(256, P.attn_workspace_size(self.attn_shape, 0, 0)), dtype=torch.uint8,
                                   device=dev)
        self.ws_commit = torch.zeros(P.commit_workspace_size(self.commit_shape()), dtype=torch.uint8, device=dev)
        self.scale = 1.0 / math.sqrt(D)
        w = weights
        self.d_qkv = [P.dense_desc(d, s.qkv_dim, P.DENSE_PLAIN, w["w_qkv"][l], w["attn_norm"][l], s.rms_eps)
                      for l in range(L)]
        self.d_o = [P.dense_desc(Hq * D, d, P.DENSE_PLAIN, w["w_o"][l]) for l in range(L)]
        self.d_gu = [P.dense_desc(d, s.d_ffn, P.DENSE_SWIGLU, w["w_gu"][l], w["mlp_norm"][l], s.rms_eps)
                     for l in range(L)]
        self.d_down = [P.dense_desc(s.d_ffn, d, P.DENSE_PLAIN, w["w_down"][l]) for l in range(L)]
        # the vocabulary projection reads the final-normalised state (h_prev after the output stage's norm)
        self.d_vocab = P.dense_desc(d, s.vocab, P.DENSE_PLAIN, w["embed"])

    # -- stages ---------------------------------------------------------------
    def _forward(self, h, k_cand, v_cand, branch: str, listed: bool):
        """Calls of one forward on stream h (branch "local" or "full")."""
        s, B = self.shape, self.B
        wl = (self.work, self.n_work) if listed else (None, None)
        calls = []
        for l in range(s.num_layers):
            calls.append(P.prepare_dense(self.d_qkv[l], B, h, None, self.qkv, *wl))
            if self.fused_prep:
                prep = P.qkv_prep(self.qkv, self.w["q_norm"][l], self.w["k_norm"][l], s.rms_eps, s.rope_theta,
                                  k_cand[l], v_cand[l])
                inp = P.inputs(None, self.k_cache[l], self.v_cache[l], self.table, self.seq_lens, self.scale)
                if branch == "local":
                    calls.append(P.prepare_local_qkv(self.attn_shape, inp, prep, self.n_sink, self.window, self.attn,
                                                     self.lse, self.ws_local))
                else:
                    calls.append(P.prepare_full_qkv(self.attn_shape, inp, prep, 0, None, *wl, self.attn, self.lse,
                                                    self.ws_full))
            else:
                calls.append(P.prepare_qk_norm_rope(B, s.num_q_heads, s.num_kv_heads, s.head_dim, self.qkv,
                                                    self.w["q_norm"][l], self.w["k_norm"][l], s.rms_eps,
                                                    s.rope_theta, self.seq_lens, self.q, k_cand[l], v_cand[l], *wl))
                inp = P.inputs(self.q, self.k_cache[l], self.v_cache[l], self.table, self.seq_lens, self.scale,
                               k_cand[l], v_cand[l])
                if branch == "local":
                    calls.append(P.prepare_local(self.attn_shape, inp, self.n_sink, self.window, self.attn,
                                                 self.lse, self.ws_local))
                else:
                    calls.append(P.prepare_full(self.attn_shape, inp, 0, None, *wl, self.attn, self.lse,
                                                self.ws_full))
            calls.append(P.prepare_dense(self.d_o[l], B, self.attn, h, h, *wl))
            calls.append(P.prepare_dense(self.d_gu[l], B, h, None, self.mlp, *wl))
            calls.append(P.prepare_dense(self.d_down[l], B, self.mlp, h, h, *wl))
        return calls

    def _input(self):
        s, B = self.shape, self.B
        return [P.prepare_embed(self.w["embed"], s.vocab, s.d_model, B, self.tokens, self.emb),
                P.prepare_copy_rows(B, s.d_model, self.emb, self.h)]

    def _output(self, k_full=None, v_full=None, flags=None):
        s, B = self.shape, self.B
        return [P.prepare_rms_norm_rows(B, s.d_model, self.h, self.w["final_norm"], s.rms_eps, self.h_prev),
                P.prepare_dense(self.d_vocab, B, self.h_prev, None, self.logits),
                P.prepare_argmax(B, s.vocab, self.logits, self.next_token),
                P.prepare_commit(self.commit_shape(), self.k_cache, self.v_cache, self.table, self.seq_lens,
                                 self.k_loc, self.v_loc, k_full, v_full, flags, True, self.ws_commit)]

    def commit_shape(self) -> P.Shape:
        a = self.attn_shape
        return P.Shape(self.shape.num_layers, a.batch, a.num_q_heads, a.num_kv_heads, a.head_dim,
                       a.max_blocks_per_seq, a.max_seq_len, a.num_blocks, a.split_blocks)

    def oda_stages(self):
        """(local stage, retry stage, output stage) of one ODA step."""
        s, B = self.shape, self.B
        assert self.gate is not None
        local = self._input() + self._forward(self.h, self.k_loc, self.v_loc, "local", False)
        local.append(P.prepare_rms_norm_rows(B, s.d_model, self.h, self.w["final_norm"], s.rms_eps, self.h_local))
        local.append(P.prepare_gate(self.gate, B, self.h_prev, self.emb, self.h_local, self.tau, self.forced,
                                    self.score, self.flags, self.work, self.n_work, self.counter, self.ws_gate))
        retry = [P.prepare_copy_rows(B, s.d_model, self.emb, self.h_full, self.work, self.n_work)]
        retry += self._forward(self.h_full, self.k_full, self.v_full, "full", True)
        retry.append(P.prepare_copy_rows(B, s.d_model, self.h_full, self.h, self.work, self.n_work))
        out = self._output(self.k_full, self.v_full, self.flags)
        return local, retry, out

    def full_stages(self):
        """Native Full: every layer over its whole history, no gate."""
        return self._input() + self._forward(self.h, self.k_loc, self.v_loc, "full", False), [], self._output()

    def local_stages(self):
        """Standalone Local: every layer over S^L, no gate, no retry."""
        return self._input() + self._forward(self.h, self.k_loc, self.v_loc, "local", False), [], self._output()


class DraftDecoder:
    """Decode steps of many tenants with drafted tokens: one forward of each
    request's current token and its drafts (Full attention in every layer), the
    drafts verified, the accepted tokens committed, the next token drawn.

    Row b * T + t of the buffers is token t of request b.  Before a step, `tokens`
    [B][T] holds the last committed choice's successor (the current token) and the
    drafts, `drafts` [B][T - 1] the drafts again, `n_drafts` / `n_tokens` [B] how
    many of each are in use (set_drafts writes the four), `uniform` [B][T] the random
    numbers.  After it, `accepted` [B] and `answer` [B][T] (accepted drafts, next
    token, -1) are oda_verify_drafts' outputs, and caches, lengths and row_lens are
    ready for the next step.

    groups: (group_start, members, prefix_blocks), int32 device tensors: requests
    whose prompts share their first blocks, every request in one group (of no blocks
    if it shares none); adapters: {"w_qkv" | "w_o" | "w_gu" |
    "w_down": [LoraDesc per layer]}, any of them, chosen per request by adapter_ids
    [B] (-1: none); temperature: fp32 [B] or None; draft_probs: True to verify
    against `probs` [B][T - 1][V] (written before each step), else drafts count as
    given."""

    def __init__(self, shape: DecoderShape, weights: dict, batch: int, tokens: int, k_cache, v_cache, block_table,
                 seq_lens, max_blocks_per_seq: int, max_seq_len: int, num_blocks: int, groups, adapters: dict | None = None,
                 adapter_ids=None, temperature=None, draft_probs: bool = False):
        import torch
        s, B, T = shape, batch, tokens
        dev = k_cache.device
        self.shape, self.B, self.T, self.w = s, B, T, weights
        self.k_cache, self.v_cache, self.table, self.seq_lens = k_cache, v_cache, block_table, seq_lens
        self.temperature = temperature
        f32 = dict(dtype=torch.float32, device=dev)
        bf = dict(dtype=torch.bfloat16, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        L, d, Hq, Hkv, D, rows = s.num_layers, s.d_model, s.num_q_heads, s.num_kv_heads, s.head_dim, B * T
        self.tokens = torch.zeros(B, T, **i32)
        self.drafts = torch.zeros(B, max(1, T - 1), **i32)
        self.n_tokens = torch.full((B,), T, **i32)
        self.n_drafts = torch.full((B,), T - 1, **i32)
        self.uniform = torch.zeros(B, T, **f32)
        self.probs = torch.zeros(B, T - 1, s.vocab, **f32) if draft_probs and T > 1 else None
        self.accepted = torch.zeros(B, **i32)
        self.answer = torch.zeros(B, T, **i32)
        self.row_lens = (seq_lens[:, None] + torch.arange(T, **i32)).to(torch.int32).contiguous()
        self.h = torch.zeros(rows, d, **f32)
        self.state = torch.zeros(rows, d, **f32)       # final-normalised
        self.qkv = torch.zeros(rows, s.qkv_dim, **f32)
        self.q = torch.zeros(B, T, Hq, D, **bf)
        self.attn = torch.zeros(rows, Hq * D, **f32)
        self.mlp = torch.zeros(rows, s.d_ffn, **f32)
        self.logits = torch.zeros(B, T, s.vocab, **f32)
        self.k_cand = torch.zeros(L, B, T, Hkv, D, **bf)
        self.v_cand = torch.zeros(L, B, T, Hkv, D, **bf)
        self.scale = 1.0 / math.sqrt(D)
        self.adapters = adapters or {}
        self.row_adapters = None if adapter_ids is None else \
            adapter_ids.to(torch.int32).repeat_interleave(T).contiguous()
        if self.adapters and self.row_adapters is None:
            raise ValueError("adapters need adapter_ids")
        start, members, prefix = groups
        self.attn_shape = P.Shape(1, B, Hq, Hkv, D, max_blocks_per_seq, max_seq_len, num_blocks)
        self.commit_shape = P.Shape(L, B, Hq, Hkv, D, max_blocks_per_seq, max_seq_len, num_blocks)
        self.groups = P.prefix_groups(prefix.numel(), T, start, members, prefix, self.n_tokens)

        def zeros(n):
            return torch.zeros(max(256, n), dtype=torch.uint8, device=dev)

        self.plan = zeros(P.prefix_plan_size(self.attn_shape, self.groups))
        self.ws_attn = zeros(P.prefix_workspace_size(self.attn_shape, self.groups))
        self.ws_lora = zeros(max([P.lora_workspace_size(d, rows) for a in self.adapters.values() for d in a], default=0))
        self.ws_verify = zeros(P.verify_workspace_size(B, s.vocab, T - 1))
        self.ws_commit = zeros(P.commit_workspace_size(self.commit_shape))
        w = weights
        self.desc = dict(
            w_qkv=[P.dense_desc(d, s.qkv_dim, P.DENSE_PLAIN, w["w_qkv"][l], w["attn_norm"][l], s.rms_eps) for l in range(L)],
            w_o=[P.dense_desc(Hq * D, d, P.DENSE_PLAIN, w["w_o"][l]) for l in range(L)],
            w_gu=[P.dense_desc(d, s.d_ffn, P.DENSE_SWIGLU, w["w_gu"][l], w["mlp_norm"][l], s.rms_eps) for l in range(L)],
            w_down=[P.dense_desc(s.d_ffn, d, P.DENSE_PLAIN, w["w_down"][l]) for l in range(L)])
        self.d_vocab = P.dense_desc(d, s.vocab, P.DENSE_PLAIN, w["embed"])

    def set_drafts(self, current, drafts, n_drafts) -> None:
        """The next step's current tokens [B], drafts [B][T - 1] and their counts [B] (clamped to [0, T - 1])."""
        self.tokens[:, 0].copy_(current)
        if self.T > 1:
            self.tokens[:, 1:].copy_(drafts)
            self.drafts.copy_(drafts)
        self.n_drafts.copy_(n_drafts.clamp(0, self.T - 1))
        self.n_tokens.copy_(self.n_drafts + 1)

    def _dense(self, name: str, l: int, x, residual, y):
        rows = self.B * self.T
        if name in self.adapters:
            return P.prepare_dense_lora(self.desc[name][l], self.adapters[name][l], rows, x, residual, y, self.row_adapters,
                                        self.ws_lora)
        return P.prepare_dense(self.desc[name][l], rows, x, residual, y)

    def stages(self):
        """(forward, verification, commit) of one step, as prepared calls."""
        s, B, T = self.shape, self.B, self.T
        rows = B * T

        def inputs(l):
            return P.inputs(self.q, self.k_cache[l], self.v_cache[l], self.table, self.seq_lens, self.scale, self.k_cand[l],
                            self.v_cand[l])

        forward = [P.prepare_embed(self.w["embed"], s.vocab, s.d_model, rows, self.tokens, self.h),
                   P.prepare_prefix_plan(self.attn_shape, inputs(0), self.groups, self.plan)]
        for l in range(s.num_layers):
            forward += [
                self._dense("w_qkv", l, self.h, None, self.qkv),
                P.prepare_qk_norm_rope(rows, s.num_q_heads, s.num_kv_heads, s.head_dim, self.qkv, self.w["q_norm"][l],
                                       self.w["k_norm"][l], s.rms_eps, s.rope_theta, self.row_lens, self.q, self.k_cand[l],
                                       self.v_cand[l]),
                P.prepare_prefix_decode_attn(self.attn_shape, inputs(l), self.groups, self.plan, self.attn, None,
                                             self.ws_attn),
                self._dense("w_o", l, self.attn, self.h, self.h),
                self._dense("w_gu", l, self.h, None, self.mlp),
                self._dense("w_down", l, self.mlp, self.h, self.h)]
        forward += [P.prepare_rms_norm_rows(rows, s.d_model, self.h, self.w["final_norm"], s.rms_eps, self.state),
                    P.prepare_dense(self.d_vocab, rows, self.state, None, self.logits)]
        verify = P.verify_desc(s.vocab, T - 1, self.logits, self.drafts if T > 1 else None, self.uniform, self.probs,
                               self.n_drafts, self.temperature)
        return (forward, [P.prepare_verify_drafts(verify, B, self.accepted, self.answer, self.ws_verify)],
                [P.prepare_commit_drafts(self.commit_shape, T, self.k_cache, self.v_cache, self.table, self.seq_lens,
                                         self.k_cand, self.v_cand, self.accepted, True, self.row_lens, self.ws_commit)])


class PromptDecoder:
    """Prompts into the paged cache, a chunk of each request at a time: one forward of
    the chunk's tokens (causal attention behind what the cache holds already), their
    K/V appended layer by layer, and, of the last row of each request or of every row,
    the log probabilities of given tokens, the entropy and the first of the order.

    set_chunk(tokens, row_start, targets) gives the next chunk: rows row_start[b] ..
    row_start[b + 1] - 1 of `tokens` are request b's (none: it waits); `seq_lens` grows by
    them and then counts what the cache holds.  Decoder and DraftDecoder count the current
    token too: add 1 to the lengths before their first step.

    rows: rows of the buffers (chunks may have fewer, but the dense layers go through all of
    them, and `logits` has a row of the vocabulary for each, whatever is scored: choose them
    for the chunks that come); rings: (k_ring, v_ring, n_sink, window) to keep the direct
    rings [L][B][..] current; axis_pairs: rotary axes of `positions` [rows][axes], written
    before each chunk (None: places of the history); score: "last" or "all" rows; top:
    alternatives per scored row; native_window: of every layer (0: the whole history)."""

    def __init__(self, shape: DecoderShape, weights: dict, batch: int, rows: int, k_cache, v_cache, block_table, seq_lens,
                 max_blocks_per_seq: int, max_seq_len: int, num_blocks: int, rings=None, axis_pairs=None, score: str = "last",
                 top: int = 0, native_window: int = 0):
        import torch
        if score not in ("last", "all"):
            raise ValueError(f"score must be 'last' or 'all' (got {score!r})")
        s, B = shape, batch
        dev = k_cache.device
        self.shape, self.B, self.rows, self.w = s, B, rows, weights
        self.k_cache, self.v_cache, self.table, self.seq_lens = k_cache, v_cache, block_table, seq_lens
        self.rings, self.axis_pairs, self.native_window = rings, axis_pairs, native_window
        f32 = dict(dtype=torch.float32, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        L, d, Hq, Hkv, D = s.num_layers, s.d_model, s.num_q_heads, s.num_kv_heads, s.head_dim
        self.tokens = torch.zeros(rows, **i32)
        self.targets = torch.full((rows,), -1, **i32)
        self.row_start = torch.zeros(B + 1, **i32)
        self.positions = None if axis_pairs is None else torch.zeros(rows, len(axis_pairs), **i32)
        self.listed = torch.zeros(rows, **i32) if score == "last" else None     # scored rows
        self.n_listed = torch.zeros(1, **i32) if score == "last" else None
        self.h = torch.zeros(rows, d, **f32)
        self.state = torch.zeros(rows, d, **f32)       # final-normalised
        self.qkv = torch.zeros(rows, s.qkv_dim, **f32)
        self.q = torch.zeros(rows, Hq, D, dtype=torch.bfloat16, device=dev)
        self.attn = torch.zeros(rows, Hq * D, **f32)
        self.mlp = torch.zeros(rows, s.d_ffn, **f32)
        self.logits = torch.zeros(rows, s.vocab, **f32)
        self.logprob, self.entropy = torch.zeros(rows, **f32), torch.zeros(rows, **f32)
        self.rank = torch.zeros(rows, **i32)
        self.top_logprobs = torch.zeros(rows, top, **f32) if top else None
        self.top_tokens = torch.zeros(rows, top, **i32) if top else None
        self.scale = 1.0 / math.sqrt(D)
        self.attn_shape = P.Shape(1, B, Hq, Hkv, D, max_blocks_per_seq, max_seq_len, num_blocks)
        self.prompt_rows = P.prompt_rows(rows, self.row_start)
        self.scored = P.logprob_desc(s.vocab, top, self.logits, self.targets)

        def zeros(n):
            return torch.zeros(max(256, n), dtype=torch.uint8, device=dev)

        self.plan = zeros(P.prompt_plan_size(self.attn_shape, self.prompt_rows))
        self.ws_attn = zeros(P.prompt_workspace_size(self.attn_shape, self.prompt_rows))
        self.ws_score = zeros(P.logprob_workspace_size(self.scored, rows))

    def set_chunk(self, tokens, row_start, targets=None) -> None:
        """The next chunk: tokens [n <= rows], row_start [B + 1], targets [n] (the tokens to score, -1: none).  Starts are
        taken into [0, n] and as ascending, as the kernels take them: lengths grow by the rows that are appended; tokens
        in front of the first or behind the last request's rows are no request's, and their scores mean nothing.  A
        request that outgrows max_seq_len has NaN scores from then on."""
        import torch
        n = tokens.numel()
        if n > self.rows:
            raise ValueError(f"{n} rows in a chunk, room for {self.rows}")
        if row_start.numel() != self.B + 1:
            raise ValueError(f"{self.B} requests need {self.B + 1} row starts (got {row_start.numel()})")
        if targets is not None and targets.numel() != n:
            raise ValueError(f"{targets.numel()} targets for {n} tokens")
        self.tokens.zero_()                             # rows of no request keep a token of the vocabulary
        self.tokens[:n].copy_(tokens)
        self.targets.fill_(-1)
        if targets is not None:
            self.targets[:n].copy_(targets)
        self.row_start.copy_(row_start.clamp(0, n).cummax(0).values)
        count = self.row_start[1:] - self.row_start[:-1]
        self.seq_lens.add_(count)
        if self.listed is not None:
            order = torch.argsort((count <= 0).to(torch.int32), stable=True)[:self.rows]     # requests with rows first
            self.listed[:order.numel()].copy_(self.row_start[1:][order] - 1)
            self.n_listed.copy_((count > 0).sum())

    def stages(self):
        """(forward, scores) of one chunk, as prepared calls."""
        s, w, n = self.shape, self.w, self.rows
        Hq, Hkv, D, d = s.num_q_heads, s.num_kv_heads, s.head_dim, s.d_model
        forward = [P.prepare_embed(w["embed"], s.vocab, d, n, self.tokens, self.h),
                   P.prepare_prompt_plan(self.attn_shape, self.prompt_rows, self.seq_lens, True, self.native_window, self.plan)]
        for l in range(s.num_layers):
            rings = () if self.rings is None else (self.rings[0][l], self.rings[1][l], self.rings[2], self.rings[3])
            desc = P.append_desc(self.qkv, w["q_norm"][l], w["k_norm"][l], s.rms_eps, s.rope_theta, self.positions,
                                 self.axis_pairs)
            inp = P.inputs(self.q, self.k_cache[l], self.v_cache[l], self.table, self.seq_lens, self.scale)
            forward += [
                P.prepare_dense(P.dense_desc(d, s.qkv_dim, P.DENSE_PLAIN, w["w_qkv"][l], w["attn_norm"][l], s.rms_eps), n,
                                self.h, None, self.qkv),
                P.prepare_append_qkv(self.attn_shape, self.prompt_rows, desc, self.k_cache[l], self.v_cache[l], self.table,
                                     self.seq_lens, self.q, *rings),
                P.prepare_prompt_attn(self.attn_shape, inp, self.prompt_rows, self.plan, self.attn, None, self.ws_attn),
                P.prepare_dense(P.dense_desc(Hq * D, d, P.DENSE_PLAIN, w["w_o"][l]), n, self.attn, self.h, self.h),
                P.prepare_dense(P.dense_desc(d, s.d_ffn, P.DENSE_SWIGLU, w["w_gu"][l], w["mlp_norm"][l], s.rms_eps), n, self.h,
                                None, self.mlp),
                P.prepare_dense(P.dense_desc(s.d_ffn, d, P.DENSE_PLAIN, w["w_down"][l]), n, self.mlp, self.h, self.h)]
        listed = (self.listed, self.n_listed)
        scores = [P.prepare_rms_norm_rows(n, d, self.h, w["final_norm"], s.rms_eps, self.state, *listed),
                  P.prepare_dense(P.dense_desc(d, s.vocab, P.DENSE_PLAIN, w["embed"]), n, self.state, None, self.logits, *listed),
                  P.prepare_token_logprobs(self.scored, n, self.logprob, self.rank, self.entropy, self.top_logprobs,
                                           self.top_tokens, self.ws_score, *listed)]
        return forward, scores


def run(calls) -> None:
    for c in calls:
        c()
