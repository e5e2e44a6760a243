"""Operators that take prompts in, fp64, by definition.  TEST INFRASTRUCTURE (see
package doc).

* ``append_rows``      -- heads of a chunk's rows normed, turned and rounded, and
  their K/V in the paged cache and the rings;
* ``prompt_attention`` -- attention of a chunk's rows over the paged cache;
* ``token_logprobs``   -- log probabilities of tokens, entropy, the first of the order.
"""
from __future__ import annotations

import numpy as np

from .attention import BLOCK_SIZE, bf16_to_f64, key_rows, value_rows
from .decoder import bf16_bits, rmsnorm, round_bf16


def turn(x, positions, axis_pairs, theta):
    """Rows x [rows][heads][D] turned: pair (i, i + D/2) by p theta^(-2i/D), p the
    position [rows][axes] of the axis that the pair belongs to."""
    D = x.shape[-1]
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    angle = np.asarray(positions, dtype=np.float64)[:, axis] * theta ** (-2.0 * np.arange(D // 2) / D)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    lo, hi = x[..., :D // 2], x[..., D // 2:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def append_rows(qkv, Hq, Hkv, D, row_start, seq_lens, q_gain=None, k_gain=None, eps=0.0, theta=0.0, positions=None,
                axis_pairs=None):
    """qkv f64 [rows][(Hq + 2 Hkv) D] -> (q, k, v) f64 [rows][heads][D], not yet rounded, and the place of each row in
    its request's history with the request: (request, place) per row (-1, -1: none)."""
    R = qkv.shape[0]
    owner = np.full((R, 2), -1, dtype=np.int64)
    for b, n in enumerate(seq_lens):
        m = row_start[b + 1] - row_start[b]
        for i in range(m):
            owner[row_start[b] + i] = b, n - m + i
    x = qkv.reshape(R, Hq + 2 * Hkv, D)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    q = rmsnorm(q, q_gain, eps) if q_gain is not None else q
    k = rmsnorm(k, k_gain, eps) if k_gain is not None else k
    if theta:
        p = owner[:, 1:] if positions is None else np.asarray(positions).reshape(R, -1)
        pairs = [D // 2] if axis_pairs is None else axis_pairs
        q, k = turn(q, p, pairs, theta), turn(k, p, pairs, theta)
    return q, k, v, owner


def put_rows(k, v, owner, table, seq_lens, k_cache, v_cache, k_ring=None, v_ring=None, sink_blocks=0, ring_blocks=0):
    """Writes rows' K and V, rounded to bf16, into one layer's caches uint16 [NB][Hkv][..], and, where the ring still holds
    a row's block after its request's seq_lens positions, into the rings [B][blocks][Hkv][..]."""
    kb, vb = bf16_bits(round_bf16(k)), bf16_bits(round_bf16(v))
    D = k.shape[-1]
    for r, (b, p) in enumerate(owner):
        if b < 0:
            continue
        j, slot, blk = p // BLOCK_SIZE, p % BLOCK_SIZE, table[b, p // BLOCK_SIZE]
        k_cache[blk, :, :, slot, :] = kb[r].reshape(-1, D // 8, 8)
        v_cache[blk, :, :, slot] = vb[r]
        if k_ring is None:
            continue
        last = (seq_lens[b] - 1) // BLOCK_SIZE
        if j >= sink_blocks and j <= last - ring_blocks:
            continue
        at = j if j < sink_blocks else sink_blocks + j % ring_blocks
        k_ring[b, at, :, :, slot, :] = kb[r].reshape(-1, D // 8, 8)
        v_ring[b, at, :, :, slot] = vb[r]


def prompt_attention(q, k_cache, v_cache, table, row_start, seq_lens, scale, causal=True, window=0):
    """q uint16 bf16 [rows][Hq][D]; caches of one layer with a leading axis of 1.  Returns out f64 [rows][Hq][D], lse
    (rows of no request NaN; rows that attend nothing 0 and -infinity) and the mean absolute value behind each out."""
    R, Hq, D = q.shape
    Hkv = k_cache.shape[2]
    G = Hq // Hkv
    out, lse, mag = np.full((R, Hq, D), np.nan), np.full((R, Hq), np.nan), np.zeros((R, Hq, D))
    for b, n in enumerate(seq_lens):
        m = row_start[b + 1] - row_start[b]
        if m == 0:
            continue
        rows = slice(row_start[b], row_start[b] + m)
        if n == 0:
            out[rows], lse[rows] = 0.0, -np.inf
            continue
        place = n - m + np.arange(m)
        pos = np.arange(n)
        seen = np.ones((m, n), dtype=bool)
        if causal:
            seen = pos[None] <= place[:, None]
            if window:
                seen &= pos[None] > place[:, None] - window
        for g in range(Hkv):
            K, V = key_rows(k_cache, table, 0, b, g, pos), value_rows(v_cache, table, 0, b, g, pos)
            for h in range(g * G, (g + 1) * G):
                z = np.where(seen, scale * (bf16_to_f64(q[rows, h]) @ K.T), -np.inf)
                top = z.max(-1, keepdims=True)
                w = np.exp(z - top)
                total = w.sum(-1, keepdims=True)
                if np.isfinite(V).all():
                    out[rows, h], mag[rows, h] = (w / total) @ V, (w / total) @ np.abs(V)
                else:                              # what a row does not attend may be anything
                    for i in range(m):
                        p, x = (w / total)[i, seen[i]], V[seen[i]]
                        out[row_start[b] + i, h], mag[row_start[b] + i, h] = p @ x, p @ np.abs(x)
                lse[rows, h] = (top + np.log(total))[:, 0]
    return out, lse, mag


def token_logprobs(z, tokens, top):
    """z [rows][V].  Returns (logprob, rank, entropy, top_logprobs, top_tokens)."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, dtype=np.float64))
    R, V = z.shape
    logprob, entropy = np.full(R, np.nan), np.full(R, np.nan)
    rank = np.zeros(R, dtype=np.int64)
    best, ids = np.full((R, top), -np.inf), np.full((R, top), -1, dtype=np.int64)
    for r in range(R):
        order = np.lexsort((np.arange(V), -z[r]))
        m = z[r].max()
        t = -1 if tokens is None else tokens[r]
        if 0 <= t < V:
            rank[r] = 1 + int(np.flatnonzero(order == t)[0])
        if m == -np.inf:
            continue
        w = (z[r] == np.inf).astype(float) if m == np.inf else np.exp(z[r] - m)
        total = w.sum()
        with np.errstate(divide="ignore", invalid="ignore"):
            log = np.where(w > 0, np.log(w), -np.inf) if m == np.inf else z[r] - m
        log = log - np.log(total)
        p = w / total
        entropy[r] = -(p[p > 0] * log[p > 0]).sum()
        if 0 <= t < V:
            logprob[r] = log[t]
        for i, v in enumerate(order[:top]):
            if z[r, v] > -np.inf:
                best[r, i], ids[r, i] = log[v], v
    return logprob, rank, entropy, best, ids
