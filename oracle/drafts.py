"""Operators of a step with tenants and drafted tokens, fp64, by definition.
TEST INFRASTRUCTURE (see package doc).

* ``dense_lora``     -- a dense layer with a low-rank adapter per row;
* ``token_weights``  -- the weights a row of logits gives its tokens;
* ``verify_drafts``  -- rejection sampling of drafts by given random numbers;
* ``commit_drafts``  -- the accepted tokens' K/V into the paged cache;
* ``prefix_attention`` -- attention of several current tokens per request, each
  over the request's own history (what sharing a prefix must not change).
"""
from __future__ import annotations

import numpy as np

from .attention import BLOCK_SIZE, attend, bf16_to_f64, key_rows, value_rows


def dense_lora(x, w, a, b, scale, ids, part_rows, gain=None, eps=0.0, swiglu=False, residual=None):
    """x f64 [B][K]; w f64 [rows][K]; a f64 [A][parts r][K]; b f64 [A][rows][r].
    Returns (y, bound): bound is the sum of the absolute terms behind each y
    (for SWIGLU, of the gate and of the up sum as a pair)."""
    B, rank = x.shape[0], b.shape[2]
    part = np.repeat(np.arange(len(part_rows)), part_rows)
    rows, mag = [], []
    for i in range(B):
        v = x[i]
        if gain is not None:
            v = v / np.sqrt(np.mean(v * v) + eps) * gain
        y, m = w @ v, np.abs(w) @ np.abs(v)
        if ids[i] >= 0:
            t = (a[ids[i]] @ v).reshape(len(part_rows), rank)
            tm = (np.abs(a[ids[i]]) @ np.abs(v)).reshape(len(part_rows), rank)
            y = y + scale[ids[i]] * (b[ids[i]] * t[part]).sum(-1)
            m = m + abs(scale[ids[i]]) * (np.abs(b[ids[i]]) * tm[part]).sum(-1)
        rows.append(y)
        mag.append(m)
    y, mag = np.array(rows), np.array(mag)
    if swiglu:
        n = y.shape[1] // 2
        g, u = y[:, :n], y[:, n:]
        return g / (1 + np.exp(-g)) * u, (g, u, mag[:, :n], mag[:, n:])
    return (y if residual is None else y + residual), mag


def token_weights(z, temperature):
    """Weights of a row's tokens (unnormalised, the largest has 1), or None if no
    logit is above -infinity.  temperature > 0: exp((z - max) / temperature);
    else the first largest logit alone.  NaN counts as -infinity."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, dtype=np.float64))
    top = z.max()
    if top == -np.inf:
        return None
    if not temperature > 0:
        w = np.zeros_like(z)
        w[np.argmax(z)] = 1.0
        return w
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.exp((z - top) / temperature)
    w = np.where(np.isnan(w), 0.0, w)
    w[z == top] = 1.0
    w[z == -np.inf] = 0.0
    return w


def draw(w, u):
    """The smallest index whose cumulative weight exceeds u times the whole."""
    c = np.cumsum(w)
    past = np.flatnonzero((c > u * c[-1]) & (w > 0))
    return int(past[0]) if len(past) else int(np.flatnonzero(w > 0)[-1])


def verify_drafts(logits, drafts, u, draft_probs=None, n_drafts=None, temperature=None):
    """(n_accepted [B], tokens [B][K + 1]) of rejection sampling."""
    B, rows, V = logits.shape
    K = rows - 1
    accepted = np.zeros(B, dtype=np.int32)
    tokens = np.full((B, rows), -1, dtype=np.int32)
    for b in range(B):
        n = K if n_drafts is None else min(max(int(n_drafts[b]), 0), K)
        t = 1.0 if temperature is None else float(temperature[b])

        def probs(i):
            w = token_weights(logits[b, i], t)
            return None if w is None else w / w.sum()

        j = 0
        while j < n:
            x, p = int(drafts[b, j]), probs(j)
            if p is None or not 0 <= x < V:
                break
            q = 1.0 if draft_probs is None else max(float(np.nan_to_num(draft_probs[b, j, x], nan=0.0)), 0.0)
            if not float(u[b, j]) * q < p[x]:
                break
            tokens[b, j] = x
            j += 1
        accepted[b] = j
        p = probs(j)
        if p is None:
            continue
        if j < n and t > 0:
            if draft_probs is not None:
                q = np.asarray(draft_probs[b, j], dtype=np.float64)
                w = np.maximum(p - np.maximum(np.where(np.isnan(q), 0.0, q), 0.0), 0.0)
            else:
                w = p.copy()
                if 0 <= drafts[b, j] < V:
                    w[drafts[b, j]] = 0.0
            p = w if w.sum() > 0 else p
        tokens[b, j] = draw(p, float(u[b, K]))
    return accepted, tokens


def commit_drafts(k_cache, v_cache, block_table, seq_lens, k_cand, v_cand, n_accepted=None, advance=True):
    """In place; k_cand, v_cand [L][B][T][Hkv][D].  Returns the tokens committed per request."""
    L, B, T, Hkv, D = k_cand.shape
    counts = np.zeros(B, dtype=np.int32)
    for b in range(B):
        counts[b] = T if n_accepted is None else min(max(int(n_accepted[b]) + 1, 0), T)
        for t in range(counts[b]):
            pos = int(seq_lens[b]) - 1 + t
            if pos < 0 or pos // BLOCK_SIZE >= block_table.shape[1]:
                continue
            blk = int(block_table[b, pos // BLOCK_SIZE])
            if not 0 <= blk < k_cache.shape[1]:
                continue
            for l in range(L):
                k_cache[l, blk, :, :, pos % BLOCK_SIZE, :] = k_cand[l, b, t].reshape(Hkv, D // 8, 8)
                v_cache[l, blk, :, :, pos % BLOCK_SIZE] = v_cand[l, b, t]
        if advance:
            seq_lens[b] += counts[b]
    return counts


def prefix_attention(q, k_cache, v_cache, block_table, seq_lens, scale, n_tokens=None, k_cur=None, v_cur=None,
                     requests=None):
    """q uint16 [L][B][T][Hq][D].  Row t of request b attends positions 0 ..
    seq_lens[b] - 1 + t; with k_cur / v_cur [L][B][T][Hkv][D] the positions from
    seq_lens[b] - 1 on are the candidates, else the cache holds them.  Rows that
    are not attended (t >= n_tokens[b], other requests) are NaN."""
    L, B, T, Hq, D = q.shape
    Hkv = k_cache.shape[2]
    G = Hq // Hkv
    out = np.full((L, B, T, Hq, D), np.nan)
    lse = np.full((L, B, T, Hq), np.nan)
    for b in range(B) if requests is None else requests:
        n = int(seq_lens[b])
        for t in range(T if n_tokens is None else int(n_tokens[b])):
            cached = np.arange(n - 1 if k_cur is not None else n + t)
            for l in range(L):
                for g in range(Hkv):
                    K = key_rows(k_cache, block_table, l, b, g, cached)
                    V = value_rows(v_cache, block_table, l, b, g, cached)
                    if k_cur is not None:
                        K = np.vstack([K, bf16_to_f64(k_cur[l, b, :t + 1, g])])
                        V = np.vstack([V, bf16_to_f64(v_cur[l, b, :t + 1, g])])
                    for h in range(g * G, (g + 1) * G):
                        out[l, b, t, h], lse[l, b, t, h], _ = attend(bf16_to_f64(q[l, b, t, h]), K, V, scale)
    return out, lse
