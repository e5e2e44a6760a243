"""Pins of the oracle's draft operators (CPU): the verification keeps the target's
distribution, adapters are the dense layer with their product added to the
weight, attention rows are decode attention at their own lengths."""
import numpy as np
import pytest

import oda_synth as S
from oracle import attention as OA
from oracle import decoder as ODec
from oracle import drafts as OD


@pytest.mark.parametrize("drawn", [True, False])
def test_verification_keeps_the_target_distribution(drawn):
    """The first token's frequencies over 40,000 requests equal p, for drafts
    drawn from q and for fixed drafts (five standard deviations)."""
    g = np.random.default_rng(3)
    V, N = 7, 40000
    z = g.standard_normal(V) * 1.5
    q = np.exp(g.standard_normal(V))
    q /= q.sum()
    p = OD.token_weights(z, 0.8)
    p /= p.sum()
    x = np.searchsorted(np.cumsum(q), g.random(N)).clip(max=V - 1) if drawn else np.full(N, 2)
    logits = np.broadcast_to(z, (N, 2, V))
    probs = np.broadcast_to(q, (N, 1, V)) if drawn else None
    _, tok = OD.verify_drafts(logits, x[:, None], g.random((N, 2)), probs, None, np.full(N, 0.8))
    freq = np.bincount(tok[:, 0], minlength=V) / N
    assert np.all(np.abs(freq - p) <= 5 * np.sqrt(p * (1 - p) / N))


def test_worked_verification():
    """p = (1/2, 1/4, 1/4), q = (1/4, 1/2, 1/4): draft 1 is kept below u = 1/2; the
    residual is all on token 0."""
    z = np.log(np.array([[[2.0, 1, 1], [1, 2, 1]]]))
    q = np.array([[[0.25, 0.5, 0.25]]])
    x = np.array([[1]])
    acc, tok = OD.verify_drafts(z, x, np.array([[0.49, 0.26]]), q)
    assert acc[0] == 1 and tok.tolist() == [[1, 1]]          # next: cumulative 1/4, 3/4, 1
    acc, tok = OD.verify_drafts(z, x, np.array([[0.51, 0.99]]), q)
    assert acc[0] == 0 and tok.tolist() == [[0, -1]]


def test_greedy_verification_is_the_argmax():
    g = np.random.default_rng(4)
    z = g.standard_normal((5, 4, 50))
    x = z[:, :3].argmax(-1)
    x[2, 1] = (x[2, 1] + 1) % 50
    acc, tok = OD.verify_drafts(z, x, g.random((5, 4)), None, None, np.zeros(5))
    assert acc.tolist() == [3, 3, 1, 3, 3]
    for b in range(5):
        assert tok[b, :acc[b] + 1].tolist() == z[b, :acc[b] + 1].argmax(-1).tolist()
        assert (tok[b, acc[b] + 1:] == -1).all()


def test_adapter_is_a_change_of_the_weight():
    g = np.random.default_rng(5)
    K, parts, r = 24, [5, 3], 8
    w, x, gain = g.standard_normal((8, K)), g.standard_normal((3, K)), 1 + 0.1 * g.standard_normal(K)
    a, b, s = g.standard_normal((2, 16, K)), g.standard_normal((2, 8, r)), np.array([0.5, 2.0])
    y, _ = OD.dense_lora(x, w, a, b, s, [1, -1, 0], parts, gain, 1e-6)
    for i, ad in enumerate([1, -1, 0]):
        full = w.copy()
        if ad >= 0:
            full[:5] += s[ad] * b[ad, :5] @ a[ad, :r]
            full[5:] += s[ad] * b[ad, 5:] @ a[ad, r:]
        np.testing.assert_allclose(y[i], full @ ODec.rmsnorm(x[i], gain, 1e-6), rtol=1e-12, atol=1e-12)


def test_rows_of_a_request_are_decode_attention():
    L, B, T, Hq, Hkv, D = 1, 2, 3, 4, 2, 64
    seq = np.array([20, 5], dtype=np.int32)
    table, nb = S.paged_block_table(S.rng(6, S.STREAM_TABLE), seq + T, None)
    k, v = S.kv_cache(6, L, nb, Hkv, D)
    q = S.normal_bf16(S.rng(6, S.STREAM_Q), (L, B, T, Hq, D))
    out, lse = OD.prefix_attention(q, k, v, table, seq, 0.125)
    kc = S.normal_bf16(S.rng(6, S.STREAM_KCUR), (L, B, T, Hkv, D))
    vc = S.normal_bf16(S.rng(6, S.STREAM_VCUR), (L, B, T, Hkv, D))
    cand, _ = OD.prefix_attention(q, k, v, table, seq, 0.125, k_cur=kc, v_cur=vc)
    for t in range(T):
        ref, ref_lse, _ = OA.decode_attention(q[:, :, t], k, v, table, seq + t, OA.full_set, 0.125)
        np.testing.assert_allclose(out[:, :, t], ref, rtol=1e-13, atol=1e-13)
        np.testing.assert_allclose(lse[:, :, t], ref_lse, rtol=1e-13, atol=1e-13)
    # candidates equal the same rows read from the cache once they are committed
    OD.commit_drafts(k, v, table, seq.copy(), kc, vc, advance=False)
    again, _ = OD.prefix_attention(q, k, v, table, seq, 0.125)
    np.testing.assert_allclose(again, cand, rtol=1e-13, atol=1e-13)
