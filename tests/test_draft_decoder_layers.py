"""Steps of DraftDecoder with adapters whose rank differs between layers, and with
drafts verified against their probabilities, against the oracle."""
import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_f32, dev_i32, dev_u16
from oracle import drafts as OD
from test_draft_decoder import STEP_REL_L2, Tenants, _bits, _rel_l2

pytestmark = pytest.mark.gpu


def _remake(t, descs, draft_probs=False):
    """The same requests under other adapters or another kind of draft."""
    from paper_2609_20734_amd import decoder as PD
    t.dec = PD.DraftDecoder(t.shape, t.dec.w, t.B, t.T, t.dk, t.dv, t.dec.table, t.dseq, t.mb, t.mb * 16, t.nb, t.groups, descs,
                            dev_i32(t.ids), dev_f32(t.temps), draft_probs)


def _step(t, current, drafts, counts, u):
    t.set(current, drafts, counts, u)
    for st in t.dec.stages():
        for c in st:
            c()
    torch.cuda.synchronize()


@pytest.mark.parametrize("ranks", [(8, 64), (40, 8)])
def test_ranks_differ_between_layers(ranks):
    """The second layer's adapters have the larger rank, or the smaller."""
    t = Tenants(seed=11, adapters=())
    g, d, F = S.rng(11, 92), t.shape.d_model, t.shape.d_ffn
    HD, KD = t.shape.num_q_heads * t.shape.head_dim, t.shape.num_kv_heads * t.shape.head_dim
    sizes = dict(w_qkv=(d, [HD, KD, KD]), w_gu=(d, [F, F]))
    descs, layers = {}, {}
    for name, (K, parts) in sizes.items():
        layers[name] = []
        for r in ranks:
            a = S.normal_bf16(g, (2, len(parts) * r, K), K ** -0.5)
            b = S.normal_bf16(g, (2, sum(parts), r), 0.5 * r ** -0.5)
            sc = (0.5 + g.random(2)).astype(np.float32)
            layers[name].append((a, b, sc, parts, r))
        descs[name] = [t.P.lora_desc(2, r, parts, dev_u16(a), dev_u16(b), dev_f32(sc)) for a, b, sc, parts, r in layers[name]]
    _remake(t, descs)
    plain = t.weight

    def weight(name, l, b):
        if name not in layers:
            return plain(name, l, b)
        a, bb, sc, parts, r = layers[name][l]
        t.ad = {name: (np.broadcast_to(a, (t.L, *a.shape)), np.broadcast_to(bb, (t.L, *bb.shape)),
                       np.broadcast_to(sc, (t.L, 2)), parts, r)}
        return plain(name, l, b)

    t.weight = weight
    current = t.g.integers(0, t.V, size=t.B).astype(np.int32)
    drafts = t.g.integers(0, t.V, size=(t.B, t.T - 1)).astype(np.int32)
    counts = np.full(t.B, t.T - 1, dtype=np.int32)
    _step(t, current, drafts, counts, np.full((t.B, t.T), 0.5, np.float32))
    logits = t.dec.logits.cpu().numpy()
    for b in range(t.B):
        k, v = t.k.copy(), t.v.copy()
        for i, token in enumerate([int(current[b])] + drafts[b].tolist()):
            assert _rel_l2(logits[b, i], t.token(b, token, int(t.seq[b]) + i, k, v)) <= STEP_REL_L2, (b, i)


def _draw(t, q):
    return np.array([[t.g.choice(t.V, p=r.astype(np.float64) / r.astype(np.float64).sum()) for r in rows] for rows in q],
                    dtype=np.int32)


def _verified_steps(t, current, proposals, steps=4):
    """Steps with drafts and probabilities of `proposals(current)`; (accepted, in use) of every request and step."""
    seen = []
    for _ in range(steps):
        drafts, q = proposals(current)
        counts = t.g.integers(0, t.T, size=t.B).astype(np.int32)
        u = t.g.random((t.B, t.T)).astype(np.float32) * np.float32(0.999)
        t.dec.probs.copy_(torch.from_numpy(q))
        before = t.dseq.cpu().numpy()
        _step(t, current, drafts, counts, u)
        acc, tok = t.dec.accepted.cpu().numpy(), t.dec.answer.cpu().numpy()
        want = OD.verify_drafts(t.dec.logits.cpu().numpy(), drafts, u, q, counts, t.temps)
        np.testing.assert_array_equal(acc, want[0])
        np.testing.assert_array_equal(tok, want[1])
        OD.commit_drafts(t.k, t.v, t.dec.table.cpu().numpy(), t.seq, _bits(t.dec.k_cand), _bits(t.dec.v_cand), acc)
        np.testing.assert_array_equal(t.dseq.cpu().numpy(), t.seq)
        np.testing.assert_array_equal(t.seq, before + acc + 1)
        seen += [(int(a), int(n)) for a, n in zip(acc, counts)]
        current = tok[np.arange(t.B), acc].astype(np.int32)
    return seen


def test_drafts_with_unlike_probabilities():
    """draft_probs=True, drafts of a model that knows nothing: most are refused, and their successors drawn from what the
    target has over the draft's probabilities."""
    t = Tenants(seed=12, adapters=(), temps=(1.0, 0.7, 0.0, 1.5, 1.0))
    _remake(t, {}, draft_probs=True)
    assert t.dec.probs.shape == (t.B, t.T - 1, t.V)

    def proposals(_):
        q = np.exp(2.0 * t.g.standard_normal((t.B, t.T - 1, t.V)))
        q = (q / q.sum(-1, keepdims=True)).astype(np.float32)
        return _draw(t, q), q

    seen = _verified_steps(t, t.g.integers(0, t.V, size=t.B).astype(np.int32), proposals)
    assert any(a < n for a, n in seen)


def test_drafts_with_their_probabilities():
    """Drafts of a model close to the target: several at a time are accepted."""
    t = Tenants(seed=13, adapters=(), temps=(1.0, 0.7, 1.3, 1.5, 1.0))
    _remake(t, {}, draft_probs=True)

    def proposals(current):
        drafts = np.zeros((t.B, t.T - 1), dtype=np.int32)
        q = np.zeros((t.B, t.T - 1, t.V), dtype=np.float32)
        for b in range(t.B):
            k, v, token = t.k.copy(), t.v.copy(), int(current[b])
            for i in range(t.T - 1):
                z = t.token(b, token, int(t.seq[b]) + i, k, v) / float(t.temps[b]) + 0.3 * t.g.standard_normal(t.V)
                w = np.exp(z - z.max())
                q[b, i] = w / w.sum()
                token = drafts[b, i] = _draw(t, q[b:b + 1, i:i + 1])[0, 0]
        return drafts, q

    seen = _verified_steps(t, t.g.integers(0, t.V, size=t.B).astype(np.int32), proposals, steps=5)
    assert max(a for a, _ in seen) >= 2
