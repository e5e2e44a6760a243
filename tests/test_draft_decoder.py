"""Whole steps of DraftDecoder (shared-prefix attention, adapters, verification,
commit) against the oracle, which runs every token of a request one after the
other with the adapter's product added to the weights; and the step captured as a
graph."""
import math

import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_f32, dev_i32, dev_u16, need_gpu
from oracle import attention as OA
from oracle import decoder as ODec
from oracle import drafts as OD

pytestmark = pytest.mark.gpu

STEP_REL_L2 = 1e-3       # the decoder steps' bar (tests/test_decoder_parity.py)


def _bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def _rel_l2(got, ref):
    return float(np.linalg.norm(got.astype(np.float64) - ref) / np.linalg.norm(ref))


class Tenants:
    """Five requests: three behind a prompt of 3 blocks, two behind one of 1 block
    (each group a tenant with its adapter, one request without), up to 3 drafts."""

    def __init__(self, seed=8, adapters=("w_qkv", "w_o", "w_gu", "w_down"), T=4, temps=(0.0, 1.0, 0.0, 0.7, 0.0)):
        P = self.P = need_gpu()
        from paper_2609_20734_amd import decoder as PD
        L, d, Hq, Hkv, D, F, V = 2, 128, 4, 2, 64, 192, 320
        self.L, self.T, self.V, self.B = L, T, V, 5
        self.shape = PD.DecoderShape(L, d, Hq, Hkv, D, F, V)
        self.w = S.decoder_weights(seed, L, d, Hq, Hkv, D, F, V)
        self.model = ODec.Model(self.w, Hq, Hkv, D)
        B = self.B
        order = [2, 0, 4, 1, 3]
        pre = [3, 3, 1, 1, 3]                              # of request 0..4
        pre = [3 if b in order[:3] else 1 for b in range(B)]
        self.seq = np.array([16 * pre[b] + n for b, n in enumerate((7, 16, 1, 30, 20))], dtype=np.int32)
        steps = 6
        self.mb = int(math.ceil((self.seq.max() + steps * T) / 16))
        self.table, self.nb = S.paged_block_table(S.rng(seed, S.STREAM_TABLE), self.seq + steps * T, self.mb)
        for group, n in ((order[:3], 3), (order[3:], 1)):
            for b in group[1:]:
                self.table[b, :n] = self.table[group[0], :n]
        self.k, self.v = S.kv_cache(seed, L, self.nb, Hkv, D)
        self.groups = tuple(dev_i32(a) for a in ([0, 3, 5], order, [3, 1]))
        self.ids = np.array([0, 1, 0, -1, 0], dtype=np.int32)
        g = S.rng(seed, 91)
        self.ad, descs = {}, {}
        sizes = dict(w_qkv=(d, [Hq * D, Hkv * D, Hkv * D], 8), w_o=(Hq * D, [d], 16), w_gu=(d, [F, F], 8), w_down=(F, [d], 24))
        for name in adapters:
            K, parts, r = sizes[name]
            a = S.normal_bf16(g, (L, 2, len(parts) * r, K), K ** -0.5)
            b = S.normal_bf16(g, (L, 2, sum(parts), r), 0.5 * r ** -0.5)
            sc = (0.5 + g.random((L, 2))).astype(np.float32)
            self.ad[name] = (a, b, sc, parts, r)
            descs[name] = [P.lora_desc(2, r, parts, dev_u16(a[l]), dev_u16(b[l]), dev_f32(sc[l])) for l in range(L)]
        self.temps = np.array(temps, dtype=np.float32)
        dw = {n: (dev_u16(x) if x.dtype == np.uint16 else dev_f32(x)) for n, x in self.w.items()}
        self.dk, self.dv, self.dseq = dev_u16(self.k), dev_u16(self.v), dev_i32(self.seq)
        self.dec = PD.DraftDecoder(self.shape, dw, B, T, self.dk, self.dv, dev_i32(self.table), self.dseq, self.mb,
                                   self.mb * 16, self.nb, self.groups, descs, dev_i32(self.ids) if adapters else None,
                                   dev_f32(self.temps))
        self.g = g

    def weight(self, name, l, b):
        w = OA.bf16_to_f64(self.w[name][l])
        if name in self.ad and self.ids[b] >= 0:
            a, bb, sc, parts, r = self.ad[name]
            a, bb, at = OA.bf16_to_f64(a[l, self.ids[b]]), OA.bf16_to_f64(bb[l, self.ids[b]]), 0
            w = w.copy()
            for p, n in enumerate(parts):
                w[at:at + n] += float(sc[l, self.ids[b]]) * bb[at:at + n] @ a[p * r:(p + 1) * r]
                at += n
        return w

    def token(self, b, token, n, k, v):
        """Logits of one token of request b at position n - 1 over the caches (which get its K/V)."""
        m = self.model
        h = m.embed([token])[0]
        for l in range(self.L):
            x = ODec.rmsnorm(h, self.w["attn_norm"][l], m.eps)
            q, kc, vc = ODec.qk_norm_rope((self.weight("w_qkv", l, b) @ x)[None], m.Hq, m.Hkv, m.D, self.w["q_norm"][l],
                                          self.w["k_norm"][l], m.eps, m.theta, [n - 1])
            blk, at = self.table[b, (n - 1) // 16], (n - 1) % 16
            k[l, blk, :, :, at, :] = ODec.bf16_bits(kc[0]).reshape(m.Hkv, m.D // 8, 8)
            v[l, blk, :, :, at] = ODec.bf16_bits(vc[0])
            out = OA.decode_attention(ODec.bf16_bits(q)[None], k[l:l + 1], v[l:l + 1], self.table[b:b + 1],
                                      np.array([n]), OA.full_set, 1 / math.sqrt(m.D))[0]
            h = h + self.weight("w_o", l, b) @ out.reshape(-1)
            x = ODec.rmsnorm(h, self.w["mlp_norm"][l], m.eps)
            gu = self.weight("w_gu", l, b) @ x
            F = len(gu) // 2
            h = h + self.weight("w_down", l, b) @ (ODec.silu(gu[:F]) * gu[F:])
        return OA.bf16_to_f64(self.w["embed"]) @ m.final_state(h)

    def plan_step(self, current, guess):
        """The step's inputs: drafts are the oracle's greedy continuation, some spoilt."""
        drafts = np.zeros((self.B, self.T - 1), dtype=np.int32)
        for b in range(self.B):
            k, v, n, tok = self.k.copy(), self.v.copy(), int(self.seq[b]), int(current[b])
            for i in range(self.T - 1):
                tok = int(np.argmax(self.token(b, tok, n + i, k, v)))
                if self.g.random() > guess:
                    tok = (tok + 7) % self.V
                drafts[b, i] = tok
        counts = self.g.integers(0, self.T, size=self.B).astype(np.int32)
        return drafts, counts, self.g.random((self.B, self.T)).astype(np.float32) * np.float32(0.999)

    def set(self, current, drafts, counts, u):
        self.dec.set_drafts(*(torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (current, drafts, counts)))
        self.dec.uniform.copy_(torch.from_numpy(u))


@pytest.mark.parametrize("adapters", [("w_qkv", "w_o", "w_gu", "w_down"), ()])
def test_steps_match_oracle(adapters):
    t = Tenants(adapters=adapters)
    stages = t.dec.stages()
    current = t.g.integers(0, t.V, size=t.B).astype(np.int32)
    accepted = []
    for step in range(4):
        drafts, counts, u = t.plan_step(current, 0.8)
        t.set(current, drafts, counts, u)
        for st in stages:
            for c in st:
                c()
        torch.cuda.synchronize()
        logits = t.dec.logits.cpu().numpy()
        kc, vc = _bits(t.dec.k_cand), _bits(t.dec.v_cand)
        acc, tok = t.dec.accepted.cpu().numpy(), t.dec.answer.cpu().numpy()
        ref_acc, ref_tok = OD.verify_drafts(logits, drafts, u, None, counts, t.temps)
        np.testing.assert_array_equal(acc, ref_acc)
        np.testing.assert_array_equal(tok, ref_tok)
        for b in range(t.B):
            k, v = t.k.copy(), t.v.copy()
            row = [int(current[b])] + drafts[b].tolist()
            for i in range(counts[b] + 1):
                ref = t.token(b, row[i], int(t.seq[b]) + i, k, v)
                assert _rel_l2(logits[b, i], ref) <= STEP_REL_L2, (step, b, i)
                top = np.sort(ref)[-2:]
                if t.temps[b] == 0 and i <= acc[b] and top[1] - top[0] > 1e-3 * max(1.0, abs(top[1])):
                    assert tok[b, i] == int(np.argmax(ref)), (step, b, i)      # as greedy decoding one by one
        # the device's own candidates, committed as the oracle does
        lens = t.seq.copy()
        OD.commit_drafts(t.k, t.v, t.table, t.seq, kc, vc, acc)
        np.testing.assert_array_equal(_bits(t.dk).reshape(t.k.shape), t.k)
        np.testing.assert_array_equal(_bits(t.dv).reshape(t.v.shape), t.v)
        np.testing.assert_array_equal(t.dseq.cpu().numpy(), t.seq)
        np.testing.assert_array_equal(t.seq, lens + acc + 1)
        np.testing.assert_array_equal(t.dec.row_lens.cpu().numpy(), t.seq[:, None] + np.arange(t.T))
        current = tok[np.arange(t.B), acc].astype(np.int32)
        accepted += acc.tolist()
    assert len(set(accepted)) >= 3           # refusals and acceptances of several lengths


def test_captured_step_replays_bit_exactly():
    t = Tenants(seed=9)
    dec = t.dec
    drafts, counts, u = t.plan_step(np.arange(t.B), 0.9)
    k0, v0, s0 = t.dk.clone(), t.dv.clone(), t.dseq.clone()
    r0 = dec.row_lens.clone()

    def reset():
        t.dk.copy_(k0)
        t.dv.copy_(v0)
        t.dseq.copy_(s0)
        dec.row_lens.copy_(r0)
        t.set(np.arange(t.B, dtype=np.int32), drafts, counts, u)

    def outputs():
        return [x.clone() for x in (dec.logits, dec.accepted, dec.answer, t.dk, t.dv, t.dseq, dec.row_lens)]

    reset()
    for st in dec.stages():
        for c in st:
            c()
    torch.cuda.synchronize()
    ref = outputs()
    reset()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for st in dec.stages():
            for c in st:
                c()
    for rep in range(3):
        reset()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outputs(), ref):
            assert torch.equal(a, b), f"replay {rep} differs from eager"
        _ = (dec.logits * 2).sum().item()


def test_one_token_a_step():
    """T = 1: no drafts, the draw alone, through the same classes."""
    t = Tenants(seed=10, T=1, temps=(0.0,) * 5)
    stages = t.dec.stages()
    current = np.arange(5, dtype=np.int32)
    for _ in range(2):
        t.set(current, np.zeros((5, 0), dtype=np.int32), np.zeros(5, dtype=np.int32), np.zeros((5, 1), dtype=np.float32))
        for st in stages:
            for c in st:
                c()
        torch.cuda.synchronize()
        logits = t.dec.logits.cpu().numpy()
        for b in range(5):
            ref = t.token(b, int(current[b]), int(t.seq[b]), t.k.copy(), t.v.copy())
            assert _rel_l2(logits[b, 0], ref) <= STEP_REL_L2
        tok = t.dec.answer.cpu().numpy()
        np.testing.assert_array_equal(tok[:, 0], logits[:, 0].argmax(-1))
        OD.commit_drafts(t.k, t.v, t.table, t.seq, _bits(t.dec.k_cand), _bits(t.dec.v_cand))
        np.testing.assert_array_equal(t.dseq.cpu().numpy(), t.seq)
        current = tok[:, 0].astype(np.int32)


def test_adapters_need_ids():
    from paper_2609_20734_amd import decoder as PD
    t = Tenants(seed=10, adapters=("w_o",))
    with pytest.raises(ValueError):
        PD.DraftDecoder(t.shape, t.dec.w, t.B, t.T, t.dk, t.dv, t.dec.table, t.dseq, t.mb, t.mb * 16, t.nb, t.groups,
                        t.dec.adapters)
