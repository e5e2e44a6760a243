"""Whole prompts through PromptDecoder (rows appended, prompt attention, scores) against
the oracle, which runs every token of a request one after the other; chunks of any
size leave the same caches; the decode steps that go on from them; a chunk captured as
a graph."""
import math

import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_f32, dev_i32, dev_u16, need_gpu
from oracle import attention as OA
from oracle import decoder as ODec
from oracle import prompt as OP

pytestmark = pytest.mark.gpu

STEP_REL_L2 = 1e-3       # the decoder steps' bar (tests/test_decoder_parity.py)


class Prompts:
    """Four requests whose prompts come in chunks of uneven sizes (some in none)."""
    chunks = [[5, 40, 0, 1], [1, 0, 17, 30], [20, 3, 16, 1]]

    def __init__(self, seed=12, score="all", top=5, window=0, rings=False, rows=48):
        P = self.P = need_gpu()
        from paper_2609_20734_amd import decoder as PD
        L, d, Hq, Hkv, D, F, V = 2, 128, 4, 2, 64, 192, 320
        self.L, self.V, self.B, self.Hkv, self.D, self.window = L, V, 4, Hkv, D, window
        self.shape = PD.DecoderShape(L, d, Hq, Hkv, D, F, V)
        self.w = S.decoder_weights(seed, L, d, Hq, Hkv, D, F, V)
        self.model = ODec.Model(self.w, Hq, Hkv, D)
        total = np.sum(self.chunks, 0) + 8
        self.mb = int(math.ceil(total.max() / 16)) + 1
        self.table, self.nb = S.paged_block_table(S.rng(seed, S.STREAM_TABLE), total, self.mb)
        self.k, self.v = S.kv_cache(seed, L, self.nb, Hkv, D)
        g = self.g = S.rng(seed, 94)
        self.tokens = [g.integers(0, V, size=int(t)) for t in np.sum(self.chunks, 0)]
        self.dw = {n: (dev_u16(x) if x.dtype == np.uint16 else dev_f32(x)) for n, x in self.w.items()}
        self.dk, self.dv, self.dseq = dev_u16(self.k), dev_u16(self.v), dev_i32(np.zeros(4))
        self.dtab = dev_i32(self.table)
        self.rings = None
        if rings:
            n = P.ring_elements(P.Shape(L, 4, Hq, Hkv, D, self.mb, self.mb * 16, self.nb), 4, 24)
            kr, vr = (torch.zeros(L, n // L, dtype=torch.int16, device="cuda") for _ in range(2))
            self.rings = (kr, vr, 4, 24)
        self.dec = PD.PromptDecoder(self.shape, self.dw, 4, rows, self.dk, self.dv, self.dtab, self.dseq, self.mb, self.mb * 16,
                                    self.nb, rings=self.rings, score=score, top=top, native_window=window)
        self.run = PD.run

    def chunk(self, c):
        """(tokens, targets, row_start) of chunk c."""
        at = np.sum(self.chunks[:c], 0).astype(int) if c else np.zeros(4, int)
        toks, tgt = [], []
        for b in range(4):
            seq = np.append(self.tokens[b], 7)
            toks += list(seq[at[b]:at[b] + self.chunks[c][b]])
            tgt += list(seq[at[b] + 1:at[b] + self.chunks[c][b] + 1])
        return toks, tgt, np.concatenate([[0], np.cumsum(self.chunks[c])])

    def set(self, c):
        toks, tgt, start = self.chunk(c)
        self.dec.set_chunk(*(torch.tensor(np.array(x), dtype=torch.int32, device="cuda") for x in (toks, start, tgt)))

    def oracle(self):
        """Logits of every token of every request, and the caches."""
        m, k, v = self.model, self.k.copy(), self.v.copy()
        logits = []
        for b in range(4):
            rows = []
            for i, tok in enumerate(self.tokens[b]):
                h = m.embed([tok])[0]
                n = i + 1
                for l in range(self.L):
                    x = ODec.rmsnorm(h, self.w["attn_norm"][l], m.eps)
                    q, kc, vc = ODec.qk_norm_rope((OA.bf16_to_f64(self.w["w_qkv"][l]) @ x)[None], m.Hq, m.Hkv, m.D,
                                                  self.w["q_norm"][l], self.w["k_norm"][l], m.eps, m.theta, [i])
                    blk, slot = self.table[b, i // 16], i % 16
                    k[l, blk, :, :, slot, :] = ODec.bf16_bits(kc[0]).reshape(m.Hkv, m.D // 8, 8)
                    v[l, blk, :, :, slot] = ODec.bf16_bits(vc[0])
                    out = OA.decode_attention(ODec.bf16_bits(q)[None], k[l:l + 1], v[l:l + 1], self.table[b:b + 1], np.array([n]),
                                              lambda n: OA.native_window_set(n, self.window), 1 / math.sqrt(m.D))[0]
                    h = h + OA.bf16_to_f64(self.w["w_o"][l]) @ out.reshape(-1)
                    x = ODec.rmsnorm(h, self.w["mlp_norm"][l], m.eps)
                    gu = OA.bf16_to_f64(self.w["w_gu"][l]) @ x
                    F = len(gu) // 2
                    h = h + OA.bf16_to_f64(self.w["w_down"][l]) @ (ODec.silu(gu[:F]) * gu[F:])
                rows.append(OA.bf16_to_f64(self.w["embed"]) @ m.final_state(h))
            logits.append(np.array(rows))
        return logits, k, v


def rel_l2(a, b):
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


@pytest.mark.parametrize("window", [0, 20])
def test_prompts_match_the_oracle(window):
    t = Prompts(window=window)
    ref, k, v = t.oracle()
    forward, scores = t.dec.stages()
    done = np.zeros(4, int)
    for c in range(3):
        t.set(c)
        t.run(forward + scores)
        torch.cuda.synchronize()
        _, tgt, start = t.chunk(c)
        want = np.concatenate([ref[b][done[b]:done[b] + t.chunks[c][b]] for b in range(4)])
        done += t.chunks[c]
        n = len(want)
        got = t.dec.logits.cpu().numpy()[:n].astype(np.float64)
        assert rel_l2(got, want) <= STEP_REL_L2, c
        # the scores are those of the logits
        lp, rank, h, best, ids = OP.token_logprobs(got, np.array(tgt), 5)
        assert np.abs(t.dec.logprob.cpu().numpy()[:n] - lp).max() <= 1e-5 + 2.0 ** -22 * np.abs(lp).max()
        np.testing.assert_array_equal(t.dec.rank.cpu().numpy()[:n], rank)
        np.testing.assert_array_equal(t.dec.top_tokens.cpu().numpy()[:n], ids)
        assert np.abs(t.dec.entropy.cpu().numpy()[:n] - h).max() <= 2e-5
        np.testing.assert_array_equal(t.dseq.cpu().numpy(), done)
    # caches: the oracle's up to rare one-step ties; nothing else is touched
    for got, want, was in ((t.dk, k, t.k), (t.dv, v, t.v)):
        got = got.cpu().numpy().view(np.uint16)
        a, b = OA.bf16_to_f64(got), OA.bf16_to_f64(want)
        assert (got != want).mean() < 5e-3 and np.abs(a - b).max() <= 2.0 ** -6 * np.abs(b).max()
        np.testing.assert_array_equal(got[want == was], was[want == was])


def test_chunks_of_any_size_leave_the_same_caches_and_scores():
    """One chunk of everything and three chunks: up to the rounding of fp32 sums."""
    a, b = Prompts(score="last"), Prompts(score="last", rows=160)
    for t, chunks in ((a, [0, 1, 2]), (b, None)):
        forward, scores = t.dec.stages()
        if chunks is None:
            t.chunks = [list(np.sum(t.chunks, 0))]
            chunks = [0]
        for c in chunks:
            t.set(c)
            t.run(forward)
        t.run(scores)
        torch.cuda.synchronize()
    for x, y in ((a.dk, b.dk), (a.dv, b.dv)):
        x, y = (OA.bf16_to_f64(u.cpu().numpy().view(np.uint16)) for u in (x, y))
        assert (x != y).mean() < 5e-3 and np.abs(x - y).max() <= 2.0 ** -6 * np.abs(y).max()
    la = a.dec.row_start[1:].long() - 1
    lb = b.dec.row_start[1:].long() - 1
    assert rel_l2(a.dec.logits[la].double().cpu().numpy(), b.dec.logits[lb].double().cpu().numpy()) <= STEP_REL_L2
    # only the last rows were scored
    assert set(a.dec.listed[:4].tolist()) == set(la.tolist()) and int(a.dec.n_listed) == 4
    rest = np.setdiff1d(np.arange(48), la.cpu().numpy())
    assert (a.dec.logits.cpu().numpy()[rest] == 0).all() and (a.dec.rank.cpu().numpy()[rest] == 0).all()


def test_requests_without_rows_are_not_scored():
    t = Prompts(score="last")
    forward, scores = t.dec.stages()
    t.set(0)
    t.run(forward + scores)
    torch.cuda.synchronize()
    assert int(t.dec.n_listed) == 3 and t.dec.listed[:3].tolist() == [4, 44, 45]


def test_decode_steps_go_on_from_a_prompt():
    """Decoder's next greedy token is the oracle's, Local through the rings the paged one's."""
    from paper_2609_20734_amd import decoder as PD
    t = Prompts(rings=True, score="last", top=1)
    forward, scores = t.dec.stages()
    for c in range(3):
        t.set(c)
        t.run(forward + scores)
    torch.cuda.synchronize()
    last = t.dec.row_start[1:].long() - 1
    first = t.dec.top_tokens[last, 0].cpu().numpy()
    ref, _, _ = t.oracle()
    assert [int(np.argmax(r[-1])) for r in ref] == first.tolist()
    # rings hold what a ring filled from the cache holds
    L, B, Hkv, D = t.L, 4, t.Hkv, t.D
    shape = t.P.Shape(1, B, 4, Hkv, D, t.mb, t.mb * 16, t.nb)
    q = dev_u16(S.normal_bf16(t.g, (1, B, 4, D)))
    ws = torch.zeros(max(256, t.P.attn_workspace_size(shape, 4, 24)), dtype=torch.uint8, device="cuda")
    for l in range(L):
        o = [torch.zeros(1, B, 4, D, device="cuda") for _ in range(2)]
        s = [torch.zeros(1, B, 4, device="cuda") for _ in range(2)]
        t.P.local_decode_attn(shape, t.P.inputs(q, t.dk[l], t.dv[l], t.dtab, t.dseq, 0.125), 4, 24, o[0], s[0], ws)
        t.P.local_decode_attn_ring(shape, t.P.inputs(q, None, None, None, t.dseq, 0.125), t.rings[0][l], t.rings[1][l], 4, 24,
                                   o[1], s[1], ws)
        torch.cuda.synchronize()
        assert torch.equal(o[0], o[1]) and torch.equal(s[0], s[1])
    # one step of native Full on the first token
    t.dseq.add_(1)
    dec = PD.Decoder(t.shape, t.dw, B, t.dk, t.dv, t.dtab, t.dseq, t.mb, t.mb * 16, t.nb, 4, 24)
    local, retry, out = dec.full_stages()
    dec.tokens.copy_(torch.from_numpy(first.astype(np.int32)))
    PD.run(local + retry + out)
    torch.cuda.synchronize()
    t.tokens = [np.append(x, f) for x, f in zip(t.tokens, first)]
    ref, _, _ = t.oracle()
    assert rel_l2(dec.logits.cpu().numpy().astype(np.float64), np.array([r[-1] for r in ref])) <= STEP_REL_L2


def test_a_chunk_as_a_graph():
    """Captured once, replayed for every chunk, with eager work between: bit for bit the eager run's."""
    a, b = Prompts(), Prompts()
    forward, scores = b.dec.stages()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = b.dec.stages()
        b.run(captured[0] + captured[1])
    ea = a.dec.stages()
    for c in range(3):
        a.set(c)
        a.run(ea[0] + ea[1])
        b.set(c)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in ((a.dec.logits, b.dec.logits), (a.dec.logprob, b.dec.logprob), (a.dec.rank, b.dec.rank),
                     (a.dec.top_tokens, b.dec.top_tokens), (a.dk, b.dk), (a.dv, b.dv), (a.dseq, b.dseq)):
            assert torch.equal(x.nan_to_num(0.0) if x.is_floating_point() else x, y.nan_to_num(0.0) if y.is_floating_point() else y)


def test_refusals():
    t = Prompts()
    with pytest.raises(ValueError):
        t.dec.set_chunk(torch.zeros(49, dtype=torch.int32), torch.zeros(5, dtype=torch.int32))
    from paper_2609_20734_amd import decoder as PD
    with pytest.raises(ValueError):
        PD.PromptDecoder(t.shape, t.dw, 4, 8, t.dk, t.dv, t.dtab, t.dseq, t.mb, t.mb * 16, t.nb, score="some")
