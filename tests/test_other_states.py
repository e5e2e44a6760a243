"""Attention of rows over other states, as a decoder beside an encoder uses it: the
states' K/V appended once (no query heads, no rotation), every step's rows appended as
queries alone and attended without a mask, their tokens scored.

Tolerances: without a norm and a rotation an append rounds alone, so its bits are the
oracle's; the attention then has its own bars (fp32 and bf16 outputs), and the scores
those of their logits."""
import math

import numpy as np
import pytest
import torch

import oda_synth as S
from harness import LSE_ABS, MAX_ABS_INTERNAL, dev_f32, dev_i32, dev_u16, need_gpu
from oracle import prompt as OP
from oracle.attention import bf16_to_f64
from oracle.decoder import bf16_bits, round_bf16

pytestmark = pytest.mark.gpu


class States:
    """B requests with states of their own length (one has none); steps of any rows."""

    def __init__(self, seed, lens, Hq, Hkv, D, V=517):
        P = self.P = need_gpu()
        self.g, self.B, self.Hq, self.Hkv, self.D, self.V = S.rng(seed, 95), len(lens), Hq, Hkv, D, V
        self.lens = np.array(lens, dtype=np.int32)
        self.mb = -(-int(self.lens.max()) // 16)
        self.table, self.nb = S.paged_block_table(S.rng(seed, S.STREAM_TABLE), np.maximum(self.lens, 1), self.mb)
        self.k, self.v = (a[0] for a in S.kv_cache(seed, 1, self.nb, Hkv, D))
        self.dk, self.dv, self.dtab, self.dlen = dev_u16(self.k), dev_u16(self.v), dev_i32(self.table), dev_i32(self.lens)
        self.shape = P.Shape(1, self.B, Hq, Hkv, D, self.mb, self.mb * 16, self.nb)
        self.scale = 1 / math.sqrt(D)
        self.w = dev_f32(0.05 * self.g.standard_normal((Hq * D, V)))

    def encode(self):
        """The states' rows into the cache, and what the oracle holds then."""
        P, start = self.P, np.concatenate([[0], np.cumsum(self.lens)])
        x = self.g.standard_normal((int(start[-1]), 2 * self.Hkv * self.D)).astype(np.float32)
        desc = P.append_desc(dev_f32(x), None, None, 0.0, 0.0)
        self.keep = (dev_i32(start), desc)
        P.prepare_append_qkv(self.shape, P.prompt_rows(len(x), self.keep[0]), desc, self.dk, self.dv, self.dtab, self.dlen, None)()
        full = np.concatenate([np.zeros((len(x), self.Hq * self.D)), x.astype(np.float64)], 1)
        _, k, v, owner = OP.append_rows(full, self.Hq, self.Hkv, self.D, start, self.lens)
        OP.put_rows(k, v, owner, self.table, self.lens, self.k, self.v)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(self.dk.cpu().numpy().view(np.uint16), self.k)
        np.testing.assert_array_equal(self.dv.cpu().numpy().view(np.uint16), self.v)

    def step(self, rows, bf16, cap):
        """Calls of a step of up to `cap` rows: queries, plan, attention, scores."""
        P = self.P
        self.start = np.concatenate([[0], np.cumsum(rows)])
        self.dstart, self.cap = dev_i32(self.start), cap
        self.x = torch.zeros(cap, self.Hq * self.D, device="cuda")
        self.tok = torch.zeros(cap, dtype=torch.int32, device="cuda")
        r = P.prompt_rows(cap, self.dstart)
        self.q = torch.zeros(cap, self.Hq, self.D, dtype=torch.bfloat16, device="cuda")
        self.out = torch.full((cap, self.Hq, self.D), -9.0, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
        self.lse = torch.full((cap, self.Hq), -9.0, device="cuda")
        self.z = torch.zeros(cap, self.V, device="cuda")
        self.lp = torch.zeros(cap, device="cuda")
        plan = torch.zeros(P.prompt_plan_size(self.shape, r), dtype=torch.uint8, device="cuda")
        ws = torch.zeros(P.prompt_workspace_size(self.shape, r), dtype=torch.uint8, device="cuda")
        desc = P.logprob_desc(self.V, 0, self.z, self.tok)
        lws = torch.zeros(P.logprob_workspace_size(desc, cap), dtype=torch.uint8, device="cuda")
        # (queries without places of their own: any length that holds the rows)
        places = torch.full((self.B,), cap, dtype=torch.int32, device="cuda")
        own = P.Shape(1, self.B, self.Hq, self.Hkv, self.D, -(-cap // 16), -(-cap // 16) * 16, self.nb)
        self.calls = [
            P.prepare_append_qkv(own, r, P.append_desc(self.x, None, None, 0.0, 0.0), None, None, None, places, self.q),
            P.prepare_prompt_plan(self.shape, r, self.dlen, False, 0, plan),
            P.prepare_prompt_attn(self.shape, P.inputs(self.q, self.dk, self.dv, self.dtab, None, self.scale), r, plan, self.out,
                                  self.lse, ws),
        ]
        self.scores = P.prepare_token_logprobs(desc, cap, self.lp, None, None, None, None, lws)

    def fill(self):
        x = self.g.standard_normal((self.cap, self.Hq * self.D)).astype(np.float32)
        self.x.copy_(torch.from_numpy(x))
        return x.astype(np.float64)

    def run(self):
        for c in self.calls:
            c()
        self.scores()

    def check(self, x, bf16, tokens):
        n = int(self.start[-1])
        qb = bf16_bits(round_bf16(x)).reshape(self.cap, self.Hq, self.D)
        np.testing.assert_array_equal(self.q[:n].view(torch.int16).cpu().numpy().view(np.uint16), qb[:n])
        ref, rlse, mag = OP.prompt_attention(qb, self.k[None], self.v[None], self.table, self.start, self.lens, self.scale, causal=False)
        out, lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        bound = MAX_ABS_INTERNAL
        if bf16:
            bound = bound + 2.0 ** -8 * (np.abs(ref[:n]) + mag[:n])
        assert (np.abs(out[:n] - ref[:n]) <= bound).all()
        seen = np.isfinite(rlse[:n])
        np.testing.assert_array_equal(np.isneginf(lse[:n]), ~seen)
        assert np.abs(lse[:n][seen] - rlse[:n][seen]).max() <= LSE_ABS
        assert (out[n:] == -9.0).all() and (lse[n:] == -9.0).all()
        z = self.z.double().cpu().numpy()
        lp = OP.token_logprobs(z, tokens, 0)[0]
        assert np.abs(self.lp.double().cpu().numpy() - lp).max() <= 1e-5 + 2.0 ** -22 * np.abs(lp).max()


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 64), (8, 2, 128), (5, 5, 64)])
@pytest.mark.parametrize("bf16", [False, True])
def test_rows_over_an_encoders_states(Hq, Hkv, D, bf16):
    t = States(31, [75, 1, 0, 333], Hq, Hkv, D)
    t.encode()
    for rows in ([9, 4, 3, 40], [1, 1, 1, 1], [0, 0, 2, 1]):     # a prompt, one token of each, of some
        t.step(rows, bf16, cap=60)
        x, tokens = t.fill(), t.g.integers(0, t.V, size=60)
        t.tok.copy_(torch.from_numpy(tokens.astype(np.int32)))
        t.calls.append(lambda: torch.mm(t.out.float().reshape(60, -1), t.w, out=t.z))
        t.run()
        torch.cuda.synchronize()
        t.check(x, bf16, tokens)


def test_a_captured_step_with_other_rows_and_states():
    t = States(32, [120, 64, 5], 8, 4, 64)
    t.encode()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        t.step([3, 1, 2], False, cap=12)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            t.run()
    for rows, lens in (([3, 1, 2], [120, 64, 5]), ([1, 1, 1], [17, 64, 1]), ([0, 10, 2], [120, 0, 3])):
        t.start, t.lens = np.concatenate([[0], np.cumsum(rows)]), np.array(lens, dtype=np.int32)
        t.dstart.copy_(dev_i32(t.start))
        t.dlen.copy_(dev_i32(t.lens))
        x, tokens = t.fill(), t.g.integers(0, t.V, size=12)
        t.tok.copy_(torch.from_numpy(tokens.astype(np.int32)))
        t.z.copy_(dev_f32(t.g.standard_normal((12, t.V))))
        t.out.fill_(-9.0)
        t.lse.fill_(-9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        t.check(x, False, tokens)


def test_two_graphs_share_their_workspaces():
    """Two captured steps of other sizes with one workspace each for attention and scores, replayed in turn."""
    t = States(33, [2000, 900, 40], 8, 2, 64, V=40_000)
    t.encode()
    P, side = t.P, torch.cuda.Stream()
    ws = lws = None
    steps = []
    with torch.cuda.stream(side):
        for rows in ([30, 1, 2], [1, 1, 1]):
            cap = sum(rows)
            t.step(rows, False, cap)
            ws = ws if ws is not None else torch.zeros(P.prompt_workspace_size(t.shape, P.prompt_rows(cap, t.dstart)),
                                                       dtype=torch.uint8, device="cuda")
            desc = P.logprob_desc(t.V, 3, t.z, t.tok)
            lws = lws if lws is not None else torch.zeros(P.logprob_workspace_size(desc, cap), dtype=torch.uint8, device="cuda")
            top = torch.zeros(cap, 3, device="cuda"), torch.zeros(cap, 3, dtype=torch.int32, device="cuda")
            r = P.prompt_rows(cap, t.dstart)
            plan = torch.zeros(P.prompt_plan_size(t.shape, r), dtype=torch.uint8, device="cuda")
            calls = [t.calls[0], P.prepare_prompt_plan(t.shape, r, t.dlen, False, 0, plan),
                     P.prepare_prompt_attn(t.shape, P.inputs(t.q, t.dk, t.dv, t.dtab, None, t.scale), r, plan, t.out, t.lse, ws),
                     P.prepare_token_logprobs(desc, cap, t.lp, None, None, *top, lws)]
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                for c in calls:
                    c()
            steps.append((graph, calls, top, {n: getattr(t, n) for n in ("start", "cap", "x", "tok", "q", "out", "lse", "z", "lp")}))
    for _ in range(3):
        for graph, _, top, own in steps:
            t.__dict__.update(own)
            x, tokens = t.fill(), t.g.integers(0, t.V, size=t.cap)
            t.tok.copy_(torch.from_numpy(tokens.astype(np.int32)))
            z = t.g.standard_normal((t.cap, t.V)).astype(np.float32)
            t.z.copy_(torch.from_numpy(z))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            t.check(x, False, tokens)
            np.testing.assert_array_equal(top[1].cpu().numpy(), OP.token_logprobs(z.astype(np.float64), tokens, 3)[4])
