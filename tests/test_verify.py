"""oda_verify_drafts against the fp64 oracle: tokens and counts are whole numbers
and have to be equal.  (A draw changes only where u lies within the sums'
rounding, about 1e-13, of a border.)"""
import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_f32, dev_i32, need_gpu
from oracle import drafts as OD

pytestmark = pytest.mark.gpu


class Drafts:
    def __init__(self, seed, B, K, V, temps=(1.0,), q=True, std=2.5, noise=0.4):
        self.P = need_gpu()
        g = S.rng(seed, 78)
        self.g, self.B, self.K, self.V = g, B, K, V
        self.z = (std * g.standard_normal((B, K + 1, V))).astype(np.float32)
        self.t = np.resize(np.array(temps, dtype=np.float32), B)
        self.n = np.array([K - (b % 3 if K >= 3 else 0) for b in range(B)], dtype=np.int32)
        self.q = None
        self.x = np.zeros((B, K), dtype=np.int32)
        if q and K:
            e = (self.z[:, :K] + noise * g.standard_normal((B, K, V))) / np.maximum(self.t, 0.05)[:, None, None]
            e = np.exp(e - e.max(-1, keepdims=True))
            self.q = (e / e.sum(-1, keepdims=True)).astype(np.float32)
            c = np.cumsum(self.q.astype(np.float64), -1)
            r = g.random((B, K, 1)) * c[..., -1:]
            self.x = np.minimum((c <= r).sum(-1), V - 1).astype(np.int32)
        elif K:
            self.x = self.z[:, :K].argmax(-1).astype(np.int32)
            wild = g.random((B, K)) < 0.3
            self.x = np.where(wild, g.integers(0, V, size=(B, K)), self.x).astype(np.int32)
        self.u = g.random((B, K + 1)).astype(np.float32)
        self.u[self.u >= 1] = 0.5

    def upload(self):
        f = lambda a: None if a is None else dev_f32(a)  # noqa: E731
        self.dev = (dev_f32(self.z), dev_i32(self.x) if self.K else None, dev_f32(self.u), f(self.q), dev_i32(self.n),
                    dev_f32(self.t))
        self.desc = self.P.verify_desc(self.V, self.K, *self.dev)
        self.ws = torch.zeros(self.P.verify_workspace_size(self.B, self.V, self.K), dtype=torch.uint8, device="cuda")
        self.acc = torch.full((self.B,), -9, dtype=torch.int32, device="cuda")
        self.tok = torch.full((self.B, self.K + 1), -9, dtype=torch.int32, device="cuda")

    def run(self, work=None):
        wl = (None, None) if work is None else (dev_i32(work + [0] * (self.B - len(work))), dev_i32([len(work)]))
        self.P.verify_drafts(self.desc, self.B, self.acc, self.tok, self.ws, *wl)
        torch.cuda.synchronize()
        return self.acc.cpu().numpy(), self.tok.cpu().numpy()

    def oracle(self):
        return OD.verify_drafts(self.z, self.x, self.u, self.q, self.n, self.t)

    def check(self, work=None):
        self.upload()
        ra, rt = self.oracle()
        for _ in range(3):                       # the workspace's words are back at zero after every call
            a, t = self.run(work)
            rows = np.arange(self.B) if work is None else np.array([b for b in work if 0 <= b < self.B], dtype=int)
            np.testing.assert_array_equal(a[rows], ra[rows])
            np.testing.assert_array_equal(t[rows], rt[rows])
            rest = np.setdiff1d(np.arange(self.B), rows)
            assert (a[rest] == -9).all() and (t[rest] == -9).all()
        return ra, rt


@pytest.mark.parametrize("q", [True, False])
@pytest.mark.parametrize("B,K,V", [(1, 0, 1), (3, 0, 7), (2, 1, 1), (2, 1, 5), (5, 3, 63), (4, 2, 2047), (3, 4, 4097),
                                   (7, 8, 9001), (2, 5, 50257), (33, 1, 16389), (1, 4, 151936), (2, 3, 300001)])
def test_matches_oracle(B, K, V, q):
    Drafts(B * 100 + K, B, K, V, temps=(1.0, 0.0, 0.6, 1.7), q=q).check()


def test_counts_of_every_kind():
    """Many small requests: none, some and all drafts accepted, temperatures mixed."""
    t = Drafts(5, 256, 6, 40, temps=(1.0, 0.0, 0.3, 4.0, -1.0, np.nan, np.inf), noise=0.8)
    acc, _ = t.check()
    assert set(acc) >= {0, 1, 2, 3, 4}


def test_masks_infinities_and_nan():
    t = Drafts(6, 10, 3, 3001, temps=(1.0, 0.7))
    t.n[:] = 3
    low = np.finfo(np.float32).min
    t.z[0, :, ::2] = -np.inf                       # half masked
    t.z[1, :, 1::2] = low                          # by the lowest value
    t.z[2] = -np.inf                               # nothing to choose
    t.z[3] = low                                   # all at the lowest value: even
    t.z[4, 1] = -np.inf                            # the second row empty
    t.z[5, :, 100:200] = np.nan
    t.z[6] = np.nan
    t.z[7, :, 2500] = np.inf                       # one infinite logit, then two
    t.z[8, :, [17, 2999]] = np.inf
    t.z[9, :, :-1] = -np.inf                       # one token left
    acc, tok = t.check()
    assert acc[2] == 0 and tok[2, 0] == -1 and tok[6, 0] == -1
    assert all(v == 3000 or v == -1 for v in tok[9])
    t.t[:] = 0.0
    t.check()


def test_refused_where_nothing_is_left_draws_from_the_target():
    """q >= p everywhere: the residual is empty."""
    t = Drafts(7, 24, 2, 500)
    t.n[:] = 2
    t.q[:] = 1.0
    acc, tok = t.check()
    assert (acc < 2).any()


def test_ends_of_the_unit_interval():
    t = Drafts(8, 6, 2, 5003, std=4.0)
    t.n[:] = [0, 1, 2, 2, 1, 0]
    t.u[:3] = 0.0                                  # the first token with a weight
    t.u[3:] = 1 - 2.0 ** -24                       # the largest fp32 below 1
    t.z[0, 0, :50] = -np.inf
    t.z[5, 0, -50:] = -np.inf
    t.check()


def test_draft_tokens_and_counts_out_of_range():
    t = Drafts(9, 8, 3, 700)
    t.n[:] = [-5, 9, 3, 3, 3, 0, 1, 2 ** 31 - 1]
    t.x[1, 0], t.x[2, 1], t.x[3, 0], t.x[4, 2] = -1, 700, 2 ** 31 - 1, -2 ** 31
    t.check()
    t = Drafts(9, 8, 3, 700, q=False)
    t.x[1, 0], t.x[2, 1], t.x[3, 0], t.x[4, 2] = -1, 700, 2 ** 31 - 1, -2 ** 31
    t.check()


def test_draft_probabilities_that_are_none():
    t = Drafts(10, 6, 2, 900)
    t.n[:] = 2
    t.q[0, 0, :450] = np.nan
    t.q[1, 0] *= -1
    t.q[2, 0] = 0.0
    t.q[3, :, t.x[3, 0]] = np.nan
    t.check()


def test_ties_go_to_the_first():
    t = Drafts(11, 4, 2, 4099, temps=(0.0,))
    t.n[:] = 2
    t.z[:] = np.minimum(t.z, 2.0)                  # hundreds of equal largest logits
    t.x[:, 0] = t.z[:, 0].argmax(-1)
    t.x[0, 1] = t.z[0, 1].argmax(-1)
    acc, _ = t.check()
    assert acc[0] == 2 and (acc >= 1).all()


def test_listed_requests_only():
    Drafts(12, 9, 2, 1000).check(work=[7, 0, 3, -2, 9])


def test_empty_list():
    Drafts(12, 3, 2, 1000).check(work=[])


def test_optional_arrays_left_out():
    t = Drafts(13, 5, 2, 1234)
    t.n[:], t.t[:] = 2, 1.0
    t.upload()
    t.desc = t.P.verify_desc(t.V, t.K, *t.dev[:3], t.dev[3])
    ra, rt = t.oracle()
    a, tok = t.run()
    np.testing.assert_array_equal(a, ra)
    np.testing.assert_array_equal(tok, rt)


def test_unaligned_rows():
    """Logits and probabilities at any 4-byte address."""
    t = Drafts(14, 3, 2, 4095)
    t.upload()
    z = torch.zeros(t.z.size + 3, device="cuda")
    q = torch.zeros(t.q.size + 1, device="cuda")
    z[3:] = t.dev[0].flatten()
    q[1:] = t.dev[3].flatten()
    t.desc = t.P.verify_desc(t.V, t.K, z[3:], t.dev[1], t.dev[2], q[1:], t.dev[4], t.dev[5])
    ra, rt = t.oracle()
    a, tok = t.run()
    np.testing.assert_array_equal(a, ra)
    np.testing.assert_array_equal(tok, rt)


def test_workspace_serves_smaller_calls():
    """One workspace, sized for the largest vocabulary and draft count."""
    big = Drafts(15, 4, 5, 20000)
    big.upload()
    for V, K in ((20000, 5), (300, 5), (20000, 0), (4097, 2)):
        t = Drafts(16, 4, K, V)
        t.upload()
        t.ws = big.ws
        ra, rt = t.oracle()
        a, tok = t.run()
        np.testing.assert_array_equal(a, ra)
        np.testing.assert_array_equal(tok, rt)


def test_captured_call_replays():
    t = Drafts(17, 6, 4, 30011, temps=(1.0, 0.0, 0.8))
    t.upload()
    t.run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        t.P.verify_drafts(t.desc, t.B, t.acc, t.tok, t.ws)
    for rep in range(3):
        t.u = t.g.random(t.u.shape).astype(np.float32) * np.float32(0.999)
        t.dev[2].copy_(torch.from_numpy(t.u))
        t.acc.fill_(-9)
        t.tok.fill_(-9)
        g.replay()
        torch.cuda.synchronize()
        ra, rt = t.oracle()
        np.testing.assert_array_equal(t.acc.cpu().numpy(), ra)
        np.testing.assert_array_equal(t.tok.cpu().numpy(), rt)
        _ = (t.dev[0] * 2).sum().item()


def test_a_request_listed_twice():
    """Each place of the list has its own sums and words: a request listed several times gets its one result."""
    t = Drafts(41, 9, 3, 20011, temps=(1.0, 0.7, 1.3))
    t.check([2, 2, 2, 5, 2, 7, 5, 2])
    t.check([8] * 9)
    t.check()
