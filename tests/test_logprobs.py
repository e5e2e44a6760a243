"""oda_token_logprobs against the fp64 oracle.  Tokens and ranks are whole numbers and
have to be equal.  Tolerance of the rest: a lane adds up to V / 512 weights in fp32
(2^-24 of the sum each), an exponent of up to 30 is off by 30 * 2^-24, the result is
rounded once: below 1e-5 + 2^-22 of the value for V up to 60,000 and split rows."""
import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_f32, dev_i32, need_gpu
from oracle import prompt as OP

pytestmark = pytest.mark.gpu


def near(got, ref, what):
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - ref) <= 1e-5 + 2.0 ** -22 * np.abs(ref))
    assert ok.all(), f"{what}: {got[~ok][:4]} for {ref[~ok][:4]}"


class Scores:
    def __init__(self, seed, R, V, top, std=2.5):
        self.P = need_gpu()
        g = S.rng(seed, 92)
        self.g, self.R, self.V, self.top = g, R, V, top
        self.z = (std * g.standard_normal((R, V))).astype(np.float32)
        self.t = np.where(g.random(R) < 0.5, self.z.argmax(-1), g.integers(0, V, size=R)).astype(np.int32)
        self.ws = None

    def run(self, stride=0, work=None, tokens=True, lead=0):
        P, R, V, k = self.P, self.R, self.V, self.top
        wide = np.full((R, max(stride, V)), np.inf, dtype=np.float32)     # (what a row does not own is not read)
        wide[:, :V] = self.z
        flat = dev_f32(np.concatenate([np.full(lead, np.inf, dtype=np.float32), wide.reshape(-1)]))
        desc = P.logprob_desc(V, k, flat[lead:], dev_i32(self.t) if tokens else None, stride)
        if self.ws is None:
            self.ws = torch.zeros(P.logprob_workspace_size(desc, R), dtype=torch.uint8, device="cuda")
        out = [torch.full((R,), -9.0, device="cuda"), torch.full((R,), -9, dtype=torch.int32, device="cuda"),
               torch.full((R,), -9.0, device="cuda"), torch.full((R, k), -9.0, device="cuda") if k else None,
               torch.full((R, k), -9, dtype=torch.int32, device="cuda") if k else None]
        if not tokens:
            out[0] = out[1] = None
        wl = (None, None) if work is None else (dev_i32(work + [0] * (R - len(work))), dev_i32([len(work)]))
        P.token_logprobs(desc, R, *out, self.ws, *wl)
        torch.cuda.synchronize()
        return [None if o is None else o.cpu().numpy() for o in out]

    def check(self, **kw):
        ref = OP.token_logprobs(self.z, self.t, self.top)
        for _ in range(3):                       # the workspace's words are back at zero after every call
            got = self.run(**kw)
            self.same(got, ref, np.arange(self.R))
        return got

    def same(self, got, ref, rows):
        near(got[0][rows], ref[0][rows], "logprob")
        np.testing.assert_array_equal(got[1][rows], ref[1][rows])
        near(got[2][rows], ref[2][rows], "entropy")
        if self.top:
            np.testing.assert_array_equal(got[4][rows], ref[4][rows])
            near(got[3][rows], ref[3][rows], "top")


@pytest.mark.parametrize("R,V,top", [(1, 1, 0), (1, 1, 1), (3, 7, 5), (2, 5, 32), (5, 63, 20), (4, 1023, 32), (2, 4097, 1),
                                     (33, 2049, 5), (3, 50257, 20), (1, 151936, 32), (2, 300001, 7), (300, 257, 3), (1100, 40, 2)])
def test_matches_oracle(R, V, top):
    Scores(R + V, R, V, top).check()


@pytest.mark.parametrize("V,stride,lead", [(1001, 1003, 0), (1000, 1024, 1), (9001, 9003, 3)])
def test_strides_and_alignments(V, stride, lead):
    Scores(5, 6, V, 9).check(stride=stride, lead=lead)


def test_masks_infinities_and_nan():
    t = Scores(6, 14, 6001, 12)
    low = np.finfo(np.float32).min
    t.z[0, ::2] = -np.inf                          # half masked
    t.z[1, 1::2] = low                             # by the lowest value
    t.z[2] = -np.inf                               # no distribution
    t.z[3] = low                                   # all at the lowest value: even
    t.z[4, 100:200] = np.nan
    t.z[5] = np.nan
    t.z[6, 2500] = np.inf                          # one infinite logit, then three
    t.z[7, [17, 999, 5999]] = np.inf
    t.z[8, :-1] = -np.inf                          # one token left
    t.z[9, 5:] = -np.inf                           # fewer than are asked for
    t.z[10] = 0.0
    t.z[10, ::3] = -0.0                            # equal to 0
    t.z[11, 3] = 3e38                              # far above the rest
    t.z[12] = np.float32(-1e30)
    t.z[12, 70] = 1e30
    t.t[:] = [2, 1, 5, 4000, 150, 0, 2500, 999, 10, 4, 9, 3, 71, 6000]
    t.check()


def test_ties_go_to_the_lowest_index():
    t = Scores(7, 8, 20011, 32)
    t.z = np.round(t.z * 2) / 2                    # a dozen values, thousands of ties
    t.check()
    t.z[:] = 1.25                                  # all equal
    t.check()


def test_long_rows_with_few_tokens_left():
    """Masks that leave logits in a few parts of a row split over many workgroups, and ties across all of them."""
    t = Scores(16, 7, 300_001, 32)
    full = t.z.copy()
    for r, keep in enumerate(([0, 150_000, 300_000], range(70_000, 70_040), range(11, 300_001, 3_001), range(40_000, 160_000, 4_000))):
        t.z[r] = -np.inf
        t.z[r, list(keep)] = full[r, list(keep)]
    t.z[3, np.isfinite(t.z[3])] = 2.0              # thirty equal ones
    t.z[4] = -1.5                                  # all equal
    t.z[5] = np.linspace(5, -5, 300_001, dtype=np.float32)
    t.z[6] = np.round(full[6])                     # a dozen values
    t.t[:] = [150_000, 70_001, 12, 44_000, 299_999, 17, 5]
    t.check()


def test_ascending_rows_replace_every_place():
    t = Scores(8, 3, 9000, 32)
    t.z[:] = np.linspace(-5, 5, 9000, dtype=np.float32)
    t.z[1] = t.z[1, ::-1]
    t.check()


def test_tokens_outside_the_vocabulary():
    t = Scores(9, 4, 500, 3)
    t.t[:] = [-1, 500, 2 ** 31 - 1, 499]
    got = t.check()
    assert np.isnan(got[0][:3]).all() and (got[1][:3] == 0).all() and got[1][3] > 0


def test_peaked_and_flat():
    t = Scores(10, 4, 30000, 4)
    t.z[0] *= 40                                   # one token has nearly all
    t.z[1] *= 1e-3
    t.z[2, 77] = 60
    t.check()


def test_listed_rows_alone():
    t = Scores(11, 9, 5003, 6)
    ref = OP.token_logprobs(t.z, t.t, 6)
    for work in ([], [3], [8, 0, 5], [2, 2, 7], [1, 9, -1, 4]):
        got = t.run(work=work)
        rows = np.array(sorted({w for w in work if 0 <= w < 9}), dtype=int)
        t.same(got, ref, rows)
        rest = np.setdiff1d(np.arange(9), rows)
        assert (got[0][rest] == -9).all() and (got[4][rest] == -9).all()


def test_without_tokens():
    t = Scores(12, 3, 2000, 5)
    ref = OP.token_logprobs(t.z, None, 5)
    got = t.run(tokens=False)
    near(got[2], ref[2], "entropy")
    np.testing.assert_array_equal(got[4], ref[4])


def test_one_workspace_serves_calls_of_any_size():
    a, b, c = Scores(13, 2, 60000, 20), Scores(14, 700, 900, 3), Scores(15, 1, 200000, 32)
    a.check()
    for t in (b, c, a):
        t.ws = a.ws
        t.check()
    assert int(a.ws[:1024 * 128].to(torch.int64).sum()) == 0


def test_more_rows_than_a_grid_is_high():
    P = need_gpu()
    R, V = 70_000, 12
    z = torch.randn(R, V, device="cuda")
    t = torch.randint(0, V, (R,), device="cuda").int()
    lp = torch.zeros(R, device="cuda")
    desc = P.logprob_desc(V, 0, z, t)
    ws = torch.zeros(P.logprob_workspace_size(desc, R), dtype=torch.uint8, device="cuda")
    P.token_logprobs(desc, R, lp, None, None, None, None, ws)
    torch.cuda.synchronize()
    ref = torch.log_softmax(z.double(), -1).gather(1, t.long()[:, None])[:, 0]
    near(lp.cpu().numpy(), ref.cpu().numpy(), "logprob")
