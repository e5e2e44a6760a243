"""oda_append_qkv against the fp64 oracle.

Tolerance: q and k are exact values rounded to bf16 (half a step, 2^-8 of the value)
behind fp32 arithmetic: a sum of D squares, a reciprocal root, and a rotation by
factors rounded to fp32, together below 2^-19 of the pair's length.  v is rounded
alone, so its bits are the oracle's; so are all the caches' other bits."""
import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_f32, dev_i32, dev_u16, need_gpu
from oracle import prompt as OP
from oracle.attention import bf16_to_f64
from oracle.decoder import bf16_bits, round_bf16

pytestmark = pytest.mark.gpu
EPS, THETA = 1e-6, 1e6


class Append:
    def __init__(self, seed, B, Hq, Hkv, D, rows, hist, bf16=False, norm=True, theta=THETA, axis_pairs=None, positions=None,
                 sink=0, window=0, lead=0, tail=3, heads="qkv"):
        self.P = need_gpu()
        g = S.rng(seed, 91)
        self.B, self.Hq, self.Hkv, self.D, self.theta = B, Hq, Hkv, D, theta
        self.start = np.concatenate([[lead], lead + np.cumsum(rows)]).astype(np.int32)
        self.R = int(self.start[-1]) + tail
        self.seq = (np.array(rows) + np.array(hist)).astype(np.int32)
        self.mb = max(1, -(-int(self.seq.max()) // 16)) + 1
        self.max_len = self.mb * 16
        self.table, self.nb = S.paged_block_table(S.rng(seed, S.STREAM_TABLE), np.maximum(self.seq, 1), self.mb)
        self.heads = heads
        self.nq, self.nkv = (Hq if "q" in heads else 0), (Hkv if "k" in heads else 0)
        x = 1.5 * g.standard_normal((self.R, (self.nq + 2 * self.nkv) * D))
        self.bits = bf16_bits(round_bf16(x)) if bf16 else None
        self.x = bf16_to_f64(self.bits) if bf16 else x.astype(np.float32).astype(np.float64)
        self.qg = (1 + 0.1 * g.standard_normal(D)).astype(np.float32) if norm else None
        self.kg = (1 + 0.1 * g.standard_normal(D)).astype(np.float32) if norm else None
        self.axis_pairs = axis_pairs
        self.pos = positions
        if axis_pairs is not None and positions is None:
            self.pos = g.integers(0, 5000, size=(self.R, len(axis_pairs))).astype(np.int32)
        self.k, self.v = (a[0] for a in S.kv_cache(seed, 1, self.nb, Hkv, D))
        self.sb, self.rb = -(-sink // 16), (-(-window // 16) + 2 if window else 0)
        self.sink, self.window = sink, window
        self.kr = self.vr = None
        if window:
            self.kr = S.normal_bf16(g, (B, self.sb + self.rb, Hkv, D // 8, 16, 8))
            self.vr = S.normal_bf16(g, (B, self.sb + self.rb, Hkv, D, 16))
        self.q0 = S.normal_bf16(g, (self.R, Hq, D))

    def run(self, times=1):
        P = self.P
        d = lambda a: None if a is None else dev_u16(a)  # noqa: E731
        self.dk, self.dv, self.dkr, self.dvr, self.dq = d(self.k), d(self.v), d(self.kr), d(self.vr), d(self.q0)
        self.dx = dev_u16(self.bits) if self.bits is not None else dev_f32(self.x)
        f = lambda a: None if a is None else dev_f32(a)  # noqa: E731
        desc = P.append_desc(self.dx, f(self.qg), f(self.kg), EPS, self.theta,
                             None if self.pos is None else dev_i32(self.pos), self.axis_pairs)
        shape = P.Shape(1, self.B, self.Hq, self.Hkv, self.D, self.mb, self.max_len, self.nb)
        kv = (self.dk, self.dv) if self.nkv else (None, None)
        call = P.prepare_append_qkv(shape, P.prompt_rows(self.R, dev_i32(self.start)), desc, *kv, dev_i32(self.table),
                                    dev_i32(self.seq), self.dq if self.nq else None, self.dkr, self.dvr, self.sink, self.window)
        for _ in range(times):
            call()
        torch.cuda.synchronize()
        u = lambda t: None if t is None else t.cpu().numpy().view(np.uint16)  # noqa: E731
        return u(self.dq), u(self.dk), u(self.dv), u(self.dkr), u(self.dvr)

    def check(self):
        gq, gk, gv, gkr, gvr = self.run()
        rng = [(int(self.start[b]), int(self.start[b + 1])) for b in range(self.B)]
        ok = [b for b in range(self.B) if self.seq[b] >= rng[b][1] - rng[b][0] and self.seq[b] <= self.max_len]
        pad = lambda n: np.zeros((self.R, n, self.D))  # noqa: E731
        x = self.x.reshape(self.R, -1, self.D)
        full = np.concatenate([x[:, :self.nq] if self.nq else pad(self.Hq), x[:, self.nq:] if self.nkv else pad(2 * self.Hkv)], 1)
        q, k, v, owner = OP.append_rows(full.reshape(self.R, -1), self.Hq, self.Hkv, self.D, self.start, self.seq, self.qg, self.kg,
                                        EPS, self.theta, self.pos, self.axis_pairs)
        for b in range(self.B):
            if b not in ok:
                owner[rng[b][0]:rng[b][1]] = -2
        if self.nq:
            own = owner[:, 0] >= 0
            self.near(bf16_to_f64(gq[own]), q[own], "q")
            assert np.isnan(bf16_to_f64(gq[owner[:, 0] == -2])).all()
            np.testing.assert_array_equal(gq[owner[:, 0] == -1], self.q0[owner[:, 0] == -1])
        ref = [a.copy() if a is not None else None for a in (self.k, self.v, self.kr, self.vr)]
        if self.nkv:
            drop = owner[:, 0] >= 0
            for r in np.flatnonzero(drop):
                e = self.table[owner[r, 0], owner[r, 1] // 16]
                drop[r] = not 0 <= e < self.nb
            kept = np.where(drop[:, None], -1, owner)
            OP.put_rows(k, v, kept, self.table, self.seq, *ref, self.sb, self.rb)
        np.testing.assert_array_equal(gv, ref[1])
        if self.vr is not None:
            np.testing.assert_array_equal(gvr, ref[3])
        # K: the oracle's bits where nothing was written, near its value elsewhere
        for got, want, was in ((gk, ref[0], self.k), (gkr, ref[2], self.kr)):
            if was is None:
                continue
            if not self.nkv:
                np.testing.assert_array_equal(got, was)
                continue
            exact = np.full(was.shape, np.nan)
            for r, (b, p) in enumerate(kept):
                if b < 0:
                    continue
                val = k[r].reshape(self.Hkv, -1, 8)
                if was is self.k:
                    exact[self.table[b, p // 16], :, :, p % 16] = val
                    continue
                j, last = p // 16, (self.seq[b] - 1) // 16
                if j < self.sb or j > last - self.rb:
                    exact[b, j if j < self.sb else self.sb + j % self.rb, :, :, p % 16] = val
            touched = ~np.isnan(exact)
            np.testing.assert_array_equal(got[~touched], was[~touched])
            # (a pair's length is bounded by the head's: the largest of it times sqrt 2)
            err = np.abs(bf16_to_f64(got[touched]) - exact[touched])
            scale = np.sqrt(2) * np.abs(k).max()
            assert (err <= 2.0 ** -8 * np.abs(exact[touched]) + 2.0 ** -19 * scale).all()
        return gq, gk, gv, gkr, gvr

    def near(self, got, ref, what):
        h = self.D // 2
        length = np.sqrt(ref[..., :h] ** 2 + ref[..., h:] ** 2)
        bar = 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * np.concatenate([length, length], -1)
        assert (np.abs(got - ref) <= bar).all(), f"{what}: {np.abs(got - ref).max()}"


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,D,rows,hist", [
    (1, 1, 1, 64, [1], [0]),
    (1, 2, 2, 128, [1], [15]),
    (3, 6, 2, 128, [17, 0, 5], [0, 9, 14]),
    (4, 5, 1, 64, [1, 16, 15, 33], [31, 16, 1, 7]),                 # an odd number of heads of 64
    (2, 40, 8, 128, [130, 3], [5, 1000]),
    (5, 3, 3, 64, [0, 0, 48, 1, 0], [3, 0, 16, 47, 5]),
    (70, 4, 2, 64, [1 + b % 3 for b in range(70)], [7 * b for b in range(70)]),   # more than one scan of requests
])
def test_matches_oracle(B, Hq, Hkv, D, rows, hist, bf16):
    Append(31, B, Hq, Hkv, D, rows, hist, bf16=bf16, lead=2).check()


@pytest.mark.parametrize("norm,theta", [(False, 1e6), (True, 0.0), (False, 0.0), (True, 1e4)])
def test_norm_and_rotation_may_be_left_out(norm, theta):
    Append(32, 2, 4, 2, 128, [9, 20], [3, 0], norm=norm, theta=theta).check()


@pytest.mark.parametrize("D,pairs", [(128, [22, 21, 21]), (64, [8, 12, 12]), (128, [64, 0]), (64, [0, 1, 2, 29])])
def test_axes(D, pairs):
    Append(33, 2, 4, 2, D, [21, 6], [10, 0], axis_pairs=pairs).check()


def test_given_positions_of_one_axis():
    pos = np.array([[1_000_000], [0], [7], [-3], [524_287], [2]], dtype=np.int32)
    Append(34, 1, 2, 1, 128, [6], [40], positions=pos, tail=0).check()


@pytest.mark.parametrize("heads", ["q", "kv"])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_some_heads(heads, D):
    Append(35, 2, 9, 3, D, [18, 4], [3, 30], heads=heads).check()


@pytest.mark.parametrize("sink,window,rows,hist", [(4, 40, [100, 3, 1], [0, 90, 15]), (0, 1, [50, 16, 1], [9, 64, 0]),
                                                   (20, 100, [7, 300, 33], [0, 5, 400])])
def test_rings_hold_what_they_keep(sink, window, rows, hist):
    Append(36, 3, 4, 2, 64, rows, hist, sink=sink, window=window).check()


def test_bad_lengths_and_blocks():
    t = Append(37, 6, 4, 2, 128, [5, 20, 9, 40, 3, 4], [20, 3, 0, 0, 8, 0])
    t.seq[0] = t.max_len + 1                # longer than the table
    t.seq[2] = 8                            # shorter than its rows
    t.seq[5] = -5
    t.table[1, 1] = -1                      # the second block of its places
    t.table[3, 0] = t.nb
    t.check()


def test_row_starts_out_of_order_stay_inside():
    """Starts above the buffer, descending or negative: nothing outside the rows is touched."""
    t = Append(38, 4, 2, 2, 64, [4, 4, 4, 4], [0, 0, 0, 0], tail=0)
    t.start[:] = [-7, 6, 3, 900, 12]
    t.seq[:] = 64
    t.mb = 5
    t.max_len = 80
    t.table, t.nb = S.paged_block_table(S.rng(38, S.STREAM_TABLE), t.seq, t.mb)
    t.k, t.v = (a[0] for a in S.kv_cache(38, 1, t.nb, 2, 64))
    q, *_ = t.run()
    x = t.x.reshape(t.R, -1, 64)
    assert np.isfinite(bf16_to_f64(q)).all() and x.shape[0] == 16


def test_same_bits_as_the_candidate_of_a_decode_step():
    """A single row is the current token that oda_qk_norm_rope prepares (up to the sum of squares' order) and
    oda_commit_kv commits."""
    t = Append(39, 3, 4, 2, 128, [1, 1, 1], [0, 15, 100], lead=0, tail=0)
    q, k, v, _, _ = t.run()
    P = t.P
    qo = torch.zeros(3, 4, 128, dtype=torch.int16, device="cuda")
    ko, vo = (torch.zeros(3, 2, 128, dtype=torch.int16, device="cuda") for _ in range(2))
    P.qk_norm_rope(3, 4, 2, 128, t.dx, dev_f32(t.qg), dev_f32(t.kg), EPS, THETA, dev_i32(t.seq), qo, ko, vo)
    k2, v2 = dev_u16(t.k), dev_u16(t.v)
    shape = P.Shape(1, 3, 4, 2, 128, t.mb, t.max_len, t.nb)
    P.commit_kv(shape, k2, v2, dev_i32(t.table), dev_i32(t.seq), ko, vo, advance=False)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(v2.cpu().numpy().view(np.uint16), v)
    for got, want in ((q, qo), (k, k2)):
        a, b = bf16_to_f64(got), bf16_to_f64(want.cpu().numpy().view(np.uint16))
        assert (np.abs(a - b) <= 2.0 ** -7 * np.abs(b)).all() and (a != b).mean() < 5e-3


def test_padded_chunk_behind_a_long_history_and_far_places():
    """Places above 2^16 blocks' worth of elements: offsets pass 32 bits."""
    P = need_gpu()
    nb, Hkv, D = 140_000, 8, 128             # 2.3e9 elements of K
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB of device memory")
    k = torch.zeros(nb, Hkv, D // 8, 16, 8, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(nb, Hkv, D, 16, dtype=torch.bfloat16, device="cuda")
    table = torch.full((1, 4), nb - 1, dtype=torch.int32, device="cuda")
    table[0, 1] = nb - 2
    x = torch.randn(20, 3 * Hkv * D, device="cuda")
    q = torch.zeros(20, Hkv, D, dtype=torch.bfloat16, device="cuda")
    shape = P.Shape(1, 1, Hkv, Hkv, D, 4, 64, nb)
    P.append_qkv(shape, P.prompt_rows(20, dev_i32([0, 20])), P.append_desc(x, None, None, EPS, 0.0), k, v, table, dev_i32([20]), q)
    torch.cuda.synchronize()
    want = x.view(20, 3, Hkv, D).bfloat16()
    got = torch.cat([k[nb - 1], k[nb - 2]], 2)[:, :, :20].permute(2, 0, 1, 3).reshape(20, Hkv, D)
    assert torch.equal(got, want[:, 1]) and torch.equal(q, want[:, 0])
    got = torch.cat([v[nb - 1], v[nb - 2]], 2)[:, :, :20].permute(2, 0, 1)
    assert torch.equal(got, want[:, 2])
