"""oda_prefix_plan / oda_prefix_decode_attn against the fp64 oracle: groups, drafts,
splits, odd sizes, rows that are left alone, bad device data, replays.

Bars are the attention's (tests/harness.py): weights enter the product in two or three
bf16 parts (2^-18 of each is dropped) and sums are fp32, an expected error of
about 1e-6 for these inputs."""
import math

import numpy as np
import pytest
import torch

import oda_synth as S
from harness import LSE_ABS, check_close, dev_i32, dev_u16, need_gpu
from oracle import drafts as OD

pytestmark = pytest.mark.gpu


class Problem:
    """groups: list of (prefix blocks, [own lengths beyond the prefix]); a request's
    seq_lens is 16 * prefix + its own length (its first current token included)."""

    def __init__(self, seed, groups, Hq, Hkv, D, T=1, L=1, cur=True, tokens=None, pad=0, spare=3, empty=(), max_len=None,
                 poison=False):
        self.P = need_gpu()
        g = S.rng(seed, 90)
        B = sum(len(own) for _, own in groups) + spare
        self.B, self.L, self.T, self.Hq, self.Hkv, self.D, self.cur = B, L, T, Hq, Hkv, D, cur
        order = g.permutation(B)
        self.members, self.start, self.prefix = [], [0], []
        self.seq = np.full(B, 20, dtype=np.int32)
        shared, at = {}, 0
        for j, (pre, own) in enumerate(groups):
            for n in own:
                b = int(order[len(self.members)])
                self.seq[b] = 16 * pre + n
                self.members.append(b)
                shared[b] = j
            self.start.append(len(self.members))
            self.prefix.append(pre)
            for _ in range(empty[j] if j < len(empty) else 0):      # groups without members
                self.start.append(len(self.members))
                self.prefix.append(7)
        self.ntok = None if tokens is None else np.resize(np.asarray(tokens, dtype=np.int32), B)
        need = (self.seq + T + 15) // 16
        self.mb = int(need.max())
        self.max_len = max_len or self.mb * 16
        self.mb = max(self.mb, -(-self.max_len // 16))
        total = int(need.sum())
        ids = g.permutation(total + 2)
        self.nb = total + 2
        self.table = np.full((B, self.mb), -1, dtype=np.int32)
        first = {}
        for b in range(B):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += int(need[b])
            j = shared.get(b)
            if j is not None:
                pre = groups[j][0]
                if j in first:
                    self.table[b, :pre] = self.table[first[j], :pre]
                else:
                    first[j] = b
        self.k, self.v = S.kv_cache(seed, L, self.nb, Hkv, D)
        self.q = S.normal_bf16(g, (L, B, T, Hq, D))
        self.kc = S.normal_bf16(g, (L, B, T, Hkv, D)) if cur else None
        self.vc = S.normal_bf16(g, (L, B, T, Hkv, D)) if cur else None
        self.pad = pad
        self.scale = 1.0 / math.sqrt(D)
        self.flags = None
        if poison:
            self.poison()

    def counts(self):
        return np.full(self.B, self.T) if self.ntok is None else np.clip(self.ntok, 0, self.T)

    def poison(self):
        """NaN in every cache slot that no row attends."""
        used = np.zeros((self.nb, 16), dtype=bool)
        for b in range(self.B):
            n = self.seq[b] - 1 if self.cur else self.seq[b] + max(int(self.counts()[b]), 1) - 1
            pos = np.arange(n)
            used[self.table[b, pos // 16], pos % 16] = True
        for blk in range(self.nb):
            for s in np.flatnonzero(~used[blk]):
                self.k[:, blk, :, :, s, :] = 0x7fc0
                self.v[:, blk, :, :, s] = 0x7fc0

    def _cache(self, a):
        if not self.pad:
            return dev_u16(a)
        flat = np.full((self.L, a[0].size + self.pad), 0x7fc0, dtype=np.uint16)
        flat[:, :a[0].size] = a.reshape(self.L, -1)
        return dev_u16(flat)

    def upload(self):
        P = self.P
        stride = self.nb * self.Hkv * 16 * self.D + self.pad if self.pad else 0
        self.shape = P.Shape(self.L, self.B, self.Hq, self.Hkv, self.D, self.mb, self.max_len, self.nb,
                             layer_stride_kv=stride)
        up = lambda a: None if a is None else dev_u16(a)  # noqa: E731
        self.dseq, self.dtab = dev_i32(self.seq), dev_i32(self.table)
        self.dev = [dev_u16(self.q), self._cache(self.k), self._cache(self.v)]
        self.dcur = [up(self.kc), up(self.vc)]
        self.inp = P.inputs(*self.dev, self.dtab, self.dseq, self.scale, *self.dcur)
        members = np.resize(np.array(self.members + [0] * (self.B - len(self.members)), dtype=np.int32), self.B)
        self.dstart, self.dmembers, self.dprefix = dev_i32(self.start), dev_i32(members), dev_i32(self.prefix)
        self.dtok = None if self.ntok is None else dev_i32(self.ntok)
        self.dflags = None if self.flags is None else dev_i32(self.flags)
        self.groups = P.prefix_groups(len(self.prefix), self.T, self.dstart, self.dmembers, self.dprefix, self.dtok,
                                      self.dflags)
        self.plan = torch.full((P.prefix_plan_size(self.shape, self.groups),), 0x55, dtype=torch.uint8, device="cuda")
        self.ws = torch.full((P.prefix_workspace_size(self.shape, self.groups),), 0xff, dtype=torch.uint8, device="cuda")
        self.out = torch.full((self.L, self.B, self.T, self.Hq, self.D), -7.0, device="cuda")
        self.lse = torch.full((self.L, self.B, self.T, self.Hq), -7.0, device="cuda")

    def call(self):
        self.P.prefix_plan(self.shape, self.inp, self.groups, self.plan)
        self.P.prefix_decode_attn(self.shape, self.inp, self.groups, self.plan, self.out, self.lse, self.ws)

    def run(self):
        self.out.fill_(-7.0)
        self.lse.fill_(-7.0)
        self.call()
        torch.cuda.synchronize()
        return self.out.cpu().numpy(), self.lse.cpu().numpy()

    def attended(self):
        return [b for b in self.members if self.flags is None or self.flags[b]]

    def check(self, got=None, nan=()):
        out, lse = self.run() if got is None else got
        rows = np.zeros((self.B, self.T), dtype=bool)
        for b in self.attended():
            rows[b, :self.counts()[b]] = True
        for b in nan:
            assert np.isnan(out[:, b][:, rows[b]]).all() and np.isnan(lse[:, b][:, rows[b]]).all(), b
        ok = [b for b in self.attended() if b not in nan]
        ref, ref_lse = OD.prefix_attention(self.q, self.k, self.v, self.table, self.seq, self.scale, self.counts(), self.kc,
                                           self.vc, ok)
        for b in ok:
            if rows[b].any():
                check_close(out[:, b][:, rows[b]], ref[:, b][:, rows[b]], f"request {b}")
                assert np.abs(lse[:, b][:, rows[b]] - ref_lse[:, b][:, rows[b]]).max() <= LSE_ABS
        assert (out[:, ~rows] == -7.0).all() and (lse[:, ~rows] == -7.0).all()      # everything else as it was


CASES = {
    "one request, one position": dict(groups=[(0, [1])], Hq=2, Hkv=1, D=64),
    "one request without a prefix": dict(groups=[(0, [300])], Hq=8, Hkv=2, D=128),
    "own part empty": dict(groups=[(3, [1, 1])], Hq=4, Hkv=2, D=64),
    "two chats": dict(groups=[(64, [17, 40])], Hq=16, Hkv=8, D=128),
    "odd blocks": dict(groups=[(7, [5, 16, 17, 33]), (1, [15, 1, 100])], Hq=12, Hkv=4, D=128, pad=64, L=2),
    "no shared heads": dict(groups=[(9, [20, 30, 2])], Hq=2, Hkv=2, D=64),
    "groups of 5 heads": dict(groups=[(40, list(range(1, 60))), (2, [4])], Hq=10, Hkv=2, D=64),
    "groups of 16 heads": dict(groups=[(33, [10, 200, 3, 50, 70, 90])], Hq=32, Hkv=2, D=128),
    "many columns": dict(groups=[(20, [1 + 3 * i for i in range(70)])], Hq=8, Hkv=1, D=128),
    "singletons": dict(groups=[(0, [1 + 31 * i]) for i in range(20)], Hq=4, Hkv=1, D=64),
    "empty groups": dict(groups=[(5, [3, 9]), (0, []), (2, [30]), (6, [])], Hq=4, Hkv=2, D=64, empty=(2, 0, 1, 3)),
    "long prefix": dict(groups=[(1500, [9, 77])], Hq=4, Hkv=1, D=64),
    "long own parts": dict(groups=[(4, [9000, 3, 5000])], Hq=4, Hkv=1, D=128),
    "three layers": dict(groups=[(90, [40, 41, 42]), (30, [500])], Hq=8, Hkv=4, D=64, L=3),
}


@pytest.mark.parametrize("cur", [True, False])
@pytest.mark.parametrize("name", CASES)
def test_matches_oracle(name, cur):
    p = Problem(41, cur=cur, poison=True, **CASES[name])
    p.upload()
    p.check()


@pytest.mark.parametrize("cur", [True, False])
@pytest.mark.parametrize("T,Hq,Hkv,D,tokens", [
    (2, 8, 4, 64, None), (5, 8, 4, 128, [1, 2, 3, 4, 5]), (5, 4, 4, 64, [5, 0, 9, -3, 1]), (16, 16, 1, 64, None),
    (16, 5, 1, 128, [16, 7, 1]), (3, 14, 2, 64, [3, 2])])
def test_several_current_tokens(T, Hq, Hkv, D, tokens, cur):
    p = Problem(42, [(6, [1, 20, 15, 2]), (0, [1, 16, 17]), (21, [40])], Hq, Hkv, D, T=T, L=2, cur=cur, tokens=tokens,
                poison=True)
    p.upload()
    p.check()


@pytest.mark.parametrize("cur", [True, False])
def test_flagged_members_only(cur):
    for flags in ([1, 0, 0, 1, 5, 0, -1, 0, 0, 1], [0] * 10):
        p = Problem(43, [(12, [10, 20, 30, 40]), (3, [5, 6, 7])], 8, 2, 64, T=2, cur=cur)
        p.flags = np.array(flags, dtype=np.int32)
        p.upload()
        p.check()


def test_reruns_and_order_of_members_do_not_matter():
    """The same bits again; a request's rows do not depend on its place."""
    p = Problem(44, [(30, [10, 200, 31])], 8, 2, 128, T=3)
    p.upload()
    a = p.run()
    b = p.run()
    for x, y in zip(a, b):
        np.testing.assert_array_equal(x, y)
    p.members = p.members[::-1]
    p.upload()
    p.check()


def test_equals_full_attention():
    """T = 1 and no shared blocks: Full's rows."""
    p = Problem(45, [(0, [700]), (0, [33]), (0, [2000])], 8, 2, 128, spare=0)
    p.upload()
    out, lse = p.run()
    full = torch.zeros(1, p.B, 8, 128, device="cuda")
    flse = torch.zeros(1, p.B, 8, device="cuda")
    ws = torch.zeros(max(256, p.P.attn_workspace_size(p.shape, 0, 0)), dtype=torch.uint8, device="cuda")
    p.P.full_decode_attn(p.shape, p.inp, 0, None, None, None, full, flse, ws)
    torch.cuda.synchronize()
    check_close(out[:, :, 0], full.cpu().numpy())
    assert np.abs(lse[:, :, 0] - flse.cpu().numpy()).max() <= LSE_ABS


def test_masked_keys_and_large_scores():
    """Keys that score -infinity or far apart; a whole part without weight."""
    p = Problem(46, [(8, [20, 40])], 2, 1, 64, cur=True)
    inf = 0x7f80
    p.q[:, :, :, :, 0] = 0x3f80                     # q_0 = 1
    blk = p.table[p.members[0]]
    p.k[:, blk[2], :, 0, 3:9, 0] = 0x8000 | inf     # a few positions of the prefix at -infinity
    p.k[:, blk[5], :, 0, :, 0] = 0x8000 | inf       # a block of it
    own = p.table[p.members[1], 8]
    p.k[:, own, :, 0, :, 0] = 0x8000 | inf          # a block of the second request's own part
    p.k[:, blk[0], :, 1, :, 0] = 0x43c8             # one position block near +-400 per unit of q
    p.upload()
    p.check()
    for t in range(8):
        p.k[:, blk[t], :, 0, :, 0] = 0x8000 | inf   # nothing of the prefix left
    p.upload()
    p.check()


def test_lengths_and_entries_out_of_range_give_nan_rows():
    def fresh(cur=True, T=3):
        p = Problem(47, [(4, [10, 20, 30]), (2, [3, 40]), (0, [50])], 4, 2, 64, T=T, cur=cur)
        return p, p.members

    p, m = fresh()
    p.seq[m[0]], p.seq[m[1]], p.seq[m[3]], p.seq[m[5]] = 0, 4 * 16, p.max_len + 1, -2 ** 31   # 64: 63 committed, 64 shared
    p.upload()
    p.check(nan=[m[0], m[1], m[3], m[5]])
    p, m = fresh(cur=False)
    p.seq[m[2]] = p.max_len - 1                     # its third token is past the limit
    p.upload()
    p.check(nan=[m[2]])
    p, m = fresh()
    p.table[m[1], 5] = p.nb                         # an own block
    p.upload()
    p.check(nan=[m[1]])
    p, m = fresh()
    p.table[m[0], 2] = -1                           # a block of the prefix, in the table that is read
    p.upload()
    p.check(nan=m[:3])
    p, m = fresh()
    p.prefix[1] = -1
    p.upload()
    p.check(nan=m[3:5])
    p, m = fresh()
    p.prefix[1] = 10 ** 6
    p.upload()
    p.check(nan=m[3:5])
    p, m = fresh(cur=False)
    p.table[m[5], 3] = -5                           # the block that holds current tokens 50, 51 (48..63)
    p.upload()
    p.check(nan=[m[5]])


def test_members_and_starts_out_of_range_are_skipped():
    p = Problem(48, [(4, [10, 20, 30]), (2, [3, 40])], 4, 2, 64)
    drop = p.members[1]
    p.members[1] = p.B
    p.upload()
    out, lse = p.run()
    p.members.remove(p.B)
    p.check((out, lse))
    assert (out[:, drop] == -7.0).all()
    p = Problem(48, [(4, [10, 20, 30]), (2, [3, 40])], 4, 2, 64, spare=0)
    p.start = [0, 3, 10 ** 9]                       # past the members: cut off at the batch
    p.upload()
    p.check()
    p.start = [-4, 3, 5]
    p.upload()
    p.check()


def test_a_plan_of_other_sizes_gives_nan():
    p = Problem(49, [(4, [10, 20, 30])], 4, 2, 64, spare=1)
    p.upload()
    p.P.prefix_decode_attn(p.shape, p.inp, p.groups, p.plan, p.out, p.lse, p.ws)      # never planned
    torch.cuda.synchronize()
    assert torch.isnan(p.out).all() and torch.isnan(p.lse).all()
    other = Problem(49, [(4, [10, 20])], 4, 2, 64, spare=1)
    other.upload()
    other.P.prefix_plan(other.shape, other.inp, other.groups, p.plan)
    p.out.fill_(-7.0)
    p.P.prefix_decode_attn(p.shape, p.inp, p.groups, p.plan, p.out, p.lse, p.ws)
    torch.cuda.synchronize()
    assert torch.isnan(p.out).all() and torch.isnan(p.lse).all()


def test_lse_may_be_left_out_and_one_plan_serves_many_calls():
    p = Problem(50, [(4, [10, 20, 30])], 4, 2, 64, L=2)
    p.upload()
    out, _ = p.run()
    again = torch.full_like(p.out, -7.0)
    p.P.prefix_decode_attn(p.shape, p.inp, p.groups, p.plan, again, None, p.ws)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(again.cpu().numpy(), out)


def test_two_streams_share_a_plan():
    p = Problem(51, [(200, [10, 200, 300, 44])], 8, 2, 128)
    p.upload()
    want, _ = p.run()
    sides = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.full_like(p.out, -7.0) for _ in sides]
    wss = [torch.full_like(p.ws, 0xff) for _ in sides]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, o, w in zip(sides, outs, wss):
            p.P.prefix_decode_attn(p.shape, p.inp, p.groups, p.plan, o, None, w, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        np.testing.assert_array_equal(o.cpu().numpy(), want)


def test_captured_step_replays_with_growing_lengths():
    p = Problem(52, [(9, [10, 31, 16]), (0, [40])], 4, 2, 64, T=2, cur=False, max_len=400)
    p.seq[:] = np.minimum(p.seq, 300)
    p.upload()
    p.run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.call()
    for step in range(4):
        p.out.fill_(-7.0)
        p.lse.fill_(-7.0)
        g.replay()
        torch.cuda.synchronize()
        p.check((p.out.cpu().numpy(), p.lse.cpu().numpy()))
        grow = p.seq.copy()
        for i, b in enumerate(p.members):           # rows may grow up to the blocks they have
            room = int((p.table[b] >= 0).sum()) * 16 - 1
            grow[b] = min(p.seq[b] + i, room)
        p.seq = grow
        p.dseq.copy_(torch.from_numpy(p.seq))
        _ = (p.out * 2).sum().item()


def test_random_problems():
    g = np.random.default_rng(53)
    for case in range(25):
        Hkv, G, D = int(g.integers(1, 4)), int(g.integers(1, 17)), int(g.choice([64, 128]))
        T = int(g.choice([1, 1, 2, 4, 7]))
        groups = [(int(g.integers(0, 70)) if g.random() < 0.8 else 0,
                   [int(g.integers(1, 200)) for _ in range(int(g.integers(0, 9)))]) for _ in range(int(g.integers(1, 5)))]
        cur, L = bool(g.random() < 0.5), int(g.integers(1, 3))
        tokens = g.integers(0, T + 1, size=7) if g.random() < 0.5 else None
        print(f"case {case}: groups {groups} G {G} Hkv {Hkv} D {D} T {T} cur {cur} L {L}", flush=True)
        p = Problem(100 + case, groups, Hkv * G, Hkv, D, T=T, L=L, cur=cur, tokens=tokens, poison=True)
        p.upload()
        p.check()


@pytest.mark.parametrize("D,blocks,parts", [(64, 3071, 3), (64, 3074, 2), (128, 3074, 2), (128, 900, 3)])
def test_weights_of_many_columns_on_either_side_of_the_length(D, blocks, parts):
    """160 and more columns: weights of three parts below 49,152 positions, of two from there on.  Expected error: the
    fp32 sums of a few splits (3e-7) plus, for two parts, 2^-18 of each weight at most half the time (2.4e-6 rms)."""
    p = Problem(47, [(blocks, [1, 40, 3, 77, 100, 9, 16, 2, 31, 5])], 16, 1, D, poison=True, spare=1)
    assert (16 * blocks >= 49152) == (parts == 2)
    p.upload()
    got = p.run()
    p.check(got)
    ref, _ = OD.prefix_attention(p.q, p.k, p.v, p.table, p.seq, p.scale, p.counts(), p.kc, p.vc, p.attended())
    rows = p.attended()
    err = np.linalg.norm(got[0][:, rows] - ref[:, rows]) / np.linalg.norm(ref[:, rows])
    assert err <= (1e-6 if parts == 3 else 4e-6), err
