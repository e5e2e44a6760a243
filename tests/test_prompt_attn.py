"""oda_prompt_plan and oda_prompt_attn against the fp64 oracle.

Tolerances: an fp32 output takes the decode attention's bars.  A bf16 output is the
exact value off by half a step (2^-8 of it), its weights each rounded by as much: 2^-8
of the mean absolute value behind it, and the fp32 bar."""
import math

import numpy as np
import pytest
import torch

import oda_synth as S
from harness import LSE_ABS, MAX_ABS_INTERNAL, dev_i32, dev_u16, need_gpu
from oracle import prompt as OP
from oracle.attention import bf16_to_f64

pytestmark = pytest.mark.gpu


class Prompt:
    def __init__(self, seed, Hq, Hkv, D, rows, seq, causal=True, window=0, lead=0, tail=0, extra=3, scale=None):
        self.P = need_gpu()
        g = S.rng(seed, 93)
        self.g, self.B, self.Hq, self.Hkv, self.D = g, len(rows), Hq, Hkv, D
        self.causal, self.window = causal, window
        self.start = np.concatenate([[lead], lead + np.cumsum(rows)]).astype(np.int32)
        self.R = max(1, int(self.start[-1]) + tail)
        self.seq = np.array(seq, dtype=np.int32)
        self.mb = max(1, -(-int(self.seq.max()) // 16))
        self.max_len = self.mb * 16
        self.table, self.nb = S.paged_block_table(S.rng(seed, S.STREAM_TABLE), np.maximum(self.seq, 1), self.mb, extra_blocks=extra)
        self.k, self.v = S.kv_cache(seed, 1, self.nb, Hkv, D)
        self.q = S.normal_bf16(g, (self.R, Hq, D))
        self.scale = scale or 1.0 / math.sqrt(D)

    def upload(self):
        P = self.P
        self.dq, self.dk, self.dv = dev_u16(self.q), dev_u16(self.k), dev_u16(self.v)
        self.dtab, self.dseq, self.dstart = dev_i32(self.table), dev_i32(self.seq), dev_i32(self.start)
        self.shape = P.Shape(1, self.B, self.Hq, self.Hkv, self.D, self.mb, self.max_len, self.nb)
        self.rows = P.prompt_rows(self.R, self.dstart)
        self.inp = P.inputs(self.dq, self.dk, self.dv, self.dtab, None, self.scale)
        # (neither buffer needs clearing: filled with bytes that would show)
        self.plan = torch.full((P.prompt_plan_size(self.shape, self.rows),), 0xA5, dtype=torch.uint8, device="cuda")
        self.ws = torch.full((P.prompt_workspace_size(self.shape, self.rows),), 0xFF, dtype=torch.uint8, device="cuda")

    def outputs(self, bf16):
        out = torch.full((self.R, self.Hq, self.D), -9.0, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
        return out, torch.full((self.R, self.Hq), -9.0, device="cuda")

    def make_plan(self):
        self.P.prompt_plan(self.shape, self.rows, self.dseq, self.causal, self.window, self.plan)

    def run(self, bf16=False):
        self.upload()
        self.make_plan()
        return self.attend(bf16)

    def attend(self, bf16=False):
        out, lse = self.outputs(bf16)
        self.P.prompt_attn(self.shape, self.inp, self.rows, self.plan, out, lse, self.ws)
        torch.cuda.synchronize()
        return out.double().cpu().numpy(), lse.double().cpu().numpy()

    def oracle(self):
        return OP.prompt_attention(self.q, self.k, self.v, self.table, self.start, self.seq, self.scale, self.causal, self.window)

    def check(self, types=(False, True)):
        ref, rlse, mag = self.oracle()
        for bf16 in types:
            out, lse = self.run(bf16)
            self.compare(out, lse, ref, rlse, mag, bf16)
            again, lse2 = self.attend(bf16)                  # the plan serves call after call, bit for bit
            assert np.array_equal(out, again) and np.array_equal(lse, lse2)
        return ref

    def compare(self, out, lse, ref, rlse, mag, bf16, rows=None):
        own = ~np.isnan(rlse[:, 0]) if rows is None else rows
        bar = np.full(ref[own].shape, MAX_ABS_INTERNAL)
        if bf16:
            bar = bar + 2.0 ** -8 * (np.abs(ref[own]) + mag[own] * (1 + 2.0 ** -8))
        err = np.abs(out[own] - ref[own])
        assert (err <= bar).all(), (err.max(), np.unravel_index(np.argmax(err - bar), err.shape))
        none = np.isneginf(rlse[own])
        assert np.isneginf(lse[own][none]).all()
        assert (np.abs(lse[own][~none] - rlse[own][~none]) <= LSE_ABS).all()
        if rows is None:
            assert (out[~own] == -9).all() and (lse[~own] == -9).all()


@pytest.mark.parametrize("Hq,Hkv,D", [(1, 1, 64), (4, 2, 128), (5, 1, 128), (16, 2, 64), (6, 3, 64), (16, 1, 128), (8, 8, 128)])
@pytest.mark.parametrize("rows,seq", [
    ([1], [1]), ([1], [16]), ([1], [17]), ([2], [2]), ([33], [33]), ([64], [64]), ([65], [200]),
    ([1, 0, 40, 7], [1, 5, 41, 300]), ([129, 300], [129, 301])])
def test_causal(Hq, Hkv, D, rows, seq):
    Prompt(41, Hq, Hkv, D, rows, seq, lead=1, tail=2).check()


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 40, 100, 1000])
@pytest.mark.parametrize("rows,seq", [([70, 1, 200], [90, 333, 200])])
def test_window(window, rows, seq):
    Prompt(42, 4, 2, 64, rows, seq, window=window).check()


@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 64), (4, 2, 128), (16, 1, 64)])
@pytest.mark.parametrize("rows,seq", [([1], [1]), ([1, 1, 1], [0, 16, 375]), ([50, 3, 0, 17], [0, 33, 100, 15]), ([300], [31])])
def test_without_a_mask(Hq, Hkv, D, rows, seq):
    Prompt(43, Hq, Hkv, D, rows, seq, causal=False, tail=1).check()


@pytest.mark.parametrize("Hq,Hkv,rows,seq", [
    (4, 1, [8], [3001]), (4, 1, [9], [3001]), (8, 1, [16], [3333]), (8, 1, [30], [5000]), (16, 1, [48], [4100]),
    (2, 2, [1, 1, 500], [9000, 1, 700])])
def test_long_histories_are_split(Hq, Hkv, rows, seq):
    """Column counts of every wavefront grid (1, 2, 4, 8 column tiles), several ranges each."""
    Prompt(44, Hq, Hkv, 128, rows, seq).check()


def test_many_requests_of_every_size():
    rng = np.random.default_rng(3)
    rows = [int(r) for r in rng.choice([0, 1, 2, 9, 31, 64, 150], size=60)]
    seq = [r + int(h) for r, h in zip(rows, rng.integers(0, 700, size=60))]
    Prompt(45, 4, 2, 64, rows, seq).check()


def test_more_tiles_than_the_plan_has_threads():
    """1,200 requests of a row or two."""
    rows = [1 + b % 2 for b in range(1200)]
    seq = [rows[b] + b % 50 for b in range(1200)]
    Prompt(46, 2, 1, 64, rows, seq).check(types=(True,))


def test_unattended_slots_may_hold_anything():
    """NaN and infinities behind every history, in unused blocks, and between a window's requests."""
    for causal, window in ((True, 0), (True, 20), (False, 0)):
        t = Prompt(47, 4, 2, 128, [20, 1, 45], [21, 99, 150], causal=causal, window=window)
        used = np.zeros((t.nb, 16), dtype=bool)
        for b in range(t.B):
            first = t.seq[b] - (t.start[b + 1] - t.start[b])
            lo = max(0, first - window + 1) if window else 0
            for p in range(lo, t.seq[b]):
                used[t.table[b, p // 16], p % 16] = True
        for bits in (0x7FC0, 0x7F80, 0xFF80):
            for blk, slot in zip(*np.where(~used)):
                t.k[0, blk, :, :, slot] = bits
                t.v[0, blk, :, :, slot] = bits
            t.check()


def test_values_that_are_not_finite_reach_their_rows_alone():
    t = Prompt(48, 4, 2, 128, [90, 200], [120, 200])
    for b, p, d, bits in ((0, 60, 5, 0x7FC0), (0, 100, 7, 0x7F80), (1, 33, 64, 0xFF80), (1, 150, 127, 0x7F80), (1, 199, 0, 0x7FC0)):
        t.v[0, t.table[b, p // 16], 1, d, p % 16] = bits
    with np.errstate(invalid="ignore"):
        ref, rlse, mag = t.oracle()
    # rows before the value do not see it (the oracle multiplies it by 0 there)
    clean = t.v.copy()
    clean[(clean & 0x7F80) == 0x7F80] = 0
    v, t.v = t.v, clean
    base, _, mag = t.oracle()
    t.v = v
    want = base.copy()
    for b, p, d, add in ((0, 60, 5, np.nan), (0, 100, 7, np.inf), (1, 33, 64, -np.inf), (1, 150, 127, np.inf), (1, 199, 0, np.nan)):
        first = t.start[b] + max(0, p - (t.seq[b] - (t.start[b + 1] - t.start[b])))
        want[first:t.start[b + 1], 2:, d] = add
    for bf16 in (False, True):
        out, lse = t.run(bf16)
        odd = ~np.isfinite(want)
        # (an infinity times the parts of a weight, some of them 0 or negative, may be NaN)
        assert np.array_equal(np.isfinite(out), ~odd) and np.isnan(out[np.isnan(want)]).all()
        out[odd], want2 = 0.0, np.where(odd, 0.0, want)
        t.compare(out, lse, want2, rlse, np.where(odd, 0.0, mag), bf16)


def test_bad_lengths_blocks_and_their_rows():
    t = Prompt(49, 4, 2, 64, [40, 7, 30, 3, 50], [60, 100, 30, 64, 80])
    ref, rlse, mag = t.oracle()
    seq = t.seq.copy()
    t.seq[1] = t.max_len + 1
    t.seq[2] = 29                               # shorter than its rows
    t.seq[3] = -1
    t.table[0, 2] = t.nb                        # places 32..47: rows 12 on attend them
    t.table[4, 4] = -5                          # places 64..79: rows 34 on
    for bf16 in (False, True):
        out, lse = t.run(bf16)
        nan = np.zeros(t.R, dtype=bool)
        for b in (1, 2, 3):
            nan[t.start[b]:t.start[b + 1]] = True
        nan[t.start[0] + 12:t.start[1]] = True
        nan[t.start[4] + 34:t.start[5]] = True
        assert np.isnan(out[nan]).all() and np.isnan(lse[nan]).all()
        t.compare(out, lse, ref, rlse, mag, bf16, rows=~nan)
    assert seq.size == t.B


def test_a_bad_block_outside_the_window_is_not_used():
    t = Prompt(50, 2, 1, 64, [20], [200], window=30)
    ref, rlse, mag = t.oracle()
    t.table[0, :9] = -1                         # places up to 143; the first row attends 151 on
    out, lse = t.run()
    t.compare(out, lse, ref, rlse, mag, False)


def test_a_plan_of_other_sizes_gives_nan():
    t = Prompt(51, 4, 2, 64, [20, 9], [20, 40])
    t.run()
    u = Prompt(51, 4, 2, 64, [20, 9], [20, 40], tail=5)
    u.upload()
    u.plan[:t.plan.numel()] = t.plan[:min(t.plan.numel(), u.plan.numel())]
    out, lse = u.attend()
    assert np.isnan(out).all() and np.isnan(lse).all()
    u.plan.zero_()
    out, lse = u.attend(True)
    assert np.isnan(out).all() and np.isnan(lse).all()


def test_row_starts_out_of_order_stay_inside():
    t = Prompt(52, 2, 2, 64, [8, 8, 8, 8], [64, 64, 64, 64], tail=4)
    t.start[:] = [-3, 10, 4, 5000, 17]          # as ascending: 0..10, 10..10, 10..36, none
    out, lse = t.run()
    t.start[:] = [0, 10, 10, 36, 36]
    ref, rlse, mag = t.oracle()
    t.compare(out, lse, ref, rlse, mag, False)


def test_large_scores_and_values():
    """Scores of thousands, values near the largest: weights stay at most 1."""
    t = Prompt(53, 4, 2, 128, [70], [400], scale=40.0)
    t.v[:] = (bf16_to_f64(t.v) * 2.0 ** 118).astype(np.float32).view(np.uint32) >> 16
    ref, rlse, mag = t.oracle()
    for bf16 in (False, True):
        out, lse = t.run(bf16)
        # scores of up to 40 * 60 * sqrt(128) are off by their own fp32 steps (2^-24 of about 3e4, 2e-3)
        bar = 2.0 ** 118 * 4 * 8e-3 + (2.0 ** -8 * (np.abs(ref) + mag) if bf16 else 0)
        assert np.isfinite(out).all() and (np.abs(out - ref) <= bar).all()
        assert (np.abs(lse - rlse) <= 4e-3 + 2.0 ** -22 * np.abs(rlse)).all()


@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 40, 2.0 ** 90])
@pytest.mark.parametrize("rows,seq", [([3], [200]), ([300], [900])])
def test_scores_of_any_size(size, rows, seq):
    """Scores so large that the largest one takes all, whatever its product with the scale rounds to."""
    t = Prompt(60, 2, 1, 64, rows, seq)
    q, k = bf16_to_f64(t.q), bf16_to_f64(t.k)
    q[:] = 0.0
    q[..., 0] = 1.5
    k[:] = 0.0
    g = S.rng(61, 1)
    for p in range(seq[0]):                 # multiples of an eighth of `size`, one in twenty at the top
        k[0, t.table[0, p // 16], 0, 0, p % 16, 0] = size * (1.0 if g.random() < 0.05 else g.integers(0, 8) / 8)
    k[0, t.table[0, 0], 0, 0, 0, 0] = size
    t.q = (q.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    t.k = (k.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    ref, rlse, mag = t.oracle()
    for bf16 in (False, True):
        out, lse = t.run(bf16)
        t.compare(out, rlse, ref, rlse, mag, bf16)
        assert (np.abs(lse - rlse) <= LSE_ABS + 2.0 ** -22 * np.abs(rlse)).all()


def test_scores_that_grow_and_fall_along_the_history():
    """Every step raises the reference, then none does."""
    for order in (1, -1):
        t = Prompt(54, 2, 1, 64, [200], [600])
        k = bf16_to_f64(t.k)
        for p in range(600):
            w = 6.0 * (p if order > 0 else 600 - p) / 600
            blk = t.table[0, p // 16]
            k[0, blk, 0, :, p % 16] *= 0.05
            k[0, blk, 0, 0, p % 16, 0] = w
        t.k = (k.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
        q = bf16_to_f64(t.q)
        q[..., 0] = 8.0
        t.q = (q.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
        t.check()


def test_same_rows_as_decode_attention():
    """A single row per request is oda_full_decode_attn's; a chunk's last row too."""
    t = Prompt(55, 8, 2, 128, [1, 30, 1], [333, 200, 16])
    out, lse = t.run()
    last = t.start[1:] - 1
    P = t.P
    q = t.dq[torch.from_numpy(last.astype(np.int64)).cuda()].contiguous()
    o, l = torch.zeros(1, 3, 8, 128, device="cuda"), torch.zeros(1, 3, 8, device="cuda")
    ws = torch.zeros(max(256, P.attn_workspace_size(t.shape, 0, 0)), dtype=torch.uint8, device="cuda")
    P.full_decode_attn(t.shape, P.inputs(q, t.dk, t.dv, t.dtab, t.dseq, t.scale), 0, None, None, None, o, l, ws)
    torch.cuda.synchronize()
    assert np.abs(out[last] - o[0].double().cpu().numpy()).max() < 1e-5
    assert np.abs(lse[last] - l[0].double().cpu().numpy()).max() < 1e-5


def test_captured_and_replayed_with_other_lengths():
    """Plan and attention in a graph: replays follow rows and lengths that the host changes between them."""
    t = Prompt(56, 4, 2, 64, [40, 3, 20], [100, 50, 20], tail=17)
    t.upload()
    out, lse = t.outputs(False)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            t.make_plan()
            t.P.prompt_attn(t.shape, t.inp, t.rows, t.plan, out, lse, t.ws)
    for start, seq in (([0, 40, 43, 63], [100, 50, 20]), ([0, 1, 1, 2], [90, 4, 20]), ([5, 30, 80, 80], [64, 60, 3]),
                       ([0, 40, 43, 63], [100, 50, 20])):
        t.start[:], t.seq[:] = start, seq
        t.dstart.copy_(torch.from_numpy(t.start))
        t.dseq.copy_(torch.from_numpy(t.seq))
        out.fill_(-9.0)
        lse.fill_(-9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ref, rlse, mag = t.oracle()
        t.compare(out.double().cpu().numpy(), lse.double().cpu().numpy(), ref, rlse, mag, False)


def test_two_streams_share_a_plan():
    t = Prompt(57, 4, 1, 64, [300, 5], [900, 2000])
    t.upload()
    t.make_plan()
    torch.cuda.synchronize()
    a, b = t.outputs(False), t.outputs(False)
    ws2 = torch.zeros_like(t.ws)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for (out, lse), ws, st in zip((a, b), (t.ws, ws2), streams):
        t.P.prompt_attn(t.shape, t.inp, t.rows, t.plan, out, lse, ws, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ref, rlse, mag = t.oracle()
    t.compare(a[0].double().cpu().numpy(), a[1].double().cpu().numpy(), ref, rlse, mag, False)


def test_caches_beyond_32_bit_offsets():
    P = need_gpu()
    nb, Hkv, D = 140_000, 8, 128
    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GB of device memory")
    k = torch.zeros(nb, Hkv, D // 8, 16, 8, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(nb, Hkv, D, 16, dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([[nb - 1, 3, nb - 2]], dtype=torch.int32, device="cuda")
    for blk in table[0].tolist():
        k[blk].normal_()
        v[blk].normal_()
    q = torch.randn(5, Hkv, D, device="cuda").bfloat16()
    shape = P.Shape(1, 1, Hkv, Hkv, D, 3, 48, nb)
    rows = P.prompt_rows(5, dev_i32([0, 5]))
    plan = torch.zeros(P.prompt_plan_size(shape, rows), dtype=torch.uint8, device="cuda")
    ws = torch.zeros(P.prompt_workspace_size(shape, rows), dtype=torch.uint8, device="cuda")
    out = torch.zeros(5, Hkv, D, device="cuda")
    P.prompt_plan(shape, rows, dev_i32([40]), True, 0, plan)
    P.prompt_attn(shape, P.inputs(q, k, v, table, None, D ** -0.5), rows, plan, out, None, ws)
    torch.cuda.synchronize()
    kk = k[table[0].long()].double().permute(1, 0, 3, 2, 4).reshape(Hkv, 48, D)[:, :40].cpu()
    vv = v[table[0].long()].double().permute(1, 0, 3, 2).reshape(Hkv, 48, D)[:, :40].cpu()
    z = torch.matmul(q.double().cpu().transpose(0, 1), kk.transpose(1, 2)) * D ** -0.5
    z = z.masked_fill(torch.arange(40) > torch.arange(35, 40)[:, None], -math.inf)
    ref = torch.matmul(torch.softmax(z, -1), vv).transpose(0, 1)
    assert (out.double().cpu() - ref).abs().max() < MAX_ABS_INTERNAL
