"""oda_commit_drafts against the oracle, bit for bit: caches, lengths, rings, the
next step's row lengths; table entries and lengths out of range."""
import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_i32, dev_u16, need_gpu
from oracle import drafts as OD

pytestmark = pytest.mark.gpu


def _u16(t):
    return t.cpu().numpy().view(np.uint16)


class Commit:
    def __init__(self, seed, L, B, T, Hkv, D, seq, accepted, stride_pad=0):
        self.P = need_gpu()
        self.L, self.B, self.T, self.Hkv, self.D = L, B, T, Hkv, D
        self.seq = np.asarray(seq, dtype=np.int32)
        room = self.seq + T + 1
        self.mb = int(np.ceil(room.max() / 16))
        self.table, self.nb = S.paged_block_table(S.rng(seed, S.STREAM_TABLE), room, self.mb)
        ks, vs = S.kv_cache_shapes(L, self.nb, Hkv, D)
        self.k, self.v = S.kv_cache(seed, L, self.nb, Hkv, D)
        self.kc = S.normal_bf16(S.rng(seed, S.STREAM_KCUR), (L, B, T, Hkv, D))
        self.vc = S.normal_bf16(S.rng(seed, S.STREAM_VCUR), (L, B, T, Hkv, D))
        self.acc = None if accepted is None else np.asarray(accepted, dtype=np.int32)
        self.pad = stride_pad
        self.stride = self.nb * Hkv * 16 * D + stride_pad if stride_pad else 0

    def _cache(self, a):
        if not self.pad:
            return dev_u16(a)
        flat = np.full((self.L, a[0].size + self.pad), 0x7fc1, dtype=np.uint16)
        flat[:, :a[0].size] = a.reshape(self.L, -1)
        return dev_u16(flat)

    def upload(self):
        self.dk, self.dv = self._cache(self.k), self._cache(self.v)
        self.dseq, self.dtab = dev_i32(self.seq), dev_i32(self.table)
        self.dkc, self.dvc = dev_u16(self.kc), dev_u16(self.vc)
        self.dacc = None if self.acc is None else dev_i32(self.acc)
        self.shape = self.P.Shape(self.L, self.B, self.Hkv, self.Hkv, self.D, self.mb, self.mb * 16, self.nb,
                                  layer_stride_kv=self.stride)
        self.ws = torch.zeros(self.P.commit_workspace_size(self.shape), dtype=torch.uint8, device="cuda")

    def run(self, advance=True, row_lens=None, **ring):
        self.P.commit_drafts(self.shape, self.T, self.dk, self.dv, self.dtab, self.dseq, self.dkc, self.dvc, self.dacc,
                             advance, row_lens, self.ws if advance else None, **ring)
        torch.cuda.synchronize()

    def check(self):
        for got, want in ((self.dk, self.k), (self.dv, self.v)):
            got = _u16(got).reshape(self.L, -1)
            np.testing.assert_array_equal(got[:, :want[0].size], want.reshape(self.L, -1))
            assert (got[:, want[0].size:] == 0x7fc1).all()
        np.testing.assert_array_equal(self.dseq.cpu().numpy(), self.seq)


@pytest.mark.parametrize("L,B,T,Hkv,D,seq,acc", [
    (1, 1, 1, 1, 64, [1], [0]),
    (1, 1, 5, 2, 128, [40], [2]),
    (3, 4, 5, 2, 64, [1, 15, 16, 17], [4, 3, 0, -1]),
    (2, 3, 8, 8, 128, [9, 100, 31], None),
    (28, 2, 4, 8, 128, [77, 500], [3, 1]),
    (2, 5, 64, 1, 64, [1, 2, 16, 30, 47], [63, 40, 17, 99, -7]),      # several blocks; counts are clamped
    (32, 9, 3, 4, 64, [5 * i + 1 for i in range(9)], [i % 3 for i in range(9)]),
])
@pytest.mark.parametrize("advance", [True, False])
def test_matches_oracle(L, B, T, Hkv, D, seq, acc, advance):
    t = Commit(21, L, B, T, Hkv, D, seq, acc, stride_pad=(64 if L == 3 else 0))
    t.upload()
    rows = torch.full((B, T), -3, dtype=torch.int32, device="cuda") if advance else None
    t.run(advance, rows)
    OD.commit_drafts(t.k, t.v, t.table, t.seq, t.kc, t.vc, t.acc, advance)
    t.check()
    if advance:
        np.testing.assert_array_equal(rows.cpu().numpy(), t.seq[:, None] + np.arange(T))
        assert int(t.ws.to(torch.int64).sum()) == 0


def test_bad_blocks_and_lengths_drop_the_token_only():
    t = Commit(22, 2, 5, 6, 2, 64, [14, 14, 30, 5, 60], [5, 5, 5, 5, 5])
    t.table[0, 1] = -1                       # the second block of request 0's tokens
    t.table[1, 0] = t.nb                     # the first block of request 1's
    t.seq[3] = -20                           # positions before the cache
    t.seq[4] = t.mb * 16 - 2                 # the last tokens run out of the table
    t.upload()
    t.run()
    OD.commit_drafts(t.k, t.v, t.table, t.seq, t.kc, t.vc, t.acc)
    t.check()


@pytest.mark.parametrize("n_sink,window,T", [(4, 40, 5), (0, 1, 64), (20, 16, 7), (16, 100, 33)])
def test_rings_stay_current(n_sink, window, T):
    """After every commit of several steps, Local through the rings has the paged
    call's bits (rings filled once, then kept by the commits)."""
    L, B, Hkv, D, Hq = 2, 4, 2, 64, 4
    t = Commit(23, L, B, T, Hkv, D, [1 + 3 * T, 30 + 3 * T, 120, 16], None)
    rng = np.random.default_rng(5)
    t.mb = int(np.ceil((t.seq.max() + 4 * T + 2) / 16))
    t.table, t.nb = S.paged_block_table(S.rng(23, S.STREAM_TABLE), t.seq + 4 * T + 2, t.mb)
    t.k, t.v = S.kv_cache(23, L, t.nb, Hkv, D)
    t.acc = np.zeros(B, dtype=np.int32)
    t.upload()
    P = t.P
    shape = P.Shape(L, B, Hq, Hkv, D, t.mb, t.mb * 16, t.nb)
    n = P.ring_elements(shape, n_sink, window)
    kr, vr = (torch.zeros(n, dtype=torch.int16, device="cuda") for _ in range(2))
    committed = t.dseq - 1                   # the cache holds positions 0 .. n - 2
    P.ring_fill(shape, t.dk, t.dv, t.dtab, committed, n_sink, window, kr, vr)
    q = dev_u16(S.normal_bf16(S.rng(24, 1), (L, B, Hq, D)))
    ws = torch.zeros(max(256, P.attn_workspace_size(shape, n_sink, window)), dtype=torch.uint8, device="cuda")
    for step in range(4):
        t.acc = rng.integers(-1, T, size=B).astype(np.int32)
        if step == 0:
            t.acc[:] = T - 1
        t.dacc.copy_(torch.from_numpy(t.acc))
        t.kc = S.normal_bf16(rng, t.kc.shape)
        t.vc = S.normal_bf16(rng, t.vc.shape)
        t.dkc.copy_(torch.from_numpy(t.kc.view(np.int16)))
        t.dvc.copy_(torch.from_numpy(t.vc.view(np.int16)))
        t.run(True, None, k_ring=kr, v_ring=vr, n_sink=n_sink, window=window)
        OD.commit_drafts(t.k, t.v, t.table, t.seq, t.kc, t.vc, t.acc)
        t.check()
        lens = t.dseq - 1                    # every position committed so far
        a, b = (torch.zeros(L, B, Hq, D, device="cuda") for _ in range(2))
        la, lb = (torch.zeros(L, B, Hq, device="cuda") for _ in range(2))
        P.local_decode_attn(shape, P.inputs(q, t.dk, t.dv, t.dtab, lens, 0.125), n_sink, window, a, la, ws)
        P.local_decode_attn_ring(shape, P.inputs(q, None, None, None, lens, 0.125), kr, vr, n_sink, window, b, lb, ws)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and torch.equal(la, lb), step
