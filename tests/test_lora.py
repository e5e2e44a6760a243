"""oda_dense_lora_bf16 against the fp64 oracle: modes, fused parts, ranks, odd
sizes, requests without an adapter, lists, ids out of range.

Tolerance: bf16 products in fp32 are off by at most 2^-24 each, and a sum of K
terms is formed as K / 64 terms per lane or fewer, six lane steps and eight
wavefront steps, so its error is at most (K / 64 + 16 + rank) 2^-24 times the sum
of the absolute terms (the adapter's first factor's error passes through the
second with the same factor).  The factor below doubles the count for the
normalisation's factor and the products with gains and scales."""
import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_f32, dev_i32, dev_u16, need_gpu
from oracle import drafts as OD
from oracle.attention import bf16_to_f64

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, seed, K, parts, rank, adapters, B, swiglu=False, norm=False, residual=False):
        self.P = need_gpu()
        g = S.rng(seed, 77)
        n = sum(parts)
        self.K, self.parts, self.rank, self.A, self.B, self.swiglu = K, list(parts), rank, adapters, B, swiglu
        self.w = S.normal_bf16(g, (n, K), K ** -0.5)
        self.a = S.normal_bf16(g, (adapters, len(parts) * rank, K), K ** -0.5)
        self.b = S.normal_bf16(g, (adapters, n, rank), rank ** -0.5)
        self.scale = (0.5 + g.random(adapters)).astype(np.float32)
        self.x = g.standard_normal((B, K)).astype(np.float32)
        self.gain = (1 + 0.05 * g.standard_normal(K)).astype(np.float32) if norm else None
        self.out = n // 2 if swiglu else n
        self.res = g.standard_normal((B, self.out)).astype(np.float32) if residual else None
        self.ids = g.integers(-1, adapters, size=B).astype(np.int32)

    def upload(self):
        P = self.P
        self.dgain = None if self.gain is None else dev_f32(self.gain)
        self.desc = P.dense_desc(self.K, self.out, P.DENSE_SWIGLU if self.swiglu else P.DENSE_PLAIN, dev_u16(self.w),
                                 self.dgain, 1e-6)
        self.lora = P.lora_desc(self.A, self.rank, self.parts, dev_u16(self.a), dev_u16(self.b), dev_f32(self.scale))
        self.dx, self.dids = dev_f32(self.x), dev_i32(self.ids)
        self.dres = None if self.res is None else dev_f32(self.res)
        self.ws = torch.full((P.lora_workspace_size(self.lora, self.B),), 0x7f, dtype=torch.uint8, device="cuda")

    def run(self, y=None, work=None):
        y = torch.full((self.B, self.out), -7.0, device="cuda") if y is None else y
        wl = (None, None) if work is None else (dev_i32(work + [0] * (self.B - len(work))), dev_i32([len(work)]))
        self.P.dense_lora_bf16(self.desc, self.lora, self.B, self.dx, self.dres, y, self.dids, self.ws, *wl)
        torch.cuda.synchronize()
        return y.cpu().numpy()

    def check(self, got, rows=None):
        f64 = lambda v: None if v is None else v.astype(np.float64)  # noqa: E731
        ref, mag = OD.dense_lora(f64(self.x), bf16_to_f64(self.w), bf16_to_f64(self.a), bf16_to_f64(self.b),
                                 f64(self.scale), self.ids, self.parts, f64(self.gain), 1e-6, self.swiglu, f64(self.res))
        eps = 2 * (self.K / 64 + 16 + self.rank) * 2.0 ** -24
        if self.swiglu:
            g, u, mg, mu = mag
            s = 1 / (1 + np.exp(-g))
            # |d silu| <= 1.1; the device's exponential and division add a few units in the last place
            bound = eps * (1.1 * mg * np.abs(u) + np.abs(g * s) * mu) + 16 * 2.0 ** -24 * np.abs(ref) \
                + (1.1 * eps * mg) * (eps * mu)
        else:
            bound = eps * mag + 2.0 ** -23 * np.abs(ref) + (0 if self.res is None else 2.0 ** -23 * np.abs(self.res))
        rows = np.arange(self.B) if rows is None else rows
        err = np.abs(got[rows].astype(np.float64) - ref[rows])
        worst = float((err / np.maximum(bound[rows], 1e-30)).max())
        assert worst <= 1.0, f"error is {worst:.2f} of its bound"


CASES = [
    # K, parts, rank, adapters, B, swiglu, norm, residual
    (8, [1], 8, 1, 1, False, False, False),
    (8, [3], 8, 2, 5, False, True, False),
    (264, [129], 24, 3, 1, False, True, True),
    (264, [129], 24, 3, 17, False, True, True),
    (512, [64, 16, 17], 16, 4, 1, False, True, False),
    (512, [64, 16, 17], 16, 4, 9, False, True, False),
    (2048, [2048, 1024, 1024], 16, 4, 1, False, True, False),
    (2048, [2048, 1024, 1024], 16, 4, 3, False, True, False),
    (1000, [200, 100, 50, 7], 40, 5, 33, False, False, True),
    (1024, [333, 333], 128, 3, 1, True, True, False),
    (1024, [333, 333], 128, 3, 4, True, True, False),
    (1024, [700, 700], 64, 3, 40, True, True, False),
    (640, [100, 300, 200], 8, 6, 12, True, False, False),       # parts that cross gate and up
    (2048, [3000, 3000], 16, 8, 65, True, True, False),
    (6144, [512], 64, 8, 160, False, False, True),
    (1536, [70000], 8, 2, 1, False, False, False),              # one request on the tiles
    (520, [65536], 8, 2, 1, False, False, False),
]


@pytest.mark.parametrize("K,parts,rank,adapters,B,swiglu,norm,residual", CASES)
def test_matches_oracle(K, parts, rank, adapters, B, swiglu, norm, residual):
    t = Layer(3, K, parts, rank, adapters, B, swiglu, norm, residual)
    if B == 1:
        t.ids[:] = adapters - 1
    t.upload()
    got = t.run()
    t.check(got)
    np.testing.assert_array_equal(got, t.run())          # the same bits again


@pytest.mark.parametrize("B", [1, 6])
@pytest.mark.parametrize("swiglu", [False, True])
def test_no_adapter_is_the_shared_layer(B, swiglu):
    """Rows with id -1 have oda_dense_bf16's bits."""
    t = Layer(4, 512, [96, 96] if swiglu else [96], 16, 2, B, swiglu, norm=True)
    t.ids[:] = -1
    t.upload()
    y = torch.full((B, t.out), -7.0, device="cuda")
    t.P.dense_bf16(t.desc, B, t.dx, None, y)
    np.testing.assert_array_equal(t.run(), y.cpu().numpy())


@pytest.mark.parametrize("B,swiglu", [(1, False), (1, True), (7, False), (7, True)])
def test_ids_out_of_range_give_nan_rows(B, swiglu):
    t = Layer(5, 256, [40, 40] if swiglu else [40], 8, 3, B, swiglu)
    t.ids[:] = np.resize([3, -2, 0, 2 ** 31 - 1, -1, -2 ** 31, 1], B)
    t.upload()
    got = t.run()
    bad = (t.ids < -1) | (t.ids >= 3)
    assert np.isnan(got[bad]).all()
    t.ids = np.where(bad, -1, t.ids).astype(np.int32)
    if not bad.all():
        t.check(got, np.flatnonzero(~bad))


def test_listed_requests_only_and_in_place_residual():
    t = Layer(6, 768, [130], 32, 4, 24, residual=True)
    t.upload()
    work = [20, 3, 4, 11, -1, 24, 9]                      # entries outside the batch are skipped
    y = t.dres.clone()
    t.dres = y                                            # y is the residual buffer
    got = t.run(y=y, work=work)
    rows = np.array([b for b in work if 0 <= b < 24])
    t.check(got, rows)
    rest = np.setdiff1d(np.arange(24), rows)
    np.testing.assert_array_equal(got[rest], t.res[rest])


def test_empty_list_writes_nothing():
    t = Layer(7, 256, [64], 8, 2, 5)
    t.upload()
    assert (t.run(work=[]) == -7.0).all()


def test_largest_offsets():
    """An adapter past 2^31 elements of the second factor."""
    P = need_gpu()
    rows, rank, K = 1 << 18, 128, 8
    adapters = 66                                          # 66 * 2^18 * 128 > 2^31 elements
    w = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    a = torch.zeros(adapters, rank, K, dtype=torch.bfloat16, device="cuda")
    b = torch.zeros(adapters, rows, rank, dtype=torch.bfloat16, device="cuda")
    a[-1, 3, 2] = 1.0
    b[-1, :, 3] = torch.arange(rows, device="cuda").remainder(128).to(torch.bfloat16)
    for B in (1, 2):
        x = torch.zeros(B, K, device="cuda")
        x[:, 2] = 2.0
        y = torch.zeros(B, rows, device="cuda")
        lora = P.lora_desc(adapters, rank, [rows], a, b, torch.ones(adapters, device="cuda"))
        ws = torch.zeros(P.lora_workspace_size(lora, B), dtype=torch.uint8, device="cuda")
        P.dense_lora_bf16(P.dense_desc(K, rows, P.DENSE_PLAIN, w), lora, B, x, None, y,
                          torch.full((B,), adapters - 1, dtype=torch.int32, device="cuda"), ws)
        assert torch.equal(y, (2.0 * torch.arange(rows, device="cuda").remainder(128)).float().expand(B, rows))
