"""oda_prefix_decode_attn where values are near the ends of their type's range and
scores grow along the history."""
import numpy as np
import pytest
import torch

import oda_synth as S
from harness import LSE_ABS, check_close
from oracle import drafts as OD
from test_prefix import Problem

pytestmark = pytest.mark.gpu

BIG = 2.0 ** 120


def _grow(p, step):
    """Scores (in log2 units) grow by `step` a position, the same for every head."""
    p.q[:] = 0
    p.q[..., 0] = S.f32_to_bf16_bits(np.full(1, 2.0, np.float32))[0]
    per = step * np.log(2) / (2.0 * p.scale)
    for b in p.members:
        n = int(p.seq[b]) - 1 + (0 if p.cur else p.T)
        pos = np.arange(n)
        p.k[:, p.table[b, pos // 16], :, 0, pos % 16, 0] = S.f32_to_bf16_bits((per * pos).astype(np.float32))[:, None, None]
        if p.cur:
            for t in range(p.T):
                p.kc[:, b, t, :, 0] = S.f32_to_bf16_bits(np.full(1, per * (n + t), np.float32))[0]


def _scale_values(p, factor):
    def times(bits):
        return S.f32_to_bf16_bits((bits.astype(np.uint32) << 16).view(np.float32) * np.float32(factor))
    p.v = times(p.v)
    if p.cur:
        p.vc = times(p.vc)


@pytest.mark.parametrize("factor", [BIG, 2.0 ** -100])
@pytest.mark.parametrize("cur", [True, False])
@pytest.mark.parametrize("groups,Hq,Hkv,D,T", [
    ([(0, [300])], 2, 1, 64, 1), ([(20, [40, 90])], 16, 1, 128, 1), ([(20, [40, 90, 3])], 16, 1, 64, 3),
    ([(30, list(range(1, 40, 3)))], 16, 1, 128, 1)], ids=["one", "two tiles", "nine tiles", "thirteen tiles"])
@pytest.mark.parametrize("step", [0.0625, 0.5])
def test_large_and_small_values_behind_growing_scores(groups, Hq, Hkv, D, T, cur, factor, step):
    """Outputs are means of the values: as far from the end of fp32's range as these."""
    p = Problem(71, groups, Hq, Hkv, D, T=T, cur=cur, spare=1)
    _grow(p, step)
    _scale_values(p, factor)
    p.upload()
    out, lse = p.run()
    ref, ref_lse = OD.prefix_attention(p.q, p.k, p.v, p.table, p.seq, p.scale, p.counts(), p.kc, p.vc, p.members)
    rows = p.members
    check_close(out[:, rows].astype(np.float64) / factor, ref[:, rows] / factor)
    assert np.abs(lse[:, rows] - ref_lse[:, rows]).max() <= LSE_ABS
    if T == 1:                                      # what Full gives for the same rows
        full, flse = torch.zeros(1, p.B, Hq, D, device="cuda"), torch.zeros(1, p.B, Hq, device="cuda")
        ws = torch.zeros(max(256, p.P.attn_workspace_size(p.shape, 0, 0)), dtype=torch.uint8, device="cuda")
        p.P.full_decode_attn(p.shape, p.inp, 0, None, None, None, full, flse, ws)
        torch.cuda.synchronize()
        check_close(out[:, rows, 0].astype(np.float64) / factor, full.cpu().numpy()[:, rows].astype(np.float64) / factor)


@pytest.mark.parametrize("D,blocks", [(64, 3074), (128, 3074), (128, 4100)])
@pytest.mark.parametrize("peaked", [False, True])
def test_weights_of_many_columns_keep_their_bits_at_any_length(D, blocks, peaked):
    """160 columns behind 49,184 and 65,600 positions, attended evenly or at 40 positions alone.  Expected error: weights
    to 2e-7 (the exponent's fp32 rounding and the exponential's), sums of a few splits 3e-7; 16-bit weights would be
    2e-6 off."""
    p = Problem(72, [(blocks, [1, 40, 3, 77, 100, 9, 16, 2, 31, 5])], 16, 1, D, poison=True, spare=1)
    if peaked:
        g = S.rng(72, 5)
        one = S.f32_to_bf16_bits(np.ones(1, np.float32))[0]
        p.q[:] = 0
        p.q[..., 0] = one                           # scores are the keys' first dims
        first = p.members[0]
        p.k[:, :, :, 0, :, 0] = S.f32_to_bf16_bits(np.full(1, -2000.0, np.float32))[0]
        p.kc[..., 0] = S.f32_to_bf16_bits(np.full(1, -2000.0, np.float32))[0]
        for pos in g.choice(16 * blocks, 40, replace=False):
            p.k[0, p.table[first, pos // 16], 0, 0, pos % 16, 0] = S.f32_to_bf16_bits(g.random(1).astype(np.float32) * 8)[0]
    p.upload()
    out, _ = p.run()
    rows = p.members
    ref, _ = OD.prefix_attention(p.q, p.k, p.v, p.table, p.seq, p.scale, p.counts(), p.kc, p.vc, rows)
    err = np.linalg.norm(out[:, rows] - ref[:, rows]) / np.linalg.norm(ref[:, rows])
    print(f"rms error {err:.2e}", flush=True)
    assert err <= 1e-6


@pytest.mark.parametrize("groups", [[(0, [300])], [(20, [40, 90, 3, 8])], [(33, list(range(1, 40, 3)))]],
                         ids=["one tile", "four tiles", "thirteen tiles"])
@pytest.mark.parametrize("cur", [True, False])
@pytest.mark.parametrize("score", [1e4, 1e9, 1e20, 3e38, -1e4, -1e20, -3e38])
def test_scores_of_any_size(score, cur, groups):
    """All keys alike, at a score whose product with the scale is off by more than exponents hold; then every third at
    the type's lowest value; then all but a few of each request's own there.  The lse's fp32 steps are seven (two
    constants, the scale in log2 units, the reference, its product, the sum, the product back)."""
    bits = lambda x: S.f32_to_bf16_bits(np.full(1, x, np.float32))[0]  # noqa: E731
    p = Problem(73, groups, 16, 1, 64, cur=cur, spare=1)
    p.q[:] = 0
    p.q[..., 0] = bits(1.0)                         # scores are the keys' first dims
    for step in range(3):
        low = bits(-3e38)
        if step == 0:
            p.k[:, :, :, 0, :, 0] = bits(score)
        elif step == 1:
            p.k[:, :, :, 0, ::3, 0] = low
        else:
            p.k[:, :, :, 0, :, 0] = low
            for b in p.members:
                p.k[:, p.table[b, (int(p.seq[b]) - 1) // 16], :, 0, :, 0] = bits(score)
        if cur:
            p.kc[..., 0] = bits(score) if step != 1 else low
        p.upload()
        out, lse = p.run()
        ref, ref_lse = OD.prefix_attention(p.q, p.k, p.v, p.table, p.seq, p.scale, p.counts(), p.kc, p.vc, p.members)
        rows = p.members
        check_close(out[:, rows], ref[:, rows], f"step {step}")
        np.testing.assert_allclose(lse[:, rows], ref_lse[:, rows], rtol=7 * 2.0 ** -24, atol=LSE_ABS)
