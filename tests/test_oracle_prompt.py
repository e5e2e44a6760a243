"""Pins of oracle/prompt.py (no GPU)."""
import numpy as np

import oda_synth as S
from oracle import prompt as OP
from oracle.attention import bf16_to_f64, decode_attention, full_set, native_window_set
from oracle.decoder import qk_norm_rope, round_bf16


def case(seed, rows, seq, Hq=4, Hkv=2, D=64):
    start = np.concatenate([[0], np.cumsum(rows)])
    table, nb = S.paged_block_table(S.rng(seed, S.STREAM_TABLE), np.maximum(seq, 1), max(1, -(-max(seq) // 16)))
    k, v = S.kv_cache(seed, 1, nb, Hkv, D)
    return start, table, k, v, S.normal_bf16(S.rng(seed, 3), (int(start[-1]), Hq, D))


def test_a_row_is_decode_attention_of_its_length():
    rows, seq = [5, 1, 0, 20], [30, 7, 9, 20]
    start, table, k, v, q = case(1, rows, seq)
    for window in (0, 6):
        out, lse, _ = OP.prompt_attention(q, k, v, table, start, seq, 0.2, True, window)
        for b in range(4):
            for i in range(rows[b]):
                n = seq[b] - rows[b] + i + 1
                r = start[b] + i
                one, l, _ = decode_attention(q[None, r:r + 1], k, v, table[b:b + 1], [n],
                                             lambda m: native_window_set(m, window), 0.2)
                np.testing.assert_allclose(out[r], one[0, 0], atol=1e-12)
                np.testing.assert_allclose(lse[r], l[0, 0], atol=1e-12)


def test_without_a_mask_every_row_sees_all():
    rows, seq = [3, 2], [11, 0]
    start, table, k, v, q = case(2, rows, seq)
    out, lse, mag = OP.prompt_attention(q, k, v, table, start, seq, 0.2, False)
    one, l, _ = decode_attention(q[None, :1], k, v, table[:1], [11], full_set, 0.2)
    np.testing.assert_allclose(out[0], one[0, 0], atol=1e-12)
    assert (out[3:] == 0).all() and np.isneginf(lse[3:]).all()
    assert (mag[:3] >= np.abs(out[:3]) - 1e-12).all()


def test_append_is_the_decode_steps_preparation():
    g = S.rng(3, 1)
    x = g.standard_normal((4, (4 + 2 * 2) * 64))
    gain = 1 + 0.1 * g.standard_normal(64)
    start, seq = [0, 1, 1, 4], [9, 4, 20]
    q, k, v, owner = OP.append_rows(x, 4, 2, 64, start, seq, gain, gain, 1e-6, 1e6)
    rq, rk, rv = qk_norm_rope(x, 4, 2, 64, gain, gain, 1e-6, 1e6, [8, 17, 18, 19])
    for a, b in ((q, rq), (k, rk), (v, rv)):
        np.testing.assert_array_equal(round_bf16(a), b)
    assert owner.tolist() == [[0, 8], [2, 17], [2, 18], [2, 19]]


def test_axes_that_agree_are_one_axis():
    x = S.rng(4, 1).standard_normal((3, 4 * 64))
    p = np.array([[5], [0], [700]])
    one = OP.append_rows(x, 2, 1, 64, [0, 3], [3], theta=1e4, positions=p)
    three = OP.append_rows(x, 2, 1, 64, [0, 3], [3], theta=1e4, positions=np.repeat(p, 3, 1), axis_pairs=[10, 11, 11])
    np.testing.assert_array_equal(one[0], three[0])
    # and a pair follows its own axis alone
    q = np.array([[5, 1, 2], [0, 3, 4], [700, 5, 6]])
    mixed = OP.append_rows(x, 2, 1, 64, [0, 3], [3], theta=1e4, positions=q, axis_pairs=[10, 11, 11])
    np.testing.assert_array_equal(mixed[0][..., :10], one[0][..., :10])
    assert (mixed[0][..., 10:32] != one[0][..., 10:32]).any()


def test_rows_in_cache_and_ring():
    g = S.rng(5, 1)
    k, v = g.standard_normal((40, 1, 64)), g.standard_normal((40, 1, 64))
    owner = np.array([[0, 20 + i] for i in range(40)])
    kc, vc = np.zeros((4, 1, 8, 16, 8), np.uint16), np.zeros((4, 1, 64, 16), np.uint16)
    kr, vr = np.zeros((1, 4, 1, 8, 16, 8), np.uint16), np.zeros((1, 4, 1, 64, 16), np.uint16)
    table = np.array([[2, 0, 3, 1]])
    OP.put_rows(k, v, owner, table, [60], kc, vc, kr, vr, 1, 3)      # window 1..16: sink block 0, blocks 1..3 in ring 1..3
    np.testing.assert_array_equal(bf16_to_f64(kc[0, 0, :, 4]).reshape(-1), round_bf16(k[0, 0]))      # place 20: block 1
    np.testing.assert_array_equal(vr[0, 1 + 1 % 3, 0, :, 4], vc[0, 0, :, 4])
    np.testing.assert_array_equal(vr[0, 1 + 3 % 3, 0, :, 11], vc[1, 0, :, 11])                         # place 59: block 3
    assert (kc[2] == 0).all() and (kr[0, 0] == 0).all()


def test_token_logprobs_worked():
    z = np.log(np.array([[0.5, 0.25, 0.125, 0.125]]))
    lp, rank, h, best, ids = OP.token_logprobs(z, [3], 3)
    np.testing.assert_allclose([lp[0], h[0]], [np.log(0.125), 1.75 * np.log(2)], rtol=1e-12)
    assert rank[0] == 4 and ids[0].tolist() == [0, 1, 2]
    np.testing.assert_allclose(best[0], np.log([0.5, 0.25, 0.125]))
    lp, rank, h, best, ids = OP.token_logprobs([[np.inf, 1.0, np.inf], [-np.inf, np.nan, -np.inf]], [2, 0], 2)
    np.testing.assert_allclose([lp[0], h[0]], [-np.log(2), np.log(2)])
    assert rank.tolist() == [2, 1] and ids.tolist() == [[0, 2], [-1, -1]] and np.isnan(lp[1]) and np.isnan(h[1])
