"""Dense layers whose launch is large enough for the tiles of 48 or 64 rows and 32
requests (csrc/decoder.hip, launch_dense): odd row, request and K counts, lists
with ids outside the batch, nonfinite inputs and weights, adapters.

A request's sums are formed in the same order whichever tile its batch takes, so
the outputs equal those of batches of sixteen (tiles of 32 rows and 16 requests)
bit for bit; those batches are checked against the fp64 oracle with the bound of
one fp32 rounding per addition: |err| <= n 2^-24 sum_k |w x'|, n = K / 256 + 68."""
import numpy as np
import pytest
import torch

import oda_synth as S
from harness import dev_f32, dev_i32, dev_u16, need_gpu
from oracle import attention as OA
from oracle import decoder as OD

pytestmark = pytest.mark.gpu

TARGET = 256   # workgroups of one round


def _groups(N, B, tiles, edge):
    return -(-N // (tiles * edge)) * -(-B // edge)


def _rounds(N, B, rows):
    return -(-(-(-N // rows) * -(-B // 32)) // TARGET)


def _is_wide(K, N, B):
    narrow, rounds = _groups(N, B, 2, 16), _rounds(N, B, 64)
    return narrow > 2 * TARGET * rounds if rounds == 1 or K >= 4096 else narrow >= 3 * TARGET * rounds


CASES = [(8, 8000, 33), (72, 4100, 96), (40, 8191, 64), (264, 8000, 37), (1000, 5003, 61), (520, 16380, 17),
         (2088, 4113, 95), (264, 4300, 84), (1000, 8150, 160), (4104, 6100, 90)]


def test_the_cases_take_the_wide_tiles_and_their_parts_do_not():
    assert {_rounds(N, B, 48) == _rounds(N, B, 64) for _, N, B in CASES} == {True, False}   # of 48 rows and of 64
    for K, N, B in CASES:
        assert _is_wide(K, N, B) and not _is_wide(K, N, 16) and _groups(N, 16, 1, 16) > TARGET, (N, B)


def _layer(seed, K, N, B, norm, residual):
    g = S.rng(seed, S.STREAM_DECODER)
    W = S.normal_bf16(g, (N, K), K ** -0.5)
    x = (g.standard_normal((B, K)) * np.exp(4 * g.standard_normal((B, 1)))).astype(np.float32)
    gain = (1 + 0.02 * g.standard_normal(K)).astype(np.float32) if norm else None
    r = g.standard_normal((B, N)).astype(np.float32) if residual else None
    return g, W, x, gain, r


def _in_parts(run, B):
    return np.concatenate([run(b, min(b + 16, B)) for b in range(0, B, 16)])


@pytest.mark.parametrize("norm,residual", [(False, True), (True, False), (True, True)])
@pytest.mark.parametrize("K,N,B", CASES)
def test_wide_tiles(K, N, B, norm, residual):
    P = need_gpu()
    g, W, x, gain, r = _layer(K + N + B, K, N, B, norm, residual)
    desc = P.dense_desc(K, N, P.DENSE_PLAIN, dev_u16(W), dev_f32(gain) if norm else None, 1e-6)

    def run(b0, b1):
        y = torch.full((b1 - b0, N), np.nan, device="cuda")
        P.dense_bf16(desc, b1 - b0, dev_f32(x[b0:b1]), dev_f32(r[b0:b1]) if residual else None, y)
        torch.cuda.synchronize()
        return y.cpu().numpy()

    got = run(0, B)
    n = B - (B % 16 == 1)                                      # (a last part of one request is another kernel's)
    assert np.array_equal(got[:n], _in_parts(run, n))
    xn = OD.rmsnorm(x.astype(np.float64), gain, 1e-6) if norm else x.astype(np.float64)
    ref = OD.dense(W, x, gain, 1e-6, r)
    bound = (K / 256 + 68) * 2.0 ** -24 * (np.abs(xn) @ np.abs(OA.bf16_to_f64(W)).T)
    assert np.all(np.abs(got - ref) <= bound + 2.0 ** -23 * np.abs(ref))


@pytest.mark.parametrize("K,N,B", CASES[2:5])
def test_lists_and_rows_left_as_they_were(K, N, B):
    P = need_gpu()
    g, W, x, _, r = _layer(K * 3 + N, K, N, B, False, True)
    desc = P.dense_desc(K, N, P.DENSE_PLAIN, dev_u16(W))
    full = torch.empty(B, N, device="cuda")
    P.dense_bf16(desc, B, dev_f32(x), dev_f32(r), full)
    full = full.cpu().numpy()
    for count in (0, 1, 31, 32, 33, B):
        listed = [int(b) for b in g.permutation(B)[:count]]
        if count > 2:
            listed[1], listed[2] = -1, B
        y = torch.full((B, N), 7.0, device="cuda")
        P.dense_bf16(desc, B, dev_f32(x), dev_f32(r), y, dev_i32(listed + [0] * (B - count)), dev_i32([count]))
        torch.cuda.synchronize()
        done = np.array([b for b in listed if 0 <= b < B], dtype=int)
        want = np.full((B, N), 7.0, np.float32)
        want[done] = full[done]
        assert np.array_equal(y.cpu().numpy(), want), count


def test_nonfinite_values_stay_where_they_are():
    P = need_gpu()
    K, N, B = 264, 8000, 37
    g, W, x, _, _ = _layer(5, K, N, B, False, False)
    inf = int(S.f32_to_bf16_bits(np.full(1, np.inf, np.float32))[0])
    clean = torch.empty(B, N, device="cuda")
    P.dense_bf16(P.dense_desc(K, N, P.DENSE_PLAIN, dev_u16(W)), B, dev_f32(x), None, clean)
    clean = clean.cpu().numpy()
    W[70, 3] = inf
    x[20, 9], x[36, 0] = np.nan, np.inf
    y = torch.empty(B, N, device="cuda")
    P.dense_bf16(P.dense_desc(K, N, P.DENSE_PLAIN, dev_u16(W)), B, dev_f32(x), None, y)
    torch.cuda.synchronize()
    y = y.cpu().numpy()
    assert np.all(np.isnan(y[20]))
    w0 = OA.bf16_to_f64(W[:, 0])
    some = w0 != 0
    some[70] = False
    assert np.array_equal(y[36, some], np.where(w0[some] > 0, np.inf, -np.inf).astype(np.float32))
    others = np.setdiff1d(np.arange(B), [20, 36])
    assert np.array_equal(y[others, 70], np.where(x[others, 3] > 0, np.inf, -np.inf).astype(np.float32))
    keep = np.arange(N) != 70
    assert np.array_equal(y[np.ix_(others, keep)], clean[np.ix_(others, keep)])


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("K,parts,rank,B", [(264, [8000], 8, 40), (520, [2111, 5, 1987], 64, 94), (72, [8191], 24, 47),
                                              (136, [5003], 40, 61)])
def test_adapters_beside_wide_tiles(K, parts, rank, B, norm):
    P = need_gpu()
    N, A = sum(parts), 3
    assert _is_wide(K, N, B)
    g, W, x, gain, r = _layer(K + N, K, N, B, norm, True)
    a = S.normal_bf16(g, (A, len(parts) * rank, K), K ** -0.5)
    b = S.normal_bf16(g, (A, N, rank), rank ** -0.5)
    scale = (0.5 + g.random(A)).astype(np.float32)
    ids = g.integers(-1, A, size=B).astype(np.int32)
    ids[33] = A                                                # out of range: NaN
    desc = P.dense_desc(K, N, P.DENSE_PLAIN, dev_u16(W), dev_f32(gain) if norm else None, 1e-6)
    lora = P.lora_desc(A, rank, parts, dev_u16(a), dev_u16(b), dev_f32(scale))

    def run(b0, b1, adapters=True):
        n = b1 - b0
        y = torch.full((n, N), -7.0, device="cuda")
        if adapters:
            ws = torch.full((P.lora_workspace_size(lora, n),), 0x7f, dtype=torch.uint8, device="cuda")
            P.dense_lora_bf16(desc, lora, n, dev_f32(x[b0:b1]), dev_f32(r[b0:b1]), y, dev_i32(ids[b0:b1]), ws)
        else:
            P.dense_bf16(desc, n, dev_f32(x[b0:b1]), dev_f32(r[b0:b1]), y)
        torch.cuda.synchronize()
        return y.cpu().numpy()

    got = run(0, B)
    assert np.array_equal(got, _in_parts(run, B), equal_nan=True)
    assert np.all(np.isnan(got[33])) and np.all(np.isfinite(np.delete(got, 33, 0)))
    assert np.array_equal(got[ids == -1], run(0, B, False)[ids == -1])
