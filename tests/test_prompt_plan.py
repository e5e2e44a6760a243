"""The plan of oda_prompt_attn, read back: every tile's columns and blocks are covered once, and partials lie inside the
workspace, for mixes of any kind and for counts at which 32 bits would not hold the ranges of the finest cut."""
import numpy as np
import pytest
import torch

from harness import dev_i32, need_gpu

pytestmark = pytest.mark.gpu
HEADER, ITEM = 16, 12            # words


def planned(rows, seq, Hq, Hkv, D, causal=True, window=0, max_len=None):
    """(the plan's items as int32 [n][12], bytes of the workspace)."""
    P = need_gpu()
    B, R = len(rows), max(1, sum(rows))
    max_len = max_len or max(max(seq), 1)
    shape = P.Shape(1, B, Hq, Hkv, D, -(-max_len // 16), max_len, 1 << 22)
    r = P.prompt_rows(R, dev_i32(np.concatenate([[0], np.cumsum(rows)])))
    plan = torch.full((P.prompt_plan_size(shape, r),), 0xA5, dtype=torch.uint8, device="cuda")
    P.prompt_plan(shape, r, dev_i32(seq), causal, window, plan)
    torch.cuda.synchronize()
    words = plan.cpu().numpy().view(np.int32)
    n = int(words[7])
    return words[HEADER:HEADER + n * ITEM].reshape(n, ITEM), P.prompt_workspace_size(shape, r)


def check(rows, seq, Hq, Hkv, D, causal=True, window=0):
    items, ws = planned(rows, seq, Hq, Hkv, D, causal, window)
    G = Hq // Hkv
    request, row0, col0, ncols, lo, hi, place0, n, part = items[:, :9].T.astype(np.int64)
    assert (ncols >= 1).all() and (ncols <= 256).all()
    partial = part >= 0
    assert ((part + ncols)[partial] * Hkv * (D * 4 + 8) <= ws).all()
    # partials side by side, none shared
    order = np.argsort(part[partial])
    ends = (part + ncols)[partial][order]
    assert (part[partial][order][1:] >= ends[:-1]).all()
    start = np.concatenate([[0], np.cumsum(rows)])
    order = np.lexsort((lo, col0, request))
    at = 0
    for b in range(len(rows)):
        col = 0
        while col < rows[b] * G:
            i = order[at]
            assert (request[i], row0[i], col0[i]) == (b, start[b], col)
            wide, first, last = ncols[i], seq[b] - rows[b] + col // G, seq[b] - rows[b] + (col + ncols[i] - 1) // G
            blk = max(0, first - window + 1) // 16 if window else 0
            end = last // 16 + 1 if causal else -(-seq[b] // 16)
            whole = part[i] < 0
            while True:
                i = order[at]
                assert (request[i], col0[i], ncols[i], lo[i], n[i], place0[i]) == (b, col, wide, blk, seq[b], seq[b] - rows[b])
                assert hi[i] > lo[i] or end == blk
                assert whole == (part[i] < 0)
                blk = hi[i]
                at += 1
                if blk == end:
                    break
                assert not whole and (hi[i] - lo[i]) % 2 == 0 and blk < end
            col += wide
    assert at == len(items)


@pytest.mark.parametrize("Hq,Hkv,D,rows,n,causal", [
    (16, 1, 64, 100_000, 1 << 26, False), (16, 1, 64, 100_000, 1 << 26, True), (8, 1, 128, 300_000, 1 << 25, False),
    (16, 1, 64, 2_000_000, 1 << 26, True)])
def test_counts_beyond_32_bits(Hq, Hkv, D, rows, n, causal):
    """Ranges of the finest cut: 2.3e9 and more."""
    check([rows, 1], [n, 5], Hq, Hkv, D, causal)


@pytest.mark.parametrize("seed", range(24))
def test_mixes(seed):
    g = np.random.default_rng(seed)
    B = int(np.exp(g.uniform(0, np.log(300))))
    top = np.exp(g.uniform(0, np.log(3000)))
    rows = [int(r) for r in np.exp(g.uniform(-1, np.log(top + 1), size=B))]
    hist = [int(h) for h in np.exp(g.uniform(0, np.log(1 + np.exp(g.uniform(0, np.log(60000)))), size=B))]
    Hkv = int(g.choice([1, 2, 8, 16]))
    causal = bool(g.integers(0, 3))
    window = int(np.exp(g.uniform(0, 9))) if causal and g.integers(0, 2) else 0
    check(rows, [(r if causal else 0) + h for r, h in zip(rows, hist)], Hkv * int(g.choice([1, 4, 5])), Hkv, 64, causal, window)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,good", [(2 ** 31 - 1, False), (2 ** 31 - 16, False), (2 ** 31 - 64, False), (2 ** 31 - 65, True)])
def test_lengths_next_to_32_bits(n, good, causal):
    """Positions behind the last that a stage reaches are counted too: the longest lengths are out of range."""
    items, _ = planned([3], [n], 2, 1, 64, causal, max_len=2 ** 31 - 1)
    if good:
        lo, hi = items[:, 4], items[:, 5]
        assert (items[:, 7] == n).all() and lo.min() == 0 and hi.max() == -(-n // 16) and (hi > lo).all()
    else:
        assert items[:, 7].tolist() == [-1] and items[0, 3] == 6
