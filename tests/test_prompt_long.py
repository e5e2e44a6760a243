"""Long chunks through PromptDecoder, whose attention takes the widest tiles and whose dense layers thousands of rows: the
caches and scores of the same tokens in short chunks, up to the rounding of fp32 sums (the bars of
tests/test_prompt_decoder.py)."""
import numpy as np
import pytest
import torch

from oracle import attention as OA
from test_prompt_decoder import STEP_REL_L2, Prompts, rel_l2

pytestmark = pytest.mark.gpu


class Whole(Prompts):
    chunks = [[4300, 0, 37, 1]]                                     # 8,600 columns of a KV head


class Short(Prompts):
    chunks = [[700, 0, 0, 1], [900, 0, 5, 0], [1, 0, 30, 0], [1399, 0, 1, 0], [1300, 0, 1, 0]]


@pytest.mark.parametrize("window", [0, 600])
def test_a_long_chunk_is_its_short_ones(window):
    a, b = (cls(score="last", rows=4400, window=window) for cls in (Whole, Short))
    assert all(np.array_equal(x, y) for x, y in zip(a.tokens, b.tokens))
    lasts = []
    for t in (a, b):
        forward, scores = t.dec.stages()
        last = {}
        for c in range(len(t.chunks)):
            t.set(c)
            t.run(forward + scores)
            torch.cuda.synchronize()
            end = (t.dec.row_start[1:] - 1).tolist()
            for r in range(4):
                if t.chunks[c][r]:
                    last[r] = t.dec.logits[end[r]].double().cpu().numpy()
        lasts.append(last)
        assert t.dseq.tolist() == np.sum(t.chunks, 0).tolist()
    for x, y in ((a.dk, b.dk), (a.dv, b.dv)):
        x, y = (OA.bf16_to_f64(u.cpu().numpy().view(np.uint16)) for u in (x, y))
        assert np.isfinite(x).all()
        assert (x != y).mean() < 5e-3 and np.abs(x - y).max() <= 2.0 ** -6 * np.abs(y).max()
    assert lasts[0].keys() == lasts[1].keys() == {0, 2, 3}
    for r in lasts[0]:
        assert rel_l2(lasts[0][r], lasts[1][r]) <= STEP_REL_L2
