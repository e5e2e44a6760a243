"""oda_verify_drafts where the number lies within 1e-12 of a border between two tokens: the draw is fp64's.

Two tokens of weights w = exp(-d) and 1: the first is drawn iff w > u (1 + w).  For each 24-bit u the fp32 d nearest the
border is tried in extended precision, and those kept where w is off the border by a part of 1e-13 to 1e-12.  The
kernel's roundings (the exponent's product, the exponential, two sums and a product) are a few 2^-53, 1e-15."""
import numpy as np
import pytest
import torch

from harness import dev_f32, need_gpu
from oracle import drafts as OD

pytestmark = pytest.mark.gpu


def _near_borders(lo, hi):
    u = np.arange(lo, hi, dtype=np.longdouble) / np.longdouble(2 ** 24)
    d = (-np.log(u / (1 - u))).astype(np.float32)
    off = np.exp(-d.astype(np.longdouble)) * (1 - u) / u - 1
    keep = (np.abs(off) > 1e-13) & (np.abs(off) < 1e-12)
    return u[keep].astype(np.float32), d[keep], np.where(off[keep] > 0, 0, 1)


def test_numbers_next_to_a_border():
    P = need_gpu()
    u, d, want = _near_borders(2 ** 18, 2 ** 23)
    B = len(u)
    print(f"{B} numbers", flush=True)
    assert B >= 50 and 0.2 < want.mean() < 0.8
    z = np.stack([-d, np.zeros_like(d)], 1)[:, None, :].astype(np.float32)
    np.testing.assert_array_equal(OD.verify_drafts(z, np.zeros((B, 0), np.int32), u[:, None])[1][:, 0], want)
    acc = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    tok = torch.full((B, 1), -9, dtype=torch.int32, device="cuda")
    ws = torch.zeros(P.verify_workspace_size(B, 2, 0), dtype=torch.uint8, device="cuda")
    P.verify_drafts(P.verify_desc(2, 0, dev_f32(z), None, dev_f32(u[:, None])), B, acc, tok, ws)
    torch.cuda.synchronize()
    assert (acc.cpu().numpy() == 0).all()
    np.testing.assert_array_equal(tok.cpu().numpy()[:, 0], want)
