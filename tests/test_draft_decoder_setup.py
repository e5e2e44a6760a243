"""What DraftDecoder lays out before its first step, and the inputs that set_drafts
writes (CPU: no kernel runs)."""
import os

import numpy as np
import pytest
import torch

import oda_synth as S

L, D_MODEL, HQ, HKV, D, F, V = 3, 64, 2, 1, 64, 96, 40


@pytest.fixture(scope="module")
def P():
    from paper_2609_20734_amd import build as B
    if not os.path.exists(B.LIB):
        B.build()
    import paper_2609_20734_amd as P
    return P


def _bits(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)) if a.dtype == np.uint16 else torch.from_numpy(a)


def _decoder(P, T=3, ranks=(8, 8, 8), names=("w_o",), B=2):
    from paper_2609_20734_amd import decoder as PD
    w = {n: _bits(x) for n, x in S.decoder_weights(3, L, D_MODEL, HQ, HKV, D, F, V).items()}
    mb, nb = 4, 4 * B
    k = torch.zeros(L, nb, HKV, D // 8, 16, 8, dtype=torch.bfloat16)
    v = torch.zeros(L, nb, HKV, D, 16, dtype=torch.bfloat16)
    table = torch.arange(B * mb, dtype=torch.int32).view(B, mb)
    sizes = dict(w_o=(HQ * D, [D_MODEL]), w_gu=(D_MODEL, [F, F]))

    def lora(name, r):
        K, parts = sizes[name]
        return P.lora_desc(2, r, parts, torch.zeros(2, len(parts) * r, K, dtype=torch.bfloat16),
                           torch.zeros(2, sum(parts), r, dtype=torch.bfloat16), torch.ones(2))

    i32 = dict(dtype=torch.int32)
    groups = (torch.tensor([0, B], **i32), torch.arange(B, **i32), torch.tensor([0], **i32))
    return PD.DraftDecoder(PD.DecoderShape(L, D_MODEL, HQ, HKV, D, F, V), w, B, T, k, v, table, torch.full((B,), 5, **i32), mb,
                           mb * 16, nb, groups, {n: [lora(n, r) for r in ranks] for n in names}, torch.zeros(B, **i32))


@pytest.mark.parametrize("ranks", [(8, 16, 64), (128, 8, 8), (8, 72, 16)])
def test_the_adapters_workspace_serves_every_layer(P, ranks):
    """Adapters of one projection may have another rank in each layer."""
    dec = _decoder(P, ranks=ranks, names=("w_o", "w_gu"))
    need = max(P.lora_workspace_size(d, dec.B * dec.T) for a in dec.adapters.values() for d in a)
    assert dec.ws_lora.numel() >= need


@pytest.mark.parametrize("counts", [[0, 2], [-1, 1], [-2 ** 31, 3], [7, 2 ** 31 - 1]])
def test_counts_of_drafts_are_clamped_alike(P, counts):
    """Verification clamps the number of drafts to [0, T - 1]; attention has a current token more than that."""
    dec = _decoder(P)
    n = torch.tensor(counts, dtype=torch.int32)
    dec.set_drafts(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dec.T - 1, dtype=torch.int32), n)
    want = np.clip(counts, 0, dec.T - 1)
    np.testing.assert_array_equal(np.clip(dec.n_drafts.numpy(), 0, dec.T - 1), want)
    np.testing.assert_array_equal(np.clip(dec.n_tokens.numpy(), 0, dec.T), want + 1)
