"""Rings beside tables with entries that name no block: K/V of their places is dropped, from the
rings too, as the commits of single and drafted tokens do.  Tolerances as in tests/test_append.py."""
import numpy as np
import pytest
import torch

from harness import dev_i32, dev_u16
from oracle.decoder import bf16_bits, round_bf16
from test_append import Append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_places_without_a_block_are_not_in_the_rings(D, bf16):
    t = Append(61, 4, 4, 2, D, [60, 9, 1, 20], [30, 11, 36, 3], bf16=bf16, sink=16, window=40)
    t.table[0, 3] = -1                # a block of the ring, between others
    t.table[1, 0] = t.nb              # the sink's block, partly in front of the rows
    t.table[2, 2] = 2 ** 31 - 1       # a single row's
    t.check()


def test_same_rings_as_the_commit_of_a_decode_step():
    """One row per request, without norms and rotation: caches and rings are oda_commit_kv_ring's, bit for bit."""
    B, Hkv, D = 5, 2, 64
    t = Append(62, B, 4, Hkv, D, [1] * B, [0, 15, 16, 40, 77], norm=False, theta=0.0, sink=16, window=30, lead=0, tail=0)
    t.table[1, 0] = -1
    t.table[3, 2] = t.nb
    _, k, v, kr, vr = t.run()
    P = t.P
    kv = [dev_u16(bf16_bits(round_bf16(x))) for x in np.split(t.x.reshape(B, -1, D)[:, 4:], 2, axis=1)]
    was = [dev_u16(a) for a in (t.k, t.v, t.kr, t.vr)]
    shape = P.Shape(1, B, 4, Hkv, D, t.mb, t.max_len, t.nb)
    P.commit_kv_ring(shape, was[0], was[1], dev_i32(t.table), dev_i32(t.seq), *kv, advance=False, k_ring=was[2], v_ring=was[3],
                     n_sink=16, window=30)
    torch.cuda.synchronize()
    for got, want in zip((k, v, kr, vr), was):
        np.testing.assert_array_equal(got, want.cpu().numpy().view(np.uint16))
