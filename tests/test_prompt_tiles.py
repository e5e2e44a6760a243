"""The prompt attention's tests again with the tiles that a chunk of many rows gets: a
request of so many rows that the plan takes the widest tiles, and of a length that is
out of range (its rows become NaN and cost nothing), stands behind the tests' own."""
import numpy as np
import pytest

import test_prompt_attn as T
from harness import need_gpu
from oracle import prompt as OP

pytestmark = pytest.mark.gpu
CUS, COLUMNS = 256, 32       # narrow tiles: at most 2 * CUS of all KV heads together, of 32 columns


class Wide(T.Prompt):
    def __init__(self, seed, Hq, Hkv, D, rows, seq, **kw):
        more = COLUMNS * (2 * CUS // Hkv) // (Hq // Hkv) + 1
        super().__init__(seed, Hq, Hkv, D, list(rows) + [more], list(seq) + [-1], **kw)
        self.all, self.R = self.R, int(self.start[-2])

    def upload(self):
        seen, self.R = self.R, self.all
        super().upload()
        self.R = seen

    def outputs(self, bf16):
        seen, self.R = self.R, self.all
        o = super().outputs(bf16)
        self.R = seen
        return o

    def attend(self, bf16=False):
        out, lse = super().attend(bf16)
        own, end = self.start[-2:]
        assert np.isnan(out[own:end]).all() and np.isnan(lse[own:end]).all()
        assert (out[end:] == -9).all() and (lse[end:] == -9).all()
        return out[:own], lse[:own]

    def oracle(self):
        return OP.prompt_attention(self.q[:self.R], self.k, self.v, self.table, self.start[:-1], self.seq[:-1], self.scale,
                                   self.causal, self.window)


@pytest.fixture(autouse=True)
def wide(monkeypatch):
    need_gpu()
    monkeypatch.setattr(T, "Prompt", Wide)


@pytest.mark.parametrize("Hq,Hkv,D", [(1, 1, 64), (4, 2, 128), (5, 1, 128), (16, 1, 128), (8, 8, 128)])
@pytest.mark.parametrize("rows,seq", [
    ([33], [33]), ([64], [64]), ([65], [200]), ([1, 0, 40, 7], [1, 5, 41, 300]), ([129, 300], [129, 301])])
def test_causal(Hq, Hkv, D, rows, seq):
    T.test_causal(Hq, Hkv, D, rows, seq)


@pytest.mark.parametrize("window", [1, 15, 16, 17, 40, 100, 1000])
def test_window(window):
    T.test_window(window, [70, 1, 200], [90, 333, 200])


@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 64), (4, 2, 128), (16, 1, 64)])
@pytest.mark.parametrize("rows,seq", [([50, 3, 0, 17], [0, 33, 100, 15]), ([300], [31]), ([300], [63]), ([280, 290], [64, 1000])])
def test_without_a_mask(Hq, Hkv, D, rows, seq):
    T.test_without_a_mask(Hq, Hkv, D, rows, seq)


@pytest.mark.parametrize("Hq,Hkv,rows,seq", [
    (4, 1, [9], [3001]), (8, 1, [16], [3333]), (8, 1, [30], [5000]), (16, 1, [48], [4100]), (2, 2, [1, 1, 500], [9000, 1, 700])])
def test_long_histories_are_split(Hq, Hkv, rows, seq):
    T.test_long_histories_are_split(Hq, Hkv, rows, seq)


def test_unattended_slots_may_hold_anything():
    T.test_unattended_slots_may_hold_anything()


def test_values_that_are_not_finite_reach_their_rows_alone():
    T.test_values_that_are_not_finite_reach_their_rows_alone()


def test_bad_lengths_blocks_and_their_rows():
    T.test_bad_lengths_blocks_and_their_rows()


def test_a_bad_block_outside_the_window_is_not_used():
    T.test_a_bad_block_outside_the_window_is_not_used()


def test_large_scores_and_values():
    T.test_large_scores_and_values()


@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 90])
def test_scores_of_any_size(size):
    T.test_scores_of_any_size(size, [300], [900])


def test_scores_that_grow_and_fall_along_the_history():
    T.test_scores_that_grow_and_fall_along_the_history()
