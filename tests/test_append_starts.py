"""Row starts of any order in oda_append_qkv: rows, caches and rings are those of the ascending starts that they stand for,
and rows of no request keep their bits.  Tolerances as in tests/test_append.py."""
import numpy as np
import pytest

from test_append import Append

pytestmark = pytest.mark.gpu


class Given(Append):
    """The kernel gets `given`, the oracle `start`."""
    def run(self, times=1):
        seen, self.start = self.start, np.array(self.given, dtype=np.int32)
        out = super().run(times)
        self.start = seen
        return out


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("lead,rows,tail,given", [
    (0, [6, 0, 15, 0], 0, [-7, 6, 3, 900, 12]),                        # the last clamped one covers the buffer's 21 rows
    (2, [6, 0, 10, 0, 0], 3, [2, 8, 5, 18, 12, -4]),                   # rows in front and behind are no request's
    (4, [0, 17, 0, 1, 0], 2, [4, -1, 21, 20, 22, -2 ** 31]),
    (1, [1, 1, 0, 1], 7, [1, 2, 3, 3, 4])])
def test_any_order(lead, rows, tail, given, bf16):
    t = Given(63, len(rows), 4, 2, 64, rows, [3, 5, 20, 0, 9][:len(rows)], bf16=bf16, sink=16, window=20, lead=lead, tail=tail)
    t.given = given
    t.check()


def test_more_requests_than_a_scan_holds():
    """A start far ahead in the first 64 requests holds for those behind."""
    B = 150
    rows = [1 + b % 3 for b in range(70)] + [0] * 40 + [2] * 40
    t = Given(64, B, 2, 1, 128, rows, [b % 40 for b in range(B)], lead=2, tail=3)
    t.given = t.start.copy()
    t.given[71:110] = np.arange(39) - 5            # below the running largest: no rows
    t.check()
