"""The aligned fours of slots in which a commit of several tokens reads and stores
its values (csrc/oda_commit_fours.h, compiled for the host): every read is one of
the request's tokens, every token is stored once, and a request that commits
nothing reads nothing."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <vector>
#include "oda_commit_fours.h"
int main() {
  const long long far[] = {-(1ll << 31) - 1, (1ll << 31) - 2};      // seq_lens' ends, less one
  for (int i = -70; i < 70; ++i)
    for (int f = 0; f < 3; ++f)
      for (int count = 0; count <= 64; ++count) {
        const long long pos0 = f == 2 ? i : far[f] - (f ? std::max(i, 0) : std::min(i, 0));
        std::vector<int> stored(count);
        for (int t0 = oda::first_four(pos0, count); t0 < count; t0 += 4) {
          if (((pos0 + t0) & 3) != 0) return std::printf("unaligned: %lld tokens from %lld\n", (long long)count, pos0), 1;
          for (int k = 0; k < 4; ++k) {
            const int t = oda::token_read(t0, k, count);
            if (t < 0 || t >= count)
              return std::printf("token %d read of %d from position %lld on\n", t, count, pos0), 1;
            if (k >= std::max(0, -t0) && k < std::min(4, count - t0)) {
              if (t != t0 + k) return std::printf("token %d in the place of %d\n", t, t0 + k), 1;
              ++stored[t];
            }
          }
        }
        for (int t = 0; t < count; ++t)
          if (stored[t] != 1) return std::printf("token %d of %d stored %d times\n", t, count, stored[t]), 1;
      }
  return 0;
}
"""


def test_fours_cover_the_tokens_and_read_no_others(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "fours.cpp").write_text(PROGRAM)
    csrc = os.path.join(ROOT, "paper_2609_20734_amd", "csrc")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", csrc, str(tmp_path / "fours.cpp"),
                    "-o", str(tmp_path / "fours")], check=True)
    res = subprocess.run([str(tmp_path / "fours")], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0, res.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5])
def test_requests_that_commit_nothing(T):
    """n_accepted = -1 at every place within a four: caches and lengths stay as they are."""
    import numpy as np
    import torch

    from test_commit_drafts import Commit
    t = Commit(31, 2, 6, T, 2, 64, [1, 2, 3, 4, 17, 32], [-1, -1, -9, -1, -1, -1])
    t.upload()
    rows = torch.full((t.B, T), -3, dtype=torch.int32, device="cuda")
    t.run(True, rows)
    t.check()
    np.testing.assert_array_equal(rows.cpu().numpy(), t.seq[:, None] + np.arange(T))
