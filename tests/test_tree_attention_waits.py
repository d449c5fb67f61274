"""What the warps of the tree attention wait for, as far as it can be told without a GPU."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from conftest import ROOT
from paper_2607_21042_b200 import build

CSRC = os.path.join(ROOT, "paper_2607_21042_b200", "csrc")


def test_a_look_at_a_barrier_has_one_answer_for_the_warp():
    """Lanes that poll a barrier while others arrive may see different things.  Where votes of all lanes follow, a branch on a lane's own answer could leave some of them
    behind for good, so that what looks without waiting votes itself."""
    found = 0
    for path in glob.glob(os.path.join(CSRC, "*.cuh")):
        text = open(path).read()
        for at in (m.start() for m in re.finditer(r"mbarrier\.test_wait", text)):
            found += 1
            body = text[at:text.index("\n}", at)]
            assert re.search(r"return __(any|all)_sync\(0xFFFFFFFFu, done != 0\);", body), (path, body)
    assert found


def test_the_end_of_a_range_is_the_warps():
    """The error word decides whether a CTA has work; other warps may set it meanwhile, and the loop over the range votes."""
    text = open(os.path.join(CSRC, "attention_tree.cuh")).read()
    decisions = re.findall(r"u_end = ([^;]*\?)", text)
    assert decisions == ["__any_sync(0xFFFFFFFFu, *failed) ?"]


PLACES = r"""
#include <cstdio>
#include "attention_tree.cuh"
// Parts of 1 to 6 pages in every order of seven.  Places of V by turns; a tile's sums meet in the places of the last two pages when it ends.  At a page of part n all tiles
// before n may have left, or only those up to n - 2, which the part's queries wait for.
int main() {
  int len[7], ends[7];
  long pages = 0, waits = 0, lost = 0, late = 0;
  for (int x = 0; x < 279936; ++x) {                        // 6^7
    for (int n = 0, y = x; n < 7; ++n, y /= 6) len[n] = 1 + y % 6;
    int c = 0;
    for (int n = 0; n < 7; ++n) {
      bool left = false;                                    // the tile before this part is known to have left
      for (int i = 0; i < len[n]; ++i, ++c, ++pages) {
        const int tile = ttsgpt::tree_tile_in_place(n, i);
        if (tile >= 0) {
          ++waits;
          if (tile + 2 <= n - 1 || tile >= n) ++late;       // the phase may have been passed twice; or cannot end
          left = left || tile == n - 1;
        }
        const bool stands = n > 0 && ((ends[n - 1] & 3) == (c & 3) || ((ends[n - 1] - 1) & 3) == (c & 3));
        if (stands && !left) ++lost;
      }
      ends[n] = c - 1;
    }
  }
  printf("%d %ld %ld\n", pages > 0 && waits > 0, late, lost);
  return 0;
}
"""


def test_a_place_is_filled_when_the_sums_in_it_have_left(tmp_path):
    """And what is waited for is the tile just before: the barrier of one before that may have gone a phase further, which looks like none."""
    nvcc = build.nvcc_path()
    if not (shutil.which(nvcc) or os.path.exists(nvcc)):
        pytest.skip("no nvcc")
    (tmp_path / "p.cu").write_text(PLACES)
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", CSRC, "-o", str(tmp_path / "p"), str(tmp_path / "p.cu")], check=True)
    got = subprocess.run([str(tmp_path / "p")], capture_output=True, text=True, check=True).stdout
    assert got.split() == ["1", "0", "0"]
