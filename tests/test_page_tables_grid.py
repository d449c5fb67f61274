"""The grid of the page-table kernels, computed on the host: CTAs for the rows that a pass may have, up to the largest number there is."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT
from paper_2607_21042_b200 import build

PROGRAM = r"""
#include <cstdio>
#include "page_tables.cuh"
int main() {
  const int rows[] = {1, 1024, 1025, 2048, 2049, 200000, 2147482624, 2147483647};
  for (int r : rows) printf("%d %d\n", ttsgpt::page_tables_grid(16, r, 148), ttsgpt::page_tables_grid(1000, r, 148));
  return 0;
}
"""


def test_page_tables_grid(tmp_path):
    nvcc = build.nvcc_path()
    if not (shutil.which(nvcc) or os.path.exists(nvcc)):
        pytest.skip("no nvcc")
    (tmp_path / "p.cu").write_text(PROGRAM)
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "paper_2607_21042_b200", "csrc"),
                    "-o", str(tmp_path / "p"), str(tmp_path / "p.cu")], check=True)
    got = [tuple(map(int, line.split())) for line in subprocess.run([str(tmp_path / "p")], capture_output=True, text=True, check=True).stdout.splitlines()]
    # a CTA for 1024 rows up to two an SM (up to 256 requests), for 2048 rows up to one an SM
    assert got == [(1, 1), (1, 1), (2, 1), (2, 1), (3, 2), (196, 98), (296, 148), (296, 148)]
