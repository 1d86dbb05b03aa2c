"""Which token of a tile a head row belongs to: rotate's division by multiplication, the functions that the kernel and its host side
use, run on the CPU (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "rotary.cuh"
int main() {
  for (int rows = 1; rows < 512; ++rows)
    for (int tile = 1; tile <= vdn::Rotary::MAX_TILE; ++tile) {
      const unsigned m = vdn::rotary_per_row(rows, tile);
      for (int t = 0; t < tile * rows; ++t)
        if (vdn::rotary_token(t, rows, m) != t / rows) { std::printf("%d rows, tile of %d, row %d\n", rows, tile, t); return 1; }
    }
  // a tile of one token may have as many rows as there are heads
  for (int rows = 512; rows <= 2 * 65535; rows = rows * 2 - 1)
    for (int t = 0; t < rows; ++t)
      if (vdn::rotary_token(t, rows, vdn::rotary_per_row(rows, 1)) != 0) { std::printf("%d rows, row %d\n", rows, t); return 1; }
  return 0;
}
"""


def test_rows_of_a_tile_find_their_token(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("needs nvcc")
    src = tmp_path / "places.cu"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "places")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1",
                    "-I" + os.path.join(ROOT, "paper_2609_20744_b200", "csrc"), str(src), "-o", exe], check=True)
    got = subprocess.run([exe], capture_output=True, text=True)
    assert got.returncode == 0, got.stdout
