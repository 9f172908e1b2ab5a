"""Grids of the norm's gradient, checked on the host from the header that the launches use."""

import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_20818_b200", "csrc")
SOURCE = """
#include "q8_plan.h"
using namespace prm;
extern "C" {
long shifted_grid(long rows, long cols) {
  const GradForm f = grad_shifted_form(cols);
  return f.threads ? grad_shifted_grid(rows, cols, f) : 0;
}
// Widths up to `most` for which the grid breaks the kernel's rule, leaves the GPU's room or the scratch.
long bad_shifted_grids(long most, const long* rows, int n, long* first) {
  long bad = 0;
  for (long cols = 1; cols <= most; ++cols) {
    const GradForm f = grad_shifted_form(cols);
    if (!f.threads) continue;
    for (int i = 0; i < n; ++i) {
      const long grid = grad_shifted_grid(rows[i], cols, f);
      const bool apart = grid >= rows[i] || (grid >= 8 && grid % 8 == 0);
      const bool room = grid <= (long)grad_blocks(f.threads, f.nv) * kRingBlocks;
      const bool lines = std::min(grid, rows[i]) <= grad_parts(rows[i], cols);
      const bool octs = (cols + 7 + 7) / 8 <= (long)f.threads * f.nv;
      if (!(apart && room && lines && octs) && !bad++) first[0] = rows[i], first[1] = cols;
    }
  }
  return bad;
}
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", CSRC, str(d / "plan.cpp"), "-o", str(d / "plan.so")],
                   check=True)
    L = ctypes.CDLL(str(d / "plan.so"))
    L.shifted_grid.argtypes = [ctypes.c_long, ctypes.c_long]
    L.shifted_grid.restype = ctypes.c_long
    L.bad_shifted_grids.argtypes = [ctypes.c_long, ctypes.POINTER(ctypes.c_long), ctypes.c_int, ctypes.POINTER(ctypes.c_long)]
    L.bad_shifted_grids.restype = ctypes.c_long
    return L


def test_rows_of_a_block_start_alike(plan):
    """A block of the kernel for rows that start anywhere keeps the offset of its first row: its rows lie a
    multiple of eight apart, or it has only one."""
    rows = [1, 2, 7, 8, 9, 100, 143, 144, 145, 147, 148, 149, 150, 152, 160, 295, 296, 297, 300, 310, 443, 445, 500, 888,
            889, 1000, 1184, 1185, 4099, 8192, 8201, 40003, 262144, 100000007, (1 << 31) - 1]
    first = (ctypes.c_long * 2)()
    assert plan.bad_shifted_grids(16400, (ctypes.c_long * len(rows))(*rows), len(rows), first) == 0, tuple(first)
    assert plan.shifted_grid(310, 8185) == 144 and plan.shifted_grid(148, 8185) == 148
