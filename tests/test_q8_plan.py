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
// The same on a device of `sms` SMs, for all forms of the gradient and for the streamed quantiser.
long bad_grids(long most, int sms, const long* rows, int n, long* first) {
  long bad = 0;
  for (long cols = 1; cols <= most; cols += cols < 20000 ? 1 : 997) {
    const GradForm f = grad_shifted_form(cols);
    const int panels = stream_panels(cols), panel = stream_panel(cols, panels);
    for (int i = 0; i < n; ++i) {
      bool ok = true;
      if (f.threads) {
        const long grid = grad_shifted_grid(rows[i], cols, f, sms);
        ok = ok && (grid >= rows[i] || (grid >= 8 && grid % 8 == 0)) && grid <= (long)grad_blocks(f.threads, f.nv) * sms;
        ok = ok && std::min(grid, rows[i]) <= grad_parts(rows[i], cols);
      }
      for (int threads : {128, 512, 1024}) {
        const long grid = grad_grid(rows[i], cols, grad_blocks(threads, 2), sms);
        ok = ok && grid >= 1 && grid <= (long)grad_blocks(threads, 2) * sms;
      }
      for (int groups : {1, 2, 8}) {
        const long one = ring_grid(rows[i], 2, groups, 1, sms);
        ok = ok && one >= 1 && one <= sms && one <= rows[i];
        if (!stream_takes(cols, sms)) continue;
        const long grid = ring_grid(rows[i], 2, groups, panels, sms);
        ok = ok && grid >= panels && grid <= sms && grid % panels == 0;
        ok = ok && (long)panels * panel >= cols && (long)(panels - 1) * panel < cols && panel <= 8192;
        const long words = (cols + 7) / 8 * 8 + grid * panel;            // the columns' factors, the blocks' maxima
        ok = ok && words <= (std::min<long>(rows[i], kRingBlocks) + 1) * (cols + 256);
      }
      if (!ok && !bad++) first[0] = rows[i], first[1] = cols;
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
    L.bad_grids.argtypes = [ctypes.c_long, ctypes.c_int, ctypes.POINTER(ctypes.c_long), ctypes.c_int,
                            ctypes.POINTER(ctypes.c_long)]
    L.bad_grids.restype = ctypes.c_long
    return L


def test_rows_of_a_block_start_alike(plan):
    """A block of the kernel for rows that start anywhere keeps the offset of its first row: its rows lie a
    multiple of eight apart, or it has only one."""
    rows = [1, 2, 7, 8, 9, 100, 143, 144, 145, 147, 148, 149, 150, 152, 160, 295, 296, 297, 300, 310, 443, 445, 500, 888,
            889, 1000, 1184, 1185, 4099, 8192, 8201, 40003, 262144, 100000007, (1 << 31) - 1]
    first = (ctypes.c_long * 2)()
    assert plan.bad_shifted_grids(16400, (ctypes.c_long * len(rows))(*rows), len(rows), first) == 0, tuple(first)
    assert plan.shifted_grid(310, 8185) == 144 and plan.shifted_grid(148, 8185) == 148


@pytest.mark.parametrize("sms", [148, 147, 132, 74, 36, 18, 10])
def test_grids_fit_the_device(plan, sms):
    """Cooperative launches are refused where their blocks are not resident at once: a part of a GPU has fewer SMs."""
    rows = [1, 7, 16, 144, 149, 310, 1184, 8201, 262144, (1 << 31) - 1]
    first = (ctypes.c_long * 2)()
    assert plan.bad_grids(300000, sms, (ctypes.c_long * len(rows))(*rows), len(rows), first) == 0, tuple(first)
