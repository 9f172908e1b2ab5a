"""Blocks of the layer norm's gradient and the tiles' way round the pairs, checked on the host from the header that the launches use."""

import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_20818_b200", "csrc")
SOURCE = """
#include "train_plan.h"
#include <vector>
using namespace prm;
extern "C" {
// Sizes for which a launch has no block, a block has no row, more lines than the scratch has, or (rows that start anywhere) a
// thread's rows do not start alike.
long bad_parts(const long* rows, int n_rows, const long* groups, int n_groups, long most) {
  long bad = 0;
  for (long cols = 1; cols <= most; cols += cols < 300 ? 1 : 37)
    for (int i = 0; i < n_rows; ++i)
      for (int g = 0; g < n_groups; ++g)
        for (int turn : {1, 2, 4, 8, 16, 32})
          for (int blocks : {148, 296, 444, 592, 888, 1184})
            for (bool shift : {false, true}) {
              const long parts = layernorm_parts(rows[i], groups[g], cols, turn, blocks, shift);
              const bool lines = parts >= 1 && parts <= layernorm_parts_bound(rows[i], groups[g], cols);
              const bool each = (parts - 1) * turn < rows[i];
              const bool alike = !shift || parts * turn >= rows[i] || parts * turn % 8 == 0;
              bad += !(lines && each && alike);
            }
  return bad;
}
// Tiles that the pairs' walks leave out or take twice.
long bad_walk(int t0, int t1, int extra, int pairs) {
  std::vector<int> seen[2] = {std::vector<int>(t0), std::vector<int>(t1)};
  for (int pair = 0; pair < pairs; ++pair)
    for (int i = 0, which, tile; pair_tile(t0, t1, extra, pair, pairs, i, which, tile); ++i) {
      if (tile < 0 || tile >= (which ? t1 : t0)) return -1;
      ++seen[which][tile];
    }
  long bad = 0;
  for (auto& s : seen)
    for (int n : s) bad += n != 1;
  return bad;
}
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    so = str(d / "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", CSRC, str(d / "plan.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.bad_parts.restype = lib.bad_walk.restype = ctypes.c_long
    lib.bad_parts.argtypes = [ctypes.POINTER(ctypes.c_long), ctypes.c_int, ctypes.POINTER(ctypes.c_long), ctypes.c_int, ctypes.c_long]
    return lib


def longs(v):
    return (ctypes.c_long * len(v))(*v)


def test_blocks_of_the_gradient(plan):
    rows = [1, 2, 3, 7, 8, 9, 31, 100, 147, 148, 149, 295, 1000, 8191, 100000, 2 ** 31 - 1]
    groups = [1, 2, 3, 17, 64, 147, 148, 149, 592, 1184, 1185, 100000]
    assert plan.bad_parts(longs(rows), len(rows), longs(groups), len(groups), 20000) == 0


def test_every_tile_once(plan):
    r = random.Random(5)
    for _ in range(5000):
        t0, t1 = (r.choice((0, 1, r.randint(0, 80), r.randint(0, 2000))) for _ in range(2))
        pairs = min(r.choice((1, 2, 3, 36, 73, 74)), max(1, t0 + t1))
        assert plan.bad_walk(t0, t1, r.choice((0, 0, 1, 2, 7, 300)), pairs) == 0
