"""Pieces of the vocabulary and parts of k of the head's gradient, checked on the host from the header that the launches use."""

import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_20818_b200", "csrc")
SOURCE = """
#include "train_plan.h"
using namespace prm;
// What is wrong with the plan of a size, 0: nothing.
static int fault(long n, long d, long vocab) {
  const HeadGradPlan p = head_grad_plan(n, d, vocab);
  if (p.pieces < 1 || p.split < 1 || p.piece % kHeadTile || p.piece * (p.pieces - 1) >= vocab || p.piece * p.pieces < vocab) return 1;
  for (int piece : {0, 1, p.pieces - 2, p.pieces - 1}) {          // those between are as wide as these
    if (piece < 0 || piece >= p.pieces) continue;
    const long wide = std::min(p.piece, vocab - p.piece * piece);
    const int split = head_grad_split(p, wide), stages = (int)((wide + kHeadStage - 1) / kHeadStage);
    if (split < 1 || split > p.split || (piece == 0 && split != p.split)) return 2;
    int next = 0;
    for (int at = 0, s0, s1; at < split; ++at, next = s1) {
      head_part(stages, split, at, s0, s1);
      if (s0 != next || s1 <= s0) return 3;                       // a part without a stage, or stages left out
    }
    if (next != stages || wide > p.ld_g) return 4;
  }
  return p.g_bytes < (size_t)(n * p.ld_g * 2) || ((p.pieces > 1 || p.split > 1) && p.part_bytes < (size_t)(p.split * n * d * 4)) ? 5 : 0;
}
extern "C" {
int plan_fault(long n, long d, long vocab) { return fault(n, d, vocab); }
long pieces_of(long n, long d, long vocab) { return head_grad_plan(n, d, vocab).pieces; }
long split_of(long n, long d, long vocab) { return head_grad_plan(n, d, vocab).split; }
// The vocabularies first, first + step, ... of a size that have a fault.
long faults(long n, long d, long first, long last, long step) {
  long bad = 0;
  for (long v = first; v <= last; v += step) bad += fault(n, d, v) != 0;
  return bad;
}
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("head_plan")
    (d / "plan.cpp").write_text(SOURCE)
    so = str(d / "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", CSRC, str(d / "plan.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    for f in (lib.plan_fault, lib.pieces_of, lib.split_of, lib.faults):
        f.restype = ctypes.c_long
    lib.plan_fault.argtypes = lib.pieces_of.argtypes = lib.split_of.argtypes = [ctypes.c_long] * 3
    lib.faults.argtypes = [ctypes.c_long] * 5
    return lib


@pytest.mark.parametrize("n,d,vocab", [(9472, 256, 3069550), (9472, 64, 3069441), (9472, 256, 5350464), (8192, 256, 4161591),
                                       (8192, 64, 4161591), (8192, 256, 19595341)])
def test_a_last_piece_of_a_few_columns(plan, n, d, vocab):
    """Many pieces, parts of k, and a last piece with fewer stages than the others have parts."""
    assert plan.pieces_of(n, d, vocab) > 1 and plan.split_of(n, d, vocab) > 1
    assert plan.plan_fault(n, d, vocab) == 0


@pytest.mark.parametrize("n", [1, 2, 64, 100, 256, 257, 1000, 2048, 4096, 6000, 8192, 9472, 9473, 65536, 1 << 20, 1 << 27])
def test_every_part_has_a_stage(plan, n):
    """Sizes up to 2^27 each way, vocabularies one by one where they are small and around powers of two."""
    for d in (1, 64, 256, 257, 1024, 4096, 1 << 27):
        assert plan.faults(n, d, 1, 5000, 1) == 0
        assert plan.faults(n, d, 5000, 12000000, 10007) == 0
        assert plan.faults(n, d, 12000000, 1 << 27, 100003) == 0
        for k in range(12, 28):
            assert plan.faults(n, d, (1 << k) - 300, min((1 << k) + 300, 1 << 27), 1) == 0
