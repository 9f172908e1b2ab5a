"""What the gradients of layer norm and the head's loss accept, and the scratch that they ask for, decided before anything touches the
device."""

import ctypes
import os
import subprocess

import pytest

from paper_2608_20818_b200 import binding as B

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_20818_b200", "csrc")
P = 1 << 20                     # an address that is never read


def layernorm_backward(rows, cols, per, nbytes, **change):
    a = dict(gy=P, ldgy=cols, h=P, ldh=cols, mean=P, rstd=P, w=P, ldw=cols, gh=None, ldgh=0, rows=rows, cols=cols, per=per, io=0, wfp32=0,
             one=0, p=0.0, seed=1, offset=0, counter=None, gr=P, ldgr=cols, gx=None, ldgx=0, gw=P, gb=P, scratch=P, nbytes=nbytes,
             stream=None)
    return B.lib().prm_layernorm_backward(*{**a, **change}.values())


@pytest.mark.parametrize("rows,cols,per,code", [
    (4000000, 64, 1, B.PRM_ERR_WORKSPACE), (1 << 28, 256, 1, B.PRM_ERR_WORKSPACE), ((1 << 30) - 1, 8, 1, B.PRM_ERR_WORKSPACE),
    (1 << 28, 100, 8, B.PRM_ERR_WORKSPACE), (1 << 30, 100000, 1, B.PRM_ERR_SHAPE), (2 ** 31 - 8, 64, 4, B.PRM_ERR_WORKSPACE), (2 ** 31 - 1, 8, 1, B.PRM_ERR_SHAPE),
])
def test_layernorm_gradient_takes_as_many_groups_as_a_launch_has_blocks(rows, cols, per, code):
    """No scratch is given, so that what is accepted ends there."""
    assert layernorm_backward(rows, cols, per, 0) == code


LINES = """
#include "train_plan.h"
using namespace prm;
// Sizes for which a launch would leave more lines than the scratch holds.
extern "C" long beyond(const long* rows, int n_rows, const long* groups, int n_groups, long most) {
  long bad = 0;
  for (long cols = 1; cols <= most; cols += cols < 100 ? 1 : 4)
    for (int i = 0; i < n_rows; ++i)
      for (int g = 0; g < n_groups; ++g)
        for (int turn : {1, 2, 4, 8, 16, 32})
          for (int blocks : {148, 296, 444, 592, 888, 1184})
            for (bool shift : {false, true}) {
              const long lines = layernorm_lines(rows[i], groups[g], cols);
              const long parts = layernorm_parts(rows[i], groups[g], cols, turn, blocks, shift);
              // rows that start anywhere and have whole octs: the launch goes by what there is
              bad += lines < 1 || (parts > lines && !(shift && cols % 8 == 0));
            }
  return bad;
}
"""


def test_layernorm_scratch_holds_what_a_launch_leaves(tmp_path):
    (tmp_path / "lines.cpp").write_text(LINES)
    so = str(tmp_path / "lines.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", CSRC, str(tmp_path / "lines.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.beyond.restype = ctypes.c_long
    lib.beyond.argtypes = [ctypes.POINTER(ctypes.c_long), ctypes.c_int, ctypes.POINTER(ctypes.c_long), ctypes.c_int, ctypes.c_long]
    rows = [1, 2, 3, 7, 8, 9, 31, 100, 148, 1000, 8191, 2 ** 31 - 1]
    groups = [1, 2, 3, 17, 37, 64, 147, 148, 149, 592, 1184, 1185, 100000]
    assert lib.beyond((ctypes.c_long * len(rows))(*rows), len(rows), (ctypes.c_long * len(groups))(*groups), len(groups), 20000) == 0


@pytest.mark.parametrize("groups,per,cols", [(1024, 8, 8192), (4096, 16, 4096), (64, 256, 2048), (1, 8192, 4096), (300, 200, 64)])
def test_layernorm_scratch_is_in_proportion(groups, per, cols):
    """No more than two fp32 lines for each block that a device holds, or for each group."""
    nbytes = B.lib().prm_layernorm_scratch_bytes(groups * per, cols, per)
    assert nbytes <= max(groups, 1184) * 2 * cols * 4


@pytest.mark.parametrize("n,d,vocab", [(4, 64, 128), (1000, 4096, 32768), (300, 100, 700)])
@pytest.mark.parametrize("ldx", [0, 1])
def test_head_gradient_without_the_weight_s_needs_no_copy_of_x(n, d, vocab, ldx):
    """One byte less than what the rest needs is refused; rows off 16 bytes are copied all the same."""
    L = B.lib()
    all_of, copy = L.prm_head_loss_backward_scratch_bytes(n, d, vocab), L.prm_head_loss_copy_bytes(n, d)
    assert 0 < copy < all_of
    need = all_of - copy + (copy if (d + ldx) % 8 else 0)

    def call(nbytes, gw=None, scratch=P):
        return L.prm_head_loss_backward(P, P, d + ldx, P, vocab + (-vocab) % 8, 0, P, P, n, d, vocab, P, d, gw, vocab, scratch, nbytes, None)

    assert call(need - 1) == B.PRM_ERR_WORKSPACE and call(need, gw=P) == B.PRM_ERR_WORKSPACE
