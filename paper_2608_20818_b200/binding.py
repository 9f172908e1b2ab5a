"""ctypes binding of the prm C ABI (include/prm.h).

Argument marshalling only: every arithmetic step runs in the CUDA library.
The functions carry the C names; `PeriodicRowwiseMuon` bundles a handle with
a torch-allocated workspace.  Loading fails loudly when libprm.so is missing;
there is no fallback path.
"""

from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int, c_int64, c_size_t, c_uint64, c_void_p

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libprm.so")

PRM_OK = 0
PRM_ERR_ARG = -1
PRM_ERR_SHAPE = -2
PRM_ERR_ALIGN = -3
PRM_ERR_WORKSPACE = -4
PRM_ERR_CUDA = -5
PRM_ERR_DEVICE_TIMEOUT = -6
PRM_ERR_STATE = -7

PRM_OPT_GAMMA = 1
PRM_OPT_EPS_ROW = 2
PRM_OPT_EPS_NS = 3
PRM_OPT_SCALE_MODE = 4
PRM_OPT_IO_DTYPE = 5
PRM_OPT_CHECK_MODE = 6
PRM_OPT_LR = 7
PRM_OPT_WD = 8
PRM_OPT_NS_WORKSPACE_BYTES = 9
PRM_OPT_GAMMA_NS = 10
PRM_OPT_NO_REFRESH = 11
PRM_OPT_NS_GRAM_SPAN = 12
PRM_OPT_TALL_KERNEL = 13
PRM_OPT_NS_SPLIT_INPUT = 14
PRM_OPT_WIDE_KERNEL = 15

PRM_Q8_INT8 = 0
PRM_Q8_E4M3 = 1

EXPORTS = (
    "prm_create", "prm_set_option", "prm_workspace_bytes", "prm_set_workspace", "prm_step",
    "prm_step_h2d", "prm_plan", "prm_status", "prm_last_error", "prm_launch_count", "prm_destroy",
    "prm_profile", "prm_profile_read", "prm_rowstep_tall_noalloc", "prm_selftest_timeout", "prm_adamw_step",
    "prm_tall_shard_scratch_bytes", "prm_tall_shard_stats", "prm_tall_shard_apply", "prm_group_info",
    "prm_shard_rows", "prm_bucket_plan", "prm_shard_momentum_pack", "prm_refresh_gathered", "prm_refresh_segments", "prm_pipeline_model",
    "prm_partition_matrices", "prm_shape_scale",
    "prm_rmsnorm_q8", "prm_rmsnorm_q8_scratch_bytes", "prm_rmsnorm_q8_backward",
    "prm_quantize_q8", "prm_quantize_q8_scratch_bytes", "prm_matmul_q8", "prm_q8_status",
    "prm_dropout", "prm_layernorm", "prm_layernorm_scratch_bytes", "prm_layernorm_backward",
    "prm_head_loss", "prm_head_loss_scratch_bytes", "prm_head_loss_copy_bytes", "prm_head_loss_backward", "prm_head_loss_backward_scratch_bytes",
)
PRM_PROF_ROW_WIDE, PRM_PROF_ROW_TALL, PRM_PROF_PREPASS, PRM_PROF_GRAM = 0, 1, 2, 3
PRM_PROF_POLY, PRM_PROF_UPDATE, PRM_PROF_UPDATE_FINAL, PRM_PROF_GRAMSPACE, PRM_PROF_COUNT = 4, 5, 6, 7, 8
PROF_NAMES = ("row_wide", "row_tall", "prepass", "gram", "poly", "update", "update_final", "gramspace")

_lib_handle = None


class PrmError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"prm error {code}: {msg}")
        self.code = code


def lib():
    """The loaded CUDA library.  Raises if it has not been built."""
    global _lib_handle
    if _lib_handle is not None:
        return _lib_handle
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} not found: build it with `python -m paper_2608_20818_b200.build` "
            "(nvcc, sm_100a). There is no CPU fallback.")
    L = ctypes.CDLL(LIB_PATH)
    L.prm_create.argtypes = [POINTER(c_void_p), POINTER(c_int64), c_int, c_int, c_float, c_int, c_float, c_float]
    L.prm_create.restype = c_int
    L.prm_set_option.argtypes = [c_void_p, c_int, c_double]
    L.prm_set_option.restype = c_int
    L.prm_workspace_bytes.argtypes = [c_void_p]
    L.prm_workspace_bytes.restype = c_size_t
    L.prm_set_workspace.argtypes = [c_void_p, c_void_p, c_size_t]
    L.prm_set_workspace.restype = c_int
    L.prm_step.argtypes = [c_void_p, POINTER(c_void_p), POINTER(c_void_p), POINTER(c_void_p), c_int64, c_void_p]
    L.prm_step.restype = c_int
    L.prm_step_h2d.argtypes = [c_void_p, POINTER(c_void_p), POINTER(c_void_p), POINTER(c_void_p),
                               POINTER(c_void_p), c_int64, c_void_p]
    L.prm_step_h2d.restype = c_int
    L.prm_plan.argtypes = [c_void_p, c_int64, POINTER(c_int), POINTER(c_int), POINTER(c_int), POINTER(c_int)]
    L.prm_plan.restype = c_int
    L.prm_group_info.argtypes = [c_void_p, c_int, POINTER(c_int64), POINTER(c_int64), POINTER(c_int), POINTER(c_int),
                                 POINTER(c_int), POINTER(c_double)]
    L.prm_group_info.restype = c_int
    L.prm_status.argtypes = [c_void_p]
    L.prm_status.restype = c_int
    L.prm_last_error.argtypes = [c_void_p]
    L.prm_last_error.restype = c_char_p
    L.prm_launch_count.argtypes = [c_void_p]
    L.prm_launch_count.restype = c_int64
    L.prm_destroy.argtypes = [c_void_p]
    L.prm_destroy.restype = c_int
    L.prm_profile.argtypes = [c_void_p, c_int]
    L.prm_profile.restype = c_int
    L.prm_profile_read.argtypes = [c_void_p, POINTER(c_double), POINTER(c_int64), c_int]
    L.prm_profile_read.restype = c_int
    L.prm_rowstep_tall_noalloc.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_int, c_float,
                                           c_int, c_float, c_float, c_float, c_float, c_float, c_void_p,
                                           c_char_p, c_size_t]
    L.prm_rowstep_tall_noalloc.restype = c_int
    L.prm_selftest_timeout.argtypes = [c_void_p, c_double, c_void_p]
    L.prm_selftest_timeout.restype = c_int
    L.prm_adamw_step.argtypes = [c_int, POINTER(c_void_p), POINTER(c_void_p), POINTER(c_void_p), POINTER(c_void_p),
                                 POINTER(c_int64), c_int, c_float, c_float, c_float, c_float, c_float, c_int64,
                                 c_void_p]
    L.prm_adamw_step.restype = c_int
    L.prm_tall_shard_scratch_bytes.argtypes = [c_int64, c_int64]
    L.prm_tall_shard_scratch_bytes.restype = c_size_t
    L.prm_tall_shard_stats.argtypes = [c_void_p, c_void_p, c_int64, c_int64, c_int, c_float, c_int, c_void_p, c_void_p,
                                       c_size_t, c_void_p]
    L.prm_tall_shard_stats.restype = c_int
    L.prm_tall_shard_apply.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_int, c_float, c_int, c_float,
                                       c_float, c_float, c_float, c_float, c_void_p, c_void_p]
    L.prm_tall_shard_apply.restype = c_int
    L.prm_shard_rows.argtypes = [c_int64, c_int, c_int, POINTER(c_int64), POINTER(c_int64)]
    L.prm_shard_rows.restype = c_int
    L.prm_bucket_plan.argtypes = [POINTER(c_int64), c_int, c_int, c_int64, POINTER(c_int), POINTER(c_int64),
                                  POINTER(c_int), POINTER(c_int64)]
    L.prm_bucket_plan.restype = c_int
    L.prm_shard_momentum_pack.argtypes = [c_void_p, c_void_p, c_int64, c_int64, c_int64, c_int, c_float, c_int,
                                          c_void_p, c_void_p]
    L.prm_shard_momentum_pack.restype = c_int
    L.prm_refresh_gathered.argtypes = [c_void_p, POINTER(c_int), c_int, c_void_p, c_int64, POINTER(c_int64), c_int,
                                       c_int, POINTER(c_void_p), c_void_p]
    L.prm_refresh_gathered.restype = c_int
    L.prm_refresh_segments.argtypes = [c_void_p, POINTER(c_int), c_int, POINTER(c_void_p), c_int64, POINTER(c_int64),
                                       c_int, c_int, POINTER(c_void_p), c_void_p]
    L.prm_refresh_segments.restype = c_int
    L.prm_pipeline_model.argtypes = [POINTER(c_double), POINTER(c_double), c_int, POINTER(c_double), POINTER(c_double)]
    L.prm_pipeline_model.restype = c_int
    L.prm_partition_matrices.argtypes = [POINTER(c_int64), c_int, c_int, POINTER(c_int), POINTER(c_double)]
    L.prm_partition_matrices.restype = c_int
    L.prm_shape_scale.argtypes = [c_int, c_int64, c_int64]
    L.prm_shape_scale.restype = c_double
    L.prm_rmsnorm_q8.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int, c_int,
                                 c_float, c_int, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p]
    L.prm_rmsnorm_q8.restype = c_int
    L.prm_rmsnorm_q8_scratch_bytes.argtypes = [c_int64, c_int64]
    L.prm_rmsnorm_q8_scratch_bytes.restype = c_size_t
    L.prm_rmsnorm_q8_backward.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_int64,
                                          c_int64, c_int, c_int, c_float, c_void_p, c_int64, c_void_p, c_void_p,
                                          c_size_t, c_void_p]
    L.prm_rmsnorm_q8_backward.restype = c_int
    L.prm_quantize_q8_scratch_bytes.argtypes = [c_int64, c_int64]
    L.prm_quantize_q8_scratch_bytes.restype = c_size_t
    L.prm_quantize_q8.argtypes = [c_void_p, c_int64, c_int64, c_int64, c_int, c_int, c_void_p, c_void_p, c_void_p,
                                  c_int64, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_size_t, c_void_p]
    L.prm_quantize_q8.restype = c_int
    L.prm_matmul_q8.argtypes = [c_void_p, c_int64, c_int, c_void_p, c_void_p, c_int64, c_int, c_void_p, c_int64,
                                c_int64, c_int64, c_int, c_void_p, c_int64, c_int, c_void_p]
    L.prm_matmul_q8.restype = c_int
    L.prm_q8_status.argtypes = []
    L.prm_q8_status.restype = c_int
    draw = [c_double, c_uint64, c_uint64, c_void_p]          # p, seed, offset, counter
    L.prm_dropout.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int64, c_int, *draw, c_void_p, c_int64, c_void_p]
    L.prm_dropout.restype = c_int
    L.prm_layernorm.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int64,
                                c_int64, c_int, c_int, c_int, c_float, *draw, c_void_p, c_int64, c_void_p, c_int64,
                                c_void_p, c_void_p, c_void_p]
    L.prm_layernorm.restype = c_int
    L.prm_layernorm_scratch_bytes.argtypes = [c_int64, c_int64, c_int64]
    L.prm_layernorm_scratch_bytes.restype = c_size_t
    L.prm_layernorm_backward.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int64,
                                         c_void_p, c_int64, c_int64, c_int64, c_int64, c_int, c_int, c_int, *draw,
                                         c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_size_t,
                                         c_void_p]
    L.prm_layernorm_backward.restype = c_int
    for name in ("prm_head_loss_scratch_bytes", "prm_head_loss_backward_scratch_bytes"):
        getattr(L, name).argtypes = [c_int64, c_int64, c_int64]
        getattr(L, name).restype = c_size_t
    L.prm_head_loss_copy_bytes.argtypes = [c_int64, c_int64]
    L.prm_head_loss_copy_bytes.restype = c_size_t
    L.prm_head_loss.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_int, c_void_p, c_int64, c_int64, c_int64, c_void_p,
                                c_void_p, c_void_p, c_size_t, c_void_p]
    L.prm_head_loss.restype = c_int
    L.prm_head_loss_backward.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_int, c_void_p, c_void_p, c_int64,
                                         c_int64, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_size_t, c_void_p]
    L.prm_head_loss_backward.restype = c_int
    _lib_handle = L
    return L


def _check(code, handle=None):
    if code != PRM_OK:
        msg = lib().prm_last_error(handle)
        raise PrmError(code, msg.decode() if msg else "")


def prm_create(shapes, K, beta, nesterov, lr, wd):
    flat = []
    for (m, n) in shapes:
        flat += [int(m), int(n)]
    arr = (c_int64 * max(1, len(flat)))(*flat)
    h = c_void_p()
    _check(lib().prm_create(byref(h), arr, len(shapes), int(K), float(beta), int(bool(nesterov)), float(lr), float(wd)))
    return h


def prm_set_option(h, key, value):
    _check(lib().prm_set_option(h, int(key), float(value)), h)


def prm_workspace_bytes(h):
    return int(lib().prm_workspace_bytes(h))


def prm_set_workspace(h, dev_ptr, nbytes):
    _check(lib().prm_set_workspace(h, c_void_p(dev_ptr), nbytes), h)


def _ptr_array(tensors):
    return (c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def prm_step(h, params, grads, momentum, step_idx, stream=0):
    """params/grads/momentum: ctypes arrays of device pointers (see ptr_arrays)."""
    _check(lib().prm_step(h, params, grads, momentum, int(step_idx), c_void_p(stream)), h)


def prm_step_h2d(h, params, grads_dev, grads_host, momentum, step_idx, stream=0):
    _check(lib().prm_step_h2d(h, params, grads_dev, grads_host, momentum, int(step_idx), c_void_p(stream)), h)


def prm_plan(h, step_idx, n_mats):
    is_refresh, n_groups = c_int(), c_int()
    g = (c_int * n_mats)()
    o = (c_int * n_mats)()
    _check(lib().prm_plan(h, int(step_idx), byref(is_refresh), byref(n_groups), g, o), h)
    return bool(is_refresh.value), n_groups.value, list(g), list(o)


def prm_group_info(h, group):
    """{rows, cols, count, ns_batch, gram_iters, ns5_flop} of one shape group."""
    rows, cols = c_int64(), c_int64()
    count, ns_batch, gram_iters = c_int(), c_int(), c_int()
    flop = c_double()
    _check(lib().prm_group_info(h, int(group), byref(rows), byref(cols), byref(count), byref(ns_batch),
                                byref(gram_iters), byref(flop)), h)
    return {"rows": rows.value, "cols": cols.value, "count": count.value, "ns_batch": ns_batch.value,
            "gram_iters": gram_iters.value, "ns5_flop": flop.value}


def prm_status(h):
    return int(lib().prm_status(h))


def prm_last_error(h):
    msg = lib().prm_last_error(h)
    return msg.decode() if msg else ""


def prm_launch_count(h):
    return int(lib().prm_launch_count(h))


def prm_profile(h, enable):
    _check(lib().prm_profile(h, int(bool(enable))), h)


def prm_profile_read(h):
    ms = (c_double * PRM_PROF_COUNT)()
    n = (c_int64 * PRM_PROF_COUNT)()
    _check(lib().prm_profile_read(h, ms, n, PRM_PROF_COUNT), h)
    return {name: (ms[i], n[i]) for i, name in enumerate(PROF_NAMES)}


def prm_rowstep_tall_noalloc(param, grad, momentum, *, beta, nesterov, lr, wd, gamma, eps_row, scale,
                             stream=None):
    """Row step of one tall matrix for callers that cannot allocate device
    memory (no workspace, no handle): the scratch sits in a fixed array inside
    the library.  Tensors are updated in place; see include/prm.h for the size
    limit and the sharing rules of that array."""
    if len(param.shape) != 2:
        raise ValueError("param must be a 2-D matrix")
    rows, cols = param.shape
    if param.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("param must be float32 or bfloat16")
    if grad.dtype != param.dtype or momentum.dtype != torch.float32:
        raise TypeError(f"dtypes must be {param.dtype} (param, grad) and float32 (momentum)")
    if tuple(grad.shape) != tuple(param.shape) or tuple(momentum.shape) != tuple(param.shape):
        raise ValueError("param, grad and momentum must have the same shape")
    if not (param.is_contiguous() and grad.is_contiguous() and momentum.is_contiguous()):
        raise ValueError("param, grad and momentum must be contiguous")
    if param.device.type != "cuda" or grad.device != param.device or momentum.device != param.device:
        raise ValueError("param, grad and momentum must sit on the same CUDA device")
    io_fp32 = 1 if param.dtype == torch.float32 else 0
    s = (stream or torch.cuda.current_stream(param.device)).cuda_stream
    buf = ctypes.create_string_buffer(256)
    with torch.cuda.device(param.device):
        code = lib().prm_rowstep_tall_noalloc(
            c_void_p(param.data_ptr()), c_void_p(grad.data_ptr()), c_void_p(momentum.data_ptr()),
            int(rows), int(cols), io_fp32, float(beta), int(bool(nesterov)), float(lr), float(wd),
            float(gamma), float(eps_row), float(scale), c_void_p(s), buf, 256)
    if code != PRM_OK:
        raise PrmError(code, buf.value.decode())


def prm_selftest_timeout(h, limit_ms, stream=0):
    _check(lib().prm_selftest_timeout(h, float(limit_ms), c_void_p(stream)), h)


def prm_adamw_step(params, grads, exp_avg, exp_avg_sq, step, *, lr=1e-4, beta1=0.9, beta2=0.95, eps=1e-8, wd=0.01,
                   stream=None):
    """AdamW on a list of device tensors of any shape (the parameters outside
    the Muon set), in place; step is the 1-based step count."""
    n = len(params)
    if n == 0:
        return
    io_fp32 = 1 if params[0].dtype == torch.float32 else 0
    numel = (c_int64 * n)(*[p.numel() for p in params])
    s = (stream or torch.cuda.current_stream(params[0].device)).cuda_stream
    with torch.cuda.device(params[0].device):
        code = lib().prm_adamw_step(n, _ptr_array(params), _ptr_array(grads), _ptr_array(exp_avg),
                                    _ptr_array(exp_avg_sq), numel, io_fp32, float(lr), float(beta1), float(beta2),
                                    float(eps), float(wd), int(step), c_void_p(s))
    if code != PRM_OK:
        raise PrmError(code, "prm_adamw_step failed")


def prm_shard_rows(rows, world, rank):
    """(row_start, row_count) of one rank's dim-0 shard."""
    start, count = c_int64(), c_int64()
    code = lib().prm_shard_rows(int(rows), int(world), int(rank), byref(start), byref(count))
    if code != PRM_OK:
        raise PrmError(code, "prm_shard_rows: bad argument")
    return start.value, count.value


def prm_bucket_plan(shapes, world, bucket_bytes):
    """(bucket_of_mat, offset_in_segment, segment_elems per bucket)."""
    n = len(shapes)
    flat = []
    for (m, k) in shapes:
        flat += [int(m), int(k)]
    arr = (c_int64 * max(1, len(flat)))(*flat)
    bucket = (c_int * max(1, n))()
    off = (c_int64 * max(1, n))()
    seg = (c_int64 * max(1, n))()
    nb = c_int()
    code = lib().prm_bucket_plan(arr, n, int(world), int(bucket_bytes), bucket, off, byref(nb), seg)
    if code != PRM_OK:
        raise PrmError(code, "prm_bucket_plan: bad argument")
    return list(bucket)[:n], list(off)[:n], list(seg)[:nb.value]


def prm_shard_momentum_pack(grad_shard, momentum_shard, cols, reserved_elems, beta, nesterov, u_out_ptr, stream=None):
    """grad_shard, momentum_shard: (rows_local, cols) CUDA tensors (rows_local may be 0)."""
    rows_local = int(grad_shard.shape[0])
    s = stream if stream is not None else torch.cuda.current_stream(grad_shard.device).cuda_stream
    with torch.cuda.device(grad_shard.device):
        code = lib().prm_shard_momentum_pack(c_void_p(grad_shard.data_ptr()), c_void_p(momentum_shard.data_ptr()),
                                             rows_local, int(cols), int(reserved_elems),
                                             1 if grad_shard.dtype == torch.float32 else 0, float(beta),
                                             int(bool(nesterov)), c_void_p(int(u_out_ptr)), c_void_p(s))
    if code != PRM_OK:
        raise PrmError(code, "prm_shard_momentum_pack failed")


def prm_refresh_gathered(h, mats, gathered_ptr, segment_elems, offsets, world, rank, param_shard_ptrs, stream):
    n = len(mats)
    m = (c_int * max(1, n))(*[int(x) for x in mats])
    o = (c_int64 * max(1, n))(*[int(x) for x in offsets])
    p = (c_void_p * max(1, n))(*[c_void_p(int(x)) if x else None for x in param_shard_ptrs])
    _check(lib().prm_refresh_gathered(h, m, n, c_void_p(int(gathered_ptr)), int(segment_elems), o, int(world),
                                      int(rank), p, c_void_p(stream)), h)


def prm_refresh_segments(h, mats, segment_ptrs, segment_elems, offsets, world, rank, param_shard_ptrs, stream):
    """segment_ptrs: one device pointer per rank (local or peer-mapped memory)."""
    n = len(mats)
    m = (c_int * max(1, n))(*[int(x) for x in mats])
    o = (c_int64 * max(1, n))(*[int(x) for x in offsets])
    p = (c_void_p * max(1, n))(*[c_void_p(int(x)) if x else None for x in param_shard_ptrs])
    sp = (c_void_p * max(1, int(world)))(*[c_void_p(int(x)) for x in segment_ptrs])
    _check(lib().prm_refresh_segments(h, m, n, sp, int(segment_elems), o, int(world), int(rank), p,
                                      c_void_p(stream)), h)


def prm_pipeline_model(a, c):
    """(t_pipe, t_comm_exposed) of the ideal two-stage pipeline."""
    n = len(a)
    if n != len(c) or n < 1:
        raise ValueError("a and c must have the same, positive length")
    aa = (c_double * n)(*[float(x) for x in a])
    cc = (c_double * n)(*[float(x) for x in c])
    tp, te = c_double(), c_double()
    code = lib().prm_pipeline_model(aa, cc, n, byref(tp), byref(te))
    if code != PRM_OK:
        raise PrmError(code, "prm_pipeline_model: bad argument")
    return tp.value, te.value


def prm_partition_matrices(shapes, world):
    """(owner_of_mat, flop per rank): whole matrices assigned to ranks."""
    n = len(shapes)
    flat = []
    for (m, k) in shapes:
        flat += [int(m), int(k)]
    arr = (c_int64 * max(1, len(flat)))(*flat)
    owner = (c_int * max(1, n))()
    cost = (c_double * max(1, int(world)))()
    code = lib().prm_partition_matrices(arr, n, int(world), owner, cost)
    if code != PRM_OK:
        raise PrmError(code, "prm_partition_matrices: bad argument")
    return list(owner)[:n], list(cost)[:int(world)]


def prm_shape_scale(mode, rows, cols):
    """s(W) for a stored rows x cols matrix under PRM_OPT_SCALE_MODE `mode`."""
    v = float(lib().prm_shape_scale(int(mode), int(rows), int(cols)))
    if v == 0.0:
        raise PrmError(PRM_ERR_ARG, "prm_shape_scale: bad argument")
    return v


_Q8_FORMAT = {"int8": (PRM_Q8_INT8, torch.int8), "e4m3": (PRM_Q8_E4M3, torch.float8_e4m3fn)}
_Q8_CODE = {torch.int8: PRM_Q8_INT8, torch.float8_e4m3fn: PRM_Q8_E4M3}
_IO_FP32 = {torch.bfloat16: 0, torch.float32: 1}


# The 8-bit operators below are called many times per training step, on small matrices too, where the
# time on the host is what a call costs: their checks are written out on attributes that are cheap to
# read, and the reasons for a refusal are worked out by helpers that a good call does not reach.

def _on_stream(stream, inputs, call):
    """Runs call() with `stream` current, so that what it allocates belongs to that stream, and
    keeps the inputs' memory from being handed out again before the stream is done with it."""
    with torch.cuda.stream(stream):
        out = call()
    for t in inputs:
        if t is not None:
            t.record_stream(stream)
    return out


def _raw_stream(index):
    return torch._C._cuda_getCurrentRawStream(index)


def _on_device(index, fn, *args):
    """fn(*args) with device `index` current (callers test whether it is already)."""
    with torch.cuda.device(index):
        return fn(*args)


def _refuse_matrix(t, name, like):
    if t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D matrix")
    if not t.is_cuda:
        raise ValueError(f"{name} must sit on a CUDA device")
    if t.dtype not in _IO_FP32:
        raise TypeError(f"{name} must be bfloat16 or float32")
    if like is not None:
        if t.dtype != like.dtype:
            raise TypeError(f"{name} must be {like.dtype} like the matrix it goes with")
        if t.shape != like.shape:
            raise ValueError(f"{name} must have the shape {tuple(like.shape)}")
        raise ValueError(f"{name} must sit on {like.device}")


def _matrix(t, name, like=None):
    """t, a 2-D bf16 or fp32 CUDA tensor (of the type, shape and device of `like`) whose rows are
    contiguous; copied if they are not."""
    if like is None:
        if not t.is_cuda or t.dtype not in _IO_FP32 or t.dim() != 2:
            _refuse_matrix(t, name, like)
    elif t.dtype is not like.dtype or t.shape != like.shape or t.get_device() != like.get_device():
        _refuse_matrix(t, name, like)
    return t if t.stride(1) == 1 or t.shape[1] == 1 else t.contiguous()


def _refuse_vector(t, name, n, index, dtypes):
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be one of {tuple(dtypes)}")
    if t.dim() != 1 or t.shape[0] != n:
        raise ValueError(f"{name} must be a vector of {n} elements")
    raise ValueError(f"{name} must sit on cuda:{index}")


_FP32_ONLY = {torch.float32: 1}


def _vector(t, name, n, index, dtypes=_FP32_ONLY):
    """t, a contiguous vector of n elements on device `index` (copied if it is strided)."""
    if t.dtype not in dtypes or t.shape != (n,) or t.get_device() != index:
        _refuse_vector(t, name, n, index, dtypes)
    return t if n <= 1 or t.stride(0) == 1 else t.contiguous()


def _codes(rows, cols, dtype, device):
    """An uninitialised matrix of 8-bit codes whose rows start a multiple of 16 bytes apart."""
    return torch.empty_strided((rows, cols), ((cols + 15) // 16 * 16, 1), dtype=dtype, device=device)


def _format(format):
    try:
        return _Q8_FORMAT[format]
    except KeyError:
        raise ValueError('format must be "int8" or "e4m3"') from None


def _q8_check(code, what):
    raise PrmError(code, f"{what} failed (see include/prm.h for its limits)")


def prm_rmsnorm_q8(x, weight, eps, residual=None, format="int8", stream=None):
    """Root-mean-square norm of x (+ residual) in 8 bits: (codes, scale per row, h).

    x, residual: rows x cols, bf16 or fp32; weight: cols, bf16 or fp32; format "int8" or "e4m3".
    h = x + residual in x's type is what the norm is taken of and what the stream carries on; it is
    None without a residual (h = x).  codes * scale[:, None] is the norm's output."""
    if stream is not None:
        return _on_stream(stream, (x, weight, residual),
                          lambda: prm_rmsnorm_q8(x, weight, eps, residual, format))
    fmt, dtype = _format(format)
    x = _matrix(x, "x")
    rows, cols = x.shape
    index = x.get_device()
    device = x.device
    weight = _vector(weight, "weight", cols, index, _IO_FP32)
    if residual is not None:
        residual = _matrix(residual, "residual", x)
        h = torch.empty_strided((rows, cols), (cols, 1), dtype=x.dtype, device=device)
        r_ptr, ld_r, h_ptr = residual.data_ptr(), residual.stride(0), h.data_ptr()
    else:
        h = r_ptr = h_ptr = None
        ld_r = 0
    q = _codes(rows, cols, dtype, device)
    scale = torch.empty_strided((rows,), (1,), dtype=torch.float32, device=device)
    args = (x.data_ptr(), x.stride(0), r_ptr, ld_r, weight.data_ptr(), rows, cols, _IO_FP32[x.dtype],
            _IO_FP32[weight.dtype], eps, fmt, h_ptr, cols, q.data_ptr(), q.stride(0), scale.data_ptr(),
            _raw_stream(index))
    fn = (_lib_handle or lib()).prm_rmsnorm_q8
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_rmsnorm_q8")
    return q, scale, h


def prm_rmsnorm_q8_backward(grad_y, h, weight, eps, grad_h=None, stream=None):
    """Gradient of the norm at h (the sum that prm_rmsnorm_q8 returned, or its x without a residual):
    (grad_x, grad_weight).  grad_x is the gradient of x and of the residual alike; grad_h, if given,
    is what reaches h along the residual stream and is added to it."""
    if stream is not None:
        return _on_stream(stream, (grad_y, h, weight, grad_h),
                          lambda: prm_rmsnorm_q8_backward(grad_y, h, weight, eps, grad_h))
    h = _matrix(h, "h")
    grad_y = _matrix(grad_y, "grad_y", h)
    rows, cols = h.shape
    index = h.get_device()
    device = h.device
    weight = _vector(weight, "weight", cols, index, _IO_FP32)
    if grad_h is not None:
        grad_h = _matrix(grad_h, "grad_h", h)
        gh_ptr, ld_gh = grad_h.data_ptr(), grad_h.stride(0)
    else:
        gh_ptr, ld_gh = None, 0
    L = _lib_handle or lib()
    nbytes = L.prm_rmsnorm_q8_scratch_bytes(rows, cols)
    grad_x = torch.empty_strided((rows, cols), (cols, 1), dtype=h.dtype, device=device)
    grad_w = torch.empty_strided((cols,), (1,), dtype=weight.dtype, device=device)
    scratch = torch.empty_strided((nbytes,), (1,), dtype=torch.uint8, device=device)
    args = (grad_y.data_ptr(), grad_y.stride(0), h.data_ptr(), h.stride(0), weight.data_ptr(), gh_ptr, ld_gh, rows, cols,
            _IO_FP32[h.dtype], _IO_FP32[weight.dtype], eps, grad_x.data_ptr(), cols, grad_w.data_ptr(),
            scratch.data_ptr(), nbytes, _raw_stream(index))
    fn = L.prm_rmsnorm_q8_backward
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_rmsnorm_q8_backward")
    return grad_x, grad_w


def prm_quantize_q8(x, *, by_rows=True, by_cols=False, fold_rows=None, fold_cols=None, format="int8", stream=None):
    """8-bit codes of a bf16 or fp32 matrix: (codes by row, scale per row, codes by column, scale per
    column), None for what was not asked for.  By row it quantises x * fold_cols, by column
    x * fold_rows[:, None] (fp32 vectors, optional)."""
    if stream is not None:
        return _on_stream(stream, (x, fold_rows, fold_cols),
                          lambda: prm_quantize_q8(x, by_rows=by_rows, by_cols=by_cols, fold_rows=fold_rows,
                                                  fold_cols=fold_cols, format=format))
    fmt, dtype = _format(format)
    if not by_rows and not by_cols:
        raise ValueError("ask for codes by rows, by columns, or both")
    x = _matrix(x, "x")
    rows, cols = x.shape
    index = x.get_device()
    device = x.device
    fr_ptr = fc_ptr = None
    if fold_rows is not None:
        fold_rows = _vector(fold_rows, "fold_rows", rows, index)
        fr_ptr = fold_rows.data_ptr()
    if fold_cols is not None:
        fold_cols = _vector(fold_cols, "fold_cols", cols, index)
        fc_ptr = fold_cols.data_ptr()
    L = _lib_handle or lib()
    qr = sr = qc = sc = qr_ptr = sr_ptr = qc_ptr = sc_ptr = scratch_ptr = None
    ld = (cols + 15) // 16 * 16
    nbytes = 0
    if by_rows:
        qr = _codes(rows, cols, dtype, device)
        sr = torch.empty_strided((rows,), (1,), dtype=torch.float32, device=device)
        qr_ptr, sr_ptr = qr.data_ptr(), sr.data_ptr()
    if by_cols:
        qc = _codes(rows, cols, dtype, device)
        sc = torch.empty_strided((cols,), (1,), dtype=torch.float32, device=device)
        nbytes = L.prm_quantize_q8_scratch_bytes(rows, cols)
        scratch = torch.empty_strided((nbytes,), (1,), dtype=torch.uint8, device=device)
        qc_ptr, sc_ptr, scratch_ptr = qc.data_ptr(), sc.data_ptr(), scratch.data_ptr()
    if rows == 0:                       # nothing to point at: columns without an element have the scale 0
        return qr, sr, qc, None if sc is None else sc.zero_()
    args = (x.data_ptr(), x.stride(0), rows, cols, _IO_FP32[x.dtype], fmt, fr_ptr, fc_ptr, qr_ptr, ld, sr_ptr, qc_ptr, ld,
            sc_ptr, scratch_ptr, nbytes, _raw_stream(index))
    fn = L.prm_quantize_q8
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_quantize_q8")
    return qr, sr, qc, sc


def _q8_operand(t, r, c):
    """(matrix, its row stride, 1 if it is stored the other way round) as prm_matmul_q8 reads it;
    a matrix that lies in neither way, or unaligned, is copied."""
    s0, s1 = t.stride()
    if t.data_ptr() & 15 == 0:
        if s1 == 1 or c == 1:
            ld = s0 if r > 1 else (c + 15) // 16 * 16
            if ld & 15 == 0 and ld >= c:
                return t, ld, 0
        if s0 == 1 or r == 1:
            ld = s1 if c > 1 else (r + 15) // 16 * 16
            if ld & 15 == 0 and ld >= r:
                return t, ld, 1
    laid = _codes(r, c, t.dtype, t.device)
    laid.copy_(t)
    return laid, (c + 15) // 16 * 16, 0


def _refuse_product(a, b):
    if a.dim() != 2 or b.dim() != 2 or a.shape[1] != b.shape[0]:
        raise ValueError("a must be m x k and b k x n")
    if a.dtype not in _Q8_CODE or b.dtype != a.dtype:
        raise TypeError("a and b must both be int8 or both float8_e4m3fn")
    raise ValueError("a and b must sit on the same CUDA device")


def prm_matmul_q8(a, scale_a, b, scale_b, out_dtype=torch.bfloat16, out=None, stream=None):
    """(a @ b) * scale_a[:, None] * scale_b for 8-bit codes a (m x k) and b (k x n), both int8 or both
    float8_e4m3fn; a scale may be None.  Either operand may be a transposed view (`w.t()`).  Returns
    out: m x n, bf16 or fp32, a new matrix unless one with contiguous rows is given."""
    if stream is not None:
        return _on_stream(stream, (a, scale_a, b, scale_b, out),
                          lambda: prm_matmul_q8(a, scale_a, b, scale_b, out_dtype, out))
    index = a.get_device()
    fmt = _Q8_CODE.get(a.dtype)
    if (fmt is None or b.dtype is not a.dtype or index < 0 or b.get_device() != index or a.dim() != 2 or b.dim() != 2
            or a.shape[1] != b.shape[0]):
        _refuse_product(a, b)
    m, k = a.shape
    n = b.shape[1]
    sa_ptr = sb_ptr = None
    if scale_a is not None:
        scale_a = _vector(scale_a, "scale_a", m, index)
        sa_ptr = scale_a.data_ptr()
    if scale_b is not None:
        scale_b = _vector(scale_b, "scale_b", n, index)
        sb_ptr = scale_b.data_ptr()
    if out is None:
        if out_dtype not in _IO_FP32:
            raise TypeError("out_dtype must be bfloat16 or float32")
        out = torch.empty_strided((m, n), (n, 1), dtype=out_dtype, device=a.device)
        ld_out = n
    else:
        out_dtype = out.dtype
        if out_dtype not in _IO_FP32:
            raise TypeError("out must be bfloat16 or float32")
        if out.shape != (m, n) or out.get_device() != index:
            raise ValueError(f"out must be a {m} x {n} matrix on cuda:{index}")
        if n > 1 and out.stride(1) != 1 or m > 1 and out.stride(0) < n:
            raise ValueError("the rows of out must be contiguous and must not overlap")
        ld_out = out.stride(0) if m > 1 else n
    a, ld_a, a_t = _q8_operand(a, m, k)
    b, ld_b, b_t = _q8_operand(b, k, n)
    args = (a.data_ptr(), ld_a, a_t, sa_ptr, b.data_ptr(), ld_b, b_t, sb_ptr, m, k, n, fmt, out.data_ptr(), ld_out,
            _IO_FP32[out_dtype], _raw_stream(index))
    fn = (_lib_handle or lib()).prm_matmul_q8
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_matmul_q8")
    return out


def prm_q8_status():
    return int(lib().prm_q8_status())


# Operators of a training step around its products: dropout, layer norm, the loss of a linear head.

_INT64_ONLY = {torch.int64: 1}
_WORD = (1 << 64) - 1


def _draw(p, counter, index):
    """The counter's address; refuses what is no probability, and a counter that the kernel cannot read."""
    if not 0.0 <= p < 1.0:
        raise ValueError("p must be at least 0 and below 1")
    if counter is None:
        return None
    if counter.dtype is not torch.int64 or counter.numel() != 1 or counter.get_device() != index:
        raise ValueError(f"counter must be one int64 on cuda:{index}")
    return counter.data_ptr()


def prm_dropout(x, p, seed, offset=0, counter=None, residual=None, stream=None):
    """x (rows x cols, bf16 or fp32) with its elements dropped with probability p and the others divided by
    1 - p, plus residual.  Which ones is decided by seed, row, column and the number offset + counter (one
    int64 on the device): the same call on a gradient is the gradient."""
    if stream is not None:
        return _on_stream(stream, (x, counter, residual), lambda: prm_dropout(x, p, seed, offset, counter, residual))
    x = _matrix(x, "x")
    rows, cols = x.shape
    index = x.get_device()
    c_ptr = _draw(p, counter, index)
    r_ptr, ld_r = None, 0
    if residual is not None:
        residual = _matrix(residual, "residual", x)
        r_ptr, ld_r = residual.data_ptr(), residual.stride(0)
    out = torch.empty_strided((rows, cols), (cols, 1), dtype=x.dtype, device=x.device)
    args = (x.data_ptr(), x.stride(0), r_ptr, ld_r, rows, cols, _IO_FP32[x.dtype], p, seed & _WORD, offset & _WORD, c_ptr,
            out.data_ptr(), cols, _raw_stream(index))
    fn = (_lib_handle or lib()).prm_dropout
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_dropout")
    return out


def _affine(t, name, rows, cols, index, like=None):
    """(t, row stride, groups) of a scale or shift: a vector of cols, or groups x cols with groups dividing rows."""
    if t.shape == (cols,) and t.get_device() == index and t.is_contiguous() and (
            t.dtype in _IO_FP32 if like is None else t.dtype is like.dtype and t.shape == like.shape):
        return t, cols, 1
    if t.dtype not in _IO_FP32:
        raise TypeError(f"{name} must be bfloat16 or float32")
    if t.dim() not in (1, 2) or t.shape[-1] != cols or t.get_device() != index:
        raise ValueError(f"{name} must have {cols} columns, in one or two dimensions, on cuda:{index}")
    if like is not None and (t.dtype is not like.dtype or t.shape != like.shape):
        raise ValueError(f"{name} must have the weight's type and shape")
    groups = t.shape[0] if t.dim() == 2 else 1
    if groups == 0 or rows % groups:
        raise ValueError(f"{name}'s rows must divide the {rows} rows of the stream")
    if cols > 1 and t.stride(-1) != 1:
        t = t.contiguous()
    return t, t.stride(0) if t.dim() == 2 else cols, groups


def prm_layernorm(x, weight=None, bias=None, eps=1e-6, residual=None, add_one=False, p=0.0, seed=0, offset=0, counter=None,
                  stream=None):
    """Layer norm of h = x (dropped out with probability p, see prm_dropout) + residual: (y, h, mean, rstd).

    x, residual: rows x cols, bf16 or fp32.  weight, bias: cols, or groups x cols (each row of them for rows /
    groups neighbouring rows), bf16 or fp32, both in one shape and type, a bias without a weight: cols; add_one takes 1 + weight.
    h, in x's type, is what the norm is taken of and what the stream carries on; it is None where it is x itself.  mean and
    rstd (fp32) go to the gradient."""
    if stream is not None:
        return _on_stream(stream, (x, weight, bias, residual, counter),
                          lambda: prm_layernorm(x, weight, bias, eps, residual, add_one, p, seed, offset, counter))
    x = _matrix(x, "x")
    rows, cols = x.shape
    index = x.get_device()
    device = x.device
    c_ptr = None if p == 0 else _draw(p, counter, index)
    w_ptr = b_ptr = r_ptr = h_ptr = h = None
    ld_w = ld_b = ld_r = w_fp32 = 0
    groups = 1
    if weight is not None:
        weight, ld_w, groups = _affine(weight, "weight", rows, cols, index)
        w_ptr, w_fp32 = weight.data_ptr(), _IO_FP32[weight.dtype]
    if bias is not None:
        if weight is None and bias.dim() != 1:
            raise ValueError("a bias without a weight must be a vector")
        bias, ld_b, groups = _affine(bias, "bias", rows, cols, index, weight)
        b_ptr, w_fp32 = bias.data_ptr(), _IO_FP32[bias.dtype]
    if residual is not None:
        residual = _matrix(residual, "residual", x)
        r_ptr, ld_r = residual.data_ptr(), residual.stride(0)
    if residual is not None or p > 0:
        h = torch.empty_strided((rows, cols), (cols, 1), dtype=x.dtype, device=device)
        h_ptr = h.data_ptr()
    y = torch.empty_strided((rows, cols), (cols, 1), dtype=x.dtype, device=device)
    mean = torch.empty_strided((rows,), (1,), dtype=torch.float32, device=device)
    rstd = torch.empty_strided((rows,), (1,), dtype=torch.float32, device=device)
    args = (x.data_ptr(), x.stride(0), r_ptr, ld_r, w_ptr, ld_w, b_ptr, ld_b, rows, cols, max(1, rows // groups),
            _IO_FP32[x.dtype], w_fp32, 1 if add_one else 0, eps, p, seed & _WORD, offset & _WORD, c_ptr, h_ptr, cols,
            y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(), _raw_stream(index))
    fn = (_lib_handle or lib()).prm_layernorm
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_layernorm")
    return y, h, mean, rstd


def prm_layernorm_backward(grad_y, h, mean, rstd, weight=None, grad_h=None, add_one=False, p=0.0, seed=0, offset=0,
                           counter=None, need_weight=True, need_bias=True, stream=None):
    """Gradient of the layer norm at h (what prm_layernorm returned, or its x) with the forward call's p, seed,
    offset and counter: (grad_x, grad_residual, grad_weight, grad_bias).  grad_residual is None without
    dropout: it is grad_x.  grad_h, if given, is what reaches h along the residual stream.  grad_weight and
    grad_bias have weight's shape and type (without a weight they are fp32 vectors)."""
    if stream is not None:
        return _on_stream(stream, (grad_y, h, mean, rstd, weight, grad_h, counter),
                          lambda: prm_layernorm_backward(grad_y, h, mean, rstd, weight, grad_h, add_one, p, seed, offset,
                                                         counter, need_weight, need_bias))
    h = _matrix(h, "h")
    grad_y = _matrix(grad_y, "grad_y", h)
    rows, cols = h.shape
    index = h.get_device()
    device = h.device
    c_ptr = None if p == 0 else _draw(p, counter, index)
    mean = _vector(mean, "mean", rows, index)
    rstd = _vector(rstd, "rstd", rows, index)
    w_ptr = gh_ptr = gx_ptr = gw_ptr = gb_ptr = grad_x = grad_w = grad_b = None
    ld_w = ld_gh = 0
    groups, w_dtype, w_shape = 1, torch.float32, (cols,)
    if weight is not None:
        w_shape = weight.shape
        weight, ld_w, groups = _affine(weight, "weight", rows, cols, index)
        w_ptr, w_dtype = weight.data_ptr(), weight.dtype
    if grad_h is not None:
        grad_h = _matrix(grad_h, "grad_h", h)
        gh_ptr, ld_gh = grad_h.data_ptr(), grad_h.stride(0)
    grad_r = torch.empty_strided((rows, cols), (cols, 1), dtype=h.dtype, device=device)
    if p > 0:
        grad_x = torch.empty_strided((rows, cols), (cols, 1), dtype=h.dtype, device=device)
        gx_ptr = grad_x.data_ptr()
    if need_weight:
        grad_w = torch.empty_strided(w_shape, (1,) if len(w_shape) == 1 else (cols, 1), dtype=w_dtype, device=device)
        gw_ptr = grad_w.data_ptr()
    if need_bias:
        grad_b = torch.empty_strided(w_shape, (1,) if len(w_shape) == 1 else (cols, 1), dtype=w_dtype, device=device)
        gb_ptr = grad_b.data_ptr()
    per = max(1, rows // groups)
    L = _lib_handle or lib()
    nbytes = L.prm_layernorm_scratch_bytes(rows, cols, per)
    scratch = torch.empty_strided((nbytes,), (1,), dtype=torch.uint8, device=device)
    args = (grad_y.data_ptr(), grad_y.stride(0), h.data_ptr(), h.stride(0), mean.data_ptr(), rstd.data_ptr(), w_ptr, ld_w,
            gh_ptr, ld_gh, rows, cols, per, _IO_FP32[h.dtype], _IO_FP32[w_dtype], 1 if add_one else 0, p, seed & _WORD,
            offset & _WORD, c_ptr, grad_r.data_ptr(), cols, gx_ptr, cols, gw_ptr, gb_ptr, scratch.data_ptr(), nbytes,
            _raw_stream(index))
    fn = L.prm_layernorm_backward
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_layernorm_backward")
    if rows == 0 and groups > 1:
        for t in (grad_w, grad_b):
            if t is not None:
                t.zero_()
    return (grad_x, grad_r, grad_w, grad_b) if p > 0 else (grad_r, None, grad_w, grad_b)


def _head_operand(t, either_way):
    """(matrix, row stride, 1 if it is stored the other way round, bytes of the copy that the call makes of it) of a bf16
    matrix as the head's products read it; one whose elements lie in neither way is copied here."""
    r, c = t.shape
    s0, s1 = t.stride()
    if (s1 == 1 or c == 1) and (s0 >= c or r == 1):
        ld, transposed, rows, cols = (s0 if r > 1 else (c + 7) // 8 * 8), 0, r, c
    elif either_way and (s0 == 1 or r == 1) and (s1 >= r or c == 1):
        ld, transposed, rows, cols = (s1 if c > 1 else (r + 7) // 8 * 8), 1, c, r
    else:
        t = t.contiguous()
        ld, transposed, rows, cols = c, 0, r, c
    if t.data_ptr() & 15 == 0 and ld & 7 == 0:
        return t, ld, transposed, 0
    return t, ld, transposed, (_lib_handle or lib()).prm_head_loss_copy_bytes(rows, cols)


def _head_arguments(x, weight, labels):
    """x, its row stride, weight, its row stride, whether it is transposed, labels, bytes for copies."""
    if x.dim() != 2 or weight.dim() != 2 or x.shape[1] != weight.shape[0]:
        raise ValueError("x must be n x d and weight d x vocab")
    if x.dtype is not torch.bfloat16 or weight.dtype is not torch.bfloat16:
        raise TypeError("x and weight must be bfloat16")
    index = x.get_device()
    if index < 0 or weight.get_device() != index:
        raise ValueError("x and weight must sit on the same CUDA device")
    if x.shape[1] == 0 or weight.shape[1] == 0:
        raise ValueError("d and vocab must be at least 1")
    labels = _vector(labels, "labels", x.shape[0], index, _INT64_ONLY)
    x, ld_x, _, x_copy = _head_operand(x, False)
    weight, ld_w, w_t, w_copy = _head_operand(weight, True)
    return x, ld_x, weight, ld_w, w_t, labels, x_copy + w_copy


def prm_head_loss(x, weight, labels, stream=None):
    """Softmax cross entropy of the logits x @ weight, which are not kept: (loss, lse), fp32 vectors of n.

    x: n x d, weight: d x vocab (or the transposed view of an embedding), both bf16; labels: n int64.  A label
    outside 0..vocab-1 leaves its row out: loss 0.  lse, the logarithm of the row's sum of exponentials, goes to the
    gradient.  Matrices whose rows do not start on 16 bytes are copied first, by each call."""
    if stream is not None:
        return _on_stream(stream, (x, weight, labels), lambda: prm_head_loss(x, weight, labels))
    n, d = x.shape if x.dim() == 2 else (0, 0)
    x, ld_x, weight, ld_w, w_t, labels, copies = _head_arguments(x, weight, labels)
    vocab = weight.shape[1]
    index = x.get_device()
    loss = torch.empty_strided((n,), (1,), dtype=torch.float32, device=x.device)
    lse = torch.empty_strided((n,), (1,), dtype=torch.float32, device=x.device)
    L = _lib_handle or lib()
    nbytes = L.prm_head_loss_scratch_bytes(n, d, vocab) + copies
    scratch = torch.empty_strided((nbytes,), (1,), dtype=torch.uint8, device=x.device)
    args = (x.data_ptr(), ld_x, weight.data_ptr(), ld_w, w_t, labels.data_ptr(), n, d, vocab, loss.data_ptr(), lse.data_ptr(),
            scratch.data_ptr(), nbytes, _raw_stream(index))
    fn = L.prm_head_loss
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_head_loss")
    return loss, lse


def prm_head_loss_backward(grad_loss, x, weight, labels, lse, need_x=True, need_weight=True, stream=None):
    """Gradient of prm_head_loss from that of each row's loss (fp32, n) and its lse: (grad_x, grad_weight), bf16,
    None for what is not needed; grad_weight is stored the way weight is."""
    if stream is not None:
        return _on_stream(stream, (grad_loss, x, weight, labels, lse),
                          lambda: prm_head_loss_backward(grad_loss, x, weight, labels, lse, need_x, need_weight))
    n, d = x.shape if x.dim() == 2 else (0, 0)
    x, ld_x, weight, ld_w, w_t, labels, copies = _head_arguments(x, weight, labels)
    vocab = weight.shape[1]
    index = x.get_device()
    grad_loss = _vector(grad_loss, "grad_loss", n, index)
    lse = _vector(lse, "lse", n, index)
    gx = gw = gx_ptr = gw_ptr = None
    if need_x:
        gx = torch.empty_strided((n, d), (d, 1), dtype=torch.bfloat16, device=x.device)
        gx_ptr = gx.data_ptr()
    if need_weight:
        gw = torch.empty_strided((d, vocab), (1, d) if w_t else (vocab, 1), dtype=torch.bfloat16, device=x.device)
        gw_ptr = gw.data_ptr()
    L = _lib_handle or lib()
    nbytes = L.prm_head_loss_backward_scratch_bytes(n, d, vocab) + copies
    if not need_weight:
        nbytes -= L.prm_head_loss_copy_bytes(n, d)
    scratch = torch.empty_strided((nbytes,), (1,), dtype=torch.uint8, device=x.device)
    args = (grad_loss.data_ptr(), x.data_ptr(), ld_x, weight.data_ptr(), ld_w, w_t, labels.data_ptr(), lse.data_ptr(), n, d,
            vocab, gx_ptr, d, gw_ptr, d if w_t else vocab, scratch.data_ptr(), nbytes, _raw_stream(index))
    fn = L.prm_head_loss_backward
    code = fn(*args) if torch._C._cuda_getDevice() == index else _on_device(index, fn, *args)
    if code:
        _q8_check(code, "prm_head_loss_backward")
    return gx, gw


def prm_destroy(h):
    _check(lib().prm_destroy(h))


class PeriodicRowwiseMuon:
    """Handle + workspace.  Tensors stay owned by the caller; `step` only
    marshals their device pointers."""

    def __init__(self, shapes, K, beta=0.95, nesterov=False, lr=5e-3, wd=0.01, *, gamma=0.15,
                 eps_row=1e-8, eps_ns=1e-7, scale_mode=1, io_dtype="bf16", check_mode=False,
                 ns_workspace_bytes=None, gamma_ns=1.0, no_refresh=False, gram_span=2, tall_kernel=0,
                 split_input=False, wide_kernel=0, device="cuda"):
        self.shapes = [(int(m), int(n)) for (m, n) in shapes]
        self.device = torch.device(device)
        self.io_dtype = io_dtype
        self.h = None
        with torch.cuda.device(self.device):
            self.h = prm_create(self.shapes, K, beta, nesterov, lr, wd)
            prm_set_option(self.h, PRM_OPT_GAMMA, gamma)
            prm_set_option(self.h, PRM_OPT_EPS_ROW, eps_row)
            prm_set_option(self.h, PRM_OPT_EPS_NS, eps_ns)
            prm_set_option(self.h, PRM_OPT_SCALE_MODE, scale_mode)
            prm_set_option(self.h, PRM_OPT_IO_DTYPE, 1 if io_dtype == "fp32" else 0)
            prm_set_option(self.h, PRM_OPT_CHECK_MODE, 1 if check_mode else 0)
            prm_set_option(self.h, PRM_OPT_GAMMA_NS, gamma_ns)
            prm_set_option(self.h, PRM_OPT_NO_REFRESH, 1 if no_refresh else 0)
            prm_set_option(self.h, PRM_OPT_NS_GRAM_SPAN, int(gram_span))
            prm_set_option(self.h, PRM_OPT_TALL_KERNEL, int(tall_kernel))
            prm_set_option(self.h, PRM_OPT_NS_SPLIT_INPUT, 1 if split_input else 0)
            prm_set_option(self.h, PRM_OPT_WIDE_KERNEL, int(wide_kernel))
            if ns_workspace_bytes is not None:
                prm_set_option(self.h, PRM_OPT_NS_WORKSPACE_BYTES, ns_workspace_bytes)
            nbytes = prm_workspace_bytes(self.h)
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = (self.workspace.data_ptr() + 255) // 256 * 256
            prm_set_workspace(self.h, base, nbytes)
        self._cache_key = None
        self._arrays = None

    def ptr_arrays(self, params, grads, momentum):
        key = (tuple(t.data_ptr() for t in params), tuple(t.data_ptr() for t in grads),
               tuple(t.data_ptr() for t in momentum))
        if key != self._cache_key:
            want = torch.float32 if self.io_dtype == "fp32" else torch.bfloat16
            for i, (p, g, m) in enumerate(zip(params, grads, momentum)):
                if p.dtype != want or g.dtype != want or m.dtype != torch.float32:
                    raise TypeError(f"matrix {i}: dtypes must be {want} (params, grads) and float32 (momentum)")
                if tuple(p.shape) != self.shapes[i] or tuple(g.shape) != self.shapes[i] or tuple(m.shape) != self.shapes[i]:
                    raise ValueError(f"matrix {i}: shape mismatch")
                if not (p.is_contiguous() and g.is_contiguous() and m.is_contiguous()):
                    raise ValueError(f"matrix {i}: tensors must be contiguous")
            self._arrays = (_ptr_array(params), _ptr_array(grads), _ptr_array(momentum))
            self._cache_key = key
        return self._arrays

    def step(self, params, grads, momentum, step_idx, stream=None):
        """One optimizer step, enqueued on `stream` (default: torch's current stream)."""
        if len(params) != len(self.shapes):
            raise ValueError("wrong number of matrices")
        P, G, M = self.ptr_arrays(params, grads, momentum)
        s = (stream or torch.cuda.current_stream(self.device)).cuda_stream
        with torch.cuda.device(self.device):
            prm_step(self.h, P, G, M, step_idx, s)

    def step_h2d(self, params, grads_dev, grads_host, momentum, step_idx, stream=None):
        """Step whose gradients are first copied from (pinned) host tensors."""
        P, G, M = self.ptr_arrays(params, grads_dev, momentum)
        H = _ptr_array(grads_host)
        s = (stream or torch.cuda.current_stream(self.device)).cuda_stream
        with torch.cuda.device(self.device):
            prm_step_h2d(self.h, P, G, H, M, step_idx, s)

    def set_lr(self, lr):
        prm_set_option(self.h, PRM_OPT_LR, lr)

    def plan(self, step_idx):
        return prm_plan(self.h, step_idx, len(self.shapes))

    def groups(self):
        """One dict per shape group (see prm_group_info)."""
        n_groups = self.plan(0)[1]
        return [prm_group_info(self.h, g) for g in range(n_groups)]

    def status(self):
        return prm_status(self.h)

    def profile(self, enable=True):
        with torch.cuda.device(self.device):
            prm_profile(self.h, enable)

    def profile_read(self):
        """{class name: (milliseconds, launches)} since the last read."""
        with torch.cuda.device(self.device):
            return prm_profile_read(self.h)

    def launch_count(self):
        return prm_launch_count(self.h)

    def close(self):
        if self.h is not None:
            prm_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
