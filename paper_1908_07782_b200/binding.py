"""ctypes binding of libcombo_b200.so: same names as the C ABI, argument
marshalling only.  Tensors are torch tensors (device memory and streams come
from PyTorch); every step of the round runs inside the library's kernels.
There is no fallback: a missing library raises."""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcombo_b200.so")
_lib = None

COMBO_OK = 0
ACT_NONE, ACT_RELU, ACT_SILU = 0, 1, 2
STEP_NONE, STEP_MULTIPLY_ADD, STEP_TENSOR, STEP_TENSOR_PAIRS, STEP_TENSOR_THREADS, STEP_RESIDENT, STEP_STREAMED = range(7)
PATH_AUTO, PATH_DIRECT, PATH_STAGED, PATH_TILE, PATH_DIRECT_NAIVE = 0, 1, 2, 5, 6


class ComboError(RuntimeError):
    def __init__(self, status: int, where: str):
        lib = load()
        msg = lib.combo_status_string(status).decode()
        detail = lib.combo_last_cuda_error().decode()
        super().__init__("%s: %s%s" % (where, msg, (" (%s)" % detail) if status == 4 and detail else ""))
        self.status = status


def load():
    """Loads the shared library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libcombo_b200.so is missing (%s); build it with "
            "`python -m paper_1908_07782_b200.build` -- there is no fallback path" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u32, u64, f32 = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint32,
                                   ctypes.c_uint64, ctypes.c_float)
    sigs = {
        "combo_select_peers": [u64, u32, i32, i32, i32, vp],
        "combo_select_peers_async": [u64, u32, i32, i32, i32, vp, vp],
        "combo_segment_aggregate": [vp, vp, vp, vp, i32, i64, i32, i32, vp],
        "combo_segment_aggregate_bf16": [vp, vp, vp, vp, i32, i64, i32, i32, vp],
        "combo_segment_aggregate_sgd": [vp, vp, f32, vp, vp, vp, i32, i64, i32, i32, vp],
        "combo_segment_aggregate_cols": [vp, vp, f32, vp, i32, vp, vp, i32, i64, i32, i32, i64, i64,
                                         i64, vp],
        "combo_validate_idx": [vp, i32, i32, i32, vp, vp],
        "combo_segment_aggregate_rows": [vp, vp, i64, i32, vp, vp, i32, i64, i32, i32, i32, i32, vp],
        "combo_check_rows": [vp, i32, vp, vp],
        "combo_select_peers_online": [u64, u32, i32, i32, i32, vp, vp, vp],
        "combo_segment_aggregate_members": [vp, vp, i32, vp, vp, vp, i32, i64, i32, i32, vp],
        "combo_round_host": [vp, vp, f32, vp, i32, vp, u64, u32, i32, i32, i64, i32, i32, vp, vp, vp,
                             vp, vp, vp, vp],
        "combo_aggregation_divergence": [vp, vp, i32, vp, i32, i64, vp, vp, ctypes.c_size_t, vp],
        "combo_aggregation_divergence_noalloc": [vp, vp, i32, vp, i32, i64, vp, vp],
        "combo_grad_norm": [vp, vp, vp, i32, i32, i64, i32, f32, vp, vp, vp, ctypes.c_size_t, vp],
        "combo_grad_clip": [vp, vp, vp, vp, i32, i32, i64, i32, f32, vp, vp, vp, ctypes.c_size_t, vp],
        "combo_check_tensors": [vp, vp, vp, i32, i32, i64, i32, vp, vp],
        "combo_group_norm": [vp, i64, vp, i64, i32, vp, vp, i32, i64, vp, i32, i64, i64, i64, i32, f32, i32, vp, vp, vp,
                             ctypes.c_size_t, vp],
        "combo_group_norm_backward": [vp, i64, vp, i64, vp, i64, i32, vp, vp, i32, i64, vp, i32, i64, i64, i64, i32, i32,
                                      vp, vp, vp, vp, i64, vp, ctypes.c_size_t, vp],
        "combo_grouped_linear": [vp, i64, vp, i64, i64, vp, i64, i32, i32, vp, i32, i64, i64, i64, vp],
        "combo_grouped_linear_grad_input": [vp, i64, vp, i64, i64, vp, i64, i32, i32, vp, i32, i64, i64, i64, vp],
        "combo_grouped_linear_grad_weight": [vp, i64, vp, i64, vp, i64, i64, i32, i32, vp, i32, i64, i64, i64, vp],
        "combo_grouped_cross_entropy": [vp, i64, vp, i64, i64, i32, vp, vp, i32, i64, i64, i64, vp, vp, vp, ctypes.c_size_t, vp],
        "combo_grouped_cross_entropy_backward": [vp, i64, vp, i64, i64, i32, vp, vp, vp, vp, i64, vp, i64, i64, i32, vp, i32, i64, i64,
                                                 i64, vp, ctypes.c_size_t, vp],
        "combo_dropout": [vp, i64, vp, i64, vp, i64, i32, vp, i32, i64, i64, f32, u64, u32, u32, i32, vp],
        "combo_debug_dead_wait": [vp],
        "combo_device_status": [],
        "combo_last_kernel_path": [],
        "combo_last_step_path": [],
        "combo_version": [],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.combo_divergence_scratch_bytes.argtypes = [i32]
    lib.combo_divergence_scratch_bytes.restype = ctypes.c_size_t
    lib.combo_grad_scratch_bytes.argtypes = [i32]
    lib.combo_grad_scratch_bytes.restype = ctypes.c_size_t
    lib.combo_group_norm_scratch_bytes.argtypes = [i64, i64, i64, i32]
    lib.combo_group_norm_scratch_bytes.restype = ctypes.c_size_t
    for name in ("combo_grouped_cross_entropy_scratch_bytes", "combo_grouped_cross_entropy_least_scratch_bytes"):
        getattr(lib, name).argtypes = [i32, i64, i64, i64, i32, i32]
        getattr(lib, name).restype = ctypes.c_size_t
    lib.combo_set_kernel_path.argtypes = [i32]
    lib.combo_set_kernel_path.restype = None
    lib.combo_set_tuning.argtypes = [i32, i32]
    lib.combo_set_tuning.restype = None
    lib.combo_max_launch_columns.argtypes = []
    lib.combo_max_launch_columns.restype = ctypes.c_int64
    lib.combo_set_launch_columns.argtypes = [i64]
    lib.combo_set_launch_columns.restype = None
    lib.combo_set_launch_overlap.argtypes = [i32]
    lib.combo_set_launch_overlap.restype = None
    lib.combo_status_string.argtypes = [i32]
    lib.combo_status_string.restype = ctypes.c_char_p
    lib.combo_last_cuda_error.argtypes = []
    lib.combo_last_cuda_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current device, and its current stream's handle without making a Stream object, which takes 3 us where a small call takes
# 10.  Neither is in torch's public interface, which does where they are missing.
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream=None):
    """Handle of ``stream``, or of the current device's current stream."""
    return _raw_stream(_device()) if stream is None else stream.cuda_stream


def _check(status: int, where: str):
    if status != COMBO_OK:
        raise ComboError(status, where)


def combo_select_peers(seed: int, rnd: int, N: int, S: int, R: int, idx_out: torch.Tensor,
                       stream=None) -> torch.Tensor:
    """Peer table for (seed, round) into idx_out (int32 [N][S][R], device), on
    the current torch stream (or ``stream``)."""
    _check(load().combo_select_peers_async(seed, rnd, N, S, R, _ptr(idx_out), _stream(stream)),
           "combo_select_peers")
    return idx_out


def combo_select_peers_default_stream(seed, rnd, N, S, R, idx_out):
    """The stream-less C entry point (legacy default stream)."""
    _check(load().combo_select_peers(seed, rnd, N, S, R, _ptr(idx_out)), "combo_select_peers")
    return idx_out


def combo_segment_aggregate(params_in, params_out, weights, idx, N, P, S, R, stream=None):
    _check(load().combo_segment_aggregate(_ptr(params_in), _ptr(params_out), _ptr(weights), _ptr(idx),
                                          N, P, S, R, _stream(stream)), "combo_segment_aggregate")
    return params_out


def combo_segment_aggregate_bf16(params_in, params_out, weights, idx, N, P, S, R, stream=None):
    _check(load().combo_segment_aggregate_bf16(_ptr(params_in), _ptr(params_out), _ptr(weights),
                                               _ptr(idx), N, P, S, R, _stream(stream)),
           "combo_segment_aggregate_bf16")
    return params_out


def combo_segment_aggregate_sgd(params_in, grads, lr, params_out, weights, idx, N, P, S, R,
                                stream=None):
    _check(load().combo_segment_aggregate_sgd(_ptr(params_in), _ptr(grads), lr, _ptr(params_out),
                                              _ptr(weights), _ptr(idx), N, P, S, R, _stream(stream)),
           "combo_segment_aggregate_sgd")
    return params_out


def combo_segment_aggregate_cols(params_in, grads, lr, params_out, elem_bytes, weights, idx, N,
                                 P_total, S, R, p_begin, width, pitch, stream=None):
    _check(load().combo_segment_aggregate_cols(_ptr(params_in), _ptr(grads), lr, _ptr(params_out),
                                               elem_bytes, _ptr(weights), _ptr(idx), N, P_total, S, R,
                                               p_begin, width, pitch, _stream(stream)),
           "combo_segment_aggregate_cols")
    return params_out


def _host_bytes(flags, N):
    """N flag bytes in host memory for the C side (None stays NULL)."""
    if flags is None:
        return None, None
    buf = (ctypes.c_uint8 * N)(*[1 if bool(f) else 0 for f in flags])
    return buf, ctypes.cast(buf, ctypes.c_void_p)


def combo_segment_aggregate_rows(rows, out, out_pitch, elem_bytes, weights, idx, N, P, S, R, w_begin, n_local,
                                 stream=None):
    """Worker-sharded Eq. 3: ``rows`` is a device int64 tensor of N row addresses (local or
    peer memory), ``out`` holds the n_local hosted workers' new models, [n_local][out_pitch]."""
    _check(load().combo_segment_aggregate_rows(_ptr(rows), _ptr(out), out_pitch, elem_bytes, _ptr(weights),
                                               _ptr(idx), N, P, S, R, w_begin, n_local, _stream(stream)),
           "combo_segment_aggregate_rows")
    return out


def combo_check_rows(rows, N, stream=None) -> int:
    """0 when all N row addresses are non-null and 16-byte aligned, else 1 + the first bad row."""
    flag = torch.zeros(1, dtype=torch.int32, device=rows.device)
    _check(load().combo_check_rows(_ptr(rows), N, _stream(stream), _ptr(flag)), "combo_check_rows")
    return int(flag.item())


def combo_select_peers_online(seed, rnd, N, S, R, online, idx_out, stream=None):
    """Section 4.2: peers drawn from the online others only; ``online`` is a host
    sequence of N flags (None = all online).  Offline workers' rows become -1."""
    keep, ptr = _host_bytes(online, N)
    _check(load().combo_select_peers_online(seed, rnd, N, S, R, ptr, _ptr(idx_out), _stream(stream)),
           "combo_select_peers_online")
    return idx_out


def combo_segment_aggregate_members(params_in, params_out, weights, idx, newcomer, N, P, S, R, stream=None):
    """Eq. 3 where newcomers (host sequence of N flags, or None) aggregate without their
    own model and negative idx entries are skipped."""
    keep, ptr = _host_bytes(newcomer, N)
    _check(load().combo_segment_aggregate_members(_ptr(params_in), _ptr(params_out), params_in.element_size(),
                                                  _ptr(weights), _ptr(idx), ptr, N, P, S, R, _stream(stream)),
           "combo_segment_aggregate_members")
    return params_out


def combo_validate_idx(idx, N, S, R, dev_flag, stream=None):
    _check(load().combo_validate_idx(_ptr(idx), N, S, R, _stream(stream), _ptr(dev_flag)),
           "combo_validate_idx")
    return dev_flag


def combo_round_host(h_params_in, h_grads, lr, h_params_out, elem_bytes, h_weights, seed, rnd, rounds,
                     N, P, S, R, d_in, d_grads, d_out, d_weights, d_idx, h_idx_out=None, stream=None):
    """``rounds`` chained rounds from host tensors (pinned for speed) through
    caller-owned device buffers; returns after the result is in h_params_out."""
    _check(load().combo_round_host(_ptr(h_params_in), _ptr(h_grads), lr, _ptr(h_params_out),
                                   elem_bytes, _ptr(h_weights), seed, rnd, rounds, N, P, S, R, _ptr(d_in),
                                   _ptr(d_grads), _ptr(d_out), _ptr(d_weights), _ptr(d_idx),
                                   _ptr(h_idx_out), _stream(stream)), "combo_round_host")
    return h_params_out


def combo_divergence_scratch_bytes(N: int) -> int:
    return int(load().combo_divergence_scratch_bytes(N))


def combo_aggregation_divergence(models, mean_of, elem_bytes, weights, N, P, rho_out, scratch, stream=None):
    """Eq. 7 for all workers: rho_out (float64 [N], device) = distance of each row of
    ``models`` from the weighted mean over the rows of ``mean_of`` (or of ``models``).
    ``scratch`` is a device tensor of at least combo_divergence_scratch_bytes(N) bytes."""
    _check(load().combo_aggregation_divergence(_ptr(models), _ptr(mean_of), elem_bytes, _ptr(weights), N, P,
                                               _ptr(rho_out), _ptr(scratch),
                                               scratch.numel() * scratch.element_size(), _stream(stream)),
           "combo_aggregation_divergence")
    return rho_out


def combo_aggregation_divergence_noalloc(models, mean_of, elem_bytes, weights, N, P, rho_out, stream=None):
    """The same measurement for callers that cannot allocate device memory: the
    partial sums go to a fixed 1 MiB array inside the library instead of a
    caller-supplied scratch tensor.  At most 128 workers; all calls on a device
    share that array, so issue them on one stream."""
    _check(load().combo_aggregation_divergence_noalloc(_ptr(models), _ptr(mean_of), elem_bytes, _ptr(weights), N,
                                                       P, _ptr(rho_out), _stream(stream)),
           "combo_aggregation_divergence_noalloc")
    return rho_out


def _bytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


_SIZES = {torch.float32: 4, torch.bfloat16: 2}
_MAX_WORKERS = 8192


def _refuse(name: str, what: str):
    raise ValueError("%s: %s" % (name, what))


def _on_gpu(name, *tensors):
    """Refuses what is not on the current GPU: a kernel cannot read the host's memory, and what it is given are addresses."""
    at = None
    for t in tensors:
        if t is not None:
            d = t.get_device()
            if d != at:
                if at is not None or d < 0 or d != _device():
                    _refuse(name, "all tensors must be on the current GPU, got one on %s" % t.device)
                at = d


def _short(t, dtype, least) -> bool:
    return t is not None and (t.dtype is not dtype or t.numel() < least or not t.is_contiguous())


def _lists(name, tensors, out, begin, first, n_tensors, N, norm_out, coef_out, scratch):
    """Types, lengths and places of a table of tensors and of what is written per worker.  (None and counts out of range are
    left to the library's own refusal.)"""
    n, w = (n_tensors, N) if n_tensors >= 0 and 1 <= N <= _MAX_WORKERS else (-1, -1)
    if _short(tensors, torch.int64, n) or _short(out, torch.int64, n):
        _refuse(name, "tensors and out must be int64 addresses, %d in a row" % n)
    if _short(begin, torch.int64, n + 1):
        _refuse(name, "begin must be int64, %d in a row" % (n + 1))
    if _short(first, torch.int32, w + 1):
        _refuse(name, "first must be int32, %d in a row" % (w + 1))
    if _short(norm_out, torch.float32, w) or _short(coef_out, torch.float32, w):
        _refuse(name, "norm_out and coef_out must be float32, %d in a row" % w)
    _on_gpu(name, tensors, out, begin, first, norm_out, coef_out, scratch)


def combo_grad_scratch_bytes(N: int) -> int:
    return int(load().combo_grad_scratch_bytes(N))


def combo_grad_norm(tensors, begin, first, n_tensors, N, total, elem_bytes, max_norm, norm_out, coef_out, scratch,
                    stream=None):
    """Norm of every worker's gradient over its tensors, and the coefficient that clips it
    to ``max_norm`` (float32 [N] each, device).  ``tensors``: device int64 addresses;
    ``begin``: device int64 [n_tensors + 1] positions; ``first``: device int32 [N + 1]."""
    _lists("combo_grad_norm", tensors, None, begin, first, n_tensors, N, norm_out, coef_out, scratch)
    _check(load().combo_grad_norm(_ptr(tensors), _ptr(begin), _ptr(first), n_tensors, N, total, elem_bytes, max_norm,
                                  _ptr(norm_out), _ptr(coef_out), _ptr(scratch), _bytes(scratch), _stream(stream)),
           "combo_grad_norm")
    return norm_out


def combo_grad_clip(tensors, out, begin, first, n_tensors, N, total, elem_bytes, max_norm, norm_out, coef_out, scratch,
                    stream=None):
    """combo_grad_norm, and every tensor times its worker's coefficient, written to the
    addresses in ``out`` (device int64; may be ``tensors``)."""
    _lists("combo_grad_clip", tensors, out, begin, first, n_tensors, N, norm_out, coef_out, scratch)
    _check(load().combo_grad_clip(_ptr(tensors), _ptr(out), _ptr(begin), _ptr(first), n_tensors, N, total, elem_bytes,
                                  max_norm, _ptr(norm_out), _ptr(coef_out), _ptr(scratch), _bytes(scratch),
                                  _stream(stream)), "combo_grad_clip")
    return norm_out


def combo_check_tensors(tensors, begin, first, n_tensors, N, total, elem_bytes, stream=None) -> int:
    """0 when the table is as combo_grad_norm wants it, else 1 + a bad tensor, or
    1 + n_tensors + a bad worker."""
    _lists("combo_check_tensors", tensors, None, begin, first, n_tensors, N, None, None, None)
    flag = torch.zeros(1, dtype=torch.int32, device=begin.device)
    _check(load().combo_check_tensors(_ptr(tensors), _ptr(begin), _ptr(first), n_tensors, N, total, elem_bytes,
                                      _stream(stream), _ptr(flag)), "combo_check_tensors")
    return int(flag.item())


def _pitch(shape, stride, name, arg) -> int:
    """Elements between the positions of a channels-last [B, L, C] tensor."""
    B, L, C = shape
    pitch = stride[1] if L > 1 else stride[0] if B > 1 else C
    if (C > 1 and stride[2] != 1) or (B > 1 and stride[0] != L * pitch):
        _refuse(name, "%s: channels must be neighbours, samples L positions apart" % arg)
    return pitch


def _rows(shape, stride, name, arg) -> int:
    """Elements between the rows of a two-dimensional tensor."""
    if shape[1] > 1 and stride[1] != 1:
        _refuse(name, "%s: a row's elements must be neighbours" % arg)
    return stride[0] if shape[0] > 1 else shape[1]


def _norm_args(name, x, others, gamma, beta, begin, stats, groups):
    """What the two group norm calls check alike; size of x's elements, workers, size and pitch of the parameters."""
    shape = x.shape
    if len(shape) != 3 or x.dtype not in _SIZES:
        _refuse(name, "x must be [B, L, C], float32 or bfloat16")
    for t in others:
        if t.shape != shape or t.dtype != x.dtype:
            _refuse(name, "y (dy, dx) must be like x")
    for t in stats:
        if t is not None and (t.dtype != torch.float32 or t.numel() != shape[0] * groups or not t.is_contiguous()):
            _refuse(name, "mean and rstd must be float32 [B, groups]")
    if begin is None:
        N = 1
    else:
        N = begin.numel() - 1
        if begin.dtype != torch.int64 or not begin.is_contiguous():
            _refuse(name, "begin must be int64 [N + 1]")
    if gamma is None or beta is None:
        return _SIZES[x.dtype], N, 4, 0
    if gamma.shape != (N, shape[2]) or beta.shape != (N, shape[2]) or gamma.dtype != beta.dtype or gamma.dtype not in _SIZES:
        _refuse(name, "gamma and beta must be [N, C] of one type, float32 or bfloat16")
    pitch = _rows(gamma.shape, gamma.stride(), name, "gamma")
    if pitch != _rows(beta.shape, beta.stride(), name, "beta"):
        _refuse(name, "gamma and beta must have one pitch")
    return _SIZES[x.dtype], N, _SIZES[gamma.dtype], pitch


def combo_group_norm(x, y, gamma, beta, begin, groups, eps, act, mean, rstd, scratch, stream=None):
    """y = act(group norm of x), channels last: x, y [B, L, C]; gamma, beta [N, C] (views of flat
    parameter vectors, or None); begin: device int64 [N + 1], the workers' samples, or None for one
    worker; mean, rstd: float32 [B, groups] or None; scratch: device memory of
    combo_group_norm_scratch_bytes(B, L, C, groups) bytes."""
    name = "combo_group_norm"
    size, N, param_size, param_pitch = _norm_args(name, x, (y,), gamma, beta, begin, (mean, rstd), groups)
    B, L, C = shape = x.shape
    xp, yp = _pitch(shape, x.stride(), name, "x"), _pitch(shape, y.stride(), name, "y")
    _on_gpu(name, x, y, gamma, beta, begin, mean, rstd, scratch)
    _check(load().combo_group_norm(x.data_ptr(), xp, y.data_ptr(), yp, size, _ptr(gamma), _ptr(beta), param_size, param_pitch,
                                   _ptr(begin), N, B, L, C, groups, eps, act, _ptr(mean), _ptr(rstd), _ptr(scratch),
                                   _bytes(scratch), _stream(stream)), name)
    return y


def combo_group_norm_scratch_bytes(B: int, L: int, C: int, groups: int) -> int:
    return int(load().combo_group_norm_scratch_bytes(B, L, C, groups))


def combo_group_norm_backward(dy, x, dx, gamma, beta, begin, groups, act, mean, rstd, dgamma, dbeta, scratch,
                              stream=None):
    """Gradients of combo_group_norm: dx [B, L, C] and, per worker, dgamma and dbeta (float32
    [N, C], views of flat gradient vectors, or None), from the forward call's mean and rstd."""
    name = "combo_group_norm_backward"
    size, N, param_size, param_pitch = _norm_args(name, x, (dy, dx), gamma, beta, begin, (mean, rstd), groups)
    B, L, C = shape = x.shape
    grad_pitch = 0
    if dgamma is not None and dbeta is not None:
        if dgamma.shape != (N, C) or dbeta.shape != (N, C) or dgamma.dtype != torch.float32 or dbeta.dtype != torch.float32:
            _refuse(name, "dgamma and dbeta must be float32 [N, C]")
        grad_pitch = _rows(dgamma.shape, dgamma.stride(), name, "dgamma")
        if grad_pitch != _rows(dbeta.shape, dbeta.stride(), name, "dbeta"):
            _refuse(name, "dgamma and dbeta must have one pitch")
    dyp, xp, dxp = (_pitch(shape, t.stride(), name, arg) for t, arg in ((dy, "dy"), (x, "x"), (dx, "dx")))
    _on_gpu(name, dy, x, dx, gamma, beta, begin, mean, rstd, dgamma, dbeta, scratch)
    _check(load().combo_group_norm_backward(
        dy.data_ptr(), dyp, x.data_ptr(), xp, dx.data_ptr(), dxp, size, _ptr(gamma), _ptr(beta), param_size, param_pitch,
        _ptr(begin), N, B, L, C, groups, act, _ptr(mean), _ptr(rstd), _ptr(dgamma), _ptr(dbeta), grad_pitch,
        _ptr(scratch), _bytes(scratch), _stream(stream)), name)
    return dx


def _product_args(name, a, b, weights, begin, a_width, b_width, same):
    """Checks the operands of a grouped product: rows a [M, a_width], b [M, b_width] (widths: 1 = n_out, 2 = n_in),
    weights [N, n_out, n_in]; `same`: the two that are inputs."""
    shape, stride = weights.shape, weights.stride()
    N, n_out, n_in = shape
    M = a.shape[0]
    if a.shape != (M, shape[a_width]) or b.shape != (M, shape[b_width]):
        _refuse(name, "rows must be [M, %d] and [M, %d]" % (shape[a_width], shape[b_width]))
    if begin.dtype != torch.int64 or begin.numel() != N + 1 or not begin.is_contiguous():
        _refuse(name, "begin must be int64 [N + 1]")
    if n_in > 1 and stride[2] != 1:
        _refuse(name, "weights: a row's elements must be neighbours")
    if same[0].dtype != same[1].dtype or a.dtype not in _SIZES or b.dtype not in _SIZES or weights.dtype not in _SIZES:
        _refuse(name, "types are float32 and bfloat16, one for both inputs")
    pitches = _rows(a.shape, a.stride(), name, "rows"), _rows(b.shape, b.stride(), name, "rows")
    _on_gpu(name, a, b, weights, begin)
    return (N, M, n_in, n_out, *pitches, stride[1] if n_out > 1 else n_in, stride[0] if N > 1 else 0)


def combo_grouped_linear(x, w, y, begin, stream=None):
    """y[m] = x[m] W_w^T for every worker w's rows m (``begin``: device int64 [N + 1]).  x [M, n_in],
    w [N, n_out, n_in] (a view of flat parameter vectors, strides as they are), y [M, n_out] of x's
    type or, for bfloat16, float32."""
    name = "combo_grouped_linear"
    N, M, n_in, n_out, xp, yp, wp, ws = _product_args(name, x, y, w, begin, 2, 1, (x, w))
    _check(load().combo_grouped_linear(x.data_ptr(), xp, w.data_ptr(), wp, ws, y.data_ptr(), yp, _SIZES[x.dtype],
                                       _SIZES[y.dtype], begin.data_ptr(), N, M, n_in, n_out, _stream(stream)), name)
    return y


def combo_grouped_linear_grad_input(dy, w, dx, begin, stream=None):
    """dx[m] = dy[m] W_w: the gradient of combo_grouped_linear for its rows."""
    name = "combo_grouped_linear_grad_input"
    N, M, n_in, n_out, yp, xp, wp, ws = _product_args(name, dy, dx, w, begin, 1, 2, (dy, w))
    _check(load().combo_grouped_linear_grad_input(dy.data_ptr(), yp, w.data_ptr(), wp, ws, dx.data_ptr(), xp,
                                                  _SIZES[dy.dtype], _SIZES[dx.dtype], begin.data_ptr(), N, M, n_in, n_out,
                                                  _stream(stream)), name)
    return dx


def combo_grouped_linear_grad_weight(dy, x, dw, begin, stream=None):
    """dw[w] = sum over worker w's rows of dy[m]^T x[m]: the gradient for the weights, [N, n_out, n_in]
    (a view of flat gradient vectors), of dy's type or float32."""
    name = "combo_grouped_linear_grad_weight"
    N, M, n_in, n_out, yp, xp, wp, ws = _product_args(name, dy, x, dw, begin, 1, 2, (dy, x))
    _check(load().combo_grouped_linear_grad_weight(dy.data_ptr(), yp, x.data_ptr(), xp, dw.data_ptr(), wp, ws,
                                                   _SIZES[dy.dtype], _SIZES[dw.dtype], begin.data_ptr(), N, M, n_in, n_out,
                                                   _stream(stream)), name)
    return dw


def _loss_args(name, x, w, labels, floats, begin):
    """What the two cross entropy calls check alike: x [M, n_in], w [N, n_out, n_in], labels [M], `floats` float32 [M] or None."""
    if len(x.shape) != 2 or len(w.shape) != 3 or x.dtype not in _SIZES or w.dtype != x.dtype:
        _refuse(name, "x must be [M, n_in] and w [N, n_out, n_in] of one type, float32 or bfloat16")
    (M, n_in), shape, stride = x.shape, w.shape, w.stride()
    N, n_out = shape[0], shape[1]
    if shape[2] != n_in:
        _refuse(name, "x is %d wide, the weights %d" % (n_in, shape[2]))
    if n_in > 1 and stride[2] != 1:
        _refuse(name, "w: a row's elements must be neighbours")
    if labels.dtype != torch.int64 or labels.numel() != M or not labels.is_contiguous():
        _refuse(name, "labels must be int64 [M]")
    for t in floats:
        if t is not None and (t.dtype != torch.float32 or t.numel() != M or not t.is_contiguous()):
            _refuse(name, "loss, lse and row_grad must be float32 [M]")
    if begin.dtype != torch.int64 or begin.numel() != N + 1 or not begin.is_contiguous():
        _refuse(name, "begin must be int64 [N + 1]")
    return N, M, n_in, n_out, _rows(x.shape, x.stride(), name, "x"), stride[1] if n_out > 1 else n_in, stride[0] if N > 1 else 0


def combo_grouped_cross_entropy_scratch_bytes(N: int, M: int, n_in: int, n_out: int, elem_bytes: int, grad_bytes: int = 0) -> int:
    """Scratch of combo_grouped_cross_entropy, or, with the size of dw's elements, of its backward call."""
    return int(load().combo_grouped_cross_entropy_scratch_bytes(N, M, n_in, n_out, elem_bytes, grad_bytes))


def combo_grouped_cross_entropy_least_scratch_bytes(N: int, M: int, n_in: int, n_out: int, elem_bytes: int, grad_bytes: int = 0) -> int:
    """The least scratch that those calls take: the classes in smaller pieces, for more time (none for bfloat16 forward on 16 bytes)."""
    return int(load().combo_grouped_cross_entropy_least_scratch_bytes(N, M, n_in, n_out, elem_bytes, grad_bytes))


def combo_grouped_cross_entropy(x, w, labels, loss, lse, begin, scratch, stream=None):
    """Softmax cross entropy of x[m] W_w^T for every worker w's rows m (``begin``: device int64 [N + 1]), without
    keeping the logits: x [M, n_in], w [N, n_out, n_in] (a view of flat parameter vectors) of x's type, labels int64
    [M] (one outside the classes: the row has none); loss and lse (the logits' log-sum-exp, for the backward call)
    float32 [M]."""
    name = "combo_grouped_cross_entropy"
    N, M, n_in, n_out, xp, wp, ws = _loss_args(name, x, w, labels, (loss, lse), begin)
    _on_gpu(name, x, w, labels, loss, lse, begin, scratch)
    _check(load().combo_grouped_cross_entropy(x.data_ptr(), xp, w.data_ptr(), wp, ws, _SIZES[x.dtype], labels.data_ptr(),
                                              begin.data_ptr(), N, M, n_in, n_out, _ptr(loss), _ptr(lse), _ptr(scratch),
                                              _bytes(scratch), _stream(stream)), name)
    return loss


def combo_grouped_cross_entropy_backward(x, w, labels, lse, row_grad, dx, dw, begin, scratch, stream=None):
    """Gradients of sum_m row_grad[m] loss[m] (``row_grad`` None: of every worker's mean over its labelled rows): dx like
    x, dw [N, n_out, n_in] (a view of flat gradient vectors) float32 or x's type, from the forward call's lse."""
    name = "combo_grouped_cross_entropy_backward"
    N, M, n_in, n_out, xp, wp, ws = _loss_args(name, x, w, labels, (lse, row_grad), begin)
    if dx.shape != x.shape or dx.dtype != x.dtype:
        _refuse(name, "dx must be like x")
    if dw.shape != w.shape or dw.dtype not in _SIZES or (n_in > 1 and dw.stride(2) != 1):
        _refuse(name, "dw must be [N, n_out, n_in], float32 or x's type, a row's elements neighbours")
    dxp, stride = _rows(dx.shape, dx.stride(), name, "dx"), dw.stride()
    _on_gpu(name, x, w, labels, lse, row_grad, dx, dw, begin, scratch)
    _check(load().combo_grouped_cross_entropy_backward(
        x.data_ptr(), xp, w.data_ptr(), wp, ws, _SIZES[x.dtype], labels.data_ptr(), _ptr(lse), _ptr(row_grad), dx.data_ptr(), dxp,
        dw.data_ptr(), stride[1] if n_out > 1 else n_in, stride[0] if N > 1 else 0, _SIZES[dw.dtype], begin.data_ptr(), N, M, n_in,
        n_out, _ptr(scratch), _bytes(scratch), _stream(stream)), name)
    return dx


def combo_dropout(x, residual, y, begin, p, seed, rnd, site=0, first_worker=0, stream=None):
    """y = residual + x with every element dropped with probability p and the others scaled, x, y, residual (or None)
    [M, n]; the mask follows from (seed, round, site, worker, place among the worker's rows), ``begin``: device int64
    [N + 1], or None for one worker.  The backward pass is the same call on dy without a residual."""
    name = "combo_dropout"
    if len(x.shape) != 2 or x.dtype not in _SIZES:
        _refuse(name, "x must be [M, n], float32 or bfloat16")
    for t in (residual, y):
        if t is not None and (t.shape != x.shape or t.dtype != x.dtype):
            _refuse(name, "y and residual must be like x")
    if begin is not None and (begin.dtype != torch.int64 or begin.numel() < 2 or not begin.is_contiguous()):
        _refuse(name, "begin must be int64 [N + 1]")
    if not (0 <= seed < 1 << 64 and 0 <= rnd < 1 << 32 and 0 <= site < 1 << 32):
        _refuse(name, "seed has 64 bits, round and site 32")
    shape = x.shape
    xp, yp = _rows(shape, x.stride(), name, "x"), _rows(shape, y.stride(), name, "y")
    rp = 0 if residual is None else _rows(shape, residual.stride(), name, "residual")
    _on_gpu(name, x, residual, y, begin)
    _check(load().combo_dropout(x.data_ptr(), xp, _ptr(residual), rp, y.data_ptr(), yp, _SIZES[x.dtype], _ptr(begin),
                                1 if begin is None else begin.numel() - 1, shape[0], shape[1], p, seed, rnd, site, first_worker,
                                _stream(stream)), name)
    return y


def combo_device_status():
    _check(load().combo_device_status(), "combo_device_status")


def combo_last_kernel_path() -> int:
    return load().combo_last_kernel_path()


def combo_last_step_path() -> int:
    """Which kernels the last product or group norm call on this thread launched (STEP_*)."""
    return load().combo_last_step_path()


def combo_set_kernel_path(path: int) -> None:
    load().combo_set_kernel_path(path)


def combo_set_tuning(tile_elems: int = 0, stages: int = 0) -> None:
    load().combo_set_tuning(tile_elems, stages)


def combo_set_launch_overlap(on: bool = True) -> None:
    load().combo_set_launch_overlap(1 if on else 0)


def combo_max_launch_columns() -> int:
    return int(load().combo_max_launch_columns())


def combo_set_launch_columns(columns: int = 0) -> None:
    load().combo_set_launch_columns(columns)


def combo_debug_dead_wait(stream=None) -> None:
    """Enqueues the self-check kernel whose bounded wait runs out (see the header)."""
    _check(load().combo_debug_dead_wait(_stream(stream)), "combo_debug_dead_wait")


def combo_version() -> int:
    return load().combo_version()
