"""ctypes binding of libwpsgd.so: same names as the C ABI in include/wpsgd.h.

Argument marshalling only -- every step of the path runs in the HIP library.  PyTorch is
used for device memory (tensors) and for the current HIP stream; nothing here computes.
There is no CPU fallback: if the library is missing or cannot be loaded, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libwpsgd.so")

HINGE, LOGISTIC = 0, 1
SAMPLE_STREAM, SAMPLE_SHARDS = 0, 1
F32, BF16 = 0, 1
FP32_SUMS = 16
OK, INVALID_ARG, HIP_ERROR, WORKSPACE_TOO_SMALL, UNSUPPORTED, INCOMPLETE = 0, -1, -2, -3, -4, -5

EXPORTS = [
    "wpsgd_run_chains_workspace", "wpsgd_run_chains", "wpsgd_weights", "wpsgd_weights_rate",
    "wpsgd_benefit_margin", "wpsgd_combine_workspace", "wpsgd_combine", "wpsgd_sample_indices",
    "wpsgd_sample_indices_device", "wpsgd_strerror", "wpsgd_last_hip_error", "wpsgd_describe_plan",
    "wpsgd_stream_rows", "wpsgd_objective_workspace", "wpsgd_objective",
    "wpsgd_run_chains_from", "wpsgd_shard_indices", "wpsgd_shard_indices_device",
    "wpsgd_run_spans_workspace", "wpsgd_run_spans", "wpsgd_span_condition", "wpsgd_objective_static",
    "wpsgd_chains_status", "wpsgd_run_delay_chains_workspace", "wpsgd_run_delay_chains",
    "wpsgd_quantize", "wpsgd_block_matmul_workspace", "wpsgd_block_matmul",
    "wpsgd_softmax_loss", "wpsgd_tensor_list_bytes", "wpsgd_tensor_list_make",
    "wpsgd_grad_norm_workspace", "wpsgd_grad_norm", "wpsgd_clip_grads", "wpsgd_clipped_step",
    "wpsgd_draw_classes",
]


class _CMatrix(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("d", ctypes.c_int64), ("dense", ctypes.c_void_p),
                ("ld", ctypes.c_int64), ("dtype", ctypes.c_int), ("row_ptr", ctypes.c_void_p),
                ("col_idx", ctypes.c_void_p), ("vals", ctypes.c_void_p)]


class _CPlan(ctypes.Structure):
    _fields_ = [("threads", ctypes.c_int), ("block_steps", ctypes.c_int),
                ("prefetch", ctypes.c_int), ("state_in_hbm", ctypes.c_int),
                ("rows", ctypes.c_int), ("helpers", ctypes.c_int), ("slices", ctypes.c_int),
                ("slice_wait_us", ctypes.c_int)]


class _CBlocks(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("codes", ctypes.c_void_p), ("ld", ctypes.c_int64),
                ("exps", ctypes.c_void_p), ("ld_exps", ctypes.c_int64)]


class _CTensor(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int)]


class _CTensorList(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("chunks", ctypes.c_int64), ("elements", ctypes.c_int64), ("has_weights", ctypes.c_int)]


class _CDrawRule(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("top_k", ctypes.c_int), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("row_temperature", ctypes.c_void_p), ("row_top_k", ctypes.c_void_p), ("row_top_p", ctypes.c_void_p),
                ("row_min_p", ctypes.c_void_p)]


class WpsgdError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        msg = load().wpsgd_strerror(status).decode()
        if status == HIP_ERROR:
            msg += f" [hipError {load().wpsgd_last_hip_error()}]"
        super().__init__(f"{what}: {msg} (status {status})")


_lib = None


def load():
    """Loads libwpsgd.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_1708_04801_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    i64, f64, ci, u64, vp, sz = (ctypes.c_int64, ctypes.c_double, ctypes.c_int, ctypes.c_uint64,
                                 ctypes.c_void_p, ctypes.c_size_t)
    pm, pp = ctypes.POINTER(_CMatrix), ctypes.POINTER(_CPlan)
    L.wpsgd_run_chains_workspace.argtypes = [pm, ci, ci, pp]
    L.wpsgd_run_chains_workspace.restype = sz
    L.wpsgd_run_chains.argtypes = [pm, vp, ci, vp, f64, f64, ci, u64, vp, vp, sz, pp, vp]
    L.wpsgd_run_chains_from.argtypes = [pm, vp, ci, vp, f64, f64, ci, u64, ci, vp, vp, vp, vp, sz, pp, vp]
    L.wpsgd_chains_status.argtypes = [vp, vp]
    L.wpsgd_run_delay_chains_workspace.argtypes = [pm, ci, ci]
    L.wpsgd_run_delay_chains_workspace.restype = sz
    L.wpsgd_run_delay_chains.argtypes = [pm, vp, ci, vp, f64, f64, ci, u64, ci, ci, vp, vp, vp, vp, sz, vp]
    L.wpsgd_run_spans_workspace.argtypes = [pm, ci, ci, pp]
    L.wpsgd_run_spans_workspace.restype = sz
    L.wpsgd_run_spans.argtypes = [pm, vp, ci, vp, i64, f64, f64, ci, u64, ci, vp, vp, vp, sz, pp, vp]
    L.wpsgd_span_condition.argtypes = [ci, vp, f64, vp]
    L.wpsgd_shard_indices.argtypes = [u64, ci, ci, i64, i64, i64, vp]
    L.wpsgd_shard_indices_device.argtypes = [u64, ci, ci, i64, i64, i64, vp, vp]
    L.wpsgd_weights.argtypes = [ci, vp, f64, f64, vp]
    L.wpsgd_weights_rate.argtypes = [ci, vp, f64, vp]
    L.wpsgd_benefit_margin.argtypes = [ci, vp, f64, vp]
    L.wpsgd_combine_workspace.argtypes = [ci, i64]
    L.wpsgd_combine_workspace.restype = sz
    L.wpsgd_combine.argtypes = [vp, vp, ci, i64, vp, vp, sz, vp]
    L.wpsgd_sample_indices.argtypes = [u64, ci, i64, i64, i64, vp]
    L.wpsgd_sample_indices_device.argtypes = [u64, ci, i64, i64, i64, vp, vp]
    L.wpsgd_strerror.argtypes = [ci]
    L.wpsgd_strerror.restype = ctypes.c_char_p
    L.wpsgd_last_hip_error.argtypes = []
    L.wpsgd_describe_plan.argtypes = [pm, ci, ci, pp, ctypes.c_char_p, sz]
    L.wpsgd_stream_rows.argtypes = [pm, ci, i64, u64, vp, vp]
    L.wpsgd_objective_workspace.argtypes = [pm]
    L.wpsgd_objective_workspace.restype = sz
    L.wpsgd_objective.argtypes = [pm, vp, vp, f64, ci, vp, vp, sz, vp]
    L.wpsgd_objective_static.argtypes = [pm, vp, vp, f64, ci, vp, vp]
    pb, pl, pt = ctypes.POINTER(_CBlocks), ctypes.POINTER(_CTensorList), ctypes.POINTER(_CTensor)
    L.wpsgd_quantize.argtypes = [pm, vp, i64, ci, pb, vp]
    L.wpsgd_block_matmul_workspace.argtypes = [i64, i64, i64]
    L.wpsgd_block_matmul_workspace.restype = sz
    L.wpsgd_block_matmul.argtypes = [pb, pb, vp, i64, ci, vp, sz, vp]
    L.wpsgd_softmax_loss.argtypes = [vp, i64, i64, i64, ci, vp, vp, f64, vp, vp, i64, vp]
    L.wpsgd_tensor_list_bytes.argtypes = [pt, i64]
    L.wpsgd_tensor_list_bytes.restype = sz
    L.wpsgd_tensor_list_make.argtypes = [pt, i64, vp, sz, pl, vp]
    L.wpsgd_grad_norm_workspace.argtypes = [pl]
    L.wpsgd_grad_norm_workspace.restype = sz
    L.wpsgd_grad_norm.argtypes = [pl, vp, vp, sz, vp]
    L.wpsgd_clip_grads.argtypes = [pl, f64, vp, vp, sz, vp]
    L.wpsgd_clipped_step.argtypes = [pl, f64, f64, f64, vp, vp, sz, vp]
    L.wpsgd_draw_classes.argtypes = [vp, i64, i64, i64, ci, vp, ctypes.POINTER(_CDrawRule), vp, vp, vp]
    _lib = L
    return L


@dataclass
class Matrix:
    """Device-resident data set.  dense: float32 [m,d] tensor, or int16/uint16/bfloat16 [m,d]
    holding bfloat16 values; or CSR with int64 row_ptr, int32 col_idx, float32 vals."""
    m: int
    d: int
    dense: Optional[torch.Tensor] = None
    row_ptr: Optional[torch.Tensor] = None
    col_idx: Optional[torch.Tensor] = None
    vals: Optional[torch.Tensor] = None

    def c_struct(self) -> _CMatrix:
        c = _CMatrix()
        c.m, c.d = int(self.m), int(self.d)
        if self.dense is not None:
            t = self.dense
            assert t.is_cuda and t.dim() == 2 and t.stride(1) == 1
            c.dense = t.data_ptr()
            c.ld = t.stride(0)
            c.dtype = F32 if t.dtype == torch.float32 else BF16
            assert t.dtype in (torch.float32, torch.bfloat16, torch.int16, torch.uint16)
        else:
            assert self.row_ptr.dtype == torch.int64 and self.col_idx.dtype == torch.int32
            assert self.vals.dtype == torch.float32 and self.row_ptr.is_cuda
            c.row_ptr, c.col_idx, c.vals = (self.row_ptr.data_ptr(), self.col_idx.data_ptr(),
                                            self.vals.data_ptr())
        return c


def matrix_from_workload(w, device="cuda") -> Matrix:
    """Uploads a generated workload's data set to the GPU."""
    if w.dense is not None:
        host = torch.from_numpy(w.dense.view(np.int16) if w.dense.dtype == np.uint16 else w.dense)
        dev = host.to(device)
        if w.dense.dtype == np.uint16:
            dev = dev.view(torch.bfloat16)
        return Matrix(w.m, w.d, dense=dev)
    return Matrix(w.m, w.d, row_ptr=torch.from_numpy(w.row_ptr).to(device),
                  col_idx=torch.from_numpy(w.col_idx).to(device),
                  vals=torch.from_numpy(w.vals).to(device))


def _plan(plan):
    if plan is None:
        return None
    p = _CPlan()
    p.threads = int(plan.get("threads", 0))
    p.block_steps = int(plan.get("block_steps", 0))
    p.prefetch = int(plan.get("prefetch", 0))
    p.state_in_hbm = int(plan.get("state_in_hbm", 0))
    p.rows = int(plan.get("rows", 0))
    p.helpers = int(plan.get("helpers", 0))
    p.slices = int(plan.get("slices", 0))
    p.slice_wait_us = int(plan.get("slice_wait_us", 0))
    return ctypes.byref(p)


def _stream(stream):
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _steps(n_steps):
    return np.ascontiguousarray(np.asarray(n_steps), dtype=np.int64)


def _workspace(nbytes, device, stream=None):
    """A temporary workspace for one call.  It is allocated on torch's current stream; when the call's
    work is queued on another stream the caching allocator is told so, or it could hand the block to
    later current-stream work while that stream still uses it."""
    t = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    if stream is not None:
        with torch.cuda.device(t.device):
            t.record_stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream)))
    return t


def wpsgd_describe_plan(X: Matrix, k, loss, plan=None) -> str:
    buf = ctypes.create_string_buffer(256)
    cm = X.c_struct()
    rc = load().wpsgd_describe_plan(ctypes.byref(cm), int(k), int(loss), _plan(plan), buf, 256)
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_describe_plan")
    return buf.value.decode()


def wpsgd_run_chains_workspace(X: Matrix, k, loss, plan=None) -> int:
    cm = X.c_struct()
    return int(load().wpsgd_run_chains_workspace(ctypes.byref(cm), int(k), int(loss), _plan(plan)))


def wpsgd_run_chains(X: Matrix, y: torch.Tensor, n_steps, eta, lam, loss, seed,
                     W: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     plan=None, stream=None) -> torch.Tensor:
    """Runs the k chains; returns W (k x d float32 on the GPU).  Asynchronous on the stream."""
    n = _steps(n_steps)
    k = int(n.size)
    dev = y.device
    assert y.is_cuda and y.dtype == torch.float32 and y.numel() == X.m
    if W is None:
        W = torch.empty((k, X.d), dtype=torch.float32, device=dev)
    assert W.is_cuda and W.dtype == torch.float32 and W.is_contiguous() and W.shape == (k, X.d)
    cm = X.c_struct()
    pl = _plan(plan)
    if workspace is None:
        need = load().wpsgd_run_chains_workspace(ctypes.byref(cm), k, int(loss), pl)
        workspace = _workspace(need, dev, stream)
    rc = load().wpsgd_run_chains(ctypes.byref(cm), y.data_ptr(), k, n.ctypes.data, float(eta),
                                 float(lam), int(loss), int(seed), W.data_ptr(),
                                 workspace.data_ptr(), workspace.numel(), pl, _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_run_chains")
    return W


def wpsgd_chains_status(workspace: torch.Tensor, stream=None) -> int:
    """OK, or INCOMPLETE when chains of the last call on this workspace gave up (waits for the stream)."""
    rc = load().wpsgd_chains_status(workspace.data_ptr(), _stream(stream))
    if rc not in (OK, INCOMPLETE):
        raise WpsgdError(rc, "wpsgd_chains_status")
    return rc


def wpsgd_run_chains_from(X: Matrix, y: torch.Tensor, n_steps, eta, lam, loss, seed,
                          w_start: Optional[torch.Tensor] = None, step_offsets=None, sampling=0,
                          W: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                          plan=None, stream=None) -> torch.Tensor:
    """wpsgd_run_chains from a common start vector (d float32 on the GPU, or None for zero) and
    from per-chain positions in the sample streams (k integers, or None for zero)."""
    n = _steps(n_steps)
    k = int(n.size)
    dev = y.device
    assert y.is_cuda and y.dtype == torch.float32 and y.numel() == X.m
    if w_start is not None:
        assert w_start.is_cuda and w_start.dtype == torch.float32 and w_start.is_contiguous() and w_start.numel() == X.d
    off = None
    if step_offsets is not None:
        off = _steps(step_offsets)
        assert off.size == k
    if W is None:
        W = torch.empty((k, X.d), dtype=torch.float32, device=dev)
    assert W.is_cuda and W.dtype == torch.float32 and W.is_contiguous() and W.shape == (k, X.d)
    cm = X.c_struct()
    pl = _plan(plan)
    if workspace is None:
        need = load().wpsgd_run_chains_workspace(ctypes.byref(cm), k, int(loss), pl)
        workspace = _workspace(need, dev, stream)
    rc = load().wpsgd_run_chains_from(ctypes.byref(cm), y.data_ptr(), k, n.ctypes.data, float(eta),
                                      float(lam), int(loss), int(seed), int(sampling),
                                      w_start.data_ptr() if w_start is not None else None,
                                      off.ctypes.data if off is not None else None, W.data_ptr(),
                                      workspace.data_ptr(), workspace.numel(), pl, _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_run_chains_from")
    return W


def wpsgd_run_delay_chains_workspace(X: Matrix, k, tau) -> int:
    cm = X.c_struct()
    return int(load().wpsgd_run_delay_chains_workspace(ctypes.byref(cm), int(k), int(tau)))


def wpsgd_run_delay_chains(X: Matrix, y: torch.Tensor, n_samples, eta, lam, loss, seed, tau, check=True,
                           w_start: Optional[torch.Tensor] = None, W: Optional[torch.Tensor] = None,
                           accepted: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                           stream=None):
    """Phase 1 of delay SGD under the Check function: k servers, server i fed n_samples[i] samples.
    Returns (W, accepted): k x d float32 and k int64, both on the GPU."""
    n = _steps(n_samples)
    k = int(n.size)
    dev = y.device
    assert y.is_cuda and y.dtype == torch.float32 and y.numel() == X.m
    if w_start is not None:
        assert w_start.is_cuda and w_start.dtype == torch.float32 and w_start.is_contiguous() and w_start.numel() == X.d
    if W is None:
        W = torch.empty((k, X.d), dtype=torch.float32, device=dev)
    if accepted is None:
        accepted = torch.empty(k, dtype=torch.int64, device=dev)
    assert W.is_cuda and W.dtype == torch.float32 and W.is_contiguous() and W.shape == (k, X.d)
    assert accepted.is_cuda and accepted.dtype == torch.int64 and accepted.is_contiguous() and accepted.numel() == k
    cm = X.c_struct()
    if workspace is None:
        need = load().wpsgd_run_delay_chains_workspace(ctypes.byref(cm), k, int(tau))
        workspace = _workspace(max(int(need), 256), dev, stream)
    rc = load().wpsgd_run_delay_chains(ctypes.byref(cm), y.data_ptr(), k, n.ctypes.data, float(eta), float(lam),
                                       int(loss), int(seed), int(tau), int(bool(check)),
                                       w_start.data_ptr() if w_start is not None else None, W.data_ptr(),
                                       accepted.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_run_delay_chains")
    return W, accepted


def wpsgd_run_spans_workspace(X: Matrix, k, loss, plan=None) -> int:
    cm = X.c_struct()
    return int(load().wpsgd_run_spans_workspace(ctypes.byref(cm), int(k), int(loss), _plan(plan)))


def wpsgd_run_spans(X: Matrix, y: torch.Tensor, steps_per_span, n_spans, eta, lam, loss, seed,
                    w_start: Optional[torch.Tensor] = None, sampling=0, w_out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, plan=None, stream=None) -> torch.Tensor:
    """Periodic weighted averaging: n_spans times, chains of steps_per_span steps from the common
    vector, then the Eq. 6 weighted sum.  Returns the vector after the last span (d float32)."""
    n = _steps(steps_per_span)
    k = int(n.size)
    dev = y.device
    assert y.is_cuda and y.dtype == torch.float32 and y.numel() == X.m
    if w_start is not None:
        assert w_start.is_cuda and w_start.dtype == torch.float32 and w_start.is_contiguous() and w_start.numel() == X.d
    if w_out is None:
        w_out = torch.empty(X.d, dtype=torch.float32, device=dev)
    assert w_out.is_cuda and w_out.dtype == torch.float32 and w_out.is_contiguous() and w_out.numel() == X.d
    cm = X.c_struct()
    pl = _plan(plan)
    if workspace is None:
        need = load().wpsgd_run_spans_workspace(ctypes.byref(cm), k, int(loss), pl)
        workspace = _workspace(need, dev, stream)
    rc = load().wpsgd_run_spans(ctypes.byref(cm), y.data_ptr(), k, n.ctypes.data, int(n_spans), float(eta),
                                float(lam), int(loss), int(seed), int(sampling),
                                w_start.data_ptr() if w_start is not None else None, w_out.data_ptr(),
                                workspace.data_ptr(), workspace.numel(), pl, _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_run_spans")
    return w_out


def wpsgd_span_condition(steps_per_span, rate) -> float:
    n = _steps(steps_per_span)
    out = ctypes.c_double(0.0)
    rc = load().wpsgd_span_condition(int(n.size), n.ctypes.data, float(rate), ctypes.addressof(out))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_span_condition")
    return out.value


def wpsgd_weights(n_steps, eta, lam) -> np.ndarray:
    n = _steps(n_steps)
    a = np.zeros(n.size, dtype=np.float64)
    rc = load().wpsgd_weights(int(n.size), n.ctypes.data, float(eta), float(lam), a.ctypes.data)
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_weights")
    return a


def wpsgd_weights_rate(n_steps, rate) -> np.ndarray:
    n = _steps(n_steps)
    a = np.zeros(n.size, dtype=np.float64)
    rc = load().wpsgd_weights_rate(int(n.size), n.ctypes.data, float(rate), a.ctypes.data)
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_weights_rate")
    return a


def wpsgd_benefit_margin(n_steps, rate) -> float:
    n = _steps(n_steps)
    out = ctypes.c_double(0.0)
    rc = load().wpsgd_benefit_margin(int(n.size), n.ctypes.data, float(rate),
                                     ctypes.addressof(out))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_benefit_margin")
    return out.value


def wpsgd_combine_workspace(k, d) -> int:
    return int(load().wpsgd_combine_workspace(int(k), int(d)))


def wpsgd_combine(W: torch.Tensor, a, w_out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """w_out = sum_i a[i] * W[i,:]; returns w_out (d float32 on the GPU)."""
    assert W.is_cuda and W.dtype == torch.float32 and W.dim() == 2 and W.is_contiguous()
    k, d = W.shape
    a = np.ascontiguousarray(np.asarray(a), dtype=np.float64)
    assert a.shape == (k,)
    if w_out is None:
        w_out = torch.empty(d, dtype=torch.float32, device=W.device)
    if workspace is None:
        workspace = _workspace(wpsgd_combine_workspace(k, d), W.device, stream)
    rc = load().wpsgd_combine(W.data_ptr(), a.ctypes.data, k, d, w_out.data_ptr(),
                              workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_combine")
    return w_out


def wpsgd_objective_workspace(X: Matrix) -> int:
    cm = X.c_struct()
    return int(load().wpsgd_objective_workspace(ctypes.byref(cm)))


def wpsgd_objective(X: Matrix, y: torch.Tensor, w: torch.Tensor, lam, loss, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Returns a 2-element float64 GPU tensor: [regularised objective, error rate] of model w on (X, y)."""
    assert y.is_cuda and y.dtype == torch.float32 and y.numel() == X.m
    assert w.is_cuda and w.dtype == torch.float32 and w.numel() == X.d and w.is_contiguous()
    cm = X.c_struct()
    if out is None:
        out = torch.empty(2, dtype=torch.float64, device=y.device)
    if workspace is None:
        workspace = _workspace(wpsgd_objective_workspace(X), y.device, stream)
    rc = load().wpsgd_objective(ctypes.byref(cm), y.data_ptr(), w.data_ptr(), float(lam), int(loss), out.data_ptr(),
                                workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_objective")
    return out


def wpsgd_objective_static(X: Matrix, y: torch.Tensor, w: torch.Tensor, lam, loss, out: torch.Tensor,
                           stream=None) -> torch.Tensor:
    """wpsgd_objective without a workspace: the library's own static device area holds the partial
    sums and the call allocates nothing (`out`, two float64 on the GPU, comes from the caller)."""
    assert y.is_cuda and y.dtype == torch.float32 and y.numel() == X.m
    assert w.is_cuda and w.dtype == torch.float32 and w.numel() == X.d and w.is_contiguous()
    assert out.is_cuda and out.dtype == torch.float64 and out.numel() == 2
    cm = X.c_struct()
    rc = load().wpsgd_objective_static(ctypes.byref(cm), y.data_ptr(), w.data_ptr(), float(lam), int(loss),
                                       out.data_ptr(), _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_objective_static")
    return out


def wpsgd_sample_indices(seed, chain, n0, count, m) -> np.ndarray:
    out = np.zeros(max(int(count), 0), dtype=np.int64)
    rc = load().wpsgd_sample_indices(int(seed), int(chain), int(n0), int(count), int(m),
                                     out.ctypes.data)
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_sample_indices")
    return out


def wpsgd_shard_indices(seed, chain, k, n0, count, m) -> np.ndarray:
    out = np.zeros(max(int(count), 0), dtype=np.int64)
    rc = load().wpsgd_shard_indices(int(seed), int(chain), int(k), int(n0), int(count), int(m), out.ctypes.data)
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_shard_indices")
    return out


def wpsgd_shard_indices_device(seed, chain, k, n0, count, m, device="cuda", stream=None) -> torch.Tensor:
    out = torch.empty(max(int(count), 0), dtype=torch.int64, device=device)
    rc = load().wpsgd_shard_indices_device(int(seed), int(chain), int(k), int(n0), int(count), int(m),
                                           out.data_ptr(), _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_shard_indices_device")
    return out


def wpsgd_sample_indices_device(seed, chain, n0, count, m, device="cuda", stream=None) -> torch.Tensor:
    out = torch.empty(max(int(count), 0), dtype=torch.int64, device=device)
    rc = load().wpsgd_sample_indices_device(int(seed), int(chain), int(n0), int(count), int(m),
                                            out.data_ptr(), _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_sample_indices_device")
    return out


def wpsgd_stream_rows(X: Matrix, groups, rows_per_group, seed=0, stream=None) -> torch.Tensor:
    """Streaming ceiling probe; returns the sink tensor (asynchronous, time it with events)."""
    sink = torch.empty(int(groups) * 256, dtype=torch.float32, device=X.dense.device)
    cm = X.c_struct()
    rc = load().wpsgd_stream_rows(ctypes.byref(cm), int(groups), int(rows_per_group), int(seed),
                                  sink.data_ptr(), _stream(stream))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_stream_rows")
    return sink


# ---- a linear model with many classes ----

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


# What torch.cuda.current_stream(i).cuda_stream gives, without the 2.6 us that it takes to make an object of it; not a public name of torch, so where a torch has it no more the
# object is made.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = torch.cuda.current_device


def _handle(stream):
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _beside(like, *tensors):
    """The index of like's GPU, on which all the others have to be (None: not given)."""
    index = like.get_device()
    for t in tensors:
        assert t is None or t.get_device() == index, "operands on different devices"
    return index


def _call(f, index, stream, *args):
    """f(*args, the stream's handle), for None that of the GPU's current stream, with that GPU as the current device: a launch goes to that, and so does the
    stream 0."""
    if stream is None:
        handle = _raw_stream(index)
    else:
        assert getattr(stream, "device_index", index) == index, "a stream of another device"
        handle = _handle(stream)
    if index == _current_device():
        return f(*args, handle)
    with torch.cuda.device(index):
        return f(*args, handle)


def _new(like, shape, dtype, stream):
    """Memory for a result or a workspace, from the pool of the stream that the work is queued on.  (A block of the current stream's pool may still be
    in use by work that waits there, and is handed out again as soon as its tensor goes.)"""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(_handle(stream), like.device)):
        return like.new_empty(shape, dtype=dtype)


_CODES = (torch.float8_e4m3fn, torch.uint8, torch.int8)


@dataclass
class BlockMatrix:
    """rows x cols in 8-bit floating point, a power of two for each block of 128 elements of a row:
    codes float8_e4m3fn [rows, whole blocks] with zeros behind the last column, exps uint8 [rows, blocks, padded to whole words],
    value = code * 2^(exp - 127).  wpsgd_quantize makes one."""
    rows: int
    cols: int
    codes: torch.Tensor
    exps: torch.Tensor

    def c_struct(self) -> _CBlocks:
        codes, exps, rows, cols = self.codes, self.exps, self.rows, self.cols
        assert codes.is_cuda and exps.is_cuda and codes.dtype in _CODES and exps.dtype == torch.uint8
        (r0, c0), (r1, c1), (ld, step), (ld_exps, step_exps) = codes.shape, exps.shape, codes.stride(), exps.stride()
        assert r0 == r1 == rows and 128 * c1 >= cols and c0 >= (cols + 127) // 128 * 128
        assert step == step_exps == 1 or rows == 0 or cols == 0
        return _CBlocks(rows, cols, codes.data_ptr(), ld, exps.data_ptr(), ld_exps)


def _call_workspace(workspace, need, like, stream):
    """The caller's workspace, or a temporary one, as address and size, and the tensor itself: whoever calls holds on to it until the
    work is queued."""
    if workspace is None:
        if not need:
            return None, 0, None
        workspace = _new(like, need, torch.uint8, stream)
        return workspace.data_ptr(), need, workspace
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def wpsgd_quantize(X: Matrix, rows: Optional[torch.Tensor] = None, transpose=False, codes: Optional[torch.Tensor] = None,
                   exps: Optional[torch.Tensor] = None, stream=None) -> BlockMatrix:
    """Rows of a dense data set (all, or those that `rows`, int64 on the GPU, names) as a BlockMatrix, blocks along the
    columns; transpose=True: one row for each column of X, blocks along the rows taken."""
    cm = X.c_struct()
    source = X.dense if X.dense is not None else X.vals
    n, picked, index = X.m, None, source.get_device()
    if rows is not None:
        assert rows.dtype == torch.int64 and rows.is_contiguous() and rows.get_device() == index
        n, picked = rows.numel(), rows.data_ptr()
    r, c = (X.d, n) if transpose else (n, X.d)
    blocks = -(-c // 128)
    words = (blocks + 3) // 4 * 4
    if codes is None and exps is None:
        codes, exps = _new(source, (r, 128 * blocks), torch.float8_e4m3fn, stream), _new(source, (r, words), torch.uint8, stream)
        out = BlockMatrix(r, c, codes, exps)
        c_out = _CBlocks(r, c, codes.data_ptr(), 128 * blocks, exps.data_ptr(), words)
    else:
        _beside(source, codes, exps)
        out = BlockMatrix(r, c, codes if codes is not None else _new(source, (r, 128 * blocks), torch.float8_e4m3fn, stream),
                          exps if exps is not None else _new(source, (r, words), torch.uint8, stream))
        c_out = out.c_struct()
    rc = _call(load().wpsgd_quantize, index, stream, ctypes.byref(cm), picked, n, 1 if transpose else 0, ctypes.byref(c_out))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_quantize")
    return out


def wpsgd_block_matmul_workspace(rows_a, rows_b, cols) -> int:
    return int(load().wpsgd_block_matmul_workspace(int(rows_a), int(rows_b), int(cols)))


def wpsgd_block_matmul(A: BlockMatrix, B: BlockMatrix, out: Optional[torch.Tensor] = None, dtype=torch.bfloat16,
                       workspace: Optional[torch.Tensor] = None, stream=None, fp32_sums=False) -> torch.Tensor:
    """out[i, j] = sum_c A[i, c] B[j, c], float32 or bfloat16.  fp32_sums: bfloat16 results of fp32 sums at large sizes, too, where the 8-bit
    matrix instructions would otherwise drop products under 2^-14 of the largest of their 64."""
    index = _beside(A.codes, A.exps, B.codes, B.exps, out, workspace)
    if out is None:
        out = _new(A.codes, (A.rows, B.rows), dtype, stream)
        assert dtype in _DTYPES
    else:
        assert out.dtype in _DTYPES and out.shape == (A.rows, B.rows) and (out.numel() == 0 or out.stride(1) == 1)
    L = load()
    p, size, held = _call_workspace(workspace, L.wpsgd_block_matmul_workspace(A.rows, B.rows, A.cols), out, stream)
    rc = _call(L.wpsgd_block_matmul, index, stream, ctypes.byref(A.c_struct()), ctypes.byref(B.c_struct()), out.data_ptr(),
               out.stride(0) if A.rows > 1 else max(out.stride(0), B.rows), _DTYPES[out.dtype] | (FP32_SUMS if fp32_sums else 0), p, size)
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_block_matmul")
    return out


def _rows_of(Z):
    n, c = Z.shape
    ld, step = Z.stride()
    assert Z.is_cuda and Z.dtype in _DTYPES and (step == 1 or n * c == 0)
    return n, c, ld if n > 1 else max(ld, c)


def wpsgd_softmax_loss(Z: torch.Tensor, labels: torch.Tensor, scale=1.0, row_weights: Optional[torch.Tensor] = None,
                       loss: Optional[torch.Tensor] = None, grad=True, stream=None):
    """(loss, grad): the rows' weighted cross-entropies (float32) and the gradient of scale * sum(loss) with respect to
    the scores Z, in Z's type.  grad: True for a new tensor, a tensor to write (Z itself too), or False for none."""
    n, c, ld = _rows_of(Z)
    index = _beside(Z, labels, row_weights, loss)
    assert labels.dtype == torch.int64 and labels.is_contiguous() and labels.numel() == n
    if row_weights is not None:
        assert row_weights.dtype == torch.float32 and row_weights.is_contiguous() and row_weights.numel() == n
    if loss is None:
        loss = _new(Z, n, torch.float32, stream)
    else:
        assert loss.dtype == torch.float32 and loss.is_contiguous() and loss.numel() == n
    if grad is True:
        grad = _new(Z, (n, c), Z.dtype, stream)
        g_ptr, g_ld = grad.data_ptr(), c
    elif grad is not False and grad is not None:
        gn, gc, g_ld = _rows_of(grad)
        assert grad.dtype == Z.dtype and gn == n and gc == c and grad.get_device() == index
        g_ptr = grad.data_ptr()
    else:
        grad, g_ptr, g_ld = None, None, 0
    rc = _call(load().wpsgd_softmax_loss, index, stream, Z.data_ptr(), n, c, ld, _DTYPES[Z.dtype], labels.data_ptr(),
               row_weights.data_ptr() if row_weights is not None else None, float(scale), loss.data_ptr(), g_ptr, g_ld)
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_softmax_loss")
    return loss, grad


class TensorList:
    """A model that lies in many tensors, as the calls below take it.  Holds on to the tensors; stays valid while they stay in place."""

    def __init__(self, grads, weights, table, c_list):
        self.grads, self.weights, self.table, self.c_list = grads, weights, table, c_list


def wpsgd_tensor_list(grads, weights=None, stream=None) -> TensorList:
    """Gradients (float32 or bfloat16) and, for steps, the weights (float32) of the same sizes; all contiguous, on one GPU.
    The list is ready when the stream has come to it: a call on another stream has to wait, as for any tensor."""
    grads = list(grads)
    weights = list(weights) if weights is not None else None
    assert weights is None or len(weights) == len(grads)
    items = (_CTensor * max(len(grads), 1))()
    device = grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
    for i, g in enumerate(grads):
        assert g.is_cuda and g.device == device and g.dtype in _DTYPES and g.is_contiguous()
        w = weights[i] if weights is not None else None
        if w is not None:
            assert w.device == device and w.dtype == torch.float32 and w.is_contiguous() and w.numel() == g.numel()
        items[i] = _CTensor(g.data_ptr(), w.data_ptr() if w is not None else None, g.numel(), _DTYPES[g.dtype])
    L = load()
    need = L.wpsgd_tensor_list_bytes(items, len(grads))
    table = _new(grads[0] if grads else torch.empty(0, device=device), need, torch.uint8, stream)
    c_list = _CTensorList()
    rc = _call(L.wpsgd_tensor_list_make, table.get_device(), stream, items, len(grads), table.data_ptr(), table.numel(), ctypes.byref(c_list))
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_tensor_list_make")
    return TensorList(grads, weights, table, c_list)


def wpsgd_grad_norm_workspace(tensors: TensorList) -> int:
    return int(load().wpsgd_grad_norm_workspace(ctypes.byref(tensors.c_list)))


def _norm_call(name, tensors, args, norm, workspace, stream):
    L = load()
    index = _beside(tensors.table, norm, workspace)
    if norm is None:
        norm = _new(tensors.table, (), torch.float32, stream)
    else:
        assert norm.dtype == torch.float32 and norm.numel() == 1
    c_list = ctypes.byref(tensors.c_list)
    p, size, held = _call_workspace(workspace, L.wpsgd_grad_norm_workspace(c_list), norm, stream)
    rc = _call(getattr(L, name), index, stream, c_list, *args, norm.data_ptr(), p, size)
    if rc != OK:
        raise WpsgdError(rc, name)
    return norm


def wpsgd_grad_norm(tensors: TensorList, norm: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The norm of all the list's gradients together (one float32 on the GPU)."""
    return _norm_call("wpsgd_grad_norm", tensors, (), norm, workspace, stream)


def wpsgd_clip_grads(tensors: TensorList, max_norm, norm: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """Scales the gradients in place to a norm of at most max_norm; returns the norm they had."""
    return _norm_call("wpsgd_clip_grads", tensors, (float(max_norm),), norm, workspace, stream)


def wpsgd_clipped_step(tensors: TensorList, eta, lam, max_norm=float("inf"), norm: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """weights <- (1 - eta lam) weights - eta min(1, max_norm / norm) gradients, in place; returns the gradients' norm."""
    return _norm_call("wpsgd_clipped_step", tensors, (float(eta), float(lam), float(max_norm)), norm, workspace, stream)


def wpsgd_draw_classes(Z: torch.Tensor, u: torch.Tensor, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
                       drawn: Optional[torch.Tensor] = None, probs: Optional[torch.Tensor] = None, stream=None):
    """(drawn, probs): a class for each row of the scores Z (int64, -1 where none can be drawn) and its probability among
    the classes that were kept (float32).  u: float32 in [0, 1).  Each setting is a number, or a tensor with one for each row (float32; top_k int32)."""
    n, c, ld = _rows_of(Z)
    index = _beside(Z, u, drawn, probs)
    assert u.dtype == torch.float32 and u.is_contiguous() and u.numel() == n
    rule = _CDrawRule(1.0, 0, 1.0, 0.0)
    for name, v, dt in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                        ("min_p", min_p, torch.float32)):
        if isinstance(v, torch.Tensor):
            assert v.get_device() == index and v.dtype == dt and v.is_contiguous() and v.numel() == n
            setattr(rule, "row_" + name, v.data_ptr())
        else:
            setattr(rule, name, v)
    if drawn is None:
        drawn = _new(u, n, torch.int64, stream)
    else:
        assert drawn.dtype == torch.int64 and drawn.is_contiguous() and drawn.numel() == n
    if probs is None:
        probs = _new(u, n, torch.float32, stream)
    else:
        assert probs.dtype == torch.float32 and probs.is_contiguous() and probs.numel() == n
    rc = _call(load().wpsgd_draw_classes, index, stream, Z.data_ptr(), n, c, ld, _DTYPES[Z.dtype], u.data_ptr(), ctypes.byref(rule), drawn.data_ptr(), probs.data_ptr())
    if rc != OK:
        raise WpsgdError(rc, "wpsgd_draw_classes")
    return drawn, probs
