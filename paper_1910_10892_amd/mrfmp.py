"""ctypes binding of libmrfmp: argument marshalling only.

Function names mirror include/mrfmp.h.  Tensors are torch CUDA(HIP) tensors; the binding
passes their device pointers and the current stream's handle.  There is no fallback: if
the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np

from .build import LIB_PATH

MRF_ISGMR, MRF_TRWP = 0, 1
MRF_F32, MRF_F16, MRF_BF16 = 0, 1, 2
_lib = None
# handle of a device's current stream without a stream object around it, where torch has it (a tenth of a microsecond instead of 2.7, as much as
# a launch); looked up with the library
_raw_stream = _current_device = None


class MrfError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = mrf_last_error_detail() if status == -9 else ""
        super().__init__("%s failed: %s (status %d)%s" % (where, mrf_strerror(status), status,
                                                          " [" + detail + "]" if detail else ""))


class _CProblem(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("W", ctypes.c_int32), ("L", ctypes.c_int32),
        ("R", ctypes.c_int32),
        ("dirs", ctypes.c_void_p),
        ("K", ctypes.c_int32),
        ("unary", ctypes.c_void_p),
        ("pairwise", ctypes.c_void_p),
        ("edge_weight", ctypes.c_void_p),
        ("edge_weight_scalar", ctypes.c_float),
        ("rho", ctypes.c_void_p),
        ("pairwise_kind", ctypes.c_int32),
        ("trunc", ctypes.c_float), ("scale", ctypes.c_float),
        ("rho_edge", ctypes.c_void_p),
        ("pairwise_edge", ctypes.c_void_p),
        ("sgm_standard", ctypes.c_int32),
    ]


def library_path() -> str:
    return LIB_PATH


def load_library():
    """Load libmrfmp.so (built in-tree by paper_1910_10892_amd.build); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            "libmrfmp.so not built: run `python -m paper_1910_10892_amd.build` (needs hipcc)")
    # The tensors this binding is handed live in PyTorch's HIP runtime.  Import torch first, so
    # that the library's dependency on libamdhip64 binds to the copy torch has loaded; loaded
    # the other way round the process ends up with two runtimes and the library's own sees
    # no initialised device.
    import torch
    global _raw_stream, _current_device
    _raw_stream, _current_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    P = ctypes.POINTER(_CProblem)
    lib.mrf_workspace_bytes.restype = sz
    lib.mrf_workspace_bytes.argtypes = [P, ci, ci]
    lib.mrf_validate.restype = ci
    lib.mrf_validate.argtypes = [P, ci]
    lib.mrf_forward_window.restype = ci
    lib.mrf_forward_window.argtypes = [P, ci]
    for name in ("mrf_isgmr_forward", "mrf_trwp_forward"):
        f = getattr(lib, name)
        f.restype = ci
        f.argtypes = [P, vp, vp, vp, vp, vp, vp, sz, vp]
    for name in ("mrf_isgmr_backward", "mrf_trwp_backward"):
        f = getattr(lib, name)
        f.restype = ci
        f.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.mrf_scanline_count.restype = ctypes.c_int64
    lib.mrf_scanline_count.argtypes = [ctypes.c_int32] * 4
    lib.mrf_scanline_head.restype = ci
    lib.mrf_scanline_head.argtypes = [ctypes.c_int32] * 4 + [ctypes.c_int64] + [ctypes.POINTER(ctypes.c_int32)] * 3
    lib.mrf_strerror.restype = ctypes.c_char_p
    lib.mrf_last_error_detail.restype = ctypes.c_char_p
    lib.mrf_last_error_detail.argtypes = []
    lib.mrf_last_sweep_kernel.restype = ctypes.c_char_p
    lib.mrf_last_sweep_kernel.argtypes = [ci]
    lib.mrf_last_sweep_launch.restype = ctypes.c_char_p
    lib.mrf_last_sweep_launch.argtypes = [ci]
    lib.mrf_energy_workspace_bytes.restype = sz
    lib.mrf_energy_workspace_bytes.argtypes = [P]
    lib.mrf_energy.restype = ci
    lib.mrf_energy.argtypes = [P, vp, vp, vp, sz, vp]
    lib.mrf_energy_noalloc.restype = ci
    lib.mrf_energy_noalloc.argtypes = [P, vp, vp, vp]
    lib.mrf_softmin_l1_workspace_bytes.restype = sz
    lib.mrf_softmin_l1_workspace_bytes.argtypes = []
    lib.mrf_softmin_l1.restype = ci
    lib.mrf_softmin_l1.argtypes = [ctypes.c_int64, ctypes.c_int32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.mrf_softmin_smooth_l1.restype = ci
    lib.mrf_softmin_smooth_l1.argtypes = [ctypes.c_int64, ctypes.c_int32, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, sz, vp]
    i32, i64, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.mrf_layer_norm_workspace_bytes.restype = sz
    lib.mrf_layer_norm_workspace_bytes.argtypes = [i64, i32]
    lib.mrf_layer_norm_forward.restype = ci
    lib.mrf_layer_norm_forward.argtypes = [i64, i32, vp, ci, vp, vp, f32, vp, ci, vp, vp, vp]
    lib.mrf_layer_norm_backward.restype = ci
    lib.mrf_layer_norm_backward.argtypes = [i64, i32, vp, ci, vp, ci, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.mrf_distance_buckets.restype = ci
    lib.mrf_distance_buckets.argtypes = [i32, i64, ci, i64, i64, vp]
    lib.mrf_bucket_pairwise_workspace_bytes.restype = sz
    lib.mrf_bucket_pairwise_workspace_bytes.argtypes = [i64, i32, i32, i32]
    lib.mrf_bucket_pairwise_forward.restype = ci
    lib.mrf_bucket_pairwise_forward.argtypes = [i64, i32, i32, i32, vp, ci, vp, i64, i64, i64, vp, ci, vp]
    lib.mrf_bucket_pairwise_backward.restype = ci
    lib.mrf_bucket_pairwise_backward.argtypes = [i64, i32, i32, i32, vp, ci, ci, vp, i64, i64, i64, vp, vp, sz, vp]
    lib.mrf_softmin_logp.restype = ci
    lib.mrf_softmin_logp.argtypes = [i64, i32, vp, ci, vp, ci, vp, vp]
    lib.mrf_softmin_policy_workspace_bytes.restype = sz
    lib.mrf_softmin_policy_workspace_bytes.argtypes = []
    lib.mrf_softmin_policy.restype = ci
    lib.mrf_softmin_policy.argtypes = [i64, i32, vp, ci, vp, ci, vp, i64, vp, vp, vp, f32, f32, f32, f32, vp, vp, vp, vp, sz, vp]
    lib.mrf_softmin_policy_backward.restype = ci
    lib.mrf_softmin_policy_backward.argtypes = [i64, i32, vp, ci, vp, ci, vp, i64, vp, vp, vp, f32, f32, f32, vp, vp, vp, sz, vp]
    lib.mrf_workspace_fault.restype = ci
    lib.mrf_workspace_fault.argtypes = [vp, vp]
    lib.mrf_strerror.argtypes = [ci]
    lib.mrf_version.restype = ctypes.c_char_p
    lib.mrf_set_sweep_events.restype = ci
    lib.mrf_set_sweep_events.argtypes = [vp, vp]
    lib.mrf_tune.restype = ci
    lib.mrf_tune.argtypes = [ci, ci]
    _lib = lib
    return lib


def _dev_ptr(t, dtype_name: Optional[str] = None):
    """Device pointer of a contiguous torch tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous and on the GPU")
    if dtype_name is not None and _dtype_name(t) != dtype_name:
        raise ValueError("expected %s tensor, got %s" % (dtype_name, t.dtype))
    return ctypes.c_void_p(t.data_ptr())


_dtype_names = {}      # torch dtype -> its name without "torch." (the text costs more than the call otherwise)


def _dtype_name(t) -> str:
    name = _dtype_names.get(t.dtype)
    if name is None:
        name = _dtype_names[t.dtype] = str(t.dtype).rsplit(".", 1)[-1]
    return name


@dataclass
class MrfProblem:
    """Mirror of the C struct mrf_problem.  unary/pairwise/edge_weight are GPU tensors,
    dirs and rho are host sequences."""
    unary: object                 # [B,H,W,L] float32 GPU tensor (may be None for backward)
    pairwise: object              # [L,L] float32 GPU tensor
    dirs: Sequence                # R x (dh, dw)
    K: int
    edge_weight: object = None    # [R,B,H,W] float32 GPU tensor or None
    edge_weight_scalar: float = 1.0
    rho: Optional[Sequence] = None
    pairwise_kind: int = 0
    trunc: float = 0.0
    scale: float = 1.0
    shape: Optional[tuple] = None  # (B,H,W,L); taken from unary when given
    rho_edge: object = None       # [R,B,H,W] float32 GPU tensor or None (TRWP: rho per directed edge)
    pairwise_edge: object = None  # [R,B,H,W,L,L] float32 GPU tensor or None (pairwise potentials per edge)
    sgm_standard: bool = False    # standard single-pass SGM (Eq. sgm_old) instead of the revised update; forward, K = 1

    def __post_init__(self):
        if self.shape is None:
            self.shape = tuple(int(v) for v in self.unary.shape)
        self._dirs = np.ascontiguousarray(np.asarray(self.dirs, np.int32).reshape(-1, 2))
        self._rho = None if self.rho is None else np.ascontiguousarray(
            np.broadcast_to(np.asarray(self.rho, np.float32), (self._dirs.shape[0],)))

    @property
    def R(self):
        return int(self._dirs.shape[0])

    def c_struct(self) -> _CProblem:
        B, H, W, L = self.shape
        c = _CProblem()
        c.B, c.H, c.W, c.L, c.R, c.K = B, H, W, L, self.R, int(self.K)
        c.dirs = self._dirs.ctypes.data
        c.unary = _dev_ptr(self.unary, "float32")
        c.pairwise = _dev_ptr(self.pairwise, "float32")
        c.edge_weight = _dev_ptr(self.edge_weight, "float32")
        c.edge_weight_scalar = float(self.edge_weight_scalar)
        c.rho = None if self._rho is None else self._rho.ctypes.data
        c.pairwise_kind = int(self.pairwise_kind)
        c.trunc, c.scale = float(self.trunc), float(self.scale)
        c.rho_edge = _dev_ptr(self.rho_edge, "float32")
        c.pairwise_edge = _dev_ptr(self.pairwise_edge, "float32")
        c.sgm_standard = 1 if self.sgm_standard else 0
        return c


def _stream_handle(stream):
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    if _raw_stream is not None:
        return _raw_stream(_current_device())
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def mrf_strerror(status: int) -> str:
    return load_library().mrf_strerror(int(status)).decode()


def mrf_last_error_detail() -> str:
    return load_library().mrf_last_error_detail().decode()


def mrf_last_sweep_kernel(backward: bool) -> str:
    return load_library().mrf_last_sweep_kernel(1 if backward else 0).decode()


def mrf_last_sweep_launch(backward: bool) -> str:
    return load_library().mrf_last_sweep_launch(1 if backward else 0).decode()


def mrf_version() -> str:
    return load_library().mrf_version().decode()


def mrf_tune(knob: int, value: int) -> int:
    return int(load_library().mrf_tune(int(knob), int(value)))


def mrf_set_sweep_events(start_event, stop_event) -> int:
    """start_event / stop_event: torch.cuda.Event(enable_timing=True) that have been recorded
    once (so that their HIP handles exist), or None, None to clear."""
    h = lambda e: None if e is None else ctypes.c_void_p(e.cuda_event)
    return int(load_library().mrf_set_sweep_events(h(start_event), h(stop_event)))


def mrf_validate(prob: MrfProblem, algo: int) -> int:
    c = prob.c_struct()
    return int(load_library().mrf_validate(ctypes.byref(c), int(algo)))


def mrf_forward_window(prob: MrfProblem, algo: int) -> int:
    c = prob.c_struct()
    return int(load_library().mrf_forward_window(ctypes.byref(c), int(algo)))


def mrf_workspace_bytes(prob: MrfProblem, algo: int, backward: bool) -> int:
    c = prob.c_struct()
    return int(load_library().mrf_workspace_bytes(ctypes.byref(c), int(algo), int(bool(backward))))


def mrf_scanline_count(H: int, W: int, dh: int, dw: int) -> int:
    return int(load_library().mrf_scanline_count(H, W, dh, dw))


def mrf_scanline_head(H: int, W: int, dh: int, dw: int, t: int):
    y, x, n = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    rc = load_library().mrf_scanline_head(H, W, dh, dw, t, ctypes.byref(y), ctypes.byref(x), ctypes.byref(n))
    if rc != 0:
        raise MrfError(rc, "mrf_scanline_head")
    return y.value, x.value, n.value


def _forward(name, prob, cost, labels, p, q, messages, workspace, stream):
    c = prob.c_struct()
    rc = getattr(load_library(), name)(
        ctypes.byref(c), _dev_ptr(cost, "float32"), _dev_ptr(labels, "uint8"), _dev_ptr(p, "uint8"),
        _dev_ptr(q, "uint8"), _dev_ptr(messages, "float32"), _dev_ptr(workspace),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if rc != 0:
        raise MrfError(rc, name)


def _backward(name, prob, grad_cost, p, q, grad_unary, grad_edge_weight, grad_pairwise, workspace, stream):
    c = prob.c_struct()
    rc = getattr(load_library(), name)(
        ctypes.byref(c), _dev_ptr(grad_cost, "float32"), _dev_ptr(p, "uint8"), _dev_ptr(q, "uint8"),
        _dev_ptr(grad_unary, "float32"), _dev_ptr(grad_edge_weight, "float32"),
        _dev_ptr(grad_pairwise, "float32"), _dev_ptr(workspace),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if rc != 0:
        raise MrfError(rc, name)


def mrf_isgmr_forward(prob, cost, labels, p, q, messages, workspace, stream=None):
    _forward("mrf_isgmr_forward", prob, cost, labels, p, q, messages, workspace, stream)


def mrf_trwp_forward(prob, cost, labels, p, q, messages, workspace, stream=None):
    _forward("mrf_trwp_forward", prob, cost, labels, p, q, messages, workspace, stream)


def mrf_isgmr_backward(prob, grad_cost, p, q, grad_unary, grad_edge_weight, grad_pairwise, workspace,
                       stream=None):
    _backward("mrf_isgmr_backward", prob, grad_cost, p, q, grad_unary, grad_edge_weight, grad_pairwise,
              workspace, stream)


def mrf_trwp_backward(prob, grad_cost, p, q, grad_unary, grad_edge_weight, grad_pairwise, workspace,
                      stream=None):
    _backward("mrf_trwp_backward", prob, grad_cost, p, q, grad_unary, grad_edge_weight, grad_pairwise,
              workspace, stream)


def _ws_size(workspace) -> int:
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def mrf_energy_workspace_bytes(prob) -> int:
    c = prob.c_struct()
    return int(load_library().mrf_energy_workspace_bytes(ctypes.byref(c)))


def mrf_energy(prob, labels, energy, workspace, stream=None):
    """labels [B,H,W] uint8, energy [B] float64 (assigned), workspace uint8 tensor."""
    c = prob.c_struct()
    rc = load_library().mrf_energy(ctypes.byref(c), _dev_ptr(labels, "uint8"), _dev_ptr(energy, "float64"),
                                   _dev_ptr(workspace), _ws_size(workspace), _stream_handle(stream))
    if rc != 0:
        raise MrfError(rc, "mrf_energy")


def mrf_energy_noalloc(prob, labels, energy, stream=None):
    """mrf_energy without a workspace argument (the library's own fixed scratch; batch <= 64)."""
    c = prob.c_struct()
    rc = load_library().mrf_energy_noalloc(ctypes.byref(c), _dev_ptr(labels, "uint8"), _dev_ptr(energy, "float64"),
                                           _stream_handle(stream))
    if rc != 0:
        raise MrfError(rc, "mrf_energy_noalloc")


def mrf_softmin_l1_workspace_bytes() -> int:
    return int(load_library().mrf_softmin_l1_workspace_bytes())


def mrf_softmin_l1(cost, target, mask, disparity, loss, grad_cost, workspace, stream=None):
    """cost [..., L] float32, target [...] float32, mask [...] uint8 or None, disparity [...] float32 or
    None, loss [1] float64, grad_cost like cost or None."""
    L = int(cost.shape[-1])
    n = int(cost.numel() // L)
    rc = load_library().mrf_softmin_l1(n, L, _dev_ptr(cost, "float32"), _dev_ptr(target, "float32"),
                                       _dev_ptr(mask, "uint8"), _dev_ptr(disparity, "float32"),
                                       _dev_ptr(loss, "float64"), _dev_ptr(grad_cost, "float32"),
                                       _dev_ptr(workspace), _ws_size(workspace), _stream_handle(stream))
    if rc != 0:
        raise MrfError(rc, "mrf_softmin_l1")


def mrf_softmin_smooth_l1(cost, target, mask, beta, disparity, loss, grad_cost, workspace, stream=None):
    """mrf_softmin_l1 with the smooth L1 loss (threshold beta > 0)."""
    L = int(cost.shape[-1])
    n = int(cost.numel() // L)
    rc = load_library().mrf_softmin_smooth_l1(n, L, _dev_ptr(cost, "float32"), _dev_ptr(target, "float32"),
                                              _dev_ptr(mask, "uint8"), ctypes.c_float(beta), _dev_ptr(disparity, "float32"),
                                              _dev_ptr(loss, "float64"), _dev_ptr(grad_cost, "float32"),
                                              _dev_ptr(workspace), _ws_size(workspace), _stream_handle(stream))
    if rc != 0:
        raise MrfError(rc, "mrf_softmin_smooth_l1")


# ---- learning operators: element types and sizes come from the tensors, which have to fit each other (ValueError)

_TYPES = {"float32": MRF_F32, "float16": MRF_F16, "bfloat16": MRF_BF16}


def _type_of(t, what) -> int:
    code = _TYPES.get(_dtype_name(t))
    if code is None:
        raise ValueError("%s must be float32, float16 or bfloat16, got %s" % (what, t.dtype))
    return code


def _ptr(t, dtype_name: Optional[str]):
    """_dev_ptr for an argument that is declared a pointer: the plain address."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous and on the GPU")
    if dtype_name is not None and _dtype_name(t) != dtype_name:
        raise ValueError("expected %s tensor, got %s" % (dtype_name, t.dtype))
    return t.data_ptr()


def _same_size(what, t, *shape):
    if t is not None and t.shape != shape:      # (a torch.Size is a tuple)
        raise ValueError("%s has shape %s, expected %s" % (what, tuple(t.shape), shape))


def _size(n) -> int:
    # (an argument that does not fit its 32 bits would lose the others on the way to the library)
    if n > 0x7fffffff:
        raise ValueError("sizes of the last indices are at most 2^31 - 1, got %d" % n)
    return int(n)


def _checked(rc, name):
    if rc != 0:
        raise MrfError(rc, name)


def mrf_layer_norm_workspace_bytes(n_rows: int, C: int) -> int:
    return int(load_library().mrf_layer_norm_workspace_bytes(int(n_rows), int(C)))


def mrf_layer_norm_forward(x, gamma, beta, eps, y, mean, rstd, stream=None):
    """x [..., C] float32, float16 or bfloat16, gamma and beta [C] float32 or None, y like x (or float32), mean and rstd
    [...] float32 or None."""
    C, rows = _size(x.shape[-1]), tuple(x.shape[:-1])
    _same_size("y", y, *x.shape)
    for name, t in (("gamma", gamma), ("beta", beta)):
        _same_size(name, t, C)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _same_size(name, t, *rows)
    _checked(load_library().mrf_layer_norm_forward(
        math.prod(rows), C, _ptr(x, None), _type_of(x, "x"), _ptr(gamma, "float32"), _ptr(beta, "float32"), float(eps),
        _ptr(y, None), _type_of(y, "y"), _ptr(mean, "float32"), _ptr(rstd, "float32"), _stream_handle(stream)),
        "mrf_layer_norm_forward")


def mrf_layer_norm_backward(grad_y, x, gamma, mean, rstd, grad_x, grad_gamma, grad_beta, workspace, stream=None):
    """grad_y [..., C] of y's type, x, gamma, mean, rstd of the forward call; grad_x like x, grad_gamma and grad_beta [C] float32,
    each of the three or None."""
    C, rows = _size(x.shape[-1]), tuple(x.shape[:-1])
    _same_size("grad_y", grad_y, *x.shape)
    _same_size("grad_x", grad_x, *x.shape)
    for name, t in (("gamma", gamma), ("grad_gamma", grad_gamma), ("grad_beta", grad_beta)):
        _same_size(name, t, C)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _same_size(name, t, *rows)
    if grad_x is not None and grad_x.dtype != x.dtype:
        raise ValueError("grad_x must be %s like x, got %s" % (x.dtype, grad_x.dtype))
    _checked(load_library().mrf_layer_norm_backward(
        math.prod(rows), C, _ptr(grad_y, None), _type_of(grad_y, "grad_y"), _ptr(x, None), _type_of(x, "x"), _ptr(gamma, "float32"),
        _ptr(mean, "float32"), _ptr(rstd, "float32"), _ptr(grad_x, None), _ptr(grad_gamma, "float32"),
        _ptr(grad_beta, "float32"), _ptr(workspace, None), _ws_size(workspace), _stream_handle(stream)), "mrf_layer_norm_backward")


def mrf_distance_buckets(n_buckets: int, far_distance: int, first_offset: int, n_offsets: int, two_sided: bool = True):
    """Host array [n_offsets] int32: bucket of the offsets first_offset, first_offset + 1, .. (see the header)."""
    out = np.empty(max(int(n_offsets), 0), np.int32)
    _checked(load_library().mrf_distance_buckets(int(n_buckets), int(far_distance), int(bool(two_sided)), int(first_offset),
                                                 int(n_offsets), out.ctypes.data), "mrf_distance_buckets")
    return out


def mrf_bucket_pairwise_workspace_bytes(n_groups: int, Q: int, K: int, n_buckets: int) -> int:
    return int(load_library().mrf_bucket_pairwise_workspace_bytes(int(n_groups), int(Q), int(K), int(n_buckets)))


def _bucket_sizes(table, out, heads_last):
    """Groups, rows, columns and buckets of a table [..., n_buckets] (heads_last: [n_buckets, ...]) and a matrix [..., Q, K]."""
    groups = tuple(out.shape[:-2])
    NB = _size(table.shape[0] if heads_last else table.shape[-1])
    _same_size("table", table, *((NB, *groups) if heads_last else (*groups, NB)))
    return math.prod(groups), _size(out.shape[-2]), _size(out.shape[-1]), NB


def mrf_bucket_pairwise_forward(table, bucket_of, first_offset, out, query_offset=0, heads_last=False, stream=None):
    """table [..., n_buckets] float32 (heads_last: [n_buckets, ...]), bucket_of [n] int32 on the GPU for the offsets from
    first_offset on, out [..., Q, K] float32, float16 or bfloat16."""
    G, Q, K, NB = _bucket_sizes(table, out, heads_last)
    _checked(load_library().mrf_bucket_pairwise_forward(
        G, Q, K, NB, _ptr(table, "float32"), int(bool(heads_last)), _ptr(bucket_of, "int32"), int(first_offset),
        int(bucket_of.numel()), int(query_offset), _ptr(out, None), _type_of(out, "out"), _stream_handle(stream)),
        "mrf_bucket_pairwise_forward")


def mrf_bucket_pairwise_backward(grad_out, bucket_of, first_offset, grad_table, workspace, query_offset=0, heads_last=False, stream=None):
    """grad_out [..., Q, K], grad_table like the table of the forward call."""
    G, Q, K, NB = _bucket_sizes(grad_table, grad_out, heads_last)
    _checked(load_library().mrf_bucket_pairwise_backward(
        G, Q, K, NB, _ptr(grad_out, None), _type_of(grad_out, "grad_out"), int(bool(heads_last)), _ptr(bucket_of, "int32"),
        int(first_offset), int(bucket_of.numel()), int(query_offset), _ptr(grad_table, "float32"), _ptr(workspace, None),
        _ws_size(workspace), _stream_handle(stream)), "mrf_bucket_pairwise_backward")


def _label_bytes(labels) -> int:
    size = {"uint8": 1, "int32": 4}.get(_dtype_name(labels))
    if size is None:
        raise ValueError("labels must be uint8 or int32, got %s" % labels.dtype)
    return size


def mrf_softmin_logp(cost, labels, logp, stream=None):
    """cost [..., L] float32, float16 or bfloat16, labels [...] uint8 (L <= 256) or int32, logp [...] float32."""
    pixels, L = tuple(cost.shape[:-1]), _size(cost.shape[-1])
    _same_size("labels", labels, *pixels)
    _same_size("logp", logp, *pixels)
    _checked(load_library().mrf_softmin_logp(math.prod(pixels), L, _ptr(cost, None), _type_of(cost, "cost"), _ptr(labels, None),
                                             _label_bytes(labels), _ptr(logp, "float32"), _stream_handle(stream)), "mrf_softmin_logp")


def mrf_softmin_policy_workspace_bytes() -> int:
    return int(load_library().mrf_softmin_policy_workspace_bytes())


def _policy_sizes(cost, labels, advantage, old_logp, ref_logp, mask, logp, grad_cost, pixels_per_advantage):
    """Pixels, labels and pixels per advantage of tensors that fit each other."""
    pixels, L = tuple(cost.shape[:-1]), _size(cost.shape[-1])
    n, per = math.prod(pixels), int(pixels_per_advantage)
    for name, t in (("labels", labels), ("old_logp", old_logp), ("ref_logp", ref_logp), ("mask", mask), ("logp", logp)):
        _same_size(name, t, *pixels)
    _same_size("grad_cost", grad_cost, *cost.shape)
    if grad_cost is not None and grad_cost.dtype != cost.dtype:
        raise ValueError("grad_cost must be %s like cost, got %s" % (cost.dtype, grad_cost.dtype))
    if per >= 1 and int(advantage.numel()) != -(-n // per):
        raise ValueError("advantage has %d entries, expected %d" % (advantage.numel(), -(-n // per)))
    return n, L, per


def mrf_softmin_policy(cost, labels, advantage, old_logp, ref_logp, mask, clip_low, clip_high, kl_weight, loss, logp, grad_cost,
                       workspace, pixels_per_advantage=1, grad_scale=1.0, stream=None):
    """cost [..., L] float32, float16 or bfloat16, labels [...] uint8 or int32, advantage float32 with an entry per
    pixels_per_advantage pixels, old_logp and ref_logp [...] float32 or None, mask [...] uint8 or None, loss [3] float32, logp
    [...] float32 or None, grad_cost like cost or None."""
    n, L, per = _policy_sizes(cost, labels, advantage, old_logp, ref_logp, mask, logp, grad_cost, pixels_per_advantage)
    _same_size("loss", loss, 3)
    _checked(load_library().mrf_softmin_policy(
        n, L, _ptr(cost, None), _type_of(cost, "cost"), _ptr(labels, None), _label_bytes(labels), _ptr(advantage, "float32"), per,
        _ptr(old_logp, "float32"), _ptr(ref_logp, "float32"), _ptr(mask, "uint8"), float(clip_low), float(clip_high),
        float(kl_weight), float(grad_scale), _ptr(loss, "float32"), _ptr(logp, "float32"), _ptr(grad_cost, None),
        _ptr(workspace, None), _ws_size(workspace), _stream_handle(stream)), "mrf_softmin_policy")


def mrf_softmin_policy_backward(cost, labels, advantage, old_logp, ref_logp, mask, clip_low, clip_high, kl_weight, grad_loss, grad_cost,
                                workspace, pixels_per_advantage=1, stream=None):
    """As mrf_softmin_policy; grad_loss float32 of one entry on the GPU, grad_cost like cost."""
    n, L, per = _policy_sizes(cost, labels, advantage, old_logp, ref_logp, mask, None, grad_cost, pixels_per_advantage)
    if int(grad_loss.numel()) != 1:
        raise ValueError("grad_loss has %d entries, expected 1" % grad_loss.numel())
    for t, name in ((cost, None), (labels, None), (advantage, "float32"), (old_logp, "float32"), (ref_logp, "float32"), (mask, "uint8"),
                    (grad_loss, "float32"), (grad_cost, None), (workspace, None)):
        _ptr(t, name)
    _policy_backward((n, L, per, _type_of(cost, "cost"), _label_bytes(labels), float(clip_low), float(clip_high), float(kl_weight)), cost, labels,
                     advantage, old_logp, ref_logp, mask, grad_loss, grad_cost, workspace, stream)


def _policy_backward(given, cost, labels, advantage, old_logp, ref_logp, mask, grad_loss, grad_cost, workspace, stream=None):
    """The call itself, of tensors that have been checked; `given`: pixels, labels, pixels per advantage, codes of the costs' and labels' types,
    and the three numbers."""
    n, L, per, cost_type, label_bytes, clip_low, clip_high, kl_weight = given
    _checked(load_library().mrf_softmin_policy_backward(
        n, L, cost.data_ptr(), cost_type, labels.data_ptr(), label_bytes, advantage.data_ptr(), per,
        None if old_logp is None else old_logp.data_ptr(), None if ref_logp is None else ref_logp.data_ptr(),
        None if mask is None else mask.data_ptr(), clip_low, clip_high, kl_weight, grad_loss.data_ptr(),
        None if grad_cost is None else grad_cost.data_ptr(), None if workspace is None else workspace.data_ptr(),
        _ws_size(workspace), _stream_handle(stream)), "mrf_softmin_policy_backward")


def mrf_workspace_fault(workspace, stream=None) -> int:
    """0, or -11 if a wait between wavefronts ran out in the last call that used this workspace
    (synchronises the stream)."""
    return int(load_library().mrf_workspace_fault(_dev_ptr(workspace), _stream_handle(stream)))
