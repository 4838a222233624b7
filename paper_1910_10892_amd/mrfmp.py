"""ctypes binding of libmrfmp: argument marshalling only.

Function names mirror include/mrfmp.h.  Tensors are torch CUDA(HIP) tensors; the binding
passes their device pointers and the current stream's handle.  There is no fallback: if
the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
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
_device_now = None      # the current device without asking whether there is one: for calls that have a tensor on it
_int32 = _float32 = None      # torch's types, with the library


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


class _CAttention(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Q", "K", "Hq", "Hk", "D", "type")] + [
        ("scale", ctypes.c_float),
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
        ("first_offset", ctypes.c_int64), ("last_offset", ctypes.c_int64), ("query_offset", ctypes.c_int64),
        ("query_offsets", ctypes.c_void_p), ("q_lengths", ctypes.c_void_p), ("k_lengths", ctypes.c_void_p),
        ("table", ctypes.c_void_p), ("bucket_of", ctypes.c_void_p),
        ("map_offset", ctypes.c_int64), ("n_offsets", ctypes.c_int64),
        ("n_buckets", ctypes.c_int32), ("heads_last", ctypes.c_int32),
    ]


class _CHeadRotation(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "Hq", "Hk", "D", "type")] + [
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("gamma_q", ctypes.c_void_p), ("gamma_k", ctypes.c_void_p),
        ("eps", ctypes.c_float), ("rotary", ctypes.c_int32), ("interleaved", ctypes.c_int32),
        ("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p),
        ("n_axes", ctypes.c_int32), ("position_offset", ctypes.c_int64),
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
    global _raw_stream, _current_device, _device_now, _int32, _float32
    _raw_stream, _current_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device
    _device_now = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _int32, _float32 = torch.int32, torch.float32
    _codes.update({torch.float32: MRF_F32, torch.float16: MRF_F16, torch.bfloat16: MRF_BF16})
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
    A, R = ctypes.POINTER(_CAttention), ctypes.c_char_p      # (a rotation's description goes as its packed bytes)
    lib.mrf_attention_workspace_bytes.restype = sz
    lib.mrf_attention_workspace_bytes.argtypes = [A, ci]
    lib.mrf_attention_forward.restype = ci
    lib.mrf_attention_forward.argtypes = [A, vp, vp, vp, sz, vp]
    lib.mrf_attention_backward.restype = ci
    lib.mrf_attention_backward.argtypes = [A, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.mrf_head_rotation_workspace_bytes.restype = sz
    lib.mrf_head_rotation_workspace_bytes.argtypes = [i64, i32, i32, i32]
    lib.mrf_head_rotation_forward.restype = ci
    lib.mrf_head_rotation_forward.argtypes = [R, vp, vp, vp]
    lib.mrf_head_rotation_backward.restype = ci
    lib.mrf_head_rotation_backward.argtypes = [R, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.mrf_gated_scan_states.restype = i64
    lib.mrf_gated_scan_states.argtypes = [i64]
    lib.mrf_gated_scan_workspace_bytes.restype = sz
    lib.mrf_gated_scan_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mrf_gated_scan_forward.restype = ci
    lib.mrf_gated_scan_forward.argtypes = [i64, i64, i64, ci, vp, vp, vp, vp, ci, ci, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.mrf_gated_scan_backward.restype = ci
    lib.mrf_gated_scan_backward.argtypes = [i64, i64, i64, ci, vp, vp, vp, vp, vp, vp, ci, ci, vp, vp, vp, vp, vp, vp, sz, vp]
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


# ---- sequence operators: inputs may be parts of a projection (any strides, the last index dense).  A description is packed in one go and a tensor looked at once:
# small calls cost what their checks do.

_INT64_MIN, _INT64_MAX = -(1 << 63), (1 << 63) - 1
_ATTENTION = struct.Struct("@7if3P9q3q5P2q2i")
_ROTATION = struct.Struct("@6i2P6q2Pf2i2Piq")
_TWO_STRIDES = ctypes.c_int64 * 2
_BACKWARD_KEEPS_TABLE = 2      # MRF_BACKWARD_KEEPS_TABLE
_codes = {}      # torch dtype -> code of an element type


def _code_of(dtype) -> int:
    """Code of an element type (filled with the library, which imports torch)."""
    code = _codes.get(dtype)
    if code is None:
        raise ValueError("tensors must be float32, float16 or bfloat16, got %s" % dtype)
    return code


def _packed(form, *values) -> bytes:
    """A description's bytes."""
    try:
        return form.pack(*values)
    except struct.error as e:
        raise ValueError("offsets have 64 bits: %s" % e) from None


def _device_of(t):
    """The current device, on which the first tensor of a call has to be, as all others (the call goes to its stream)."""
    at = t.get_device()
    if at < 0 or at != _device_now():
        raise ValueError("tensors must be on the current GPU")
    return at


def _refused(t, what, shape, dtype, at):
    if t.get_device() != at:
        raise ValueError("%s must be on the current GPU" % what)
    if t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (what, dtype, t.dtype))
    if shape is not None and t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (what, tuple(t.shape), tuple(shape)))
    raise ValueError("%s must be contiguous" % what)


def _dense(t, what, shape, dtype, at):
    """Address of a dense tensor of that shape and type (None: 0)."""
    if t is None:
        return 0
    if t.get_device() != at or t.dtype != dtype or (shape is not None and t.shape != shape) or not t.is_contiguous():
        _refused(t, what, shape, dtype, at)
    return t.data_ptr()


def _strides(t, what, shape, dtype, at):
    """Strides of a tensor of that shape and type whose last index is dense."""
    if t.get_device() != at or t.dtype != dtype or t.shape != shape:
        _refused(t, what, shape, dtype, at)
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] > 1 and t.numel():
        raise ValueError("the last index of %s must be dense" % what)
    return strides[:-1]


def _stream_at(stream, at):
    """Handle of a stream, or of the current one of the current device."""
    return _raw_stream(at) if stream is None and _raw_stream is not None else _stream_handle(stream)


def _scratch(workspace, at):
    """Address and bytes of a workspace."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != at or not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous and on the current GPU")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


class MrfAttention:
    """Mirror of the C struct mrf_attention: q [B,Q,Hq,D], k and v [B,K,Hk,D] of one type at any strides (last index dense), table
    [Hq,n_buckets] float32 (heads_last: [n_buckets,Hq]) or None, bucket_of [n] int32 for the offsets from map_offset on, query_offsets,
    q_lengths, k_lengths [B] int32 or None, first_offset and last_offset numbers or None (no bound).  Made once, it can be called again while
    its tensors live (it holds them)."""

    def __init__(self, q, k, v, scale, *, first_offset=None, last_offset=None, query_offset=0, query_offsets=None, q_lengths=None, k_lengths=None,
                 table=None, bucket_of=None, map_offset=0, heads_last=False):
        load_library()
        if q.dim() != 4 or k.dim() != 4:
            raise ValueError("q and k must be [batch, token, head, entry]")
        at, dtype = _device_of(q), q.dtype
        B, Q, Hq, D = q.shape
        _, K, Hk, _ = k.shape
        keys = (B, K, Hk, D)
        strides = (*_strides(q, "q", q.shape, dtype, at), *_strides(k, "k", keys, dtype, at), *_strides(v, "v", keys, dtype, at))
        n = offsets = 0
        if table is not None:
            if bucket_of is None or table.dim() != 2:
                raise ValueError("a table must be two-dimensional, and needs bucket_of")
            n, offsets = table.shape[0] if heads_last else table.shape[-1], bucket_of.numel()
        if max(B, Q, K, Hq, D, n) > 0x7fffffff:
            raise ValueError("sizes are at most 2^31 - 1")
        of_batch = (B,)
        i32, f32 = _int32, _float32
        self.c = _CAttention.from_buffer_copy(_packed(
            _ATTENTION, B, Q, K, Hq, Hk, D, _code_of(dtype), scale, q.data_ptr(), k.data_ptr(), v.data_ptr(), *strides,
            _INT64_MIN if first_offset is None else int(first_offset), _INT64_MAX if last_offset is None else int(last_offset), int(query_offset),
            _dense(query_offsets, "query_offsets", of_batch, i32, at), _dense(q_lengths, "q_lengths", of_batch, i32, at),
            _dense(k_lengths, "k_lengths", of_batch, i32, at), _dense(table, "table", (n, Hq) if heads_last else (Hq, n), f32, at),
            0 if table is None else _dense(bucket_of, "bucket_of", None, i32, at), int(map_offset), offsets, n, 1 if heads_last else 0))
        self.shape, self.at, self.dtype, self.table_shape = (B, Q, K, Hq, Hk, D), at, dtype, None if table is None else table.shape
        self._kept = (q, k, v, query_offsets, q_lengths, k_lengths, table, bucket_of)


def mrf_attention_workspace_bytes(att: MrfAttention, backward: bool, grad_table: bool = True) -> int:
    """grad_table: whether the backward call is given one (it then needs room for sums by offset)."""
    return int(load_library().mrf_attention_workspace_bytes(ctypes.byref(att.c), 0 if not backward else 1 if grad_table else _BACKWARD_KEEPS_TABLE))


def mrf_attention_forward(att: MrfAttention, out, lse, workspace, stream=None):
    """out [B,Q,Hq,D] like q, lse [B,Hq,Q] float32 or None."""
    B, Q, K, Hq, Hk, D = att.shape
    at = att.at
    if at != _device_now():
        raise ValueError("tensors must be on the current GPU")
    _checked(_lib.mrf_attention_forward(
        ctypes.byref(att.c), _dense(out, "out", (B, Q, Hq, D), att.dtype, at), _dense(lse, "lse", (B, Hq, Q), _float32, at), *_scratch(workspace, at),
        _stream_at(stream, at)), "mrf_attention_forward")


def mrf_attention_backward(att: MrfAttention, grad_out, out, lse, grad_q, grad_k, grad_v, grad_table, workspace, stream=None):
    """grad_out and out [B,Q,Hq,D], lse [B,Hq,Q] of the forward call; grad_q, grad_k, grad_v of the shapes of q, k, v (dense), grad_table like
    the table, each or None."""
    B, Q, K, Hq, Hk, D = att.shape
    at, dtype, queries, keys = att.at, att.dtype, (B, Q, Hq, D), (B, K, Hk, D)
    if at != _device_now():
        raise ValueError("tensors must be on the current GPU")
    if grad_table is not None and att.table_shape is None:
        raise ValueError("grad_table without a table")
    _checked(_lib.mrf_attention_backward(
        ctypes.byref(att.c), _dense(grad_out, "grad_out", queries, dtype, at), _dense(out, "out", queries, dtype, at),
        _dense(lse, "lse", (B, Hq, Q), _float32, at), _dense(grad_q, "grad_q", queries, dtype, at), _dense(grad_k, "grad_k", keys, dtype, at),
        _dense(grad_v, "grad_v", keys, dtype, at), _dense(grad_table, "grad_table", att.table_shape, _float32, at), *_scratch(workspace, at),
        _stream_at(stream, at)), "mrf_attention_backward")


def _head_rotation(q, k, gamma_q, gamma_k, eps, inv_freq, positions, position_offset, interleaved):
    """The C struct (its bytes) of tensors that fit each other, their shapes, type and device."""
    load_library()
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be [batch, token, head, entry]")
    at, dtype, f32 = _device_of(q), q.dtype, _float32
    queries = q.shape
    B, T, Hq, D = queries
    Hk = k.shape[2]
    keys, entries, axes = (B, T, Hk, D), (D,), 1
    if positions is not None:
        if positions.dim() == 3:
            axes = positions.shape[2]
        places = _dense(positions, "positions", (B, T, axes) if positions.dim() == 3 else (B, T), _int32, at)
    else:
        places = 0
    if max(B, T, Hq, Hk, D) > 0x7fffffff or (inv_freq is not None and inv_freq.numel() > 0x3fffffff):
        raise ValueError("sizes are at most 2^31 - 1")
    packed = _packed(
        _ROTATION, B, T, Hq, Hk, D, _code_of(dtype), q.data_ptr(), k.data_ptr(), *_strides(q, "q", queries, dtype, at), *_strides(k, "k", keys, dtype, at),
        _dense(gamma_q, "gamma_q", entries, f32, at), _dense(gamma_k, "gamma_k", entries, f32, at), eps, 0 if inv_freq is None else 2 * inv_freq.numel(),
        1 if interleaved else 0, _dense(inv_freq, "inv_freq", None, f32, at), places, axes, int(position_offset))
    return packed, queries, keys, dtype, at


def mrf_head_rotation_forward(q, k, gamma_q, gamma_k, eps, inv_freq, out_q, out_k, positions=None, position_offset=0, interleaved=False, stream=None):
    """q [B,T,Hq,D] and k [B,T,Hk,D] of one type at any strides (last index dense), gamma_q, gamma_k [D] float32 or None, inv_freq [pairs that turn]
    float32 or None (none), out_q and out_k of their shapes, positions [B,T] or [B,T,axes] int32 or None (the token's place)."""
    packed, queries, keys, dtype, at = _head_rotation(q, k, gamma_q, gamma_k, eps, inv_freq, positions, position_offset, interleaved)
    _checked(_lib.mrf_head_rotation_forward(packed, _dense(out_q, "out_q", queries, dtype, at), _dense(out_k, "out_k", keys, dtype, at), _stream_at(stream, at)),
             "mrf_head_rotation_forward")


def mrf_head_rotation_workspace_bytes(n_tokens: int, Hq: int, Hk: int, D: int) -> int:
    return int(load_library().mrf_head_rotation_workspace_bytes(int(n_tokens), int(Hq), int(Hk), int(D)))


def mrf_head_rotation_backward(grad_out_q, grad_out_k, q, k, gamma_q, gamma_k, eps, inv_freq, grad_q, grad_k, grad_gamma_q, grad_gamma_k, workspace,
                               positions=None, position_offset=0, interleaved=False, stream=None):
    """Arguments of the forward call; grad_out_q, grad_out_k, grad_q, grad_k dense, of the shapes of q and k, grad_gamma_q, grad_gamma_k [D] float32;
    gradients that are not asked for are None."""
    packed, queries, keys, dtype, at = _head_rotation(q, k, gamma_q, gamma_k, eps, inv_freq, positions, position_offset, interleaved)
    entries = queries[3:]
    _checked(_lib.mrf_head_rotation_backward(
        packed, _dense(grad_out_q, "grad_out_q", queries, dtype, at), _dense(grad_out_k, "grad_out_k", keys, dtype, at),
        _dense(grad_q, "grad_q", queries, dtype, at), _dense(grad_k, "grad_k", keys, dtype, at), _dense(grad_gamma_q, "grad_gamma_q", entries, _float32, at),
        _dense(grad_gamma_k, "grad_gamma_k", entries, _float32, at), *_scratch(workspace, at), _stream_at(stream, at)), "mrf_head_rotation_backward")


def mrf_gated_scan_states(T: int) -> int:
    return int(load_library().mrf_gated_scan_states(int(T)))


def mrf_gated_scan_workspace_bytes(n_outer: int, T: int, n_inner: int) -> int:
    return int(load_library().mrf_gated_scan_workspace_bytes(int(n_outer), int(T), int(n_inner)))


def _scan_input(t, what, shape, dtype, at):
    """Address and strides (None: dense) of x or z."""
    strides = _strides(t, what, shape, dtype, at)
    return t.data_ptr(), None if t.is_contiguous() else _TWO_STRIDES(*strides)


def mrf_gated_scan_forward(x, z, initial, lengths, y, final, states, workspace, complement=True, reverse=False, stream=None):
    """x and z [outer,T,inner] of one type at any strides (last index dense), y dense like them, initial and final [outer,inner] float32 or None (final may be
    initial), lengths [outer] int32 or None, states [outer,mrf_gated_scan_states(T),inner] float32 or None."""
    load_library()
    if x.dim() != 3:
        raise ValueError("x must be [row, step, channel]")
    at, dtype, shape, f32 = _device_of(x), x.dtype, x.shape, _float32
    outer, T, inner = shape
    ends = (outer, inner)
    _checked(_lib.mrf_gated_scan_forward(
        outer, T, inner, _code_of(dtype), *_scan_input(x, "x", shape, dtype, at), *_scan_input(z, "z", shape, dtype, at), 1 if complement else 0,
        1 if reverse else 0, _dense(initial, "initial", ends, f32, at), _dense(lengths, "lengths", (outer,), _int32, at), _dense(y, "y", shape, dtype, at),
        _dense(final, "final", ends, f32, at), 0 if states is None else _dense(states, "states", (outer, mrf_gated_scan_states(T), inner), f32, at),
        *_scratch(workspace, at), _stream_at(stream, at)), "mrf_gated_scan_forward")


def mrf_gated_scan_backward(grad_y, grad_final, x, z, lengths, states, grad_x, grad_z, grad_initial, workspace, complement=True, reverse=False, stream=None):
    """grad_y, grad_x, grad_z dense like x, grad_final and grad_initial [outer,inner] float32; states of the forward call; gradients that are not
    asked for are None, and grad_final may be."""
    load_library()
    if x.dim() != 3:
        raise ValueError("x must be [row, step, channel]")
    at, dtype, shape, f32 = _device_of(x), x.dtype, x.shape, _float32
    outer, T, inner = shape
    ends = (outer, inner)
    _checked(_lib.mrf_gated_scan_backward(
        outer, T, inner, _code_of(dtype), _dense(grad_y, "grad_y", shape, dtype, at), _dense(grad_final, "grad_final", ends, f32, at),
        *_scan_input(x, "x", shape, dtype, at), *_scan_input(z, "z", shape, dtype, at), 1 if complement else 0, 1 if reverse else 0,
        _dense(lengths, "lengths", (outer,), _int32, at), _dense(states, "states", (outer, mrf_gated_scan_states(T), inner), f32, at),
        _dense(grad_x, "grad_x", shape, dtype, at), _dense(grad_z, "grad_z", shape, dtype, at), _dense(grad_initial, "grad_initial", ends, f32, at),
        *_scratch(workspace, at), _stream_at(stream, at)), "mrf_gated_scan_backward")


def mrf_workspace_fault(workspace, stream=None) -> int:
    """0, or -11 if a wait between wavefronts ran out in the last call that used this workspace
    (synchronises the stream)."""
    return int(load_library().mrf_workspace_fault(_dev_ptr(workspace), _stream_handle(stream)))
