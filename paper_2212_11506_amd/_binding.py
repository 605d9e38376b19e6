"""ctypes marshalling for the C ABI of ``libbhtsne.so`` (argument passing only).

Tensors must be contiguous CUDA (HIP) tensors of the documented dtypes; their
data pointers and the current torch stream are handed to the library.  There
is no fallback: when the shared library is missing the import of a function
fails loudly.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = os.path.join(_HERE, "lib", "libbhtsne.so")

BHTSNE_OK, BHTSNE_EINVAL, BHTSNE_EWORKSPACE, BHTSNE_ENONFINITE, BHTSNE_EDEVICE = 0, -1, -2, -3, -4
BHTSNE_EINPUT, BHTSNE_ECAPACITY = -5, -6
ORDER_MORTON, ORDER_BFS, ORDER_AUTO = 0, 1, 2  # point orders of a layout (bhtsne_layout_build_ordered)
PHASES = ("bbox_morton", "sort", "tree", "repulsive", "attractive", "update")


class BhtsneError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class _Csr(C.Structure):
    _fields_ = [("n", C.c_int64), ("nnz", C.c_int64), ("row_ptr", C.c_void_p),
                ("col", C.c_void_p), ("val", C.c_void_p)]


class _Layout(C.Structure):
    _fields_ = [("n", C.c_int64), ("nnz", C.c_int64), ("mem", C.c_void_p), ("bytes", C.c_size_t),
                ("tiles", C.c_int64), ("items", C.c_int64), ("entries", C.c_int64), ("windows", C.c_int64),
                ("segments", C.c_int64), ("order", C.c_int64), ("magic", C.c_uint64)]


class _Stats(C.Structure):
    _fields_ = [("Z", C.c_double), ("interactions", C.c_int64), ("nodes", C.c_int64),
                ("bbox", C.c_double * 4), ("r_span", C.c_double), ("device_flags", C.c_uint32),
                ("max_depth", C.c_int32)]


class _Timing(C.Structure):
    _fields_ = [("ms", C.c_double * 6), ("count", C.c_int64 * 6)]


_lib = None


def library_path() -> str:
    return _LIB


def load_library():
    """Load the HIP library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB):
        raise ImportError(f"{_LIB} is missing: build it with paper_2212_11506_amd/build.py")
    lib = C.CDLL(_LIB)
    vp, i64, f32, f64p = C.c_void_p, C.c_int64, C.c_float, C.POINTER(C.c_double)
    sigs = {
        "bhtsne_workspace_size": (C.c_size_t, [i64, i64]),
        "bhtsne_gradient": (C.c_int, [vp, C.POINTER(_Csr), f32, f32, vp, f64p, vp, C.c_size_t, vp]),
        "bhtsne_step": (C.c_int, [vp, C.POINTER(_Csr), f32, f32, f32, f32, f32, vp, vp, vp, f64p, vp,
                                  C.c_size_t, vp]),
        "bhtsne_get_stats": (C.c_int, [vp, C.POINTER(_Stats), vp]),
        "bhtsne_layout_size": (C.c_size_t, [i64, i64]),
        "bhtsne_layout_build": (C.c_int, [C.POINTER(_Csr), vp, vp, C.c_size_t, C.POINTER(_Layout), vp,
                                          C.c_size_t, vp]),
        "bhtsne_layout_build_ordered": (C.c_int, [C.POINTER(_Csr), vp, C.c_int, vp, C.c_size_t, C.POINTER(_Layout),
                                                  vp, C.c_size_t, vp]),
        "bhtsne_gradient_layout": (C.c_int, [vp, C.POINTER(_Layout), f32, f32, vp, f64p, vp, C.c_size_t, vp]),
        "bhtsne_step_layout": (C.c_int, [vp, C.POINTER(_Layout), f32, f32, f32, f32, f32, vp, vp, vp, f64p, vp,
                                         C.c_size_t, vp]),
        "bhtsne_status_string": (C.c_char_p, [C.c_int]),
        "bhtsne_timing_enable": (C.c_int, [C.c_int]),
        "bhtsne_timing_phases": (C.c_int, [C.c_uint32]),
        "bhtsne_z_exact": (C.c_int, [vp, i64, C.POINTER(C.c_double), vp, C.c_size_t, vp]),
        "bhtsne_kl": (C.c_int, [vp, C.POINTER(_Csr), C.c_double, C.POINTER(C.c_double), vp, C.c_size_t, vp]),
        "bhtsne_timing_read": (C.c_int, [C.POINTER(_Timing), C.c_int]),
        "bhtsne_affinities_workspace_size": (C.c_size_t, [i64, C.c_int32]),
        "bhtsne_workspace_size_f64": (C.c_size_t, [i64, i64]),
        "bhtsne_gradient_f64": (C.c_int, [vp, C.POINTER(_Csr), C.c_double, C.c_double, vp, f64p, vp, C.c_size_t,
                                          vp]),
        "bhtsne_step_f64": (C.c_int, [vp, C.POINTER(_Csr), C.c_double, C.c_double, C.c_double, C.c_double,
                                      C.c_double, vp, vp, vp, f64p, vp, C.c_size_t, vp]),
        "bhtsne_affinities": (C.c_int, [vp, vp, i64, C.c_int32, C.c_double, vp, vp, vp, i64,
                                        C.POINTER(C.c_int64), vp, vp, C.c_size_t, vp]),
        "bhtsne_noalloc_max_bytes": (C.c_size_t, []),
        "bhtsne_step_noalloc": (C.c_int, [vp, C.POINTER(_Csr), f32, f32, f32, f32, f32, vp, vp, vp, f64p, vp]),
        "bhtsne_layout_size_f64": (C.c_size_t, [i64, i64]),
        "bhtsne_layout_build_f64": (C.c_int, [C.POINTER(_Csr), vp, vp, C.c_size_t, C.POINTER(_Layout), vp,
                                              C.c_size_t, vp]),
        "bhtsne_gradient_layout_f64": (C.c_int, [vp, C.POINTER(_Layout), C.c_double, C.c_double, vp, f64p, vp,
                                                 C.c_size_t, vp]),
        "bhtsne_step_layout_f64": (C.c_int, [vp, C.POINTER(_Layout), C.c_double, C.c_double, C.c_double,
                                             C.c_double, C.c_double, vp, vp, vp, f64p, vp, C.c_size_t, vp]),
        "bhtsne_workspace_size_3d": (C.c_size_t, [i64, i64]),
        "bhtsne_gradient_3d": (C.c_int, [vp, C.POINTER(_Csr), f32, f32, vp, f64p, vp, C.c_size_t, vp]),
        "bhtsne_step_3d": (C.c_int, [vp, C.POINTER(_Csr), f32, f32, f32, f32, f32, vp, vp, vp, f64p, vp,
                                     C.c_size_t, vp]),
        "bhtsne_layout_size_3d": (C.c_size_t, [i64, i64]),
        "bhtsne_layout_build_3d": (C.c_int, [C.POINTER(_Csr), vp, vp, C.c_size_t, C.POINTER(_Layout), vp,
                                             C.c_size_t, vp]),
        "bhtsne_gradient_layout_3d": (C.c_int, [vp, C.POINTER(_Layout), f32, f32, vp, f64p, vp, C.c_size_t, vp]),
        "bhtsne_step_layout_3d": (C.c_int, [vp, C.POINTER(_Layout), f32, f32, f32, f32, f32, vp, vp, vp, f64p, vp,
                                            C.c_size_t, vp]),
        "bhtsne_debug_sort_3d": (C.c_int, [vp, i64, vp, vp, vp, f64p, vp, C.c_size_t, vp]),
        "bhtsne_debug_tree_3d": (C.c_int, [vp, i64, f32, C.POINTER(C.c_int64), vp, vp, vp, vp, vp, vp, vp, vp,
                                           C.c_size_t, vp]),
        "bhtsne_debug_walk": (C.c_int, [vp, i64, C.c_int, f32, C.c_int, vp, f64p, C.POINTER(C.c_uint64), vp,
                                        C.c_size_t, vp]),
        "bhtsne_debug_sort": (C.c_int, [vp, i64, vp, vp, vp, f64p, vp, C.c_size_t, vp]),
        "bhtsne_debug_tree": (C.c_int, [vp, i64, f32, C.POINTER(C.c_int64), vp, vp, vp, vp, vp, vp, vp,
                                        C.c_size_t, vp]),
        "bhtsne_layer_norm": (C.c_int, [vp, i64, vp, vp, i64, i64, C.c_double, C.c_int, C.c_int, vp, i64, vp, vp, vp]),
        "bhtsne_layer_norm_workspace_size": (C.c_size_t, [i64, i64]),
        "bhtsne_layer_norm_backward": (C.c_int, [vp, i64, vp, i64, vp, vp, vp, i64, i64, C.c_int, C.c_int, vp, i64,
                                                 vp, vp, vp, C.c_size_t, vp]),
        "bhtsne_orthogonalise_workspace_size": (C.c_size_t, [i64, i64, i64]),
        "bhtsne_orthogonalise": (C.c_int, [vp, i64, i64, i64, C.c_int, f64p, C.c_int, C.c_double, vp, vp, C.c_size_t,
                                           vp]),
        "bhtsne_muon_step": (C.c_int, [vp, vp, vp, i64, i64, i64, C.c_int, C.c_double, C.c_double, C.c_int,
                                       C.c_double, C.c_double, f64p, C.c_int, C.c_double, vp, C.c_size_t, vp]),
        "bhtsne_gated_layer": (C.c_int, [vp, i64, vp, i64, vp, i64, i64, i64, i64, C.c_int, C.c_int, vp, i64, vp, i64, vp,
                                         i64, vp]),
        "bhtsne_gated_layer_workspace_size": (C.c_size_t, [i64, i64, i64, C.c_int]),
        "bhtsne_gated_layer_backward": (C.c_int, [vp, i64] * 6 + [i64, i64, i64, C.c_int, C.c_int] + [vp, i64] * 3
                                        + [vp, C.c_size_t, vp]),
        "bhtsne_quantise_rows": (C.c_int, [vp, i64, i64, i64, C.c_int, vp, i64, vp, vp]),
        "bhtsne_linear_i8_workspace_size": (C.c_size_t, [i64, i64]),
        "bhtsne_linear_i8": (C.c_int, [vp, i64, C.c_int, vp, vp, i64, vp, vp, i64, i64, i64, C.c_int, C.c_int, vp, i64, vp,
                                       C.c_size_t, vp]),
        "bhtsne_distil_loss_workspace_size": (C.c_size_t, [i64, i64]),
        "bhtsne_distil_loss": (C.c_int, [vp, i64, i64, i64, vp, i64, vp, i64, i64, C.c_double, C.c_int, C.c_int, vp, vp, vp,
                                         C.c_size_t, vp]),
        "bhtsne_distil_loss_kept": (C.c_int, [vp, i64, i64, i64, vp, i64, vp, i64, i64, C.c_double, C.c_int, C.c_int, vp, vp, vp,
                                              vp, C.c_size_t, vp]),
        "bhtsne_distil_loss_backward": (C.c_int, [vp, vp, i64, i64, i64, vp, i64, vp, i64, i64, vp, C.c_double, C.c_int,
                                                  C.c_int, vp, i64, vp]),
        "bhtsne_distil_loss_backward_kept": (C.c_int, [vp, vp, i64, i64, i64, vp, i64, vp, i64, i64, vp, vp, C.c_double, C.c_int,
                                                       C.c_int, vp, i64, vp]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().bhtsne_status_string(int(status)).decode()


def _check(rc: int, where: str):
    if rc != BHTSNE_OK:
        raise BhtsneError(rc, where)


def _ptr(t: Optional[torch.Tensor], dtype=None, where="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{where} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{where} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{where} must be {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


class Csr:
    """Device CSR matrix P (int64 row_ptr, int32 col, float32 val)."""

    def __init__(self, row_ptr: torch.Tensor, col: torch.Tensor, val: torch.Tensor):
        self.row_ptr, self.col, self.val = row_ptr, col, val
        self.n = int(row_ptr.numel()) - 1
        self.nnz = int(col.numel())
        self._s = _Csr(self.n, self.nnz, _ptr(row_ptr, torch.int64, "row_ptr").value,
                       _ptr(col, torch.int32, "col").value if self.nnz else None,
                       _ptr(val, torch.float32, "val").value if self.nnz else None)

    @classmethod
    def from_numpy(cls, row_ptr, col, val, device="cuda"):
        return cls(torch.as_tensor(row_ptr, dtype=torch.int64).to(device),
                   torch.as_tensor(col, dtype=torch.int32).to(device),
                   torch.as_tensor(val, dtype=torch.float32).to(device))

    @property
    def struct(self):
        return C.byref(self._s)


class CsrF64(Csr):
    """Device CSR matrix P with fp64 values, for the fp64 variant (same
    struct layout as Csr: bhtsne_csr_f64)."""

    def __init__(self, row_ptr: torch.Tensor, col: torch.Tensor, val: torch.Tensor):
        self.row_ptr, self.col, self.val = row_ptr, col, val
        self.n = int(row_ptr.numel()) - 1
        self.nnz = int(col.numel())
        self._s = _Csr(self.n, self.nnz, _ptr(row_ptr, torch.int64, "row_ptr").value,
                       _ptr(col, torch.int32, "col").value if self.nnz else None,
                       _ptr(val, torch.float64, "val").value if self.nnz else None)

    @classmethod
    def from_numpy(cls, row_ptr, col, val, device="cuda"):
        return cls(torch.as_tensor(row_ptr, dtype=torch.int64).to(device),
                   torch.as_tensor(col, dtype=torch.int32).to(device),
                   torch.as_tensor(val, dtype=torch.float64).to(device))


def workspace_size_f64(n: int, nnz: int) -> int:
    return int(load_library().bhtsne_workspace_size_f64(int(n), int(nnz)))


def gradient_f64(Y: torch.Tensor, P: "CsrF64", theta: float, exaggeration: float = 1.0,
                 grad: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 return_z: bool = True):
    """bhtsne_gradient_f64: returns (grad fp64, Z or None)."""
    lib = load_library()
    if not isinstance(P, (CsrF64, LayoutF64)):
        raise TypeError("gradient_f64 takes P as a CsrF64 or a LayoutF64")
    if grad is None:
        grad = torch.empty_like(Y)
    ws = workspace if workspace is not None else torch.empty(workspace_size_f64(P.n, P.nnz), dtype=torch.uint8,
                                                             device=Y.device)
    z = C.c_double(0.0)
    fn = lib.bhtsne_gradient_layout_f64 if isinstance(P, LayoutF64) else lib.bhtsne_gradient_f64
    rc = fn(_ptr(Y, torch.float64, "Y"), P.struct, float(theta), float(exaggeration),
            _ptr(grad, torch.float64, "grad"), C.byref(z) if return_z else None,
            _ptr(ws, None, "workspace"), ws.numel(), _stream())
    _check(rc, fn.__name__)
    return grad, (z.value if return_z else None)


def step_f64(Y: torch.Tensor, P: "CsrF64", theta: float, exaggeration: float, learning_rate: float,
             momentum: float, min_gain: float, update: torch.Tensor, gains: torch.Tensor,
             grad: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
             return_z: bool = False):
    """bhtsne_step_f64: one fp64 iteration in place on Y, update and gains."""
    lib = load_library()
    if not isinstance(P, (CsrF64, LayoutF64)):
        raise TypeError("step_f64 takes P as a CsrF64 or a LayoutF64")
    ws = workspace if workspace is not None else torch.empty(workspace_size_f64(P.n, P.nnz), dtype=torch.uint8,
                                                             device=Y.device)
    z = C.c_double(0.0)
    fn = lib.bhtsne_step_layout_f64 if isinstance(P, LayoutF64) else lib.bhtsne_step_f64
    rc = fn(_ptr(Y, torch.float64, "Y"), P.struct, float(theta), float(exaggeration),
            float(learning_rate), float(momentum), float(min_gain),
            _ptr(update, torch.float64, "update"), _ptr(gains, torch.float64, "gains"),
            _ptr(grad, torch.float64, "grad"), C.byref(z) if return_z else None,
            _ptr(ws, None, "workspace"), ws.numel(), _stream())
    _check(rc, fn.__name__)
    return z.value if return_z else None


def workspace_size(n: int, nnz: int) -> int:
    return int(load_library().bhtsne_workspace_size(int(n), int(nnz)))


def _workspace(n, nnz, ws):
    need = workspace_size(n, nnz)
    if need == 0:
        raise BhtsneError(BHTSNE_EINVAL, "workspace_size")
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    return ws, need


class Layout:
    """A locality layout of P (relabelled copy in device memory) for the *_layout calls.
    order: None (bhtsne_layout_build, the automatic choice) or one of
    ORDER_MORTON, ORDER_BFS, ORDER_AUTO (bhtsne_layout_build_ordered)."""

    def __init__(self, P: Csr, Y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 order: Optional[int] = None):
        lib = load_library()
        self.n, self.nnz = P.n, P.nnz
        need = int(lib.bhtsne_layout_size(P.n, P.nnz))
        if need == 0:
            raise BhtsneError(BHTSNE_EINVAL, "bhtsne_layout_size")
        self.mem = torch.empty(need, dtype=torch.uint8, device="cuda")
        ws, _ = _workspace(P.n, P.nnz, workspace)
        self._s = _Layout()
        if order is None:
            rc = lib.bhtsne_layout_build(P.struct, _ptr(Y, torch.float32, "Y"), _ptr(self.mem), need,
                                         C.byref(self._s), _ptr(ws), ws.numel(), _stream())
            _check(rc, "bhtsne_layout_build")
        else:
            rc = lib.bhtsne_layout_build_ordered(P.struct, _ptr(Y, torch.float32, "Y"), int(order), _ptr(self.mem),
                                                 need, C.byref(self._s), _ptr(ws), ws.numel(), _stream())
            _check(rc, "bhtsne_layout_build_ordered")

    @property
    def order(self) -> int:
        """ORDER_MORTON or ORDER_BFS: the point order the copy was built in."""
        return int(self._s.order)

    @property
    def tiles(self) -> int:
        return int(self._s.tiles)

    @property
    def items(self) -> int:
        return int(self._s.items)

    @property
    def entries(self) -> int:
        return int(self._s.entries)

    @property
    def windows(self) -> int:
        return int(self._s.windows)

    @property
    def segments(self) -> int:
        return int(self._s.segments)

    @property
    def struct(self):
        return C.byref(self._s)


class LayoutF64(Layout):
    """A locality layout of an fp64 P (CsrF64) for the fp64 variant's calls:
    relabelled rows with fp64 values, then the sliced copy over 8192-point
    windows or, without tile locality, windowed segments."""

    def __init__(self, P: "CsrF64", Y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        lib = load_library()
        if not isinstance(P, CsrF64):
            raise TypeError("LayoutF64 takes P as a CsrF64")
        self.n, self.nnz = P.n, P.nnz
        need = int(lib.bhtsne_layout_size_f64(P.n, P.nnz))
        if need == 0:
            raise BhtsneError(BHTSNE_EINVAL, "bhtsne_layout_size_f64")
        self.mem = torch.empty(need, dtype=torch.uint8, device="cuda")
        ws = workspace if workspace is not None else torch.empty(workspace_size_f64(P.n, P.nnz), dtype=torch.uint8,
                                                                 device="cuda")
        self._s = _Layout()
        rc = lib.bhtsne_layout_build_f64(P.struct, _ptr(Y, torch.float64, "Y"), _ptr(self.mem), need,
                                         C.byref(self._s), _ptr(ws), ws.numel(), _stream())
        _check(rc, "bhtsne_layout_build_f64")


def layout_size(n: int, nnz: int) -> int:
    return int(load_library().bhtsne_layout_size(int(n), int(nnz)))


def gradient(Y: torch.Tensor, P, theta: float, exaggeration: float = 1.0,
             grad: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
             return_z: bool = True):
    """bhtsne_gradient (P a Csr) or bhtsne_gradient_layout (P a Layout): returns (grad, Z or None)."""
    lib = load_library()
    if grad is None:
        grad = torch.empty_like(Y)
    ws, _ = _workspace(P.n, P.nnz, workspace)
    z = C.c_double(0.0)
    fn = lib.bhtsne_gradient_layout if isinstance(P, Layout) else lib.bhtsne_gradient
    rc = fn(_ptr(Y, torch.float32, "Y"), P.struct, float(theta), float(exaggeration),
                             _ptr(grad, torch.float32, "grad"), C.byref(z) if return_z else None,
                             _ptr(ws, None, "workspace"), ws.numel(), _stream())
    _check(rc, fn.__name__)
    return grad, (z.value if return_z else None)


def z_exact(Y: torch.Tensor, workspace: Optional[torch.Tensor] = None) -> float:
    """bhtsne_z_exact: the exact normaliser over all ordered pairs i != j."""
    lib = load_library()
    n = Y.shape[0]
    ws, _ = _workspace(n, 0, workspace)
    z = C.c_double(0.0)
    _check(lib.bhtsne_z_exact(_ptr(Y, torch.float32, "Y"), n, C.byref(z), _ptr(ws, None, "workspace"),
                              ws.numel(), _stream()), "bhtsne_z_exact")
    return z.value


def kl(Y: torch.Tensor, P: "Csr", Z: float, workspace: Optional[torch.Tensor] = None) -> float:
    """bhtsne_kl: KL(P || Q) over P's stored entries for the given normaliser Z."""
    lib = load_library()
    if not isinstance(P, Csr):
        raise TypeError("kl takes P as a Csr")
    ws, _ = _workspace(P.n, 0, workspace)
    out = C.c_double(0.0)
    _check(lib.bhtsne_kl(_ptr(Y, torch.float32, "Y"), P.struct, float(Z), C.byref(out),
                         _ptr(ws, None, "workspace"), ws.numel(), _stream()), "bhtsne_kl")
    return out.value


def affinities_workspace_size(n: int, k: int) -> int:
    return int(load_library().bhtsne_affinities_workspace_size(int(n), int(k)))


def affinities(knn_idx: torch.Tensor, knn_dist: torch.Tensor, perplexity: float,
               workspace: Optional[torch.Tensor] = None, capacity: Optional[int] = None,
               sigma2: bool = False):
    """bhtsne_affinities: the symmetric P of k-nearest-neighbour lists
    (knn_idx int32 [n, k], knn_dist float32 [n, k]) at the given perplexity.
    Returns (Csr, sigma^2 fp64 [n] or None).  Output arrays hold `capacity`
    entries (default 2 n k, the most P can have) and are trimmed to nnz."""
    lib = load_library()
    n, k = int(knn_idx.shape[0]), int(knn_idx.shape[1])
    if tuple(knn_dist.shape) != (n, k):
        raise ValueError("knn_idx and knn_dist must have the same shape")
    need = affinities_workspace_size(n, k)
    if need == 0:
        raise BhtsneError(BHTSNE_EINVAL, "bhtsne_affinities_workspace_size")
    ws = workspace if workspace is not None else torch.empty(need, dtype=torch.uint8, device=knn_idx.device)
    cap = 2 * n * k if capacity is None else int(capacity)
    dev = knn_idx.device
    row_ptr = torch.empty(n + 1, dtype=torch.int64, device=dev)
    col = torch.empty(max(cap, 1), dtype=torch.int32, device=dev)
    val = torch.empty(max(cap, 1), dtype=torch.float32, device=dev)
    s2 = torch.empty(n, dtype=torch.float64, device=dev) if sigma2 else None
    nnz = C.c_int64(0)
    rc = lib.bhtsne_affinities(_ptr(knn_idx, torch.int32, "knn_idx"), _ptr(knn_dist, torch.float32, "knn_dist"),
                               n, k, float(perplexity), _ptr(row_ptr, torch.int64, "row_ptr"),
                               _ptr(col, torch.int32, "col"), _ptr(val, torch.float32, "val"), cap,
                               C.byref(nnz), _ptr(s2, torch.float64, "sigma2"), _ptr(ws, None, "workspace"),
                               ws.numel(), _stream())
    if rc == BHTSNE_ECAPACITY:
        raise BhtsneError(rc, f"bhtsne_affinities (needs {nnz.value} entries)")
    _check(rc, "bhtsne_affinities")
    m = nnz.value
    return Csr(row_ptr, col[:m], val[:m]), s2


def step(Y: torch.Tensor, P, theta: float, exaggeration: float, learning_rate: float,
         momentum: float, min_gain: float, update: torch.Tensor, gains: torch.Tensor,
         grad: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
         return_z: bool = False):
    """bhtsne_step (P a Csr) or bhtsne_step_layout (P a Layout): Y, update and gains are
    updated in place; returns Z or None."""
    lib = load_library()
    ws, _ = _workspace(P.n, P.nnz, workspace)
    z = C.c_double(0.0)
    fn = lib.bhtsne_step_layout if isinstance(P, Layout) else lib.bhtsne_step
    rc = fn(_ptr(Y, torch.float32, "Y"), P.struct, float(theta), float(exaggeration),
                         float(learning_rate), float(momentum), float(min_gain),
                         _ptr(update, torch.float32, "update"), _ptr(gains, torch.float32, "gains"),
                         _ptr(grad, torch.float32, "grad"), C.byref(z) if return_z else None,
                         _ptr(ws, None, "workspace"), ws.numel(), _stream())
    _check(rc, fn.__name__)
    return z.value if return_z else None


def noalloc_max_bytes() -> int:
    return int(load_library().bhtsne_noalloc_max_bytes())


def step_noalloc(Y: torch.Tensor, P: "Csr", theta: float, exaggeration: float, learning_rate: float,
                 momentum: float, min_gain: float, update: torch.Tensor, gains: torch.Tensor,
                 grad: Optional[torch.Tensor] = None, return_z: bool = False):
    """bhtsne_step_noalloc: bhtsne_step on the library's fixed scratch array
    (no workspace, nothing allocated); Y, update and gains change in place."""
    lib = load_library()
    if not isinstance(P, Csr):
        raise TypeError("step_noalloc takes P as a Csr")
    z = C.c_double(0.0)
    rc = lib.bhtsne_step_noalloc(_ptr(Y, torch.float32, "Y"), P.struct, float(theta), float(exaggeration),
                                 float(learning_rate), float(momentum), float(min_gain),
                                 _ptr(update, torch.float32, "update"), _ptr(gains, torch.float32, "gains"),
                                 _ptr(grad, torch.float32, "grad"), C.byref(z) if return_z else None, _stream())
    _check(rc, "bhtsne_step_noalloc")
    return z.value if return_z else None


def get_stats(workspace: torch.Tensor, check: bool = True) -> dict:
    lib = load_library()
    s = _Stats()
    rc = lib.bhtsne_get_stats(_ptr(workspace, None, "workspace"), C.byref(s), _stream())
    if check:
        _check(rc, "bhtsne_get_stats")
    return {"Z": s.Z, "interactions": s.interactions, "nodes": s.nodes, "bbox": list(s.bbox),
            "r_span": s.r_span, "device_flags": s.device_flags, "max_depth": s.max_depth, "status": rc}


def timing_enable(on: bool = True):
    _check(load_library().bhtsne_timing_enable(1 if on else 0), "bhtsne_timing_enable")


def timing_phases(names=None):
    """Phases that record events while timing is on (None: all of them)."""
    mask = (1 << len(PHASES)) - 1 if names is None else sum(1 << PHASES.index(p) for p in set(names))
    _check(load_library().bhtsne_timing_phases(mask), "bhtsne_timing_phases")


def timing_read(reset: bool = True) -> dict:
    t = _Timing()
    _check(load_library().bhtsne_timing_read(C.byref(t), 1 if reset else 0), "bhtsne_timing_read")
    return {name: (t.ms[k], t.count[k]) for k, name in enumerate(PHASES)}


def debug_sort(Y: torch.Tensor, workspace: Optional[torch.Tensor] = None):
    """(codes, sorted_codes, perm, params[10]) as tensors / list."""
    lib = load_library()
    n = Y.shape[0]
    ws, _ = _workspace(n, 0, workspace)
    codes = torch.empty(n, dtype=torch.int64, device=Y.device)
    scodes = torch.empty(n, dtype=torch.int64, device=Y.device)
    perm = torch.empty(n, dtype=torch.int32, device=Y.device)
    params = (C.c_double * 10)()
    rc = lib.bhtsne_debug_sort(_ptr(Y, torch.float32, "Y"), n, _ptr(codes), _ptr(scodes), _ptr(perm),
                               params, _ptr(ws), ws.numel(), _stream())
    _check(rc, "bhtsne_debug_sort")
    return codes, scodes, perm, list(params)


def debug_tree(Y: torch.Tensor, theta: float = 0.5, workspace: Optional[torch.Tensor] = None) -> dict:
    """Tree arrays (pre-order) truncated to the node count, on the device."""
    lib = load_library()
    n = Y.shape[0]
    ws, _ = _workspace(n, 0, workspace)
    dev = Y.device
    level = torch.empty(2 * n, dtype=torch.uint8, device=dev)
    kind = torch.empty(2 * n, dtype=torch.uint8, device=dev)
    begin = torch.empty(2 * n, dtype=torch.int32, device=dev)
    end = torch.empty(2 * n, dtype=torch.int32, device=dev)
    summ = torch.empty((2 * n, 4), dtype=torch.float32, device=dev)
    meta = torch.empty(2 * n, dtype=torch.int32, device=dev)
    nn = C.c_int64(0)
    rc = lib.bhtsne_debug_tree(_ptr(Y, torch.float32, "Y"), n, float(theta), C.byref(nn), _ptr(level),
                               _ptr(kind), _ptr(begin), _ptr(end), _ptr(summ), _ptr(meta), _ptr(ws),
                               ws.numel(), _stream())
    _check(rc, "bhtsne_debug_tree")
    k = nn.value
    return {"nodes": k, "level": level[:k], "kind": kind[:k], "begin": begin[:k], "end": end[:k],
            "summary": summ[:k], "meta": meta[:k]}


# ---------------------------------------------------------------- 3-D embeddings
def workspace_size_3d(n: int, nnz: int) -> int:
    return int(load_library().bhtsne_workspace_size_3d(int(n), int(nnz)))


def _workspace_3d(n, nnz, ws):
    need = workspace_size_3d(n, nnz)
    if need == 0:
        raise BhtsneError(BHTSNE_EINVAL, "workspace_size_3d")
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    return ws


def _check_3d(Y):
    if Y.dim() != 2 or Y.shape[1] != 3:
        raise ValueError("a 3-D embedding is an n x 3 tensor")


class Layout3(Layout):
    """A locality layout of P for 3-D embeddings (bhtsne_layout_build_3d): the
    relabelled rows and their sliced copy over 8192-point windows of 3-D
    points.  With tiles == 0 (no tile locality) the 3-D calls refuse it and
    the plain Csr serves."""

    def __init__(self, P: Csr, Y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        lib = load_library()
        if Y is not None:
            _check_3d(Y)
        self.n, self.nnz = P.n, P.nnz
        need = int(lib.bhtsne_layout_size_3d(P.n, P.nnz))
        if need == 0:
            raise BhtsneError(BHTSNE_EINVAL, "bhtsne_layout_size_3d")
        self.mem = torch.empty(need, dtype=torch.uint8, device="cuda")
        ws = _workspace_3d(P.n, P.nnz, workspace)
        self._s = _Layout()
        rc = lib.bhtsne_layout_build_3d(P.struct, _ptr(Y, torch.float32, "Y"), _ptr(self.mem), need,
                                        C.byref(self._s), _ptr(ws), ws.numel(), _stream())
        _check(rc, "bhtsne_layout_build_3d")


def layout_size_3d(n: int, nnz: int) -> int:
    return int(load_library().bhtsne_layout_size_3d(int(n), int(nnz)))


def gradient_3d(Y: torch.Tensor, P: "Csr", theta: float, exaggeration: float = 1.0,
                grad: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                return_z: bool = True):
    """bhtsne_gradient_3d (P a Csr) or bhtsne_gradient_layout_3d (P a Layout3):
    returns (grad n x 3, Z or None)."""
    lib = load_library()
    _check_3d(Y)
    if isinstance(P, Layout) and not isinstance(P, Layout3):
        raise TypeError("gradient_3d takes P as a Csr or a Layout3")
    if grad is None:
        grad = torch.empty_like(Y)
    ws = _workspace_3d(P.n, P.nnz, workspace)
    z = C.c_double(0.0)
    fn = lib.bhtsne_gradient_layout_3d if isinstance(P, Layout3) else lib.bhtsne_gradient_3d
    rc = fn(_ptr(Y, torch.float32, "Y"), P.struct, float(theta), float(exaggeration),
            _ptr(grad, torch.float32, "grad"), C.byref(z) if return_z else None,
            _ptr(ws, None, "workspace"), ws.numel(), _stream())
    _check(rc, fn.__name__)
    return grad, (z.value if return_z else None)


def step_3d(Y: torch.Tensor, P: "Csr", theta: float, exaggeration: float, learning_rate: float,
            momentum: float, min_gain: float, update: torch.Tensor, gains: torch.Tensor,
            grad: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
            return_z: bool = False):
    """bhtsne_step_3d (P a Csr) or bhtsne_step_layout_3d (P a Layout3): one
    iteration in place on Y, update and gains (n x 3)."""
    lib = load_library()
    _check_3d(Y)
    if isinstance(P, Layout) and not isinstance(P, Layout3):
        raise TypeError("step_3d takes P as a Csr or a Layout3")
    ws = _workspace_3d(P.n, P.nnz, workspace)
    z = C.c_double(0.0)
    fn = lib.bhtsne_step_layout_3d if isinstance(P, Layout3) else lib.bhtsne_step_3d
    rc = fn(_ptr(Y, torch.float32, "Y"), P.struct, float(theta), float(exaggeration),
            float(learning_rate), float(momentum), float(min_gain),
            _ptr(update, torch.float32, "update"), _ptr(gains, torch.float32, "gains"),
            _ptr(grad, torch.float32, "grad"), C.byref(z) if return_z else None,
            _ptr(ws, None, "workspace"), ws.numel(), _stream())
    _check(rc, fn.__name__)
    return z.value if return_z else None


def debug_sort_3d(Y: torch.Tensor, workspace: Optional[torch.Tensor] = None):
    """(codes, sorted_codes, perm, params[14]) of a 3-D embedding."""
    lib = load_library()
    _check_3d(Y)
    n = Y.shape[0]
    ws = _workspace_3d(n, 0, workspace)
    codes = torch.empty(n, dtype=torch.int64, device=Y.device)
    scodes = torch.empty(n, dtype=torch.int64, device=Y.device)
    perm = torch.empty(n, dtype=torch.int32, device=Y.device)
    params = (C.c_double * 14)()
    rc = lib.bhtsne_debug_sort_3d(_ptr(Y, torch.float32, "Y"), n, _ptr(codes), _ptr(scodes), _ptr(perm),
                                  params, _ptr(ws), ws.numel(), _stream())
    _check(rc, "bhtsne_debug_sort_3d")
    return codes, scodes, perm, list(params)


def debug_tree_3d(Y: torch.Tensor, theta: float = 0.5, workspace: Optional[torch.Tensor] = None) -> dict:
    """Octree arrays (pre-order) truncated to the node count, on the device."""
    lib = load_library()
    _check_3d(Y)
    n = Y.shape[0]
    ws = _workspace_3d(n, 0, workspace)
    dev = Y.device
    level = torch.empty(2 * n, dtype=torch.uint8, device=dev)
    kind = torch.empty(2 * n, dtype=torch.uint8, device=dev)
    begin = torch.empty(2 * n, dtype=torch.int32, device=dev)
    end = torch.empty(2 * n, dtype=torch.int32, device=dev)
    summ = torch.empty((2 * n, 4), dtype=torch.float32, device=dev)
    thr = torch.empty(2 * n, dtype=torch.float32, device=dev)
    meta = torch.empty(2 * n, dtype=torch.int32, device=dev)
    nn = C.c_int64(0)
    rc = lib.bhtsne_debug_tree_3d(_ptr(Y, torch.float32, "Y"), n, float(theta), C.byref(nn), _ptr(level),
                                  _ptr(kind), _ptr(begin), _ptr(end), _ptr(summ), _ptr(thr), _ptr(meta),
                                  _ptr(ws), ws.numel(), _stream())
    _check(rc, "bhtsne_debug_tree_3d")
    k = nn.value
    return {"nodes": k, "level": level[:k], "kind": kind[:k], "begin": begin[:k], "end": end[:k],
            "summary": summ[:k], "threshold": thr[:k], "meta": meta[:k]}


def debug_walk(Y: torch.Tensor, theta: float = 0.5, form: int = -1):
    """(F_rep, Z, interactions) of a 2-D or 3-D fp32 embedding through one form of the repulsive walk: -1 the
    one its size takes, 0 one wave a group of 64 points (2-D), 1 one wave a group, loading ahead."""
    lib = load_library()
    n, dim = Y.shape
    ws = _workspace_3d(n, 0, None) if dim == 3 else _workspace(n, 0, None)[0]
    frep = torch.empty_like(Y)
    Z, inter = C.c_double(0.0), C.c_uint64(0)
    rc = lib.bhtsne_debug_walk(_ptr(Y, torch.float32, "Y"), n, dim, float(theta), int(form), _ptr(frep), C.byref(Z),
                               C.byref(inter), _ptr(ws), ws.numel(), _stream())
    _check(rc, "bhtsne_debug_walk")
    return frep, Z.value, inter.value


# ------------------------------------------------------------------ operators of a trained map
# Their smallest calls run a few microseconds on the GPU, so marshalling is kept short: one look at a tensor where
# nothing is wrong, and what depends on plain numbers alone is worked out once for them.
class _Matrices(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64), ("batch_stride", C.c_int64)]


_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}  # BHTSNE_F32, BHTSNE_F16, BHTSNE_BF16
_written = torch.autograd.graph.increment_version  # a graph that has saved the tensor must not use it any more
_forward = torch.autograd.forward_ad
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


_current_gpu = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _home(t: torch.Tensor, where: str) -> int:
    """The GPU that a call runs on: the current one, which holds all its tensors."""
    gpu = t.get_device()
    if gpu < 0:
        raise ValueError(f"{where} must be a GPU tensor")
    if gpu != _current_gpu():
        raise ValueError(f"{where} is on GPU {gpu}, the current one is {_current_gpu()}: call under torch.cuda.device({gpu})")
    return gpu


def _stream_of(gpu: int) -> int:
    """The current stream of a GPU."""
    return _raw_stream(gpu) if _raw_stream else torch.cuda.current_stream(gpu).cuda_stream


def _type(t: torch.Tensor, where: str) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"{where} must be float32, float16 or bfloat16, got {t.dtype}")
    return kind


def _refuse(t: torch.Tensor, where: str, shape, dtype, gpu: int):
    if not t.is_cuda:
        raise ValueError(f"{where} must be a GPU tensor")
    if t.get_device() != gpu:
        raise ValueError(f"{where} is on GPU {t.get_device()}, the others on {gpu}")
    if t.dtype != dtype:
        raise ValueError(f"{where} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{where} must be {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{where} must be contiguous inside a row")


def _no_tangent(t: torch.Tensor, where: str):
    if _forward.unpack_dual(t).tangent is not None:
        raise ValueError(f"{where} has a tangent, which the call would lose: it has no derivative in forward mode")


def _rows(t: torch.Tensor, where: str, shape, dtype, gpu: int) -> int:
    """Checks a matrix with unit stride inside a row; the stride between its rows."""
    if _forward._current_level >= 0:
        _no_tangent(t, where)
    if not (t.get_device() == gpu and t.dtype == dtype and t.shape == shape):
        _refuse(t, where, shape, dtype, gpu)
    row, inside = t.stride()
    if inside != 1 and shape[1] > 1:
        _refuse(t, where, shape, dtype, gpu)
    return row if shape[0] > 1 else shape[1]


def _vector(t: Optional[torch.Tensor], where: str, size: int, gpu: int, dtype=None) -> Optional[int]:
    if t is None:
        return None
    if _forward._current_level >= 0:
        _no_tangent(t, where)
    if t.get_device() == gpu and t.numel() == size and t.is_contiguous() and (dtype is None or t.dtype == dtype):
        return t.data_ptr()
    if t.numel() != size:
        raise ValueError(f"{where} must have {size} values, got {t.numel()}")
    _ptr(t, dtype, where)
    raise ValueError(f"{where} is on GPU {t.get_device()}, the others on {gpu}")


def _workspace_bytes(t: torch.Tensor, gpu: int) -> int:
    if t.get_device() != gpu or not t.is_contiguous():
        _ptr(t, None, "workspace")
        raise ValueError(f"workspace is on GPU {t.get_device()}, the others on {gpu}")
    return t.numel() * t.element_size()


def _param_type(weight, bias, dtype) -> int:
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError(f"weight and bias must have one type, got {weight.dtype} and {bias.dtype}")
    p = weight if weight is not None else bias
    return _type(p, "weight") if p is not None else _TYPES[dtype]


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5, out: Optional[torch.Tensor] = None):
    """bhtsne_layer_norm over the rows of x (n x d, rows any distance apart): (y, mean, rstd); out may be x.

    y's gradient goes to x, weight and bias through bhtsne_layer_norm_backward (once); mean and rstd have none, and
    neither has a call with out."""
    if torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad)
                                    or (bias is not None and bias.requires_grad)):
        if out is not None:
            raise ValueError("out has no gradient: leave it out, or call under torch.no_grad()")
        return _LayerNorm.apply(x, weight, bias, eps)
    return _layer_norm(x, weight, bias, eps, out)


def _layer_norm(x, weight, bias, eps, out=None):
    lib = load_library()
    if x.dim() != 2:
        raise ValueError(f"x must be n x d, got {tuple(x.shape)}")
    shape, dtype, kind = x.shape, x.dtype, _type(x, "x")
    n, d = shape
    gpu = _home(x, "x")
    x_stride = _rows(x, "x", shape, dtype, gpu)
    if out is None:
        y, y_stride = torch.empty_like(x) if x_stride == d else x.new_empty(shape), d
    else:
        y, y_stride = out, _rows(out, "out", shape, dtype, gpu)
    mean, rstd = x.new_empty((2, n), dtype=torch.float32).unbind(0)
    rc = lib.bhtsne_layer_norm(x.data_ptr(), x_stride, _vector(weight, "weight", d, gpu), _vector(bias, "bias", d, gpu), n, d,
                               eps, kind, _param_type(weight, bias, dtype), y.data_ptr(), y_stride, mean.data_ptr(),
                               rstd.data_ptr(), _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_layer_norm")
    if out is not None:
        _written(out)
    return y, mean, rstd


class _LayerNorm(torch.autograd.Function):
    """layer_norm as a node of torch's graph."""

    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = _layer_norm(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias_type = bias.dtype if bias is not None else None
        ctx.mark_non_differentiable(mean, rstd)
        ctx.set_materialize_grads(False)
        return y, mean, rstd

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, _mean, _rstd):
        if dy is None:
            return None, None, None, None
        x, weight, mean, rstd = ctx.saved_tensors
        n, d = x.shape
        if (d > 1 and dy.stride(1) != 1) or (n > 1 and 0 < dy.stride(0) < d):
            dy = dy.contiguous()
        dx, dweight, dbias = _layer_norm_backward(dy, x, weight, mean, rstd, ctx.bias_type)
        return dx, dweight if weight is not None else None, dbias if ctx.bias_type is not None else None, None


@functools.lru_cache(maxsize=256)
def layer_norm_workspace_size(n: int, d: int) -> int:
    return int(load_library().bhtsne_layer_norm_workspace_size(int(n), int(d)))


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor,
                        rstd: torch.Tensor, dx: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None):
    """bhtsne_layer_norm_backward: (dx, dweight, dbias), the last two of weight's type (x's without a weight);
    dx may be dy or x.  The results have no gradient of their own."""
    return _layer_norm_backward(dy, x, weight, mean, rstd, None, dx, workspace)


def _layer_norm_backward(dy, x, weight, mean, rstd, bias_type=None, dx=None, workspace=None):
    lib = load_library()
    if x.dim() != 2:
        raise ValueError(f"x must be n x d, got {tuple(x.shape)}")
    shape, dtype, kind = x.shape, x.dtype, _type(x, "x")
    n, d = shape
    gpu = _home(x, "x")
    need = layer_norm_workspace_size(n, d)
    if need == 0:
        raise BhtsneError(BHTSNE_EINVAL, "bhtsne_layer_norm_workspace_size")
    x_stride, dy_stride = _rows(x, "x", shape, dtype, gpu), _rows(dy, "dy", shape, dtype, gpu)
    given = dx
    if dx is None:
        dx, dx_stride = torch.empty_like(x) if x_stride == d else x.new_empty(shape), d
    else:
        dx_stride = _rows(dx, "dx", shape, dtype, gpu)
    if workspace is None:
        workspace = x.new_empty(need, dtype=torch.uint8)
    else:
        need = _workspace_bytes(workspace, gpu)
    if weight is not None:
        _type(weight, "weight")
    ptype = weight.dtype if weight is not None else bias_type if bias_type is not None else dtype
    dweight, dbias = x.new_empty((2, d), dtype=ptype).unbind(0)
    rc = lib.bhtsne_layer_norm_backward(dy.data_ptr(), dy_stride, x.data_ptr(), x_stride, _vector(weight, "weight", d, gpu),
                                        _vector(mean, "mean", n, gpu, torch.float32),
                                        _vector(rstd, "rstd", n, gpu, torch.float32), n, d, kind, _TYPES[ptype],
                                        dx.data_ptr(), dx_stride, dweight.data_ptr(), dbias.data_ptr(),
                                        workspace.data_ptr(), need, _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_layer_norm_backward")
    if given is not None:
        _written(given)
    return dx, dweight, dbias


def _matrices(t: torch.Tensor, where: str, shape, dtype, gpu: int) -> _Matrices:
    if _forward._current_level >= 0:
        _no_tangent(t, where)
    if not (t.get_device() == gpu and t.dtype == dtype and t.shape == shape):
        _refuse(t, where, shape, dtype, gpu)
    stride = t.stride()
    if stride[-1] != 1 and shape[-1] > 1:
        _refuse(t, where, shape, dtype, gpu)
    return _Matrices(t.data_ptr(), stride[-2] if shape[-2] > 1 else shape[-1], stride[0] if len(shape) == 3 else 0)


def _matrix_sizes(t: torch.Tensor, where: str):
    shape = t.shape
    if len(shape) == 2:
        return 1, shape[0], shape[1]
    if len(shape) == 3:
        return tuple(shape)
    raise ValueError(f"{where} must be rows x cols or batch x rows x cols, got {tuple(shape)}")


@functools.lru_cache(maxsize=64)
def _flat_coefficients(flat, steps: int):
    if len(flat) == 3:
        flat = flat * max(1, steps)
    if len(flat) != 3 * steps and steps > 0:
        raise ValueError(f"coefficients must be one (a, b, c) or {steps} of them")
    return (C.c_double * len(flat))(*flat)


def _coefficients(coefficients, steps: int):
    """None, one (a, b, c) for every step, or one for each, as they are now: kept by their values alone."""
    if coefficients is None:
        return None
    try:
        flat = tuple(map(float, coefficients))
    except (TypeError, ValueError, RuntimeError):  # not numbers: rows of them
        flat = []
        for row in coefficients:
            if isinstance(row, (list, tuple)) or getattr(row, "ndim", 0) > 0:
                flat.extend(map(float, row))
            else:
                flat.append(float(row))
    return _flat_coefficients(tuple(flat), int(steps))


@functools.lru_cache(maxsize=256)
def orthogonalise_workspace_size(batch: int, rows: int, cols: int) -> int:
    return int(load_library().bhtsne_orthogonalise_workspace_size(int(batch), int(rows), int(cols)))


def _orthogonal_workspace(sizes, like, ws, gpu: int):
    if ws is not None:
        return ws, _workspace_bytes(ws, gpu)
    need = orthogonalise_workspace_size(*sizes)
    if need == 0:
        raise BhtsneError(BHTSNE_EINVAL, "bhtsne_orthogonalise_workspace_size")
    return like.new_empty(need, dtype=torch.uint8), need


def orthogonalise(G: torch.Tensor, steps: int = 5, coefficients=None, eps: float = 1e-7,
                  out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """bhtsne_orthogonalise of G (rows x cols, or batch x rows x cols); out may be G.  It has no gradient, and refuses a G
    whose graph torch records."""
    lib = load_library()
    if G.requires_grad and torch.is_grad_enabled():
        raise ValueError("orthogonalise has no gradient: take G.detach(), or call under torch.no_grad()")
    sizes = _matrix_sizes(G, "G")
    kind, shape, dtype, gpu = _type(G, "G"), G.shape, G.dtype, _home(G, "G")
    g = _matrices(G, "G", shape, dtype, gpu)
    O = out if out is not None else torch.empty_like(G, memory_format=torch.contiguous_format)
    o = _matrices(O, "out", shape, dtype, gpu)
    ws, nbytes = _orthogonal_workspace(sizes, G, workspace, gpu)
    rc = lib.bhtsne_orthogonalise(C.byref(g), *sizes, kind, _coefficients(coefficients, steps), steps, eps, C.byref(o),
                                  ws.data_ptr(), nbytes, _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_orthogonalise")
    if out is not None:
        _written(out)
    return O


def muon_step(W: torch.Tensor, G: torch.Tensor, M: torch.Tensor, learning_rate: float, momentum: float = 0.95,
              nesterov: bool = True, weight_decay: float = 0.0, scale: Optional[float] = None, steps: int = 5,
              coefficients=None, eps: float = 1e-7, workspace: Optional[torch.Tensor] = None) -> None:
    """bhtsne_muon_step: one step in place on the weights W and the fp32 momentum M (rows x cols, or batch x rows x
    cols), outside of torch's graph as an optimiser's.  scale: None is sqrt(max(1, rows / cols))."""
    lib = load_library()
    sizes = _matrix_sizes(W, "W")
    kind, shape, gpu = _type(W, "W"), W.shape, _home(W, "W")
    w, g = _matrices(W, "W", shape, W.dtype, gpu), _matrices(G, "G", shape, W.dtype, gpu)
    m = _matrices(M, "M", shape, torch.float32, gpu)
    if scale is None:
        scale = max(1.0, sizes[1] / max(1, sizes[2])) ** 0.5
    ws, nbytes = _orthogonal_workspace(sizes, W, workspace, gpu)
    rc = lib.bhtsne_muon_step(C.byref(w), C.byref(g), C.byref(m), *sizes, kind, learning_rate, momentum, bool(nesterov),
                              weight_decay, scale, _coefficients(coefficients, steps), steps, eps, ws.data_ptr(), nbytes,
                              _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_muon_step")
    _written((W, M))


# ------------------------------------------------------------------ dense operators of a trained map
_ACTIVATIONS = {"silu": 0, "gelu": 1}  # BHTSNE_SILU, BHTSNE_GELU
_I8 = 3


def _activation(name: str) -> int:
    kind = _ACTIVATIONS.get(name)
    if kind is None:
        raise ValueError(f"activation must be one of {sorted(_ACTIVATIONS)}, got {name!r}")
    return kind


def _layer_sizes(x: torch.Tensor, gate: torch.Tensor):
    if x.dim() != 2 or gate.dim() != 2:
        raise ValueError(f"x must be n x d and gate f x d, got {tuple(x.shape)} and {tuple(gate.shape)}")
    return x.shape[0], x.shape[1], gate.shape[0]


def gated_layer(x: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, activation: str = "silu", keep: bool = False,
                out: Optional[torch.Tensor] = None):
    """bhtsne_gated_layer: h = act(x gate^T) (x up^T) of x (n x d) and the weights gate and up (f x d, a row a feature);
    with keep (h, a, b), a = x gate^T and b = x up^T being what the backward pass takes.

    h's gradient goes to x, gate and up through bhtsne_gated_layer_backward (once); a and b have none, and neither has a
    call with out.  A backward pass that is captured in a graph wants leaves that no graph recorded outside of the capture
    still holds, as every one of torch's does."""
    if torch.is_grad_enabled() and (x.requires_grad or gate.requires_grad or up.requires_grad):
        if out is not None:
            raise ValueError("out has no gradient: leave it out, or call under torch.no_grad()")
        h, a, b = _GatedLayer.apply(x, gate, up, activation)
        return (h, a, b) if keep else h
    if out is not None:
        _no_gradient(out, "a gated_layer with out")
    h, a, b = _gated_layer(x, gate, up, activation, keep, out)
    return (h, a, b) if keep else h


def _gated_layer(x, gate, up, activation, keep, out=None):
    lib = load_library()
    n, d, f = _layer_sizes(x, gate)
    act, dtype, kind, gpu = _activation(activation), x.dtype, _type(x, "x"), _home(x, "x")
    x_stride = _rows(x, "x", x.shape, dtype, gpu)
    gate_stride, up_stride = _rows(gate, "gate", (f, d), dtype, gpu), _rows(up, "up", (f, d), dtype, gpu)
    h_stride = f if out is None else _rows(out, "out", (n, f), dtype, gpu)
    h = out if out is not None else x.new_empty((n, f))
    a, b = (x.new_empty((n, f)), x.new_empty((n, f))) if keep else (None, None)
    rc = lib.bhtsne_gated_layer(x.data_ptr(), x_stride, gate.data_ptr(), gate_stride, up.data_ptr(), up_stride, n, d, f, act, kind,
                                h.data_ptr(), h_stride, a.data_ptr() if keep else None, f, b.data_ptr() if keep else None, f,
                                _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_gated_layer")
    if out is not None:
        _written(out)
    return h, a, b


class _GatedLayer(torch.autograd.Function):
    """gated_layer as a node of torch's graph."""

    @staticmethod
    def forward(ctx, x, gate, up, activation):
        h, a, b = _gated_layer(x, gate, up, activation, True)
        ctx.save_for_backward(x, gate, up, a, b)
        ctx.activation = activation
        ctx.mark_non_differentiable(a, b)
        ctx.set_materialize_grads(False)  # a's and b's would be arrays of zeros, as large as they are
        return h, a, b

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, _a, _b):
        if dh is None:
            return None, None, None, None
        x, gate, up, a, b = ctx.saved_tensors
        if (dh.shape[1] > 1 and dh.stride(1) != 1) or (dh.shape[0] > 1 and 0 < dh.stride(0) < dh.shape[1]):
            dh = dh.contiguous()
        return (*_gated_layer_backward(dh, x, gate, up, a, b, ctx.activation, ctx.needs_input_grad[:3]), None)


@functools.lru_cache(maxsize=256)
def gated_layer_workspace_size(n: int, d: int, f: int, dtype: torch.dtype = torch.float32) -> int:
    return int(load_library().bhtsne_gated_layer_workspace_size(int(n), int(d), int(f), _TYPES[dtype]))


def gated_layer_backward(dh: torch.Tensor, x: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, a: torch.Tensor, b: torch.Tensor,
                         activation: str = "silu", workspace: Optional[torch.Tensor] = None):
    """bhtsne_gated_layer_backward: (dx, dgate, dup) from a and b as gated_layer kept them.  The results have no gradient
    of their own."""
    return _gated_layer_backward(dh, x, gate, up, a, b, activation, (True, True, True), workspace)


def _gated_layer_backward(dh, x, gate, up, a, b, activation, wanted, workspace=None):
    lib = load_library()
    n, d, f = _layer_sizes(x, gate)
    act, dtype, kind, gpu = _activation(activation), x.dtype, _type(x, "x"), _home(x, "x")
    need = gated_layer_workspace_size(n, d, f, dtype)
    if need == 0:
        raise BhtsneError(BHTSNE_EINVAL, "bhtsne_gated_layer_workspace_size")
    wide, tall = (n, f), (f, d)
    strides = (_rows(dh, "dh", wide, dtype, gpu), _rows(x, "x", x.shape, dtype, gpu), _rows(gate, "gate", tall, dtype, gpu),
               _rows(up, "up", tall, dtype, gpu), _rows(a, "a", wide, dtype, gpu), _rows(b, "b", wide, dtype, gpu))
    if workspace is None:
        workspace = x.new_empty(need, dtype=torch.uint8)
    else:
        need = _workspace_bytes(workspace, gpu)
    dx = x.new_empty((n, d)) if wanted[0] else None
    dgate, dup = (x.new_empty(tall) if w else None for w in wanted[1:])
    rc = lib.bhtsne_gated_layer_backward(dh.data_ptr(), strides[0], x.data_ptr(), strides[1], gate.data_ptr(), strides[2],
                                         up.data_ptr(), strides[3], a.data_ptr(), strides[4], b.data_ptr(), strides[5], n, d, f,
                                         act, kind, dx.data_ptr() if wanted[0] else None, d,
                                         dgate.data_ptr() if wanted[1] else None, d, dup.data_ptr() if wanted[2] else None, d,
                                         workspace.data_ptr(), need, _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_gated_layer_backward")
    return dx, dgate, dup


def quantise_rows(x: torch.Tensor):
    """bhtsne_quantise_rows: (q, scale), int8 values of x's shape and a fp32 scale for each row."""
    lib = load_library()
    _no_gradient(x, "quantise_rows")
    if x.dim() != 2:
        raise ValueError(f"x must be n x d, got {tuple(x.shape)}")
    n, d = x.shape
    kind, gpu = _type(x, "x"), _home(x, "x")
    stride = _rows(x, "x", x.shape, x.dtype, gpu)
    q, scale = x.new_empty((n, d), dtype=torch.int8), x.new_empty(n, dtype=torch.float32)
    rc = lib.bhtsne_quantise_rows(x.data_ptr(), stride, n, d, kind, q.data_ptr(), d, scale.data_ptr(), _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_quantise_rows")
    return q, scale


def _no_gradient(t: torch.Tensor, where: str):
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{where} has no gradient: detach its tensors, or call under torch.no_grad()")


@functools.lru_cache(maxsize=256)
def linear_i8_workspace_size(n: int, d: int) -> int:
    return int(load_library().bhtsne_linear_i8_workspace_size(int(n), int(d)))


def linear_i8(x: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, x_scale: Optional[torch.Tensor] = None,
              bias: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """bhtsne_linear_i8: x_scale_i w_scale_j sum_k x_ik w_jk + bias_j of x (n x d) and int8 weights w (f x d, a row a
    feature, as quantise_rows gives them).  x is int8 with x_scale, or of another type without: its rows are then quantised
    on the way.  dtype: of the result, None is out's, x's, or float32 for an int8 x; bias is of that type or float32.  It
    has no gradient, and refuses inputs whose graph torch records."""
    lib = load_library()
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError(f"x must be n x d and w f x d, got {tuple(x.shape)} and {tuple(w.shape)}")
    for t in (x, w_scale, x_scale, bias, out):
        if t is not None:
            _no_gradient(t, "linear_i8")
    (n, d), f = x.shape, w.shape[0]
    whole, gpu = x.dtype == torch.int8, _home(x, "x")
    if whole != (x_scale is not None):
        raise ValueError("an int8 x comes with its x_scale, another without")
    x_kind = _I8 if whole else _type(x, "x")
    if out is not None and dtype is not None and out.dtype != dtype:
        raise ValueError(f"out must be {dtype}, got {out.dtype}")
    if dtype is None:
        dtype = out.dtype if out is not None else torch.float32 if whole else x.dtype
    kind = _TYPES.get(dtype)
    if kind is None:
        raise ValueError(f"dtype must be float32, float16 or bfloat16, got {dtype}")
    x_stride, w_stride = _rows(x, "x", x.shape, x.dtype, gpu), _rows(w, "w", (f, d), torch.int8, gpu)
    out_stride = f if out is None else _rows(out, "out", (n, f), dtype, gpu)
    result = out if out is not None else x.new_empty((n, f), dtype=dtype)
    bias_kind = kind
    if bias is not None:
        bias_kind = _TYPES.get(bias.dtype)
        if bias_kind not in (kind, 0):
            raise ValueError(f"bias must be {dtype} or float32, got {bias.dtype}")
    need = 0
    if workspace is not None:
        need = _workspace_bytes(workspace, gpu)
    elif not whole:
        need = linear_i8_workspace_size(n, d)
        if need == 0:
            raise BhtsneError(BHTSNE_EINVAL, "bhtsne_linear_i8_workspace_size")
        if need > 256:
            workspace = x.new_empty(need, dtype=torch.uint8)
    rc = lib.bhtsne_linear_i8(x.data_ptr(), x_stride, x_kind, _vector(x_scale, "x_scale", n, gpu, torch.float32), w.data_ptr(), w_stride,
                              _vector(w_scale, "w_scale", f, gpu, torch.float32), _vector(bias, "bias", f, gpu), n, d, f, kind,
                              bias_kind, result.data_ptr(), out_stride, workspace.data_ptr() if workspace is not None else None, need,
                              _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_linear_i8")
    if out is not None:
        _written(out)
    return result


def _lists(logits: torch.Tensor, idx: torch.Tensor, teacher: torch.Tensor):
    """Checks what both directions of distil_loss take: the arguments from logits to k, and the two types."""
    if logits.dim() != 2 or idx.dim() != 2:
        raise ValueError(f"logits must be n x v and idx n x k, got {tuple(logits.shape)} and {tuple(idx.shape)}")
    (n, v), k = logits.shape, idx.shape[1]
    kind, gpu = _type(logits, "logits"), _home(logits, "logits")
    teacher_kind = _type(teacher, "teacher")
    if teacher_kind not in (kind, 0):
        raise ValueError(f"teacher must be {logits.dtype} or float32, got {teacher.dtype}")
    args = (logits.data_ptr(), _rows(logits, "logits", logits.shape, logits.dtype, gpu), n, v, idx.data_ptr(),
            _rows(idx, "idx", (n, k), torch.int32, gpu), teacher.data_ptr(), _rows(teacher, "teacher", (n, k), teacher.dtype, gpu), k)
    return args, kind, teacher_kind, gpu


@functools.lru_cache(maxsize=256)
def distil_loss_workspace_size(n: int, v: int) -> int:
    return int(load_library().bhtsne_distil_loss_workspace_size(int(n), int(v)))


def distil_loss(logits: torch.Tensor, idx: torch.Tensor, teacher: torch.Tensor, temperature: float = 1.0,
                workspace: Optional[torch.Tensor] = None, keep: bool = False):
    """bhtsne_distil_loss: (loss, lse), n values each, of logits (n x v) against the teacher's logits (n x k) of the classes
    idx (n x k int32; outside [0, v): absent); with keep (loss, lse, kept), kept (n x 2) being what lse is rounded from, for the
    backward pass of rows with a large lse.

    loss's gradient goes to the logits through bhtsne_distil_loss_backward_kept (once); lse and kept have none, and the teacher
    neither: one whose graph torch records is refused.  For a captured backward pass see gated_layer."""
    _no_gradient(teacher, "the teacher of distil_loss")
    if logits.requires_grad and torch.is_grad_enabled():
        loss, lse, kept = _DistilLoss.apply(logits, idx, teacher, float(temperature), workspace)
    else:
        loss, lse, kept = _distil_loss(logits, idx, teacher, temperature, workspace, keep)
    return (loss, lse, kept) if keep else (loss, lse)


def _distil_loss(logits, idx, teacher, temperature, workspace=None, keep=False):
    lib = load_library()
    args, kind, teacher_kind, gpu = _lists(logits, idx, teacher)
    n, v = logits.shape
    loss, lse = logits.new_empty(n, dtype=torch.float32), logits.new_empty(n, dtype=torch.float32)  # two: each may be changed in place
    kept = logits.new_empty((n, 2), dtype=torch.float32) if keep else None
    if workspace is not None:
        need = _workspace_bytes(workspace, gpu)
    else:
        need = distil_loss_workspace_size(n, v)
        if need > 256:
            workspace = logits.new_empty(need, dtype=torch.uint8)
    rc = lib.bhtsne_distil_loss_kept(*args, temperature, kind, teacher_kind, loss.data_ptr(), lse.data_ptr(),
                                     kept.data_ptr() if keep else None, workspace.data_ptr() if workspace is not None else None,
                                     need, _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_distil_loss")
    return loss, lse, kept


class _DistilLoss(torch.autograd.Function):
    """distil_loss as a node of torch's graph."""

    @staticmethod
    def forward(ctx, logits, idx, teacher, temperature, workspace):
        loss, lse, kept = _distil_loss(logits, idx, teacher, temperature, workspace, True)
        ctx.save_for_backward(logits, idx, teacher, lse, kept)
        ctx.temperature = temperature
        ctx.mark_non_differentiable(lse, kept)
        ctx.set_materialize_grads(False)
        return loss, lse, kept

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss, _lse, _kept):
        if dloss is None:
            return None, None, None, None, None
        logits, idx, teacher, lse, kept = ctx.saved_tensors
        return distil_loss_backward(dloss.contiguous(), logits, idx, teacher, lse, ctx.temperature, kept=kept), None, None, None, None


def distil_loss_backward(dloss: torch.Tensor, logits: torch.Tensor, idx: torch.Tensor, teacher: torch.Tensor, lse: torch.Tensor,
                         temperature: float = 1.0, dlogits: Optional[torch.Tensor] = None,
                         kept: Optional[torch.Tensor] = None) -> torch.Tensor:
    """bhtsne_distil_loss_backward: the gradient of the logits, of their type; dlogits may be the logits.  From lse as
    distil_loss gave it, which is off by its rounding, |lse| 2^-24; with kept as well that counts no more.  The result has no
    gradient of its own."""
    lib = load_library()
    args, kind, teacher_kind, gpu = _lists(logits, idx, teacher)
    n, v = logits.shape
    stride = v if dlogits is None else _rows(dlogits, "dlogits", logits.shape, logits.dtype, gpu)
    out = dlogits if dlogits is not None else logits.new_empty((n, v))
    rc = lib.bhtsne_distil_loss_backward_kept(_vector(dloss, "dloss", n, gpu, torch.float32), *args,
                                              _vector(lse, "lse", n, gpu, torch.float32), _vector(kept, "kept", 2 * n, gpu, torch.float32),
                                              temperature, kind, teacher_kind, out.data_ptr(), stride, _stream_of(gpu))
    if rc:
        _check(rc, "bhtsne_distil_loss_backward")
    if dlogits is not None:
        _written(dlogits)
    return out
