"""ctypes binding of include/nk_rows.h (layers whose weight is chosen row by row).  Same names,
argument marshalling only; tensors are used for their pointers, the caller owns every buffer."""
from __future__ import annotations

import ctypes

from . import binding
from .binding import BF16, F32, ROW_MAJOR, NkError, _ptr

GROUPED_ROWS, GROUPED_WEIGHTS = 0, 1

EXPORTS = ["nk_grouped_create", "nk_grouped_workspace_bytes", "nk_grouped_run", "nk_grouped_check",
           "nk_grouped_kernel_name", "nk_grouped_last_cuda_error", "nk_grouped_destroy",
           "nk_route_create", "nk_route_workspace_bytes", "nk_route_run", "nk_route_backward", "nk_route_dispatch",
           "nk_route_combine", "nk_route_combine_backward", "nk_route_check", "nk_route_kernel_name",
           "nk_route_last_cuda_error", "nk_route_destroy",
           "nk_lora_create", "nk_lora_workspace_bytes", "nk_lora_run", "nk_lora_check", "nk_lora_kernel_name",
           "nk_lora_last_cuda_error", "nk_lora_destroy"]


class GroupedDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("groups", "rows", "N", "K")]
                + [(n, ctypes.c_int32) for n in ("kind", "in_dtype", "out_dtype", "layout_b", "beta", "device")]
                + [(n, ctypes.c_int64) for n in ("lda", "ldb", "ldc", "stride_g")])


class RouteDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("tokens", "experts", "topk", "width", "ld_logits", "ld_tokens", "ld_slots")]
                + [(n, ctypes.c_int32) for n in ("logits_dtype", "dtype", "renormalise", "device")])


class LoraDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("rows", "N", "K", "rank", "adapters", "requests")]
                + [(n, ctypes.c_int32) for n in ("in_dtype", "out_dtype", "layout", "device")]
                + [(n, ctypes.c_int64) for n in ("ldx", "ldw", "ldy")])


_lib = None


def lib():
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        for family, desc in (("grouped", GroupedDesc), ("route", RouteDesc), ("lora", LoraDesc)):
            create = getattr(L, f"nk_{family}_create")
            create.restype, create.argtypes = ctypes.c_int, [ctypes.POINTER(desc), ctypes.POINTER(vp)]
            for name, result in (("workspace_bytes", sz), ("check", ctypes.c_int), ("destroy", ctypes.c_int),
                                 ("kernel_name", ctypes.c_char_p), ("last_cuda_error", ctypes.c_char_p)):
                f = getattr(L, f"nk_{family}_{name}")
                f.restype, f.argtypes = result, [vp]
        L.nk_grouped_run.restype = ctypes.c_int
        L.nk_grouped_run.argtypes = [vp] * 6 + [sz, vp]
        L.nk_lora_run.restype = ctypes.c_int
        L.nk_lora_run.argtypes = [vp] * 10 + [sz, vp]
        L.nk_route_run.restype = ctypes.c_int
        L.nk_route_run.argtypes = [vp] * 7 + [sz, vp]
        for name, pointers in (("backward", 4), ("dispatch", 3), ("combine", 4), ("combine_backward", 6)):
            f = getattr(L, f"nk_route_{name}")
            f.restype, f.argtypes = ctypes.c_int, [vp] * (pointers + 2)
        _lib = L
    return _lib


def exported_symbols():
    L = lib()
    return [s for s in EXPORTS if hasattr(L, s)]


def _bytes(workspace, workspace_bytes):
    if workspace_bytes is not None:
        return workspace_bytes
    return 0 if workspace is None else workspace.nbytes


class _Handle:
    """create / workspace_bytes / check / destroy of one family of plans."""
    family = ""

    def _create(self, desc):
        self.desc = desc
        self._h = ctypes.c_void_p()
        self._check(getattr(lib(), f"nk_{self.family}_create")(ctypes.byref(desc), ctypes.byref(self._h)))
        self._raw = self._h.value

    def _check(self, status):
        if status != 0:
            msg = lib().nk_status_str(status).decode()
            if self._h:
                extra = getattr(lib(), f"nk_{self.family}_last_cuda_error")(self._h).decode()
                if extra:
                    msg += f" ({extra})"
            raise NkError(status, msg)

    @property
    def workspace_bytes(self) -> int:
        return getattr(lib(), f"nk_{self.family}_workspace_bytes")(self._h)

    @property
    def kernel_name(self) -> str:
        return getattr(lib(), f"nk_{self.family}_kernel_name")(self._h).decode()

    def check(self):
        self._check(getattr(lib(), f"nk_{self.family}_check")(self._h))

    def destroy(self):
        if self._h:
            getattr(lib(), f"nk_{self.family}_destroy")(self._h)
            self._h = ctypes.c_void_p()
            self._raw = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class GroupedPlan(_Handle):
    """nk_grouped: products grouped by expert over ragged groups of rows (GROUPED_ROWS), or the
    gradient of their weights (GROUPED_WEIGHTS)."""
    family = "grouped"

    def __init__(self, groups, rows, N, K, kind=GROUPED_ROWS, in_dtype=BF16, out_dtype=F32, layout_b=ROW_MAJOR,
                 beta=0, device=0, lda=0, ldb=0, ldc=0, stride_g=0):
        self._create(GroupedDesc(groups, rows, N, K, kind, in_dtype, out_dtype, layout_b, beta, device,
                                 lda, ldb, ldc, stride_g))

    def run(self, A, B, C, offsets, workspace=None, workspace_bytes=None, stream=None):
        """offsets: device INT32 [groups + 1]; never read by the host."""
        status = _lib.nk_grouped_run(self._raw, _ptr(A), _ptr(B), _ptr(C), _ptr(offsets), _ptr(workspace),
                                      _bytes(workspace, workspace_bytes), stream)
        if status:
            self._check(status)


class RoutePlan(_Handle):
    """nk_route: choice of experts and gates, the rows' way to their experts' order and back, and the gradients."""
    family = "route"

    def __init__(self, tokens, experts, topk, width=0, logits_dtype=F32, dtype=BF16, renormalise=1, device=0,
                 ld_logits=0, ld_tokens=0, ld_slots=0):
        self._create(RouteDesc(tokens, experts, topk, width, ld_logits, ld_tokens, ld_slots, logits_dtype, dtype,
                               renormalise, device))

    def run(self, logits, gates, experts, offsets, slots, workspace=None, workspace_bytes=None, stream=None):
        status = _lib.nk_route_run(self._raw, _ptr(logits), _ptr(gates), _ptr(experts), _ptr(offsets), _ptr(slots),
                                    _ptr(workspace), _bytes(workspace, workspace_bytes), stream)
        if status:
            self._check(status)

    def backward(self, logits, experts, dgates, dlogits, stream=None):
        status = _lib.nk_route_backward(self._raw, _ptr(logits), _ptr(experts), _ptr(dgates), _ptr(dlogits), stream)
        if status:
            self._check(status)

    def dispatch(self, X, slots, Xs, stream=None):
        status = _lib.nk_route_dispatch(self._raw, _ptr(X), _ptr(slots), _ptr(Xs), stream)
        if status:
            self._check(status)

    def combine(self, Ys, slots, Y, gates=None, stream=None):
        """gates None: plain sum, the gradient of dispatch."""
        status = _lib.nk_route_combine(self._raw, _ptr(Ys), _ptr(slots), _ptr(gates), _ptr(Y), stream)
        if status:
            self._check(status)

    def combine_backward(self, dY, Ys, slots, gates, dYs, dgates, stream=None):
        status = _lib.nk_route_combine_backward(self._raw, _ptr(dY), _ptr(Ys), _ptr(slots), _ptr(gates), _ptr(dYs),
                                                 _ptr(dgates), stream)
        if status:
            self._check(status)


class LoraPlan(_Handle):
    """nk_lora: a shared projection with the low-rank adapters of many requests beside it."""
    family = "lora"

    def __init__(self, rows, N, K, rank, adapters, requests, in_dtype=BF16, out_dtype=F32, layout=ROW_MAJOR, device=0,
                 ldx=0, ldw=0, ldy=0):
        self._create(LoraDesc(rows, N, K, rank, adapters, requests, in_dtype, out_dtype, layout, device, ldx, ldw, ldy))

    def run(self, X, W, A, B, scale, offsets, adapter, Y, workspace=None, workspace_bytes=None, stream=None):
        """offsets (INT32 [requests + 1]), adapter (INT32 [requests]) and scale (FP32 [adapters]) are on the device."""
        status = _lib.nk_lora_run(self._raw, _ptr(X), _ptr(W), _ptr(A), _ptr(B), _ptr(scale), _ptr(offsets), _ptr(adapter),
                                   _ptr(Y), _ptr(workspace), _bytes(workspace, workspace_bytes), stream)
        if status:
            self._check(status)
