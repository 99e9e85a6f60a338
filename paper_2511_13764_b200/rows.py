"""ctypes binding of include/nk_rows.h (layers whose weight is chosen row by row).  Same names,
argument marshalling only; tensors are used for their pointers, the caller owns every buffer."""
from __future__ import annotations

import ctypes

from . import binding
from .binding import BF16, F32, ROW_MAJOR, NkError, _ptr

GROUPED_ROWS, GROUPED_WEIGHTS = 0, 1

EXPORTS = ["nk_grouped_create", "nk_grouped_workspace_bytes", "nk_grouped_run", "nk_grouped_check",
           "nk_grouped_kernel_name", "nk_grouped_last_cuda_error", "nk_grouped_destroy"]


class GroupedDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("groups", "rows", "N", "K")]
                + [(n, ctypes.c_int32) for n in ("kind", "in_dtype", "out_dtype", "layout_b", "beta", "device")]
                + [(n, ctypes.c_int64) for n in ("lda", "ldb", "ldc", "stride_g")])


_lib = None


def lib():
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        for family, desc in (("grouped", GroupedDesc),):
            create = getattr(L, f"nk_{family}_create")
            create.restype, create.argtypes = ctypes.c_int, [ctypes.POINTER(desc), ctypes.POINTER(vp)]
            for name, result in (("workspace_bytes", sz), ("check", ctypes.c_int), ("destroy", ctypes.c_int),
                                 ("kernel_name", ctypes.c_char_p), ("last_cuda_error", ctypes.c_char_p)):
                f = getattr(L, f"nk_{family}_{name}")
                f.restype, f.argtypes = result, [vp]
        L.nk_grouped_run.restype = ctypes.c_int
        L.nk_grouped_run.argtypes = [vp] * 6 + [sz, vp]
        _lib = L
    return _lib


def exported_symbols():
    L = lib()
    return [s for s in EXPORTS if hasattr(L, s)]


def _bytes(workspace, workspace_bytes):
    if workspace_bytes is not None:
        return workspace_bytes
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


class _Handle:
    """create / workspace_bytes / check / destroy of one family of plans."""
    family = ""

    def _create(self, desc):
        self.desc = desc
        self._h = ctypes.c_void_p()
        self._check(getattr(lib(), f"nk_{self.family}_create")(ctypes.byref(desc), ctypes.byref(self._h)))

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
        status = lib().nk_grouped_run(self._h, _ptr(A), _ptr(B), _ptr(C), _ptr(offsets), _ptr(workspace),
                                      _bytes(workspace, workspace_bytes), stream)
        if status:
            self._check(status)
