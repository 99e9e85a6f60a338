"""ctypes binding of include/nk_mx.h (4-bit floating-point operands).  Same names, argument marshalling only;
tensors are used for their pointers, the caller owns every buffer."""
from __future__ import annotations

import ctypes

from . import binding
from .binding import BF16, EPI_NONE, F32
from .rows import _Handle

MXF4, NVF4 = 0, 1

EXPORTS = ["nk_pack_create", "nk_pack_data_bytes", "nk_pack_scales_bytes", "nk_pack_workspace_bytes", "nk_pack_scale",
           "nk_pack_run", "nk_pack_values", "nk_pack_check", "nk_pack_kernel_name", "nk_pack_last_cuda_error", "nk_pack_destroy",
           "nk_mx_create", "nk_mx_workspace_bytes", "nk_mx_run", "nk_mx_check", "nk_mx_kernel_name", "nk_mx_last_cuda_error",
           "nk_mx_destroy"]


class PackDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("rows", "K", "batch", "groups", "ldx", "stride_x")]
                + [(n, ctypes.c_int32) for n in ("format", "in_dtype", "value_dtype", "transposed", "device")])


class MxDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int64) for n in ("rows", "N", "K", "groups", "ldc")]
                + [(n, ctypes.c_int32) for n in ("format", "out_dtype", "epilogue", "beta", "device")])


_lib = None


def _ptr(x):
    """As binding's, with fewer steps for tensors: a small call's arguments take as long as its launch."""
    return None if x is None else x if x.__class__ is int else x.data_ptr()


def _bytes(workspace, workspace_bytes):
    if workspace_bytes is not None:
        return workspace_bytes
    return 0 if workspace is None else workspace.nbytes


def lib():
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        for family, desc, sizes in (("pack", PackDesc, ("data_bytes", "scales_bytes", "workspace_bytes")), ("mx", MxDesc, ("workspace_bytes",))):
            create = getattr(L, f"nk_{family}_create")
            create.restype, create.argtypes = ctypes.c_int, [ctypes.POINTER(desc), ctypes.POINTER(vp)]
            for name, result in [(n, sz) for n in sizes] + [("check", ctypes.c_int), ("destroy", ctypes.c_int),
                                                            ("kernel_name", ctypes.c_char_p), ("last_cuda_error", ctypes.c_char_p)]:
                f = getattr(L, f"nk_{family}_{name}")
                f.restype, f.argtypes = result, [vp]
        for name, arguments in (("pack_scale", [vp] * 4 + [sz, vp]), ("pack_run", [vp] * 7), ("pack_values", [vp] * 7),
                                ("mx_run", [vp] * 11 + [sz, vp])):
            f = getattr(L, f"nk_{name}")
            f.restype, f.argtypes = ctypes.c_int, arguments
        _lib = L
    return _lib


def exported_symbols():
    L = lib()
    return [s for s in EXPORTS if hasattr(L, s)]


class _MxHandle(_Handle):
    def _create(self, desc):
        lib()
        super()._create(desc)


class PackPlan(_MxHandle):
    """nk_pack: matrices into 4-bit elements and block scales, along their rows or (transposed) their columns."""
    family = "pack"

    def __init__(self, rows, K, format=NVF4, in_dtype=BF16, value_dtype=F32, batch=1, groups=0, transposed=0, device=0, ldx=0,
                 stride_x=0):
        self._create(PackDesc(rows, K, batch, groups, ldx, stride_x, format, in_dtype, value_dtype, transposed, device))

    @property
    def data_bytes(self) -> int:
        return _lib.nk_pack_data_bytes(self._raw)

    @property
    def scales_bytes(self) -> int:
        return _lib.nk_pack_scales_bytes(self._raw)

    def tensor_scale(self, X, scale, workspace=None, workspace_bytes=None, stream=None):
        """scale: device FP32 [batch], written (nk_pack_scale)."""
        status = _lib.nk_pack_scale(self._raw, _ptr(X), _ptr(scale), _ptr(workspace), _bytes(workspace, workspace_bytes), stream)
        if status:
            self._check(status)

    def run(self, X, data, scales, scale=None, offsets=None, stream=None):
        status = _lib.nk_pack_run(self._raw, _ptr(X), _ptr(scale), _ptr(offsets), _ptr(data), _ptr(scales), stream)
        if status:
            self._check(status)

    def values(self, data, scales, Y, scale=None, offsets=None, stream=None):
        """What the packed arrays stand for."""
        status = _lib.nk_pack_values(self._raw, _ptr(data), _ptr(scales), _ptr(scale), _ptr(offsets), _ptr(Y), stream)
        if status:
            self._check(status)


class MxPlan(_MxHandle):
    """nk_mx: products of packed operands, of all rows with one weight (groups = 0) or grouped by expert."""
    family = "mx"

    def __init__(self, rows, N, K, groups=0, format=NVF4, out_dtype=F32, epilogue=EPI_NONE, beta=0, device=0, ldc=0):
        self._create(MxDesc(rows, N, K, groups, ldc, format, out_dtype, epilogue, beta, device))

    def run(self, A, A_scales, B, B_scales, C, scale_a=None, scale_b=None, bias=None, offsets=None, workspace=None,
            workspace_bytes=None, stream=None):
        """scale_a, scale_b: the operands' tensor scales (device FP32; scale_b and bias by group)."""
        status = _lib.nk_mx_run(self._raw, _ptr(A), _ptr(A_scales), _ptr(B), _ptr(B_scales), _ptr(scale_a), _ptr(scale_b), _ptr(bias),
                                 _ptr(offsets), _ptr(C), _ptr(workspace), _bytes(workspace, workspace_bytes), stream)
        if status:
            self._check(status)
