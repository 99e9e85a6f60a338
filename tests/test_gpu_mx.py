"""nk_mx on the GPU against the formats' definitions and a product in 64 bits.

Tolerance, for an element c = alpha sum_k a_k b_k with S = |alpha| sum_k |a_k b_k|: products are exact; the tensor core adds 64 of them to an FP32
accumulator with bits of the smaller terms dropped, 2^-22 of the sum's size at most a step; sums of accumulators, the scales' product
and the epilogue round to nearest, a few 2^-24.  steps of 64: at most 32 for an FP32 result, 256 for a 16-bit one.  Then half a step of the
result's type.
"""
import numpy as np
import pytest
import torch

import paper_2511_13764_b200 as nk
from mx_testlib import quantise, tensor_scale, values

pytestmark = pytest.mark.gpu

FORMATS = {"mxf4": nk.MXF4, "nvf4": nk.NVF4}
TYPES = {"f32": (nk.F32, torch.float32), "bf16": (nk.BF16, torch.bfloat16), "f16": (nk.F16, torch.float16)}


def stream():
    return torch.cuda.current_stream().cuda_stream


def normal(*shape, seed=0, scale=1.0, kind="bf16"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(TYPES[kind][1])


class Packed:
    """A matrix (or a batch of them) packed on the GPU, and what it stands for in 64 bits."""

    def __init__(self, x, fmt, transposed=0, offsets=None, kind="bf16"):
        batch, rows, K = x.shape if x.dim() == 3 else (1, *x.shape)
        groups = 0 if offsets is None else len(offsets) - 1
        self.plan = nk.PackPlan(rows, K, format=FORMATS[fmt], in_dtype=TYPES[kind][0], batch=batch, groups=groups, transposed=transposed)
        self.data = torch.empty(self.plan.data_bytes, dtype=torch.uint8, device="cuda")
        self.scales = torch.full((self.plan.scales_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
        self.scale, ts = None, [1.0] * batch
        z = x.double().numpy().reshape(batch, rows, K)
        if fmt == "nvf4":
            ts = [tensor_scale(m) for m in z]
            self.scale = torch.tensor(ts, dtype=torch.float32, device="cuda")
        self.offsets = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
        self.plan.run(x.cuda(), self.data, self.scales, scale=self.scale, offsets=self.offsets, stream=stream())
        self.plan.check()
        out = []
        for m, t in zip(z, ts):
            m = m.T.copy() if transposed else m
            codes, bytes_, _ = quantise(m, fmt, t)
            out.append(values(codes, bytes_, fmt, t, m.shape[1]))
        self.values = torch.from_numpy(np.stack(out) if x.dim() == 3 else out[0]).cuda()


def bound(a, b, K, out, y):
    """What an element may be off by (see above); a, b: the values."""
    S = a.abs() @ b.abs().transpose(-1, -2)
    steps = min(-(-K // 64), 32 if out == "f32" else 256)
    rel = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[out]
    return (steps * 2.0 ** -22 + (K // 2048 + 4) * 2.0 ** -24) * S + rel * y.abs() + (2.0 ** -25 if out == "f16" else 0.0)


def run(A, B, N, K, fmt, out, groups=0, bias=None, relu=False, beta=0, c=None, ldc=0, offsets=None, rows=None):
    rows = A.values.shape[0] if rows is None else rows
    plan = nk.MxPlan(rows, N, K, groups=groups, format=FORMATS[fmt], out_dtype=TYPES[out][0], epilogue=nk.EPI_BIAS_RELU if relu else nk.EPI_NONE,
                     beta=beta, ldc=ldc)
    width = ldc or N
    C = torch.full((rows * width + 64,), 7.0, dtype=TYPES[out][1], device="cuda")
    if c is not None:
        C[:rows * width].view(rows, width)[:, :N] = c
    ws = torch.full((max(1, plan.workspace_bytes),), 0xFF, dtype=torch.uint8, device="cuda")
    plan.run(A.data, A.scales, B.data, B.scales, C, scale_a=A.scale, scale_b=B.scale, bias=bias, offsets=offsets, workspace=ws, stream=stream())
    plan.check()
    assert (C[rows * width:] == 7.0).all(), "written behind the end"
    C = C[:rows * width].view(rows, width)
    assert (C[:, N:] == 7.0).all()
    return C[:, :N].double()


def check(rows, N, K, fmt, out, **more):
    A, B = Packed(normal(rows, K, seed=rows + K), fmt), Packed(normal(N, K, seed=N, scale=0.1), fmt)
    got = run(A, B, N, K, fmt, out, **more)
    y = A.values @ B.values.t()
    tol = bound(A.values, B.values, K, out, y)
    bad = ~((got - y).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, first {bad.nonzero()[:4].tolist()}, got {got[bad][:4].tolist()}, want {y[bad][:4].tolist()}"


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("rows,N,K", [(32, 256, 256), (1, 8, 64), (1, 256, 8), (2, 40, 72), (16, 128, 512), (17, 136, 264), (33, 264, 1000), (64, 256, 256),
                                      (65, 520, 328), (100, 256, 4096), (128, 512, 256), (129, 256, 256), (160, 256, 512), (192, 256, 256),
                                      (200, 248, 776), (256, 256, 256), (257, 256, 2048), (300, 1000, 520), (1000, 776, 1032)])
def test_sizes(fmt, rows, N, K):
    check(rows, N, K, fmt, "f32")


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,N,K", [(5, 264, 640), (300, 264, 4360), (2000, 2056, 512), (4099, 1024, 2056)])
def test_results(fmt, out, rows, N, K):
    check(rows, N, K, fmt, out)
