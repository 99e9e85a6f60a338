"""nk_mx on the GPU against the formats' definitions and a product in 64 bits.

Tolerance, for an element c = alpha sum_k a_k b_k with S = |alpha| sum_k |a_k b_k|: products are exact; the tensor core adds 64 of them to an FP32
accumulator with bits of the smaller terms dropped, 2^-22 of the sum's size at most a step; sums of accumulators, the scales' product
and the epilogue round to nearest, a few 2^-24.  steps of 64: at most 128 for an FP32 result, 256 for a 16-bit one.  Then half a step of the
result's type.
"""
import numpy as np
import pytest
import torch

import paper_2511_13764_b200 as nk
from mx_testlib import groups_width, one_groups_tiles, quantise, tensor_scale, values

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
    steps = min(-(-K // 64), 128 if out == "f32" else 256)
    rel = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[out]
    return (steps * 2.0 ** -22 + (K // 8192 + 4) * 2.0 ** -24) * S + rel * y.abs() + (2.0 ** -25 if out == "f16" else 0.0)


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


GROUPS = [[0, 5], [0, 0, 130, 130, 131, 300, 300], [7, 20, 20, 290], [0, 0], [128, 256, 300], [0, 64, 129, 193, 300], list(range(0, 301, 4)) + [300]]


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("offsets", GROUPS)
@pytest.mark.parametrize("N,K,out", [(264, 136, "f32"), (136, 520, "bf16"), (8, 72, "f16"), (520, 64, "bf16")])
def test_grouped(fmt, offsets, N, K, out):
    rows, groups = 300, len(offsets) - 1
    A = Packed(normal(rows, K, seed=K), fmt, offsets=offsets)
    B = Packed(normal(groups, N, K, seed=N, scale=0.1), fmt)
    got = run(A, B, N, K, fmt, out, groups=groups, offsets=A.offsets)
    seen = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        y = A.values[lo:hi] @ B.values[g].t()
        assert ((got[lo:hi] - y).abs() <= bound(A.values[lo:hi], B.values[g], K, out, y)).all(), g
        seen[lo:hi] = True
    assert (got[~seen] == 7.0).all(), "rows outside all groups are not touched"


@pytest.mark.parametrize("sizes", [[1000, 3, 0, 400, 65, 130], [2000, 1], [1, 1, 1, 700]])
def test_grouped_tiles_of_every_width(sizes):
    """Groups of several tiles: cut evenly in steps of 64, scales that begin inside 128 rows."""
    offsets = [0]
    for n in sizes:
        offsets.append(offsets[-1] + n)
    rows, N, K = offsets[-1], 776, 264
    A, B = Packed(normal(rows, K, seed=1), "nvf4", offsets=offsets), Packed(normal(len(sizes), N, K, seed=2), "nvf4")
    got = run(A, B, N, K, "nvf4", "f32", groups=len(sizes), offsets=A.offsets)
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        y = A.values[lo:hi] @ B.values[g].t()
        assert ((got[lo:hi] - y).abs() <= bound(A.values[lo:hi], B.values[g], K, "f32", y)).all(), g


@pytest.mark.parametrize("offsets", [[0, 200, 100, 300], [-5, 100, 200, 300], [0, 100, 400, 500]])
def test_bad_offsets_are_clamped_and_reported(offsets):
    top, clamped = 0, []
    for o in offsets:
        top = max(top, min(o, 300))
        clamped.append(top)
    A, B = Packed(normal(300, 64, seed=1), "mxf4", offsets=clamped), Packed(normal(3, 64, 64, seed=2), "mxf4")
    plan = nk.MxPlan(300, 64, 64, groups=3, format=nk.MXF4)
    C = torch.full((300, 64), 7.0, device="cuda")
    plan.run(A.data, A.scales, B.data, B.scales, C, offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"), stream=stream())
    with pytest.raises(nk.NkError) as e:
        plan.check()
    assert e.value.status == 1
    plan.check()
    for g, (lo, hi) in enumerate(zip(clamped, clamped[1:])):
        y = A.values[lo:hi] @ B.values[g].t()
        assert ((C[lo:hi].double() - y).abs() <= bound(A.values[lo:hi], B.values[g], 64, "f32", y)).all()


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,N,K,groups", [(50, 136, 200, 0), (300, 264, 1032, 0), (300, 264, 136, 3)])
@pytest.mark.parametrize("relu,bias,beta", [(True, True, 0), (True, False, 0), (False, False, 1), (True, True, 1)])
def test_epilogues(out, rows, N, K, groups, relu, bias, beta):
    offsets = [0, 100, 100, 300] if groups else None
    A = Packed(normal(rows, K, seed=3), "nvf4", offsets=offsets)
    B = Packed(normal(*((groups, N, K) if groups else (N, K)), seed=4, scale=0.1), "nvf4")
    b = normal(*((groups, N) if groups else (N,)), seed=5, kind="f32").cuda() if bias else None
    old = normal(rows, N, seed=6, kind=out).cuda() if beta else None
    got = run(A, B, N, K, "nvf4", out, groups=groups, bias=b, relu=relu, beta=beta, c=old, ldc=N + 16, offsets=A.offsets)
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:]) if groups else [(0, rows)]):
        v = B.values[g] if groups else B.values
        y = A.values[lo:hi] @ v.t()
        tol = bound(A.values[lo:hi], v, K, out, torch.zeros_like(y))
        if bias:
            y = y + (b[g] if groups else b).double()
        if beta:
            y = y + old[lo:hi].double()
        # (the additions round to nearest: 2^-23 of what is added)
        more = 2.0 ** -23 * (2.0 * y.abs() + (b.abs().max() if bias else 0.0) + (old[lo:hi].double().abs() if beta else 0.0))
        y = torch.relu(y) if relu else y
        rel = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[out]
        assert ((got[lo:hi] - y).abs() <= tol + more + rel * y.abs()).all()


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("rows,N,K", [(33, 264, 136), (333, 520, 776), (1000, 64, 264)])
def test_gradients_of_a_layer(fmt, rows, N, K):
    """dX = dY . W and dW = dY^T . X from operands packed along their columns; the length of dW's contraction is any number."""
    x, w, dy = normal(rows, K, seed=1), normal(N, K, seed=2, scale=0.1), normal(rows, N, seed=3)
    a, b = Packed(dy, fmt), Packed(w, fmt, transposed=1)
    got = run(a, b, K, N, fmt, "f32")
    y = a.values @ b.values.t()
    assert ((got - y).abs() <= bound(a.values, b.values, N, "f32", y)).all()
    a, b = Packed(dy, fmt, transposed=1), Packed(x, fmt, transposed=1)
    got = run(a, b, K, rows, fmt, "f32")
    y = a.values @ b.values.t()
    assert ((got - y).abs() <= bound(a.values, b.values, rows, "f32", y)).all()
    # against differences: <dY, X . W^T> changes along W by <dW, V>, as the products of the packed operands themselves do (they are linear)
    xt, dyt = b.values.t(), a.values.t()
    v = normal(N, K, seed=9).double().cuda()
    h = 0.5

    def loss(m):
        return (dyt * (xt @ m.t())).sum()
    slope = (loss(w.double().cuda() + h * v) - loss(w.double().cuda() - h * v)) / (2 * h)
    assert abs((got * v).sum() - slope) <= (bound(a.values, b.values, rows, "f32", y) * v.abs()).sum() + 1e-9 * slope.abs()


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("out,K", [("f32", 65536), ("f32", 2304), ("f32", 8448), ("bf16", 40000), ("f16", 20000)])
@pytest.mark.parametrize("rows", [16, 300])
def test_long_sums_of_one_sign(fmt, out, K, rows):
    """The error of an accumulator goes one way: sums over it are taken in FP32."""
    A, B = Packed(normal(rows, K, seed=1).abs(), fmt), Packed(normal(264, K, seed=2, scale=1.0 / K).abs(), fmt)
    got = run(A, B, 264, K, fmt, out)
    y = A.values @ B.values.t()
    assert ((got - y).abs() <= bound(A.values, B.values, K, out, y)).all()
    if out == "f32":
        assert ((got - y) / y).abs().max() <= 2.0 ** -20


@pytest.mark.parametrize("rows,N,K", [(16, 256, 16384), (1, 8, 8192), (64, 1024, 16384), (40, 264, 10000), (300, 256, 33000)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_cut_tiles(rows, N, K, out):
    """Few tiles and a long contraction: cut along it.  The same bits every time, and the counters are zero again."""
    A, B = Packed(normal(rows, K, seed=1), "nvf4"), Packed(normal(N, K, seed=2, scale=0.1), "nvf4")
    plan = nk.MxPlan(rows, N, K, out_dtype=TYPES[out][0])
    assert plan.workspace_bytes > 0
    ws = torch.full((plan.workspace_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
    results = []
    for _ in range(20):
        C = torch.empty(rows, N, dtype=TYPES[out][1], device="cuda")
        plan.run(A.data, A.scales, B.data, B.scales, C, scale_a=A.scale, scale_b=B.scale, workspace=ws, stream=stream())
        results.append(C)
    plan.check()
    assert all(torch.equal(results[0], r) for r in results)
    y = A.values @ B.values.t()
    assert ((results[0].double() - y).abs() <= bound(A.values, B.values, K, out, y)).all()
    with pytest.raises(nk.NkError) as e:
        plan.run(A.data, A.scales, B.data, B.scales, C, scale_a=A.scale, scale_b=B.scale, workspace=ws[:-16], stream=stream())
    assert e.value.status == 4


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_what_is_not_finite_stays_in_its_row_and_feature(fmt):
    rows, N, K, offsets = 200, 264, 200, [0, 90, 200]
    x, w = normal(rows, K, seed=1), normal(2, N, K, seed=2)
    A0, B0 = Packed(x, fmt, offsets=offsets), Packed(w, fmt)
    clean = run(A0, B0, N, K, fmt, "f32", groups=2, offsets=A0.offsets)
    scale_a, scale_b = A0.scale, B0.scale
    x[77, 13], w[1, 100, 7] = float("nan"), float("inf")
    for P, m, s in ((A0, x, scale_a), (B0, w, scale_b)):    # the same tensor scales, so that all else stays as it is
        P.plan.run(m.cuda(), P.data, P.scales, scale=s, offsets=P.offsets, stream=stream())
    got = run(A0, B0, N, K, fmt, "f32", groups=2, offsets=A0.offsets)
    hit = torch.zeros(rows, N, dtype=torch.bool, device="cuda")
    hit[77] = True
    hit[90:, 100] = True
    assert got[hit].isnan().all() and torch.equal(got[~hit], clean[~hit])


def test_rows_behind_the_last_and_scales_nobody_wrote():
    """Scales and data of rows that are not there may hold anything, NaN patterns among them."""
    A, B = Packed(normal(130, 72, seed=1), "nvf4"), Packed(normal(136, 72, seed=2), "nvf4")
    y = A.values @ B.values.t()
    # rows 130 .. 255 of A's tiles, 136 .. 255 of B's
    for P, n in ((A, 130), (B, 136)):
        t = P.scales.view(-1, 32, 4, 4)                      # 512-byte tiles: r % 32, r / 32, c
        C = t.shape[0] // 2
        r = torch.arange(n - 128, 128, device="cuda")
        for c in range(C):
            t[C + c, r % 32, r // 32, :] = 0x7F
    got = run(A, B, 136, 72, "nvf4", "f32")
    assert ((got - y).abs() <= bound(A.values, B.values, 72, "f32", y)).all()


def test_tensor_scales_that_are_left_out():
    x, w = normal(40, 128, seed=1), normal(64, 128, seed=2)
    out = []
    for s in (None, 0.25):
        P = []
        for m in (x, w):
            p = Packed(m, "nvf4")
            p.scale = None if s is None else torch.tensor([s], device="cuda")
            p.plan.run(m.cuda(), p.data, p.scales, scale=p.scale, stream=stream())
            codes, bytes_, _ = quantise(m.double().numpy(), "nvf4", 1.0 if s is None else s)
            p.values = torch.from_numpy(values(codes, bytes_, "nvf4", 1.0 if s is None else s, 128)).cuda()
            P.append(p)
        got = run(*P, 64, 128, "nvf4", "f32")
        y = P[0].values @ P[1].values.t()
        assert ((got - y).abs() <= bound(P[0].values, P[1].values, 128, "f32", y)).all()
        out.append(got)


def test_streams_graphs_and_plans_destroyed_early():
    A, B = Packed(normal(300, 512, seed=1), "nvf4"), Packed(normal(520, 512, seed=2), "nvf4")
    want = run(A, B, 520, 512, "nvf4", "bf16")
    # two plans at once on two streams, destroyed with work queued
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    results = []
    torch.cuda.synchronize()
    for s in (a, b) * 4:
        plan = nk.MxPlan(300, 520, 512, out_dtype=nk.BF16)
        C = torch.zeros(300, 520, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(max(1, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for _ in range(10):
            plan.run(A.data, A.scales, B.data, B.scales, C, scale_a=A.scale, scale_b=B.scale, workspace=ws, stream=s.cuda_stream)
        plan.destroy()
        results.append((C, ws))
    torch.cuda.synchronize()
    assert all(torch.equal(C.double(), want) for C, _ in results)
    # a cut plan in a graph, replayed on other inputs
    A, B = Packed(normal(20, 16384, seed=1), "mxf4"), Packed(normal(264, 16384, seed=2), "mxf4")
    plan = nk.MxPlan(20, 264, 16384, format=nk.MXF4)
    C, ws = torch.empty(20, 264, device="cuda"), torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            plan.run(A.data, A.scales, B.data, B.scales, C, workspace=ws, stream=stream())
    plan.destroy()
    for seed in (5, 6):
        other = Packed(normal(20, 16384, seed=seed), "mxf4")
        A.data.copy_(other.data)
        A.scales.copy_(other.scales)
        graph.replay()
        torch.cuda.synchronize()
        y = other.values @ B.values.t()
        assert ((C.double() - y).abs() <= bound(other.values, B.values, 16384, "f32", y)).all()


def test_cut_plans_at_once_and_without_counters():
    """Cut plans on two streams beside each other; a plan that finds no counters left cuts nothing."""
    A, B = Packed(normal(16, 16384, seed=1), "nvf4"), Packed(normal(256, 16384, seed=2), "nvf4")
    y = A.values @ B.values.t()
    tol = bound(A.values, B.values, 16384, "f32", y)
    plans = [nk.MxPlan(16, 256, 16384) for _ in range(1040)]
    names = [p.kernel_name for p in plans]
    assert not names[0].endswith("_uncut") and names[-1].endswith("_uncut") and plans[-1].workspace_bytes == 0
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    work = []
    torch.cuda.synchronize()
    for i, p in enumerate((plans[0], plans[1], plans[-1])):
        C, ws = torch.empty(16, 256, device="cuda"), torch.empty(max(1, p.workspace_bytes), dtype=torch.uint8, device="cuda")
        work.append((C, ws))
    torch.cuda.synchronize()
    for _ in range(30):
        for i, p in enumerate((plans[0], plans[1], plans[-1])):
            p.run(A.data, A.scales, B.data, B.scales, work[i][0], scale_a=A.scale, scale_b=B.scale, workspace=work[i][1], stream=side[i % 2].cuda_stream)
    torch.cuda.synchronize()
    for p in plans:
        p.destroy()
    assert torch.equal(work[0][0], work[1][0])
    assert all(((C.double() - y).abs() <= tol).all() for C, _ in work)


def test_results_beyond_32_bits():
    """More than 2^31 elements of C, and a group whose rows begin there."""
    rows, N, K, first = 70016, 32768, 64, 69950
    A, B = Packed(normal(rows, K, seed=1), "mxf4", offsets=[0, first, rows]), Packed(normal(2, N, K, seed=2), "mxf4")
    plan = nk.MxPlan(rows, N, K, groups=2, format=nk.MXF4, out_dtype=nk.BF16)
    C = torch.empty(rows, N, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(1, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
    plan.run(A.data, A.scales, B.data, B.scales, C, offsets=A.offsets, workspace=ws, stream=stream())
    plan.check()
    for r in (0, 1, 65535, 65536, first - 1, first, rows - 1):
        a, b = A.values[r:r + 1], B.values[int(r >= first)]
        y = a @ b.t()
        assert ((C[r:r + 1].double() - y).abs() <= bound(a, b, K, "bf16", y)).all(), r


def test_no_rows_and_refusals():
    plan = nk.MxPlan(0, 64, 64)
    plan.run(None, None, None, None, None, stream=stream())
    plan.check()
    for status, args in ((1, dict(rows=-1)), (1, dict(N=0)), (1, dict(K=0)), (3, dict(N=12)), (3, dict(ldc=68)), (1, dict(ldc=56)), (1, dict(format=2)),
                         (2, dict(out_dtype=nk.S32)), (1, dict(epilogue=2)), (1, dict(beta=2)), (1, dict(groups=-1)), (2, dict(groups=2000)),
                         (5, dict(device=99)), (2, dict(rows=(1 << 31) - 10))):
        with pytest.raises(nk.NkError) as e:
            nk.MxPlan(**{**dict(rows=32, N=64, K=64), **args})
        assert e.value.status == status, args
    A, B = Packed(normal(32, 64, seed=1), "nvf4"), Packed(normal(64, 64, seed=2), "nvf4")
    C, off, bias = torch.empty(32, 64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(64, device="cuda")
    plan, grouped, mx = nk.MxPlan(32, 64, 64), nk.MxPlan(32, 64, 64, groups=1), nk.MxPlan(32, 64, 64, format=nk.MXF4)
    for status, call in ((1, lambda: plan.run(None, A.scales, B.data, B.scales, C)), (1, lambda: plan.run(A.data, A.scales, B.data, None, C)),
                         (1, lambda: plan.run(A.data, A.scales, B.data, B.scales, None)), (1, lambda: plan.run(A.data, A.scales, B.data, B.scales, C, offsets=off)),
                         (1, lambda: grouped.run(A.data, A.scales, B.data, B.scales, C)), (1, lambda: plan.run(A.data, A.scales, B.data, B.scales, C, bias=bias)),
                         (1, lambda: mx.run(A.data, A.scales, B.data, B.scales, C, scale_a=A.scale)), (3, lambda: plan.run(A.data[8:], A.scales, B.data, B.scales, C)),
                         (3, lambda: plan.run(A.data, A.scales, B.data, B.scales, C.data_ptr() + 4))):
        with pytest.raises(nk.NkError) as e:
            call()
        assert e.value.status == status


LARGEST = torch.finfo(torch.float32).max


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("groups", [0, 3])
@pytest.mark.parametrize("relu", [False, True])
def test_tensor_scales_whose_product_is_beyond_the_range(out, groups, relu):
    """Each operand's scale is in range, their product is not: rows of zeros stay zeros, results that fit come out.  (A step more for the second
    scale's rounding, 2^-24, which the bound's four hold.)"""
    rows, N, K = 300, 264, 136
    offsets = [0, 100, 100, 300] if groups else None
    x, w = normal(rows, K, seed=1, scale=2.0 ** 74), normal(*((groups, N, K) if groups else (N, K)), seed=2, scale=2.0 ** 74)
    x[0::3] *= 2.0 ** -14
    x[1::3] = 0.0
    x[2] = 2.0 ** 40                                        # every block rounds to zero
    w[..., 0::2, :] *= 2.0 ** -14
    w[..., 5, :] = 0.0
    if groups:
        w[0] *= 2.0 ** -80                                  # one group's scale is ordinary beside the others'
    A, B = Packed(x, "nvf4", offsets=offsets), Packed(w, "nvf4")
    assert torch.isinf(A.scale * B.scale).any() and torch.isfinite(A.scale).all() and torch.isfinite(B.scale).all()
    bias = normal(*((groups, N) if groups else (N,)), seed=5, kind="f32").cuda() * 2.0 ** 100 if relu else None
    got = run(A, B, N, K, "nvf4", out, groups=groups, relu=relu, bias=bias, offsets=A.offsets)
    small = 0
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:]) if groups else [(0, rows)]):
        a, b = A.values[lo:hi], B.values[g] if groups else B.values
        plain = a @ b.t()
        y = plain + (bias[g] if groups else bias).double() if relu else plain
        tol = bound(a, b, K, out, y) + (2.0 ** -23 * (y.abs() + 2.0 ** 103) if relu else 0.0)
        y = torch.relu(y) if relu else y
        fits, over = y.abs() + tol <= LARGEST * (1 - 2.0 ** -8), y.abs() - tol > LARGEST * (1 + 2.0 ** -8)
        assert ((got[lo:hi] - y).abs() <= tol)[fits].all(), g
        assert torch.equal(got[lo:hi][over], torch.sign(y[over]) * torch.inf), g
        if not relu:
            assert (got[lo:hi][plain == 0] == 0).all(), g
        small += int((fits & (plain != 0)).sum())
    assert small > 1000


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("groups", [0, 2])
@pytest.mark.parametrize("ea,eb", [(-75, -75), (-74, -73), (-47, -100), (-98, -49)])
def test_tensor_scales_whose_product_is_below_the_range(out, groups, ea, eb):
    """A caller's small scales: their product is zero or has lost bits, the results have not.  (2^-149 and 2^-134: the types' smallest steps.)"""
    ta, tb = 169 * 2.0 ** (ea - 7), 203 * 2.0 ** (eb - 7)
    rows, N, K = 200, 264, 4096
    offsets = [0, 90, 200] if groups else None
    A = Packed(normal(rows, K, seed=1), "nvf4", offsets=offsets)
    B = Packed(normal(*((groups, N, K) if groups else (N, K)), seed=2), "nvf4")
    for P, seed, t in ((A, 3, ta), (B, 4, tb)):
        shape = (rows, K) if P is A else (groups, N, K) if groups else (N, K)
        m = (normal(*shape, seed=seed).clamp(-3, 3).double() * 800 * t).to(torch.bfloat16)
        P.scale = torch.full((groups if P is B and groups else 1,), t, dtype=torch.float32, device="cuda")
        P.plan.run(m.cuda(), P.data, P.scales, scale=P.scale, offsets=P.offsets, stream=stream())
        z = m.double().numpy().reshape(-1, K)
        codes, bytes_, _ = quantise(z, "nvf4", t)
        P.values = torch.from_numpy(values(codes, bytes_, "nvf4", t, K)).cuda().reshape(shape)
    got = run(A, B, N, K, "nvf4", out, groups=groups, offsets=A.offsets)
    least = 2.0 ** -149 if out == "f32" else 2.0 ** -134
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:]) if groups else [(0, rows)]):
        a, b = A.values[lo:hi], B.values[g] if groups else B.values
        y = a @ b.t()
        assert ((got[lo:hi] - y).abs() <= bound(a, b, K, out, y) + least).all(), g
        assert (y.abs() > 2.0 ** -126).any()


class OnDevice:
    """A matrix (or a batch) made and packed on the GPU; its values are read back (both compared with the definitions in test_gpu_pack.py)."""

    def __init__(self, *shape, fmt="nvf4", seed=0, offsets=None, change=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn(*shape, generator=g, device="cuda")
        x = (x if change is None else change(x)).to(torch.bfloat16)
        batch, rows, K = shape if len(shape) == 3 else (1, *shape)
        groups = 0 if offsets is None else len(offsets) - 1
        plan = nk.PackPlan(rows, K, format=FORMATS[fmt], batch=batch, groups=groups)
        self.data = torch.empty(plan.data_bytes, dtype=torch.uint8, device="cuda")
        self.scales = torch.full((plan.scales_bytes,), 0xFF, dtype=torch.uint8, device="cuda")
        self.offsets = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
        self.scale = None
        if fmt == "nvf4":
            self.scale, ws = torch.empty(batch, device="cuda"), torch.empty(max(1, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
            plan.tensor_scale(x, self.scale, workspace=ws, stream=stream())
        plan.run(x, self.data, self.scales, scale=self.scale, offsets=self.offsets, stream=stream())
        y = torch.zeros(*shape, device="cuda")
        plan.values(self.data, self.scales, y, scale=self.scale, offsets=self.offsets, stream=stream())
        plan.check()
        self.values = y.double()


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("rows,N,K", [(16, 256, 16384), (300, 256, 33000), (1300, 1096, 264), (2000, 2056, 8448), (5537, 1712, 9216)])
def test_scales_of_any_size_in_tiles_of_every_kind(out, rows, N, K):
    """Cut tiles, sums of accumulators, wide tiles: other scales of the same packed operands, powers of two apart, give the same numbers that power of two
    apart, but for a second rounding of the scales' product and what the type's smallest step takes.  (Where `want` has been rounded to 16 bits, too:
    2^-23 apart, two numbers on either side of the middle of a step go to its two ends, which are 2^-7 of the smaller apart, two half steps.)"""
    A, B = OnDevice(rows, K, seed=1, change=lambda x: x * (torch.arange(rows, device="cuda") % 5 > 0)[:, None]), OnDevice(N, K, seed=2)
    plain = run(A, B, N, K, "nvf4", "f32", rows=rows)
    ta, tb = A.scale, B.scale
    rel, least = {"f32": (2.0 ** -22, 2.0 ** -149), "bf16": (2.0 ** -8 + 2.0 ** -20, 2.0 ** -134)}[out]
    for a, b in ((-64, -64), (-12, -88), (80, 80), (100, 40)):
        A.scale, B.scale = ta * 2.0 ** a, tb * 2.0 ** b
        if K < 8192 or out == "f32":
            want = plain * 2.0 ** (a + b)
        else:                                               # (16-bit sums have longer accumulators: another order)
            A.scale, B.scale = ta, tb
            want = run(A, B, N, K, "nvf4", "bf16", rows=rows) * 2.0 ** (a + b)
            A.scale, B.scale = ta * 2.0 ** a, tb * 2.0 ** b
            rel = 2 * 2.0 ** -8 + 2.0 ** -20
        got = run(A, B, N, K, "nvf4", out, rows=rows)
        over = want.abs() > LARGEST
        assert torch.equal(got[over], torch.sign(want[over]) * torch.inf)
        rest = ~over & (want.abs() < LARGEST * (1 - 2.0 ** -7))
        assert ((got - want).abs() <= rel * want.abs() + least)[rest].all(), (a, b)
        assert (got[::5] == 0).all()


def pairs_of_sms():
    return torch.cuda.get_device_properties(0).multi_processor_count // 2


def compare_whole(A, B, rows, N, K, fmt, out, more=False):
    """The whole of C with the product in 64 bits; `more`: bias, ReLU and beta, rows further apart than they are long."""
    bias = old = None
    if more:
        g = torch.Generator(device="cuda").manual_seed(7)
        bias, old = torch.randn(N, generator=g, device="cuda"), torch.randn(rows, N, generator=g, device="cuda").to(TYPES[out][1])
    got = run(A, B, N, K, fmt, out, rows=rows, bias=bias, relu=more, beta=int(more), c=old, ldc=N + 8 if more else 0)
    y = A.values @ B.values.t()
    tol = bound(A.values, B.values, K, out, torch.zeros_like(y))
    if more:
        # (two additions that round to nearest: 2^-23 of what is added)
        tol += 2.0 ** -23 * (y.abs() + bias.double().abs() + old.double().abs())
        y = torch.relu(y + bias.double() + old.double())
    tol += {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[out] * y.abs()
    bad = ~((got - y).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, first {bad.nonzero()[:4].tolist()}, got {got[bad][:4].tolist()}, want {y[bad][:4].tolist()}"


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("out,more", [("f32", False), ("bf16", False), ("f16", False), ("f32", True), ("bf16", True)])
@pytest.mark.parametrize("rows,N,K,width", [(4096, 4096, 520, 256), (4096, 4096, 2056, 256), (3500, 4104, 264, 256), (2100, 2568, 776, 192), (2500, 2056, 520, 192),
                                            (1300, 4104, 520, 192), (1300, 2488, 208, 192), (1600, 2568, 264, 128)])
def test_wide_tiles(fmt, out, more, rows, N, K, width):
    """Tiles of every width, several of them to most pairs: accumulators that share columns follow each other, rows' scales begin in the middle of 128."""
    assert one_groups_tiles(rows, N, K, pairs_of_sms()) == (width, 1), "this size no longer takes the tiles that it is here for"
    compare_whole(OnDevice(rows, K, fmt=fmt, seed=rows), OnDevice(N, K, fmt=fmt, seed=N), rows, N, K, fmt, out, more)


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("out,more,rows,N,K,width,parts", [
    ("f32", False, 2000, 2056, 8448, 256, 1), ("f32", False, 2560, 4096, 8448, 256, 1), ("f32", True, 2500, 4096, 8704, 256, 1), ("bf16", False, 2560, 4096, 16640, 256, 3),
    ("f16", False, 2000, 2056, 16640, 256, 1), ("f16", False, 2600, 2568, 16640, 256, 1), ("bf16", True, 2900, 2056, 16640, 192, 1), ("f32", False, 1000, 2056, 8448, 128, 1), ("f32", False, 3000, 1544, 8448, 192, 1), ("bf16", True, 3000, 1544, 16640, 256, 3),
    # cut, too; 16-bit results of one accumulator or of two
    ("f32", False, 3848, 1248, 15016, 256, 4), ("f32", False, 5537, 1712, 9216, 256, 3), ("bf16", False, 3848, 1248, 15016, 256, 4), ("f16", True, 5537, 1712, 9216, 256, 3)])
def test_sums_and_cuts_of_wide_tiles(fmt, out, more, rows, N, K, width, parts):
    assert one_groups_tiles(rows, N, K, pairs_of_sms()) == (width, parts), "this size no longer takes the tiles that it is here for"
    compare_whole(OnDevice(rows, K, fmt=fmt, seed=rows), OnDevice(N, K, fmt=fmt, seed=N), rows, N, K, fmt, out, more)


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("K", [264, 1032])
@pytest.mark.parametrize("sizes,width", [([1300, 1300], 192), ([1500, 3, 700, 900], 256), ([2500, 2500, 3, 0, 1500], 256), ([200, 190, 180, 0, 170], 128), ([60, 64, 1], 64), ([20, 0, 32], 32)])
def test_grouped_tiles_of_each_width(fmt, out, K, sizes, width):
    N, offsets = 2056, [0]
    for n in sizes:
        offsets.append(offsets[-1] + n)
    assert groups_width(sizes, N, K, pairs_of_sms()) == width, "these loads no longer take the tiles that they are here for"
    rows, G = offsets[-1], len(sizes)
    A, B = OnDevice(rows, K, fmt=fmt, seed=1, offsets=offsets), OnDevice(G, N, K, fmt=fmt, seed=2)
    got = run(A, B, N, K, fmt, out, groups=G, offsets=A.offsets, rows=rows)
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        y = A.values[lo:hi] @ B.values[g].t()
        assert ((got[lo:hi] - y).abs() <= bound(A.values[lo:hi], B.values[g], K, out, y)).all(), g


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("rows", [64, 512])
@pytest.mark.parametrize("K", [4096, 8192, 65536])
@pytest.mark.parametrize("kind", ["normal", "one sign", "spread"])
def test_error_of_fp32_results(fmt, rows, K, kind):
    """The errors that nk_mx.h states (2-norm: 2.5e-8, 1e-7, 1.2e-6), within twice.  Spread: blocks that differ by ten powers of two."""
    def change(x):
        if kind == "one sign":
            return x.abs()
        if kind == "spread":
            e = torch.randint(-5, 6, (x.shape[0], K // 32), generator=torch.Generator().manual_seed(x.shape[0])).cuda()
            return x * (2.0 ** e).repeat_interleave(32, 1)
        return x
    A, B = OnDevice(rows, K, fmt=fmt, seed=1, change=change), OnDevice(520, K, fmt=fmt, seed=2, change=change)
    got = run(A, B, 520, K, fmt, "f32", rows=rows)
    y = A.values @ B.values.t()
    error = float((got - y).norm() / y.norm())
    assert error <= 2 * {"normal": 2.5e-8, "one sign": 1e-7, "spread": 1.2e-6}[kind], error
