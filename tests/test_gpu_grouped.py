"""Products grouped by expert (nk_grouped) against the formula in 64 bits: ragged and empty groups, every
operand layout and type, strides, accumulation, the gradients, and what the call refuses.

Tolerances are those of the dense GEMM's parity tests, for the same reasons: FP32 accumulation of exact
products, so |c - y| <= 1e-5 * max sum |a b|, plus half a unit in the last place of a 16-bit result."""
import numpy as np
import pytest
import torch

import paper_2511_13764_b200 as nk
from nk_testlib import TOL_BF16_REL, TOL_F16_ABS, TOL_F16_REL, TOL_REL_SMAX

TYPES = {"bf16": (nk.BF16, torch.bfloat16), "f16": (nk.F16, torch.float16), "f32": (nk.F32, torch.float32)}
SENTINEL = 7.0


def offsets_of(sizes, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(sizes)]), dtype=torch.int32)


def rand(shape, kind, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float32) * scale).to(TYPES[kind][1])


def padded(x, ld, fill=float("nan")):
    """x as a strided view of rows of ld elements; what lies between is `fill`."""
    if ld == x.shape[-1]:
        return x.cuda().contiguous()
    buf = torch.full((*x.shape[:-1], ld), fill, dtype=x.dtype)
    buf[..., :x.shape[-1]] = x
    return buf.cuda()


def close(got, want, size, kind):
    """size: the largest sum of |products| of any element."""
    want, got = want.cpu(), got.double().cpu()
    tol = TOL_REL_SMAX * size + {"bf16": TOL_BF16_REL, "f16": TOL_F16_REL, "f32": 0.0}[kind] * want.abs() + (TOL_F16_ABS if kind == "f16" else 0)
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: got {got[bad][0]} want {want[bad][0]}"


def scratch(plan):
    return torch.full((max(16, plan.workspace_bytes),), 255, dtype=torch.uint8, device="cuda")


def run_rows(sizes, N, K, kind="bf16", out="bf16", layout="row", first=0, spare=0, lda=0, ldb=0, ldc=0, gap=0, beta=0, seed=0, spoil=True):
    """One forward product; returns (C rows of the groups as float64, formula, sum of |products|)."""
    gen = torch.Generator().manual_seed(seed)
    G, rows = len(sizes), first + sum(sizes) + spare
    off = offsets_of(sizes, first)
    A = rand((rows, K), kind, gen)
    if spoil:                                    # rows of no group must not matter
        A[:first] = float("nan")
        A[first + sum(sizes):] = float("inf")
    W = rand((G, K, N), kind, gen, K ** -0.5)
    stored = W if layout == "row" else W.transpose(1, 2).contiguous()
    lda, ldb, ldc = lda or K, ldb or stored.shape[2], ldc or N
    stride = stored.shape[1] * ldb + gap
    wbuf = torch.full((G * stride,), float("nan"), dtype=W.dtype)
    for g in range(G):
        view = wbuf[g * stride: g * stride + stored.shape[1] * ldb].view(stored.shape[1], ldb)
        view[:, : stored.shape[2]] = stored[g]
    C = torch.full((rows, ldc), SENTINEL, dtype=TYPES[out][1])
    if beta:
        C[:, :N] = rand((rows, N), out, gen)
    before = C.clone()
    plan = nk.GroupedPlan(G, rows, N, K, in_dtype=TYPES[kind][0], out_dtype=TYPES[out][0], beta=beta,
                          layout_b=nk.ROW_MAJOR if layout == "row" else nk.TRANSPOSED, lda=lda, ldb=ldb, ldc=ldc, stride_g=stride)
    dC = C.cuda()
    dA, dW, dO = padded(A, lda), wbuf.cuda(), off.cuda()
    plan.run(dA, dW, dC, dO, workspace=scratch(plan), stream=torch.cuda.current_stream().cuda_stream)
    plan.check()
    got = dC.cpu()
    want = torch.zeros(rows, N, dtype=torch.float64)
    size = 1e-30
    for g in range(G):
        lo, hi = int(off[g]), int(off[g + 1])
        a, w = A[lo:hi].double().cuda(), W[g].double().cuda()
        want[lo:hi] = (a @ w).cpu()
        if hi > lo:
            size = max(size, float((a.abs() @ w.abs()).max()))
    lo, hi = first, first + sum(sizes)
    if beta:
        want[lo:hi] += before[lo:hi, :N].double()
        size += float(before[lo:hi, :N].double().abs().max()) if hi > lo else 0
    # nothing but the groups' rows and columns was written
    assert torch.equal(got[:lo].nan_to_num(3), before[:lo].nan_to_num(3)) and torch.equal(got[hi:], before[hi:])
    assert torch.equal(got[:, N:], before[:, N:])
    close(got[lo:hi, :N], want[lo:hi], size, out)
    return plan


def run_weights(sizes, N, K, kind="bf16", out="f32", first=0, spare=0, lda=0, ldb=0, ldc=0, gap=0, beta=0, seed=0, poison=None):
    gen = torch.Generator().manual_seed(seed)
    G, rows = len(sizes), first + sum(sizes) + spare
    off = offsets_of(sizes, first)
    A, B = rand((rows, K), kind, gen), rand((rows, N), kind, gen)
    for x in (A, B):
        x[:first] = float("nan")
        x[first + sum(sizes):] = float("inf")
    if poison is not None:                       # a whole group of NaN must stay in its own gradient
        A[off[poison]:off[poison + 1]] = float("nan")
        B[off[poison]:off[poison + 1]] = float("inf")
    lda, ldb, ldc = lda or K, ldb or N, ldc or N
    stride = K * ldc + gap
    C = torch.full((G * stride,), SENTINEL, dtype=TYPES[out][1])
    view = lambda t, g: t[g * stride: g * stride + K * ldc].view(K, ldc)   # noqa: E731
    if beta:
        for g in range(G):
            view(C, g)[:, :N] = rand((K, N), out, gen)
    before = C.clone()
    plan = nk.GroupedPlan(G, rows, N, K, kind=nk.GROUPED_WEIGHTS, in_dtype=TYPES[kind][0], out_dtype=TYPES[out][0], beta=beta,
                          lda=lda, ldb=ldb, ldc=ldc, stride_g=stride)
    dC = C.cuda()
    dA, dB, dO = padded(A, lda), padded(B, ldb), off.cuda()
    plan.run(dA, dB, dC, dO, workspace=scratch(plan), stream=torch.cuda.current_stream().cuda_stream)
    plan.check()
    got = dC.cpu()
    for g in range(G):
        lo, hi = int(off[g]), int(off[g + 1])
        c, old = view(got, g), view(before, g)
        assert torch.equal(c[:, N:], old[:, N:])
        assert torch.equal(got[g * stride + K * ldc:(g + 1) * stride], before[g * stride + K * ldc:(g + 1) * stride])
        if g == poison:
            assert c[:, :N].isnan().all() or hi == lo
            continue
        a, b = A[lo:hi].double().cuda(), B[lo:hi].double().cuda()
        want = (a.t() @ b).cpu()
        size = float((a.abs().t() @ b.abs()).max()) if hi > lo else 1e-30
        if beta:
            want = want + old[:, :N].double()
            size += float(old[:, :N].double().abs().max())
        close(c[:, :N], want, size, out)
    return plan


GROUPS = {
    "one_row": [1],
    "single_group": [300],
    "tile_edges": [255, 256, 257, 1, 0, 33],
    "empty_first_last": [0, 40, 0, 0, 17, 0],
    "all_empty": [0, 0, 0],
    "many_small": [(i * 7) % 5 for i in range(97)],
    "one_takes_all": [0] * 9 + [700] + [0] * 6,
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(GROUPS))
@pytest.mark.parametrize("layout", ["row", "transposed"])
def test_rows_of_ragged_groups(name, layout):
    run_rows(GROUPS[name], 264, 200, layout=layout, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("beta", [0, 1])
def test_rows_types_layouts_strides(kind, out, layout, beta):
    run_rows([5, 130, 0, 64], 328, 136, kind=kind, out=kind if out == "same" else out, layout=layout, first=11, spare=9,
             lda=152, ldb=344, ldc=336, gap=40, beta=beta, seed=2)


@pytest.mark.gpu
@pytest.mark.parametrize("N,K", [(8, 8), (8, 4096), (1000, 8), (256, 64), (520, 1032), (1024, 2048)])
def test_rows_sizes(N, K):
    for layout in ("row", "transposed"):
        run_rows([3, 1, 0, 70, 2], N, K, out="f32", layout=layout, seed=3)


@pytest.mark.gpu
def test_rows_many_tiles():
    # more tiles than CTA pairs, more than eight row tiles in a group
    run_rows([2600, 513, 1, 900], 1288, 512, seed=4)
    run_rows([2600, 513, 1, 900], 1288, 512, layout="transposed", kind="f16", out="f16", seed=4)


@pytest.mark.gpu
def test_rows_most_groups():
    gen = np.random.default_rng(5)
    run_rows(gen.integers(0, 4, 1024).tolist(), 136, 72, seed=5)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 2, 40])
def test_rows_cut_along_k(rows):
    """Few tiles and a long contraction: K splits, their partial sums added in the same order on every run."""
    gen = torch.Generator().manual_seed(6)
    A, W = rand((rows, 8192), "bf16", gen).cuda(), rand((1, 8192, 512), "bf16", gen, 0.01).cuda()
    off = torch.tensor([0, rows], dtype=torch.int32).cuda()
    plan = nk.GroupedPlan(1, rows, 512, 8192, out_dtype=nk.F32)
    outs = []
    ws = scratch(plan)
    for _ in range(20):
        C = torch.full((rows, 512), float("nan"), device="cuda")
        plan.run(A, W, C, off, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
        outs.append(C)
    plan.check()
    assert all(torch.equal(outs[0], c) for c in outs)
    close(outs[0], A.double() @ W[0].double(), float((A.double().abs() @ W[0].double().abs()).max()), "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,N,K", [([2560], 2048, 2048), ([700, 1, 900, 0, 650, 300], 2048, 1536), ([9600, 40], 512, 4096)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_rows_last_wave_cut(sizes, N, K, out):
    """A few tiles behind full waves of them: only the last wave's are cut along k."""
    run_rows(sizes, N, K, out=out, seed=7)
    run_rows(sizes, N, K, kind="f16", out="f16" if out == "bf16" else "f32", layout="transposed", beta=1, seed=8)


@pytest.mark.gpu
def test_more_plans_than_counters():
    """A plan that finds no counters left runs without cutting tiles, and gives them back to nobody."""
    plans = [nk.GroupedPlan(1, 40, 512, 8192, out_dtype=nk.F32) for _ in range(1030)]
    assert plans[0].workspace_bytes > 0 and plans[-1].workspace_bytes == 0
    gen = torch.Generator().manual_seed(9)
    A, W = rand((40, 8192), "bf16", gen).cuda(), rand((1, 8192, 512), "bf16", gen, 0.01).cuda()
    off = torch.tensor([0, 40], dtype=torch.int32).cuda()
    want, size = A.double() @ W[0].double(), float((A.double().abs() @ W[0].double().abs()).max())
    for plan in (plans[0], plans[-1]):
        C = torch.full((40, 512), float("nan"), device="cuda")
        plan.run(A, W, C, off, workspace=scratch(plan), stream=torch.cuda.current_stream().cuda_stream)
        plan.check()
        close(C, want, size, "f32")
    for plan in plans:
        plan.destroy()
    assert nk.GroupedPlan(1, 40, 512, 8192).workspace_bytes > 0


@pytest.mark.gpu
def test_plan_without_counters_says_so():
    plans = [nk.GroupedPlan(1, 40, 512, 8192, out_dtype=nk.F32) for _ in range(1025)]
    late = nk.LoraPlan(40, 64, 64, 8, 1, 1), nk.LoraPlan(4000, 64, 64, 8, 1, 1)
    for plan in (plans[-1],) + late:
        assert plan.kernel_name.endswith("_uncut")
    assert not plans[0].kernel_name.endswith("_uncut")
    for plan in (*plans, *late):
        plan.destroy()
    again = nk.LoraPlan(4000, 64, 64, 8, 1, 1), nk.GroupedPlan(1, 40, 512, 8192)
    assert not any(plan.kernel_name.endswith("_uncut") for plan in again)


@pytest.mark.gpu
def test_plan_destroyed_with_runs_queued():
    """The next plan of cut tiles, on another stream, does not count in the words of the runs that are left."""
    gen = torch.Generator().manual_seed(20)
    W = rand((1, 8192, 512), "bf16", gen, 0.01).cuda()
    A = [rand((40, 8192), "bf16", gen).cuda() for _ in range(2)]
    off = torch.tensor([0, 40], dtype=torch.int32).cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    bytes_ = nk.GroupedPlan(1, 40, 512, 8192, out_dtype=nk.F32).workspace_bytes
    ws = [torch.full((bytes_,), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = [a.double() @ W[0].double() for a in A]
    size = [float((a.double().abs() @ W[0].double().abs()).max()) for a in A]
    for _ in range(5):
        outs = [[torch.full((40, 512), float("nan"), device="cuda") for _ in range(30)] for _ in range(2)]
        torch.cuda.synchronize()
        for i in range(2):
            plan = nk.GroupedPlan(1, 40, 512, 8192, out_dtype=nk.F32)
            for C in outs[i]:
                plan.run(A[i], W, C, off, workspace=ws[i], stream=streams[i].cuda_stream)
            plan.destroy()
        torch.cuda.synchronize()
        for i in range(2):
            for C in outs[i]:
                close(C, want[i], size[i], "f32")


@pytest.mark.gpu
def test_graph_outlives_its_plan():
    """A captured run goes on working, and goes on counting in words of its own, when its plan is gone."""
    gen = torch.Generator().manual_seed(21)
    A, W = rand((40, 8192), "bf16", gen).cuda(), rand((1, 8192, 512), "bf16", gen, 0.01).cuda()
    off = torch.tensor([0, 40], dtype=torch.int32).cuda()
    want, size = A.double() @ W[0].double(), float((A.double().abs() @ W[0].double().abs()).max())
    plan = nk.GroupedPlan(1, 40, 512, 8192, out_dtype=nk.F32)
    ws, C, D = scratch(plan), torch.empty(40, 512, device="cuda"), torch.empty(40, 512, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run(A, W, C, off, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
    plan.destroy()
    other, side = nk.GroupedPlan(1, 40, 512, 8192, out_dtype=nk.F32), torch.cuda.Stream()
    ws2 = scratch(other)
    torch.cuda.synchronize()
    for _ in range(20):
        C.fill_(float("nan"))
        D.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(10):
            graph.replay()
            other.run(A, W, D, off, workspace=ws2, stream=side.cuda_stream)
        torch.cuda.synchronize()
        close(C, want, size, "f32")
        close(D, want, size, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(GROUPS))
def test_weights_of_ragged_groups(name):
    run_weights(GROUPS[name], 264, 200, seed=11)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("beta", [0, 1])
def test_weights_types_strides(kind, out, beta):
    run_weights([5, 130, 0, 64, 65, 79, 80], 328, 136, kind=kind, out=kind if out == "same" else out, first=11, spare=9,
                lda=152, ldb=344, ldc=336, gap=40, beta=beta, seed=12)


@pytest.mark.gpu
@pytest.mark.parametrize("N,K", [(8, 8), (8, 1000), (1000, 8), (256, 256), (520, 296), (1024, 2048)])
def test_weights_sizes(N, K):
    run_weights([3, 1, 0, 70, 2], N, K, seed=13)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,poison", [([37, 5, 50], 1), ([64, 7, 9], 1), ([1, 1, 1], 1), ([15, 16, 17], 2), ([100, 0, 31], 0)])
def test_weights_neighbours_of_nan(sizes, poison):
    run_weights(sizes, 136, 264, poison=poison, seed=14)


@pytest.mark.gpu
def test_weights_many_tiles():
    run_weights([2049, 0, 700, 33, 1], 1288, 1032, out="bf16", seed=15)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,N,K", [([16384], 256, 256), ([9001], 64, 520), ([3000, 0, 5000, 7], 304, 264), ([0, 4097, 0], 1032, 1032)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_weights_cut_along_the_rows(sizes, N, K, out):
    """Few tiles and many rows: the parts of a tile are added in the same order on every run."""
    run_weights(sizes, N, K, out=out, seed=16)
    run_weights(sizes, N, K, kind="f16", out="f16" if out == "bf16" else "f32", beta=1, seed=17)
    gen = torch.Generator().manual_seed(18)
    rows, off = sum(sizes), offsets_of(sizes).cuda()
    A, B = rand((rows, K), "bf16", gen).cuda(), rand((rows, N), "bf16", gen).cuda()
    plan = nk.GroupedPlan(len(sizes), rows, N, K, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32)
    ws, outs = scratch(plan), []
    for _ in range(10):
        C = torch.full((len(sizes), K, N), float("nan"), device="cuda")
        plan.run(A, B, C, off, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
        outs.append(C)
    plan.check()
    assert all(torch.equal(outs[0], c) for c in outs)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1024, 8192])
def test_fp32_sums_do_not_drift(rows):
    """Sums of thousands of rows are as good as FP32 arithmetic: relative 2-norm error within 1e-6 (chunks of 512 rows, each
    32 truncated additions of at most 2^-23 of the running sum, on average half of that over a sum that grows: 32 / 3 * 2^-23)."""
    gen = torch.Generator().manual_seed(19)
    A, B = rand((rows, 256), "bf16", gen).cuda(), rand((rows, 512), "bf16", gen).cuda()
    plan = nk.GroupedPlan(1, rows, 512, 256, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32)
    C = torch.empty(1, 256, 512, device="cuda")
    plan.run(A, B, C, torch.tensor([0, rows], dtype=torch.int32).cuda(), workspace=scratch(plan), stream=torch.cuda.current_stream().cuda_stream)
    plan.check()
    want = A.double().t() @ B.double()
    assert float((C[0].double() - want).norm() / want.norm()) <= 32 / 3 * 2.0 ** -23


def positive(shape, kind, seed, scale):
    """Values of one sign, half to three halves of `scale` (the truncated bits of their sums all go one way)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return ((torch.rand(shape, generator=g, device="cuda") + 0.5) * scale).to(TYPES[kind][1])


def drift(got, want):
    """Mean relative error; what rounding the results to FP16 leaves of it: 2^-11 / sqrt(12) at most for one, so six times that
    over the root of their number."""
    return float(((got.double() - want) / want).mean().abs()), 6 * 2.0 ** -11 / np.sqrt(12 * want.numel())


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["rows", "rows_t", "weights"])
def test_long_sums_of_16_bit_results_do_not_drift(form):
    """2^18 products of one sign to an FP16 result, 2^14 truncated additions where one accumulator takes them all: the mean error
    stays within 2^-15, an eighth of what the rounding of one result to FP16 may be off on average of its spacing (2^-12)."""
    long_, st = 1 << 18, torch.cuda.current_stream().cuda_stream
    # about a wave of whole tiles: those of one group
    if form == "weights":
        N, K = 2304, 2304
        A, B = positive((long_, K), "f16", 1, 2.0 ** -6), positive((long_, N), "f16", 2, 2.0 ** -2)
        A *= torch.linspace(0.5, 1, K, device="cuda").half()
        plan = nk.GroupedPlan(1, long_, N, K, kind=nk.GROUPED_WEIGHTS, in_dtype=nk.F16, out_dtype=nk.F16)
        C, off = torch.empty(K, N, dtype=torch.float16, device="cuda"), torch.tensor([0, long_], dtype=torch.int32).cuda()
        want = A[:, :64].double().t() @ B[:, :256].double()
    else:
        rows, N = 1024, 2560
        A = positive((rows, long_), "f16", 3, 2.0 ** -6)
        A *= torch.linspace(0.5, 1, rows, device="cuda").half()[:, None]
        B = positive((long_, N) if form == "rows" else (N, long_), "f16", 4, 2.0 ** -2)
        plan = nk.GroupedPlan(1, rows, N, long_, in_dtype=nk.F16, out_dtype=nk.F16, layout_b=nk.ROW_MAJOR if form == "rows" else nk.TRANSPOSED)
        C, off = torch.empty(rows, N, dtype=torch.float16, device="cuda"), torch.tensor([0, rows], dtype=torch.int32).cuda()
        want = A[:64].double() @ (B[:, :256].double() if form == "rows" else B[:256].double().t())
    plan.run(A, B, C, off, workspace=scratch(plan), stream=st)
    plan.check()
    off_by, rounding = drift(C[:64, :256], want)
    assert off_by <= 2.0 ** -15 + rounding, (off_by, rounding)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["row", "transposed"])
def test_rows_of_several_chunks(kind, layout):
    """Contractions around a whole number of chunks (64 k-blocks of 64), whole tiles and cut ones."""
    for K in (4096, 4104, 8192, 8200, 16384, 20488):
        run_rows([300, 0, 1, 70], 520, K, kind=kind, out=kind, layout=layout, beta=1, seed=22)
    run_rows([5000, 3900], 1032, 4168, kind=kind, out=kind, layout=layout, seed=23)
    run_rows([5000, 3900], 1032, 8264, kind=kind, out=kind, layout=layout, seed=23)


@pytest.mark.gpu
def test_weights_of_very_many_rows():
    """A tile of 3.75 million k-blocks is cut like one of 3.1 million: 1.2 times its time, not that of one pair alone (74 times)."""
    times = []
    for rows in (200_000_000, 240_000_000):
        A, off = torch.ones(rows, 8, dtype=torch.bfloat16, device="cuda"), torch.tensor([0, rows], dtype=torch.int32).cuda()
        plan = nk.GroupedPlan(1, rows, 8, 8, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32)
        C, ws = torch.empty(8, 8, device="cuda"), scratch(plan)
        marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
        marks[0].record()
        for mark in marks[1:]:
            plan.run(A, A, C, off, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
            mark.record()
        plan.check()
        times.append(marks[1].elapsed_time(marks[2]))
        assert (C == rows).all()                 # (whole numbers below 2^24 and then multiples of 64: every sum is exact)
        del A
    assert times[1] <= 5 * times[0], times


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_weights_of_several_chunks(kind):
    run_weights([4096, 4097, 8192, 8193, 0, 20000, 16384], 1032, 1288, kind=kind, out=kind, beta=1, seed=24)


@pytest.mark.gpu
def test_rows_neighbours_of_nan():
    """Infinities and NaN of a row or a weight stay in the rows they belong to."""
    gen = torch.Generator().manual_seed(16)
    A, W = rand((90, 64), "bf16", gen), rand((3, 64, 72), "bf16", gen)
    A[40] = float("nan")
    W[2] = float("inf")
    off = torch.tensor([0, 30, 60, 90], dtype=torch.int32)
    plan = nk.GroupedPlan(3, 90, 72, 64, out_dtype=nk.F32)
    C = torch.zeros(90, 72, device="cuda")
    plan.run(A.cuda(), W.cuda(), C, off.cuda(), workspace=scratch(plan), stream=torch.cuda.current_stream().cuda_stream)
    plan.check()
    C = C.cpu()
    keep = [i for i in range(60) if i != 40]
    assert C[keep].isfinite().all() and C[40].isnan().all() and not C[60:].isfinite().any()


@pytest.mark.gpu
def test_gradients_against_differences():
    """d/ds of sum(G * (X + s E) W) and of sum(G * X (W + s E)): the loss is linear in s, so the difference
    quotient of the 64-bit formula is exact up to its rounding."""
    gen = torch.Generator().manual_seed(17)
    sizes, N, K = [3, 0, 61], 40, 72
    rows, off = 64, offsets_of(sizes)
    X, W, dY = rand((rows, K), "bf16", gen), rand((3, K, N), "bf16", gen), rand((rows, N), "bf16", gen)
    st = torch.cuda.current_stream().cuda_stream
    dX, dW = torch.empty(rows, K, device="cuda"), torch.empty(3, K, N, device="cuda")
    back = nk.GroupedPlan(3, rows, K, N, layout_b=nk.TRANSPOSED, out_dtype=nk.F32)
    back.run(dY.cuda(), W.cuda(), dX, off.cuda(), workspace=scratch(back), stream=st)
    grad = nk.GroupedPlan(3, rows, N, K, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32)
    grad.run(X.cuda(), dY.cuda(), dW, off.cuda(), workspace=scratch(grad), stream=st)
    back.check(), grad.check()

    def loss(x, w):
        y = torch.cat([x[off[g]:off[g + 1]] @ w[g] for g in range(3)])
        return float((y * dY.double()).sum())

    x, w = X.double(), W.double()
    h = 2.0 ** -6
    for _ in range(5):
        ex, ew = torch.randn(x.shape, generator=gen).double(), torch.randn(w.shape, generator=gen).double()
        for grad_of, num in ((float((dX.cpu().double() * ex).sum()), (loss(x + h * ex, w) - loss(x - h * ex, w)) / (2 * h)),
                             (float((dW.cpu().double() * ew).sum()), (loss(x, w + h * ew) - loss(x, w - h * ew)) / (2 * h))):
            # n terms of size about sqrt(contraction) each carry a relative FP32 accumulation error below 1e-5
            n = dX.numel() + dW.numel()
            assert abs(grad_of - num) <= 1e-5 * np.sqrt(n) * 10 * np.sqrt(max(sizes)), (grad_of, num)


@pytest.mark.gpu
@pytest.mark.parametrize("off", [[0, 50, 20, 90], [-5, 30, 60, 90], [0, 30, 60, 95], [0, -1, 200, 3], [90, 60, 30, 0]])
def test_offsets_that_break_the_rule_are_reported(off):
    """The kernel clamps them: nothing outside the arrays is touched, and the check says so once."""
    gen = torch.Generator().manual_seed(18)
    A, W, B = rand((90, 64), "bf16", gen).cuda(), rand((3, 64, 72), "bf16", gen).cuda(), rand((90, 72), "bf16", gen).cuda()
    o = torch.tensor(off, dtype=torch.int32).cuda()
    st = torch.cuda.current_stream().cuda_stream
    for plan, args, shape in ((nk.GroupedPlan(3, 90, 72, 64, out_dtype=nk.F32), (A, W), (90, 72)),
                              (nk.GroupedPlan(3, 90, 72, 64, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32), (A, B), (3, 64, 72))):
        C = torch.full((int(np.prod(shape)) + 512,), SENTINEL, device="cuda")
        plan.run(*args, C[256:], o, workspace=scratch(plan), stream=st)
        with pytest.raises(nk.NkError) as e:
            plan.check()
        assert e.value.status == 1 and "offsets" in str(e.value)
        plan.check()
        assert (C[:256] == SENTINEL).all() and (C[-256:] == SENTINEL).all()


@pytest.mark.gpu
def test_no_rows():
    plan = nk.GroupedPlan(4, 0, 64, 32)
    off = torch.zeros(5, dtype=torch.int32, device="cuda")
    plan.run(None, None, None, off, workspace=scratch(plan))
    plan.check()
    grad = nk.GroupedPlan(4, 0, 64, 32, kind=nk.GROUPED_WEIGHTS)
    C = torch.full((4, 32, 64), SENTINEL, device="cuda")
    grad.run(None, None, C, off, workspace=scratch(grad))
    grad.check()
    assert (C == 0).all()


@pytest.mark.gpu
def test_other_stream_and_new_pointers():
    """A plan follows the pointers and the stream of each call."""
    gen = torch.Generator().manual_seed(19)
    plan = nk.GroupedPlan(2, 50, 40, 64, out_dtype=nk.F32)
    ws = scratch(plan)
    side = torch.cuda.Stream()
    for _ in range(3):
        A, W = rand((50, 64), "bf16", gen).cuda(), rand((2, 64, 40), "bf16", gen).cuda()
        off = torch.tensor([0, 20, 50], dtype=torch.int32).cuda()
        C = torch.zeros(50, 40, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        plan.run(A, W, C, off, workspace=ws, stream=side.cuda_stream)
        side.synchronize()
        want = torch.cat([A[:20].double() @ W[0].double(), A[20:].double() @ W[1].double()])
        close(C, want, float((A.double().abs() @ W.double().abs().sum(0)).max()), "f32")


@pytest.mark.gpu
def test_run_refusals():
    plan = nk.GroupedPlan(2, 50, 40, 64)
    x = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    c = torch.zeros(1 << 16, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    ws = scratch(plan)
    for args, kw, status in (((None, x, c, off), dict(workspace=ws), 1), ((x, x, None, off), dict(workspace=ws), 1),
                             ((x, x, c, None), dict(workspace=ws), 1), ((x[1:], x, c, off), dict(workspace=ws), 3),
                             ((x, x[4:], c, off), dict(workspace=ws), 3), ((x, x, c[1:], off), dict(workspace=ws), 3),
                             ((x, x, c, off), dict(), 4), ((x, x, c, off), dict(workspace=ws, workspace_bytes=plan.workspace_bytes - 1), 4)):
        with pytest.raises(nk.NkError) as e:
            plan.run(*args, **kw)
        assert e.value.status == status


REFUSED = [
    (dict(groups=0), 1), (dict(rows=-1), 1), (dict(N=0), 1), (dict(K=-8), 1), (dict(kind=2), 1), (dict(in_dtype=9), 1),
    (dict(in_dtype=nk.F32), 2), (dict(in_dtype=nk.S8), 2), (dict(in_dtype=nk.E4M3), 2), (dict(out_dtype=nk.F16), 1),
    (dict(layout_b=7), 1), (dict(layout_b=nk.BLOCKED32), 2), (dict(kind=nk.GROUPED_WEIGHTS, layout_b=nk.TRANSPOSED), 2),
    (dict(beta=2), 1), (dict(groups=1025), 2), (dict(N=12), 3), (dict(K=20), 3), (dict(lda=36), 3), (dict(lda=24), 1),
    (dict(ldb=8), 1), (dict(ldc=8), 1), (dict(stride_g=64), 1), (dict(stride_g=4100), 3), (dict(rows=1 << 31), 2),
    (dict(rows=(1 << 31) - 8192, N=1 << 20), 2),
]


@pytest.mark.parametrize("kw,status", REFUSED)
def test_descriptor_refusals_need_no_device(kw, status):
    args = dict(groups=2, rows=50, N=64, K=32)
    args.update(kw)
    with pytest.raises(nk.NkError) as e:
        nk.GroupedPlan(**args)
    assert e.value.status == status


def test_null_handles():
    from paper_2511_13764_b200 import rows
    L = rows.lib()
    assert L.nk_grouped_create(None, None) == 1
    assert L.nk_grouped_workspace_bytes(None) == 0 and L.nk_grouped_check(None) == 1 and L.nk_grouped_destroy(None) == 0
    assert L.nk_grouped_run(None, None, None, None, None, None, 0, None) == 1
    assert L.nk_grouped_kernel_name(None) == b"" and L.nk_grouped_last_cuda_error(None) == b""
