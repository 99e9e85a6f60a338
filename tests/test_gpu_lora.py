"""The adapters of many requests beside a shared projection (nk_lora) against the formula in 64 bits.

Tolerance: that of the dense GEMM (1e-5 of the largest sum of |products|, half a unit in the last place of a 16-bit
result) on both products; X . A_a enters the second product as FP32 or as two 16-bit numbers, off by at most 2^-16 of
itself, so 2^-16 * scale * sum |X . A_a| |B_a| is added."""
import numpy as np
import pytest
import torch

import paper_2511_13764_b200 as nk
from nk_testlib import TOL_BF16_REL, TOL_F16_ABS, TOL_F16_REL, TOL_REL_SMAX

TYPES = {"bf16": (nk.BF16, torch.bfloat16), "f16": (nk.F16, torch.float16), "f32": (nk.F32, torch.float32)}
SENTINEL = 7.0


def rand(shape, kind, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float32) * scale).to(TYPES[kind][1])


def strided(x, ld):
    buf = torch.full((x.shape[0], ld), float("nan"), dtype=x.dtype)
    buf[:, : x.shape[1]] = x
    return buf.cuda()


def make(sizes, N, K, r, L, kind, first=0, spare=0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    rows = first + sum(sizes) + spare
    off = torch.tensor(np.concatenate([[first], first + np.cumsum(sizes)]), dtype=torch.int32)
    which = torch.randint(0, L, (len(sizes),), generator=gen, dtype=torch.int32)
    return (rand((rows, K), kind, gen), rand((K, N), kind, gen, K ** -0.5), rand((L, K, r), kind, gen, K ** -0.5),
            rand((L, r, N), kind, gen, r ** -0.5), 0.5 + torch.rand(L, generator=gen), off, which)


def run(data, layout="row", out="f32", ldx=0, ldw=0, ldy=0, check=True):
    X, W, A, B, scale, off, which = data
    rows, K = X.shape
    N, r, L = W.shape[1], A.shape[2], A.shape[0]
    kind = "bf16" if X.dtype == torch.bfloat16 else "f16"
    t = layout == "transposed"
    Ws, As, Bs = (m.transpose(-1, -2).contiguous() if t else m for m in (W, A, B))
    plan = nk.LoraPlan(rows, N, K, r, L, len(which), in_dtype=TYPES[kind][0], out_dtype=TYPES[out][0],
                       layout=nk.TRANSPOSED if t else nk.ROW_MAJOR, ldx=ldx, ldw=ldw, ldy=ldy)
    Y = torch.full((rows, ldy or N), SENTINEL, dtype=TYPES[out][1], device="cuda")
    ws = torch.full((plan.workspace_bytes,), 255, dtype=torch.uint8, device="cuda")
    args = (strided(X, ldx or K), strided(Ws, ldw or Ws.shape[1]), As.cuda(), Bs.cuda(), scale.cuda(), off.cuda(), which.cuda())
    plan.run(*args, Y, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
    if check:
        plan.check()
    assert (Y[:, N:] == SENTINEL).all()
    return Y[:, :N].cpu(), plan


def want_of(data):
    """Formula, and the tolerance's size terms."""
    X, W, A, B, scale, off, which = data
    x, w = X.double().cuda(), W.double().cuda()
    y, size, h16 = x @ w, x.abs() @ w.abs(), torch.zeros(X.shape[0], W.shape[1], dtype=torch.float64, device="cuda")
    for q, a in enumerate(which.tolist()):
        lo, hi = int(off[q]), int(off[q + 1])
        if 0 <= a < A.shape[0] and hi > lo:
            f, g, s = A[a].double().cuda(), B[a].double().cuda(), float(scale[a])
            h = x[lo:hi] @ f
            y[lo:hi] += s * h @ g
            size[lo:hi] += s * (x[lo:hi].abs() @ f.abs()) @ g.abs()
            h16[lo:hi] = 2.0 ** -16 * s * h.abs() @ g.abs()
    return y.cpu(), float(size.max()), h16.cpu()


def close(got, data, out):
    y, size, h16 = want_of(data)
    tol = TOL_REL_SMAX * size + h16 + {"bf16": TOL_BF16_REL, "f16": TOL_F16_REL, "f32": 0.0}[out] * y.abs() + (TOL_F16_ABS if out == "f16" else 0)
    bad = ~((got.double() - y).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: got {got[bad][0]} want {y[bad][0]}"


SHAPES = {
    "one_row": [1],
    "step": [1] * 16,
    "step_many": [1] * 300,
    "one_prompt": [700],
    "mixed": [1, 1, 200, 0, 1, 1, 1, 90, 1, 17, 1],
    "edges": [255, 1, 256, 257, 0, 8, 9, 7],
    "short": [5, 8, 3, 0, 0, 12, 2, 9],
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("rank", [8, 16, 40, 128])
def test_requests(name, layout, rank):
    data = make(SHAPES[name], 264, 328, rank, 5, "bf16", seed=1)
    got, _ = run(data, layout)
    close(got, data, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("name", ["step", "mixed"])
def test_types_strides_and_rows_outside(kind, out, layout, name):
    data = make(SHAPES[name], 520, 136, 24, 3, kind, first=7, spare=5, seed=2)
    got, _ = run(data, layout, out, ldx=152, ldw=544 if layout == "row" else 144, ldy=536)
    close(got, data, out)


@pytest.mark.gpu
@pytest.mark.parametrize("N,K", [(8, 8), (8, 4096), (1000, 8), (4096, 1024), (1032, 2056)])
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("sizes", [[1, 1, 1, 1], [60, 1, 130]])
def test_sizes(N, K, layout, sizes):
    data = make(sizes, N, K, 16, 2, "bf16", seed=3)
    got, _ = run(data, layout)
    close(got, data, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["one_prompt", "mixed", "edges", "short"])
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rank", [8, 40, 128])
def test_sixteen_bit_results(name, layout, kind, rank):
    data = make(SHAPES[name], 264, 328, rank, 5, kind, seed=8)
    got, _ = run(data, layout, kind)
    close(got, data, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("out", ["same", "f32"])
@pytest.mark.parametrize("rank", [40, 72, 104, 128])
@pytest.mark.parametrize("K", [8, 64, 72, 128, 192, 776, 832])
def test_short_contraction_high_rank(layout, kind, out, rank, K):
    """Fewer k-blocks in X . W than in the adapters' product, requests that share tiles, tiles of one request."""
    out = kind if out == "same" else out
    for sizes in (SHAPES["edges"], [40, 30, 25, 9, 300, 33]):
        data = make(sizes, 264, K, rank, 5, kind, seed=12)
        got, plan = run(data, layout, out)
        assert plan.kernel_name.startswith("lora_many")
        close(got, data, out)


@pytest.mark.gpu
@pytest.mark.parametrize("K", [1344, 2112, 3200, 4160])
def test_short_last_part_high_rank(K):
    """Few tiles, cut along k, the last part the shortest."""
    for sizes in ([20, 25], [12, 200, 33, 11]):
        data = make(sizes, 264, K, 128, 3, "bf16", seed=13)
        got, plan = run(data, "row", "bf16")
        assert plan.kernel_name.startswith("lora_many")
        close(got, data, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_many_tiles_and_a_cut_last_wave(layout, out):
    data = make([1, 1500, 1, 1, 3, 700, 9, 1, 360], 2056, 1096, 72, 4, "bf16", seed=9)
    got, _ = run(data, layout, out)
    close(got, data, out)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["row", "transposed"])
def test_a_long_prompt_among_many_short_requests(layout):
    """Whatever the plan's average, a long request beside many of one row is right, and where it may be long it has the tensor cores."""
    for sizes, rank, name in (([1] * 200 + [1400], 16, "lora_few"), ([1] * 200 + [1400], 64, "lora_many"),
                              ([0] * 500 + [700] + [0] * 99, 32, "lora_few"), ([1] * 500 + [3000] + [1] * 523, 40, "lora_many")):
        data = make(sizes, 264, 200, rank, 5, "bf16", seed=18)
        got, plan = run(data, layout, "bf16")
        assert plan.kernel_name.startswith(name)
        close(got, data, "bf16")
    # (nothing runs: 8 rows to a request on average, 7000 to one if it comes so)
    assert nk.LoraPlan(8023, 4096, 4096, 128, 32, 1024, layout=nk.TRANSPOSED).kernel_name.startswith("lora_many")
    assert nk.LoraPlan(240, 4096, 4096, 64, 1, 1, layout=nk.TRANSPOSED).kernel_name.startswith("lora_many")


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["row", "transposed"])
def test_most_requests(layout):
    gen = np.random.default_rng(10)
    data = make(gen.integers(0, 3, 1024).tolist(), 72, 136, 8, 60, "bf16", seed=10)
    got, _ = run(data, layout)
    close(got, data, "f32")
    data = make([int(x) for x in gen.integers(0, 25, 400)], 72, 136, 24, 7, "bf16", seed=11)
    got, _ = run(data, layout, "bf16")
    close(got, data, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["step", "mixed", "one_prompt"])
@pytest.mark.parametrize("layout", ["row", "transposed"])
def test_requests_without_an_adapter(name, layout):
    data = make(SHAPES[name], 264, 328, 16, 4, "bf16", seed=4)
    which = data[6]
    which[::2] = -1
    which[-1] = 4                                    # one past the last adapter
    got, _ = run(data, layout)
    close(got, data, "f32")
    which[:] = -1
    got, _ = run(data, layout)
    close(got, data, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["step", "mixed"])
@pytest.mark.parametrize("layout", ["row", "transposed"])
def test_nan_stays_with_its_request(name, layout):
    """An adapter of infinities or NaN reaches the rows of its own requests only, and no row without one."""
    data = make(SHAPES[name], 264, 328, 16, 6, "bf16", seed=5)
    X, W, A, B, scale, off, which = data
    A[1] = float("nan")
    B[2] = float("inf")
    which[0] = -1
    which[1] = 1
    X[int(off[4]):int(off[5])] = float("nan")
    got, _ = run(data, layout)
    bad = torch.zeros(X.shape[0], dtype=torch.bool)
    for q, a in enumerate(which.tolist()):
        if a in (1, 2) or q == 4:
            bad[int(off[q]):int(off[q + 1])] = True
    assert got[~bad].isfinite().all()
    assert not got[bad].isfinite().any()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("out", ["f16", "f32"])
@pytest.mark.parametrize("rank", [8, 40, 128])
@pytest.mark.parametrize("size", [2.0 ** -30, 2.0 ** -17, 2.0 ** -10, 1.0, 2.0 ** 18])
def test_fp16_adapters_of_any_size(layout, out, rank, size):
    """The adapters' part alone (W = 0), scale X . A_a from far below FP16's smallest number to far above its largest, rows of
    a request up to 2^11 apart: every row is as good as FP32 sums and two FP16 numbers of its own scale make it, in short requests and long.
    Of a row: 1e-5 of its largest sum of |products| (what the other tests allow of the largest row's), 2^-21 of its largest
    |scale X . A_a| times the sums of |B_a|, and half a unit in the last place of the result."""
    sizes = [300, 9, 8, 1, 20, 256]
    data = make(sizes, 264, 328, rank, 4, "f16", seed=14)
    X, W, A, B, scale, off, which = data
    W.zero_()
    X.mul_(2.0 ** -(torch.arange(X.shape[0]) % 12).to(X.dtype)[:, None])
    scale.mul_(size)
    if out == "f16" and size > 1:
        B.mul_(1.0 / 512)
    got, plan = run(data, layout, out)
    assert plan.kernel_name.startswith("lora_many")
    for q, a in enumerate(which.tolist()):
        lo, hi, s = int(off[q]), int(off[q + 1]), float(scale[a])
        x, f, g = X[lo:hi].double(), A[a].double(), B[a].double()
        h = s * x @ f
        want, sums = h @ g, (s * (x.abs() @ f.abs()) @ g.abs()).amax(1, keepdim=True)
        tol = TOL_REL_SMAX * sums + 2.0 ** -21 * h.abs().amax(1, keepdim=True) * g.abs().sum(0)
        if out == "f16":
            tol = tol + TOL_F16_REL * want.abs() + TOL_F16_ABS
        bad = ~((got[lo:hi].double() - want).abs() <= tol)
        assert not bad.any(), f"request {q}: {int(bad.sum())} of {bad.numel()} off, got {got[lo:hi][bad][0]} want {want[bad][0]}"


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("out", ["f16", "f32"])
def test_fp16_nan_stays_with_its_request(layout, out):
    data = make(SHAPES["edges"], 264, 328, 40, 9, "f16", seed=15)
    X, W, A, B, scale, off, which = data
    which.copy_(torch.arange(8))
    A[2] = float("nan")
    B[3] = float("inf")
    scale[6] = float("inf")
    X[int(off[7]):int(off[8])] = float("nan")
    X[3] = float("inf")                              # one row of the first request
    got, _ = run(data, layout, out)
    bad = torch.zeros(X.shape[0], dtype=torch.bool)
    bad[3] = True
    for q in (2, 3, 6, 7):
        bad[int(off[q]):int(off[q + 1])] = True
    assert got[~bad].isfinite().all() and not got[bad].isfinite().any()
    data[2][2], data[3][3], data[4][6] = 0, 0, 0
    keep = ~bad
    clean = tuple(d.clone() for d in data)
    clean[0][bad] = 0
    want, size, h16 = want_of(clean)
    tol = TOL_REL_SMAX * size + h16 + (TOL_F16_REL * want.abs() + TOL_F16_ABS if out == "f16" else 0)
    assert ((got.double() - want).abs() <= tol)[keep].all()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("K", [4096, 4104, 8192, 8264, 20488])
def test_contractions_of_several_chunks(layout, kind, K):
    data = make([1, 300, 7, 40, 256, 9], 520, K, 40, 3, kind, seed=16)
    got, _ = run(data, layout, kind)
    close(got, data, kind)


@pytest.mark.gpu
def test_long_sums_of_16_bit_results_do_not_drift():
    """2^17 products of one sign to an FP16 result, the adapter's among them: a mean error within 2^-15 (an eighth of half of FP16's spacing),
    and what is left of the rounding of the results."""
    rows, N, K, g = 1024, 2560, 1 << 17, torch.Generator(device="cuda").manual_seed(17)

    def positive(*shape, scale):
        return ((torch.rand(shape, generator=g, device="cuda") + 0.5) * scale).half()

    X, W, A, B = positive(rows, K, scale=2.0 ** -6), positive(K, N, scale=2.0 ** -2), positive(1, K, 8, scale=2.0 ** -8), positive(1, 8, N, scale=2.0 ** -3)
    X *= torch.linspace(0.5, 1, rows, device="cuda").half()[:, None]
    scale, off, which = torch.ones(1, device="cuda"), torch.tensor([0, rows], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    plan = nk.LoraPlan(rows, N, K, 8, 1, 1, in_dtype=nk.F16, out_dtype=nk.F16)
    Y, ws = torch.empty(rows, N, dtype=torch.float16, device="cuda"), torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    plan.run(X, W, A, B, scale, off, which, Y, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
    plan.check()
    x = X[:64].double()
    want = x @ W[:, :256].double() + x @ A[0].double() @ B[0, :, :256].double()
    off_by = float(((Y[:64, :256].double() - want) / want).mean().abs())
    assert off_by <= 2.0 ** -15 + 6 * 2.0 ** -11 / np.sqrt(12 * want.numel())


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["row", "transposed"])
@pytest.mark.parametrize("name", ["step", "mixed", "edges"])
def test_gradient_of_the_rows(layout, name):
    """dX of sum(dY * Y) by the same call with N and K exchanged, the other layout and A and B in each other's place; the loss is
    linear in X, so the difference quotient of the 64-bit formula is exact up to its rounding."""
    K, N, r, L = 328, 264, 24, 4
    X, W, A, B, scale, off, which = make(SHAPES[name], N, K, r, L, "bf16", seed=19)
    which[0] = -1
    dY = rand((X.shape[0], N), "bf16", torch.Generator().manual_seed(20))
    Ws, As, Bs = (m if layout == "row" else m.transpose(-1, -2).contiguous() for m in (W, A, B))     # as the forward pass keeps them
    plan = nk.LoraPlan(X.shape[0], K, N, r, L, len(which), layout=nk.TRANSPOSED if layout == "row" else nk.ROW_MAJOR)
    dX = torch.full((X.shape[0], K), float("nan"), device="cuda")
    ws = torch.full((plan.workspace_bytes,), 255, dtype=torch.uint8, device="cuda")
    plan.run(dY.cuda(), Ws.cuda(), Bs.cuda(), As.cuda(), scale.cuda(), off.cuda(), which.cuda(), dX, workspace=ws,
             stream=torch.cuda.current_stream().cuda_stream)
    plan.check()
    back = (dY, W.t().contiguous(), B.transpose(1, 2).contiguous(), A.transpose(1, 2).contiguous(), scale, off, which)
    close(dX.cpu(), back, "f32")
    loss = lambda x: float((want_of((x, W, A, B, scale, off, which))[0] * dY.double()).sum())   # noqa: E731
    for seed in range(3):
        e = torch.randn(X.shape, generator=torch.Generator().manual_seed(seed)).double()
        terms = dX.cpu().double() * e
        # every element of dX within 1e-5 of its largest sum of |products| (and 2^-16 of the adapter's part of it): the errors of many elements
        # add up at most like their sizes
        size = want_of(back)[1]
        num = (loss(X.double() + e) - loss(X.double() - e)) / 2
        assert abs(num - float(terms.sum())) <= (TOL_REL_SMAX + 2.0 ** -16) * size * float(e.abs().sum())


@pytest.mark.gpu
def test_same_bits_every_time():
    data = make(SHAPES["mixed"], 264, 4096, 16, 4, "bf16", seed=6)
    first, _ = run(data)
    for _ in range(10):
        again, _ = run(data)
        assert torch.equal(first, again)


@pytest.mark.gpu
@pytest.mark.parametrize("off", [[0, 50, 20, 90], [-5, 30, 60, 90], [0, 30, 60, 95], [90, 60, 30, 0]])
def test_offsets_that_break_the_rule_are_reported(off):
    data = list(make([30, 30, 30], 72, 64, 16, 2, "bf16", seed=7))
    data[5] = torch.tensor(off, dtype=torch.int32)
    _, plan = run(data, check=False)
    with pytest.raises(nk.NkError) as e:
        plan.check()
    assert e.value.status == 1 and "offsets" in str(e.value)
    plan.check()


@pytest.mark.gpu
def test_no_rows():
    plan = nk.LoraPlan(0, 64, 32, 8, 2, 3)
    plan.run(*[None] * 8)
    plan.check()


@pytest.mark.gpu
def test_run_refusals():
    plan = nk.LoraPlan(50, 64, 32, 8, 2, 3)
    x = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    f, i = torch.zeros(1 << 14, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    good = [x, x, x, x, f, i, i, f]
    for pos in range(8):
        args = list(good)
        args[pos] = None
        with pytest.raises(nk.NkError) as e:
            plan.run(*args, workspace=ws)
        assert e.value.status == 1
    for pos in (0, 1, 2, 3, 7):
        args = list(good)
        args[pos] = args[pos][1:]
        with pytest.raises(nk.NkError) as e:
            plan.run(*args, workspace=ws)
        assert e.value.status == 3
    for kw in (dict(), dict(workspace=ws, workspace_bytes=ws.numel() - 1)):
        with pytest.raises(nk.NkError) as e:
            plan.run(*good, **kw)
        assert e.value.status == 4


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), 1), (dict(N=0), 1), (dict(K=0), 1), (dict(rank=0), 1), (dict(adapters=0), 1), (dict(requests=0), 1),
    (dict(in_dtype=nk.F32), 2), (dict(in_dtype=33), 1), (dict(out_dtype=nk.F16), 1), (dict(layout=nk.BLOCKED32), 2), (dict(layout=9), 1),
    (dict(rank=136), 2), (dict(rank=12), 3), (dict(requests=1025), 2), (dict(adapters=65536), 2), (dict(N=68), 3), (dict(K=36), 3),
    (dict(ldx=24), 1), (dict(ldx=36), 3), (dict(ldw=8), 1), (dict(ldy=8), 1), (dict(rows=(1 << 24) + 1), 2),
])
def test_descriptor_refusals_need_no_device(kw, status):
    args = dict(rows=50, N=64, K=32, rank=8, adapters=2, requests=3)
    args.update(kw)
    with pytest.raises(nk.NkError) as e:
        nk.LoraPlan(**args)
    assert e.value.status == status
