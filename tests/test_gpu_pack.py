"""nk_pack on the GPU against the formats' definitions in 64 bits: every element and scale equal."""
import numpy as np
import pytest
import torch

import paper_2511_13764_b200 as nk
from mx_testlib import (BLOCK, group_places, one_zero, padded, quantise, tensor_scale, tiles_of, unpack_data, unpack_scales, values)

pytestmark = pytest.mark.gpu

FORMATS = {"mxf4": nk.MXF4, "nvf4": nk.NVF4}
TYPES = {"f32": (nk.F32, torch.float32), "bf16": (nk.BF16, torch.bfloat16), "f16": (nk.F16, torch.float16)}


def stream():
    return torch.cuda.current_stream().cuda_stream


def rows_of(rows, K, kind, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, K, generator=g) * scale * torch.exp(torch.randn(1, K, generator=g))
    x[torch.rand(rows, K, generator=g) < 0.05] = 0.0
    # ties: small multiples of a quarter
    ties = torch.rand(rows, 1, generator=g) < 0.3
    x = torch.where(ties, torch.randint(-24, 25, (rows, K), generator=g) * 0.25, x)
    return x.to(TYPES[kind][1])


def pack(x, fmt, kind, t=None, offsets=None, **more):
    rows, K = x.shape[-2:]
    plan = nk.PackPlan(rows, K, format=FORMATS[fmt], in_dtype=TYPES[kind][0], **more)
    data = torch.full((plan.data_bytes + 64,), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((plan.scales_bytes + 64,), 0xAA, dtype=torch.uint8, device="cuda")
    scale = None if t is None else torch.tensor([t], dtype=torch.float32, device="cuda").reshape(-1)
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    plan.run(x.cuda(), data, scales, scale=scale, offsets=off, stream=stream())
    plan.check()
    assert (data[plan.data_bytes:] == 0xAA).all() and (scales[plan.scales_bytes:] == 0xAA).all(), "written behind the end"
    return plan, data[:plan.data_bytes], scales[:plan.scales_bytes], scale, off


def check_values(plan, data, scales, scale, off, want, kind="f32", rows=None):
    """nk_pack_values against the values that the codes stand for (their FP32 product is exact for t of 8 bits)."""
    y = torch.full(want.shape, 7.0, dtype=TYPES[kind][1], device="cuda")
    plan.values(data, scales, y, scale=scale, offsets=off, stream=stream())
    plan.check()
    got = y.double().cpu().numpy()
    live = slice(None) if rows is None else rows
    exact = torch.from_numpy(want).to(TYPES[kind][1]).double().numpy()
    assert np.array_equal(got[live], exact[live], equal_nan=True)
    if rows is not None:
        other = np.ones(want.shape[0], bool)
        other[rows] = False
        assert (got[other] == 7.0).all()


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K", [(1, 8), (1, 64), (3, 40), (16, 4096), (127, 72), (128, 256), (129, 264), (300, 1032)])
def test_along_rows(fmt, kind, rows, K):
    x = rows_of(rows, K, kind, seed=rows + K)
    t = tensor_scale(x.double().numpy()) if fmt == "nvf4" else 1.0
    plan, data, scales, scale, _ = pack(x, fmt, kind, t if fmt == "nvf4" else None)
    codes, bytes_, _ = quantise(x.double().numpy(), fmt, t)
    assert np.array_equal(unpack_data(data.cpu().numpy(), rows, K), one_zero(codes))
    assert np.array_equal(unpack_scales(scales.cpu().numpy(), np.arange(rows), K, fmt), bytes_)
    check_values(plan, data, scales, scale, None, values(codes, bytes_, fmt, t, K))


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K", [(1, 8), (31, 64), (64, 40), (65, 136), (128, 128), (333, 264), (1000, 520)])
def test_along_columns(fmt, kind, rows, K):
    x = rows_of(rows, K, kind, seed=rows + K)
    t = tensor_scale(x.double().numpy()) if fmt == "nvf4" else 1.0
    plan, data, scales, scale, _ = pack(x, fmt, kind, t if fmt == "nvf4" else None, transposed=1)
    codes, bytes_, _ = quantise(x.double().numpy().T.copy(), fmt, t)
    assert np.array_equal(unpack_data(data.cpu().numpy(), K, rows), one_zero(codes))
    assert np.array_equal(unpack_scales(scales.cpu().numpy(), np.arange(K), rows, fmt), bytes_)
    check_values(plan, data, scales, scale, None, values(codes, bytes_, fmt, t, rows))


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("offsets", [[0, 5], [0, 0, 130, 130, 131, 300, 300], [7, 20, 20, 290], [0, 0], [128, 256, 300]])
def test_grouped_rows(fmt, offsets):
    rows, K, groups = 300, 136, len(offsets) - 1
    x = rows_of(rows, K, "bf16", seed=len(offsets))
    t = 0.0078125 if fmt == "nvf4" else 1.0
    plan, data, scales, scale, off = pack(x, fmt, "bf16", t if fmt == "nvf4" else None, offsets=offsets, groups=groups)
    codes, bytes_, _ = quantise(x.double().numpy(), fmt, t)
    live, at = group_places(offsets)
    got = data.cpu().numpy().reshape(rows, -1)
    other = np.ones(rows, bool)
    other[live] = False
    assert (got[other] == 0xAA).all(), "rows outside all groups are left alone"
    assert plan.scales_bytes == (rows // 128 + groups) * tiles_of(K, fmt) * 512
    if len(live):
        assert np.array_equal(unpack_data(got[live], len(live), K), one_zero(codes[live]))
        assert np.array_equal(unpack_scales(scales.cpu().numpy(), at, K, fmt), bytes_[live])
    check_values(plan, data, scales, scale, off, values(codes, bytes_, fmt, t, K), rows=live)


@pytest.mark.parametrize("offsets", [[0, 200, 100, 300], [-5, 100, 200, 300], [0, 100, 400, 500]])
def test_bad_offsets_are_clamped_and_reported(offsets):
    plan = nk.PackPlan(300, 64, groups=3, format=nk.MXF4)
    x = rows_of(300, 64, "bf16").cuda()
    data = torch.empty(plan.data_bytes, dtype=torch.uint8, device="cuda")
    scales = torch.empty(plan.scales_bytes, dtype=torch.uint8, device="cuda")
    plan.run(x, data, scales, offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"), stream=stream())
    with pytest.raises(nk.NkError) as e:
        plan.check()
    assert e.value.status == 1
    plan.check()                                          # reported once
    top, clamped = 0, []
    for o in offsets:
        top = max(top, min(o, 300))
        clamped.append(top)
    codes, bytes_, _ = quantise(x.double().cpu().numpy(), "mxf4")
    live, at = group_places(clamped)
    assert np.array_equal(unpack_data(data.cpu().numpy().reshape(300, -1)[live], len(live), 64), one_zero(codes[live]))
    assert np.array_equal(unpack_scales(scales.cpu().numpy(), at, 64, "mxf4"), bytes_[live])


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("transposed", [0, 1])
def test_batches_and_strides(fmt, transposed):
    """Matrices of a batch with rows further apart than they are long; each has a tensor scale of its own."""
    batch, rows, K = 3, 150, 200
    g = torch.Generator().manual_seed(5)
    store = torch.randn(batch, rows + 2, K + 24, generator=g).to(torch.bfloat16)
    plan = nk.PackPlan(rows, K, format=FORMATS[fmt], batch=batch, transposed=transposed, ldx=K + 24, stride_x=(rows + 2) * (K + 24))
    dev = store.cuda()
    data = torch.empty(plan.data_bytes, dtype=torch.uint8, device="cuda")
    scales = torch.empty(plan.scales_bytes, dtype=torch.uint8, device="cuda")
    scale, ts = None, [1.0] * batch
    if fmt == "nvf4":
        scale = torch.empty(batch, device="cuda")
        ws = torch.empty(max(1, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
        plan.tensor_scale(dev, scale, workspace=ws, stream=stream())
        ts = [tensor_scale(store[b, :rows, :K].double().numpy()) for b in range(batch)]
        assert scale.tolist() == ts
    plan.run(dev, data, scales, scale=scale, stream=stream())
    plan.check()
    outer, length = (K, rows) if transposed else (rows, K)
    per_data, per_scales = plan.data_bytes // batch, plan.scales_bytes // batch
    for b in range(batch):
        x = store[b, :rows, :K].double().numpy()
        codes, bytes_, _ = quantise(x.T.copy() if transposed else x, fmt, ts[b])
        assert np.array_equal(unpack_data(data.cpu().numpy()[b * per_data:(b + 1) * per_data], outer, length), one_zero(codes))
        assert np.array_equal(unpack_scales(scales.cpu().numpy()[b * per_scales:(b + 1) * per_scales], np.arange(outer), length, fmt), bytes_)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K", [(1, 8), (5, 24), (700, 1000), (3000, 2048)])
def test_tensor_scale(kind, rows, K):
    x = rows_of(rows, K, kind, seed=K)
    plan = nk.PackPlan(rows, K, in_dtype=TYPES[kind][0])
    ws = torch.full((max(1, plan.workspace_bytes),), 0xFF, dtype=torch.uint8, device="cuda")
    scale = torch.empty(1, device="cuda")
    for value in (None, 0.0, float("inf"), float("nan")):
        y = x.clone()
        if value == 0.0:
            y.zero_()
        elif value is not None:
            y[rows // 2, K // 2] = value
        plan.tensor_scale(y.cuda(), scale, workspace=ws, stream=stream())
        plan.check()
        if value in (None, 0.0):
            assert scale.item() == tensor_scale(y.double().numpy())
        else:
            assert np.isnan(scale.item())


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [0, 1])
def test_values_that_are_not_ordinary(fmt, kind, transposed):
    """Infinities and NaN stay in their block; the largest and smallest numbers of a type; blocks of zeros and of zeros' signs."""
    dt = TYPES[kind][1]
    x = rows_of(64, 128, kind, seed=3)
    x[0, 5], x[1, 40], x[2, 127] = float("inf"), float("-inf"), float("nan")
    x[3] = torch.finfo(dt).max
    x[4] = torch.finfo(dt).smallest_normal
    x[5] = torch.finfo(dt).smallest_normal / 4               # subnormal
    x[6], x[7] = 0.0, -0.0
    x[8, ::32] = torch.finfo(dt).max
    x[9] = -torch.finfo(dt).max
    src = x.t().contiguous() if transposed else x
    for t in ([None] if fmt == "mxf4" else [None, 2.0 ** -20, 2.0 ** 20, float("nan"), float("inf"), 0.0, -1.0]):
        plan, data, scales, _, _ = pack(src, fmt, kind, t, transposed=transposed)
        codes, bytes_, _ = quantise(x.double().numpy(), fmt, 1.0 if t is None else t)
        assert np.array_equal(unpack_data(data.cpu().numpy(), 64, 128), one_zero(codes)), t
        assert np.array_equal(unpack_scales(scales.cpu().numpy(), np.arange(64), 128, fmt), bytes_), t


@pytest.mark.parametrize("transposed", [0, 1])
def test_any_tensor_scale(transposed):
    """With a scale of 24 bits an element may differ only where the quotient is within 2^-16 of a border, a block's scale not at all here."""
    x = rows_of(256, 256, "bf16", seed=9)
    t = float(np.float32(0.0123456789))
    src = x.t().contiguous() if transposed else x
    plan, data, scales, _, _ = pack(src, "nvf4", "bf16", t, transposed=transposed)
    codes, bytes_, near = quantise(x.double().numpy(), "nvf4", t)
    assert np.array_equal(unpack_scales(scales.cpu().numpy(), np.arange(256), 256, "nvf4"), bytes_)
    wrong = unpack_data(data.cpu().numpy(), 256, 256) != one_zero(codes)
    assert not (wrong & (near > 2.0 ** -16)).any()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("transposed,rows,K", [(0, 33, 104), (1, 33, 104), (1, 4099, 24)])
def test_values_in_16_bits(kind, transposed, rows, K):
    x = rows_of(rows, K, kind, seed=rows)
    t = tensor_scale(x.double().numpy())
    plan, data, scales, scale, _ = pack(x, "nvf4", kind, t, transposed=transposed, value_dtype=TYPES[kind][0])
    z = x.double().numpy()
    codes, bytes_, _ = quantise(z.T.copy() if transposed else z, "nvf4", t)
    check_values(plan, data, scales, scale, None, values(codes, bytes_, "nvf4", t, rows if transposed else K), kind)


@pytest.mark.parametrize("transposed", [0, 1])
def test_matrices_beyond_32_bits(transposed):
    """More than 2^31 elements; the last rows are looked at."""
    rows, K = 270000, 8192
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    tail = rows_of(40, K, "bf16", seed=4)
    x[rows - 40:] = tail.cuda()
    plan = nk.PackPlan(rows, K, transposed=transposed)
    data = torch.full((plan.data_bytes,), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((plan.scales_bytes,), 0xAA, dtype=torch.uint8, device="cuda")
    scale, ws = torch.empty(1, device="cuda"), torch.empty(max(1, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
    plan.tensor_scale(x, scale, workspace=ws, stream=stream())
    plan.run(x, data, scales, scale=scale, stream=stream())
    plan.check()
    z = tail.double().numpy()
    t = tensor_scale(z)
    assert scale.item() == t
    if transposed:
        # the last 64 of the contraction of every 1000th feature (270000 is a multiple of 16: 16 blocks end there)
        f = torch.arange(0, K, 1000)
        got = data.view(K, -1)[f.cuda()][:, -(padded(rows) // 2 - (rows - 48) // 2):].cpu().numpy()
        full = np.zeros((len(f), 48))
        full[:, 8:] = z[:, f.numpy()].T
        codes, _, _ = quantise(full, "nvf4", t)
        low, high = got[:, :24] & 15, got[:, :24] >> 4
        assert np.array_equal(one_zero(np.stack([low, high], 2).reshape(len(f), 48)), one_zero(codes[:, :48]))
        assert not got[:, 24:].any()
    else:
        codes, bytes_, _ = quantise(z, "nvf4", t)
        assert np.array_equal(unpack_data(data.view(rows, -1)[rows - 40:].cpu().numpy(), 40, K), one_zero(codes))
        tiles = scales.view(-1, tiles_of(K, "nvf4") * 512)[-2:].cpu().numpy()
        at = np.arange(rows - 40, rows) - (len(scales) // (tiles_of(K, "nvf4") * 512) - 2) * 128
        assert np.array_equal(unpack_scales(tiles, at, K, "nvf4"), bytes_)


def test_no_rows_and_refusals():
    plan = nk.PackPlan(0, 64)
    assert plan.data_bytes == 0
    plan.run(None, None, None, stream=stream())
    scale = torch.empty(1, device="cuda")
    plan.tensor_scale(None, scale, stream=stream())
    plan.check()
    assert scale.item() == 2.0 ** -60
    for status, args in ((1, dict(rows=-1)), (1, dict(K=0)), (3, dict(K=12)), (3, dict(ldx=68)), (1, dict(ldx=56)), (1, dict(format=2)),
                         (2, dict(in_dtype=nk.S8)), (2, dict(value_dtype=nk.E4M3)), (2, dict(groups=2, transposed=1)),
                         (2, dict(groups=2, batch=2)), (1, dict(transposed=2)), (2, dict(groups=2000)), (1, dict(batch=2, stride_x=64)),
                         (5, dict(device=99)), (2, dict(rows=1 << 24, transposed=1))):
        with pytest.raises(nk.NkError) as e:
            nk.PackPlan(**{**dict(rows=32, K=64), **args})
        assert e.value.status == status, args
    plan = nk.PackPlan(32, 64)
    x = torch.zeros(32, 64, dtype=torch.bfloat16, device="cuda")
    data = torch.empty(plan.data_bytes + 16, dtype=torch.uint8, device="cuda")
    sc = torch.empty(plan.scales_bytes + 16, dtype=torch.uint8, device="cuda")
    off = torch.zeros(2, dtype=torch.int32, device="cuda")
    for status, call in ((1, lambda: plan.run(None, data, sc)), (1, lambda: plan.run(x, data, sc, offsets=off)), (3, lambda: plan.run(x, data[1:], sc)),
                         (3, lambda: plan.run(x, data, sc[8:])), (1, lambda: nk.PackPlan(32, 64, groups=1).run(x, data, sc)),
                         (1, lambda: nk.PackPlan(32, 64, format=nk.MXF4).run(x, data, sc, scale=scale)),
                         (2, lambda: nk.PackPlan(32, 64, format=nk.MXF4).tensor_scale(x, scale)),
                         (4, lambda: nk.PackPlan(3000, 2048).tensor_scale(x, scale)), (1, lambda: plan.values(data, None, x))):
        with pytest.raises(nk.NkError) as e:
            call()
        assert e.value.status == status


def test_in_a_graph_and_on_another_stream():
    x = rows_of(200, 512, "bf16", seed=1).cuda()
    plan = nk.PackPlan(200, 512)
    data = torch.zeros(plan.data_bytes, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(plan.scales_bytes, dtype=torch.uint8, device="cuda")
    scale = torch.empty(1, device="cuda")
    ws = torch.empty(max(1, plan.workspace_bytes), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        plan.tensor_scale(x, scale, workspace=ws, stream=stream())
        plan.run(x, data, scales, scale=scale, stream=stream())
    for seed in (2, 3):
        x.copy_(rows_of(200, 512, "bf16", seed=seed, scale=float(seed)))
        graph.replay()
        torch.cuda.synchronize()
        z = x.double().cpu().numpy()
        codes, bytes_, _ = quantise(z, "nvf4", tensor_scale(z))
        assert np.array_equal(unpack_data(data.cpu().numpy(), 200, 512), one_zero(codes))
        assert np.array_equal(unpack_scales(scales.cpu().numpy(), np.arange(200), 512, "nvf4"), bytes_)
    assert padded(512) == 512 and BLOCK["nvf4"] == 16


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed,rows,K", [(0, 1, 8), (0, 33, 104), (0, 300, 1032), (1, 33, 104), (1, 64, 24), (1, 1000, 264), (1, 4099, 24)])
def test_values_of_both_formats(fmt, kind, transposed, rows, K):
    """Reading back, whole pieces of eight and odd lengths, one chunk of a row and several."""
    x = rows_of(rows, K, "bf16", seed=rows + K)
    t = tensor_scale(x.double().numpy()) if fmt == "nvf4" else 1.0
    plan, data, scales, scale, _ = pack(x, fmt, "bf16", t if fmt == "nvf4" else None, transposed=transposed, value_dtype=TYPES[kind][0])
    z = x.double().numpy()
    codes, bytes_, _ = quantise(z.T.copy() if transposed else z, fmt, t)
    check_values(plan, data, scales, scale, None, values(codes, bytes_, fmt, t, rows if transposed else K), kind)


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("offsets", [[0, 0, 130, 130, 131, 300, 300], [7, 20, 20, 290]])
def test_values_of_groups_in_16_bits(fmt, kind, offsets):
    x = rows_of(300, 264, "bf16", seed=len(offsets))
    t = 0.0078125 if fmt == "nvf4" else 1.0
    plan, data, scales, scale, off = pack(x, fmt, "bf16", t if fmt == "nvf4" else None, offsets=offsets, groups=len(offsets) - 1, value_dtype=TYPES[kind][0])
    codes, bytes_, _ = quantise(x.double().numpy(), fmt, t)
    check_values(plan, data, scales, scale, off, values(codes, bytes_, fmt, t, 264), kind, rows=group_places(offsets)[0])


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed,rows,K", [(0, 150, 200), (1, 150, 200), (1, 77, 40)])
def test_values_of_a_batch(fmt, kind, transposed, rows, K):
    """Every matrix with its own tensor scale."""
    batch = 3
    x = torch.stack([rows_of(rows, K, "bf16", seed=b, scale=10.0 ** (b - 1)) for b in range(batch)])
    plan = nk.PackPlan(rows, K, format=FORMATS[fmt], batch=batch, transposed=transposed, value_dtype=TYPES[kind][0])
    data = torch.empty(plan.data_bytes, dtype=torch.uint8, device="cuda")
    scales = torch.empty(plan.scales_bytes, dtype=torch.uint8, device="cuda")
    ts = [tensor_scale(m.double().numpy()) if fmt == "nvf4" else 1.0 for m in x]
    scale = torch.tensor(ts, dtype=torch.float32, device="cuda") if fmt == "nvf4" else None
    plan.run(x.cuda(), data, scales, scale=scale, stream=stream())
    want = []
    for m, t in zip(x, ts):
        z = m.double().numpy()
        codes, bytes_, _ = quantise(z.T.copy() if transposed else z, fmt, t)
        want.append(values(codes, bytes_, fmt, t, rows if transposed else K))
    check_values(plan, data, scales, scale, None, np.stack(want), kind)


@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("transposed", [0, 1])
def test_values_that_are_not_ordinary_read_back(fmt, kind, transposed):
    """Blocks whose scale is a NaN, the smallest or the largest; tensor scales that make every block a NaN."""
    dt = TYPES[kind][1]
    x = rows_of(64, 128, kind, seed=3)
    x[0, 5], x[1, 40], x[2, 127] = float("inf"), float("-inf"), float("nan")
    x[3] = torch.finfo(dt).max
    x[4] = torch.finfo(dt).smallest_normal
    x[5] = torch.finfo(dt).smallest_normal / 4               # subnormal
    x[6], x[7] = 0.0, -0.0
    x[8, ::32] = torch.finfo(dt).max
    x[9] = -torch.finfo(dt).max
    src = x.t().contiguous() if transposed else x
    for t in ([None] if fmt == "mxf4" else [None, 2.0 ** -20, 2.0 ** 20, 2.0 ** -100, 2.0 ** 120, float("nan"), float("inf"), 0.0, -1.0, 2.0 ** -101, 2.0 ** 121]):
        for out in ("f32", kind):
            plan, data, scales, scale, _ = pack(src, fmt, kind, t, transposed=transposed, value_dtype=TYPES[out][0])
            legal = t is None or 2.0 ** -100 <= t <= 2.0 ** 120
            codes, bytes_, _ = quantise(x.double().numpy(), fmt, 1.0 if t is None else t if legal else float("nan"))
            assert np.array_equal(unpack_scales(scales.cpu().numpy(), np.arange(64), 128, fmt), bytes_), t
            with np.errstate(all="ignore"):
                want = values(codes, bytes_, fmt, 1.0 if t is None else t, 128)
            check_values(plan, data, scales, scale, None, want, out)
