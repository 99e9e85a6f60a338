"""Routing (nk_route): choice, gates, places, exchange of rows and all gradients, against plain 64-bit formulas.

Tolerances: a gate is exp(z - m) / sum in FP32.  z - m is rounded once (relative error of the exponential
|z - m| 2^-24), expf is good to 2 units in the last place, and at most 32 + 5 partial sums are rounded, each by 2^-24
of the sum of non-negative terms; with |z - m| <= 24 where it matters that is below (24 + 4 + 37 + 2) 2^-24 = 4e-6
of the gate.  A gradient is p (d - sum d g): the same relative error on each factor, so 1.2e-5 * p (|d| + sum |d| g)."""
import numpy as np
import pytest
import torch

import paper_2511_13764_b200 as nk
from nk_testlib import TOL_BF16_REL, TOL_F16_ABS, TOL_F16_REL

GATE_REL = 4e-6
TYPES = {"bf16": (nk.BF16, torch.bfloat16), "f16": (nk.F16, torch.float16), "f32": (nk.F32, torch.float32)}


def stream():
    return torch.cuda.current_stream().cuda_stream


def reference(z, k, renormalise):
    """Choice, gates and places in 64 bits on the CPU, straight from the definitions."""
    z = z.double()
    T, E = z.shape
    rank = torch.where(z.isnan(), torch.full_like(z, -np.inf), z)
    # NaN below minus infinity: sort by (is NaN, -value), stable
    order = torch.argsort(-rank, dim=1, stable=True)
    order = order.gather(1, torch.argsort(z.gather(1, order).isnan().int(), dim=1, stable=True))
    chosen = order[:, :k]
    picked = torch.zeros(T, E, dtype=torch.bool).scatter_(1, chosen, True)
    base = torch.where(picked, z, torch.full_like(z, -np.inf)) if renormalise else z
    p = torch.softmax(base, 1)
    nan = z.isnan().any(1, keepdim=True)
    p = torch.where(((z == -np.inf).all(1, keepdim=True)), torch.zeros_like(p), p)
    p = torch.where(nan, torch.full_like(p, np.nan), p)
    flat = chosen.reshape(-1)
    order = torch.argsort(flat, stable=True)
    slots = torch.empty_like(flat)
    slots[order] = torch.arange(flat.numel())
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), torch.bincount(flat, minlength=E).cumsum(0)])
    return chosen, p.gather(1, chosen), offsets, slots.reshape(T, k), p


def route(z, k, kind="f32", renormalise=1, ld=0):
    T, E = z.shape
    plan = nk.RoutePlan(T, E, k, logits_dtype=TYPES[kind][0], renormalise=renormalise, ld_logits=ld)
    buf = torch.full((max(T, 1), ld or E), float("nan"), dtype=TYPES[kind][1])
    buf[:T, :E] = z
    d = buf.cuda()
    out = [torch.full((T, k), -9.0, device="cuda")] + [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((T, k), (E + 1,), (T, k))]
    ws = torch.full((max(16, plan.workspace_bytes),), 255, dtype=torch.uint8, device="cuda")
    plan.run(d, *out, workspace=ws, stream=stream())
    plan.check()
    return plan, d, out


def logits(T, E, seed, kind="f32"):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, E, generator=g) * 2 + torch.randn(E, generator=g)
    return z.to(TYPES[kind][1])


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 2), (5, 3, 3), (16, 64, 2), (64, 33, 32), (65, 128, 8), (200, 1024, 32), (64, 1024, 4),
                                   (1000, 8, 1), (3001, 257, 6), (16384, 16, 2), (0, 12, 3)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("renormalise", [0, 1])
def test_route(T, E, k, kind, renormalise):
    z = logits(T, E, 100 + T + E, kind)               # 16-bit logits bring ties
    _, _, (gates, chosen, offsets, slots) = route(z, k, kind, renormalise, ld=E + 5)
    c, g, o, s, _ = reference(z, k, renormalise)
    assert torch.equal(chosen.cpu().long(), c) and torch.equal(offsets.cpu().long(), o) and torch.equal(slots.cpu().long(), s)
    assert ((gates.cpu().double() - g).abs() <= GATE_REL * g + 1e-30).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 300])
@pytest.mark.parametrize("renormalise", [0, 1])
def test_ties_masks_and_special_values(T, renormalise):
    E, k = 40, 4
    z = logits(T, E, 7)
    z[0] = 0.0                                        # all alike: the lowest indices
    z[1] = torch.where(torch.arange(E) % 2 == 0, 0.0, -0.0)   # both zeros are alike
    z[2, :] = -np.inf                                 # nothing may be chosen
    z[3, :] = -np.inf
    z[3, 17] = 1.0                                    # one left
    z[4, 10:] = -np.inf
    z[5, 3] = np.nan
    z[6] = np.nan
    z[7] = torch.finfo(torch.float32).min             # the type's lowest value is an ordinary number
    z[8, 5] = np.inf
    z[9, :38] = np.nan                                # fewer numbers than choices
    plan, d, (gates, chosen, offsets, slots) = route(z, k, renormalise=renormalise)
    c, g, o, s, p = reference(z, k, renormalise)
    assert torch.equal(chosen.cpu().long(), c) and torch.equal(offsets.cpu().long(), o) and torch.equal(slots.cpu().long(), s)
    got = gates.cpu().double()
    assert torch.equal(got.isnan(), g.isnan())
    assert ((got - g).abs().nan_to_num(0) <= GATE_REL * g.nan_to_num(0) + 1e-30).all()
    assert (got[2] == 0).all() and got[3, 0] == 1 and (got[3, 1:] == 0).all()
    dg = torch.randn(T, k, generator=torch.Generator().manual_seed(8))
    dz = torch.full((T, E), -9.0, device="cuda")
    plan.backward(d, chosen, dg.cuda(), dz, stream=stream())
    plan.check()
    dz = dz.cpu().double()
    assert (dz[2] == 0).all() and dz[[5, 6, 9]].isnan().all() and dz[8].isnan().any()
    keep = [t for t in range(T) if t not in (5, 6, 8, 9)]
    assert dz[keep].isfinite().all() and (dz[4, 10:] == 0).all()
    if renormalise:
        free = torch.ones(T, E, dtype=torch.bool).scatter_(1, c, False)
        assert (dz[keep][free[keep]] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 5, 2), (100, 64, 6), (33, 1000, 32), (2000, 128, 8)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("renormalise", [0, 1])
def test_backward_against_the_formula(T, E, k, kind, renormalise):
    z = logits(T, E, 200 + T, kind)
    plan, d, (gates, chosen, _, _) = route(z, k, kind, renormalise)
    dg = torch.randn(T, k, generator=torch.Generator().manual_seed(9))
    dz = torch.full((T, E), float("nan"), device="cuda")
    plan.backward(d, chosen, dg.cuda(), dz, stream=stream())
    plan.check()
    c, g, _, _, p = reference(z, k, renormalise)
    up = torch.zeros(T, E, dtype=torch.float64).scatter_(1, c, dg.double())
    want = p * (up - (p * up).sum(1, keepdim=True))
    tol = 1.2e-5 * p * (up.abs() + (p * up.abs()).sum(1, keepdim=True)) + 1e-30
    assert ((dz.cpu().double() - want).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("renormalise", [0, 1])
def test_backward_against_differences(renormalise):
    T, E, k = 6, 12, 3
    z = logits(T, E, 11)
    plan, d, (_, chosen, _, _) = route(z, k, renormalise=renormalise)
    dg = torch.randn(T, k, generator=torch.Generator().manual_seed(12))
    dz = torch.empty(T, E, device="cuda")
    plan.backward(d, chosen, dg.cuda(), dz, stream=stream())
    plan.check()
    c = chosen.cpu().long()

    def loss(x):
        base = x if not renormalise else torch.where(torch.zeros(T, E, dtype=torch.bool).scatter_(1, c, True), x, torch.full_like(x, -np.inf))
        return float((torch.softmax(base, 1).gather(1, c) * dg.double()).sum())

    h = 1e-4                                          # central differences: error below h^2 * third derivative (< 10) and 1e-12 / h
    for t in range(T):
        for e in range(E):
            x = z.double()
            up, down = x.clone(), x.clone()
            up[t, e] += h
            down[t, e] -= h
            assert abs((loss(up) - loss(down)) / (2 * h) - float(dz[t, e])) <= 1e-5


def places(T, k, E, seed):
    g = torch.Generator().manual_seed(seed)
    flat = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).reshape(-1)
    order = torch.argsort(flat, stable=True)
    slots = torch.empty_like(flat)
    slots[order] = torch.arange(T * k)
    return slots.reshape(T, k).int()


def strided(x, ld):
    buf = torch.full((x.shape[0], ld), float("nan"), dtype=x.dtype)
    buf[:, : x.shape[1]] = x
    return buf.cuda()


def rounding(kind, want):
    return {"bf16": TOL_BF16_REL, "f16": TOL_F16_REL}[kind] * want.abs() + (TOL_F16_ABS if kind == "f16" else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("T,k,D", [(1, 1, 8), (3, 2, 64), (17, 8, 1000), (257, 3, 136), (64, 32, 4096), (700, 2, 2048)])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("drop", [False, True])
def test_exchange_of_rows(T, k, D, kind, drop):
    g = torch.Generator().manual_seed(T + D)
    dt = TYPES[kind][1]
    slots = places(T, k, max(k, 40), T)
    if drop:                                          # dropped pairs: out of range on either side; their rows hold NaN
        gone = torch.rand(T, k, generator=g) < 0.3
        lost = slots[gone].long()
        slots = torch.where(gone, torch.where(torch.rand(T, k, generator=g) < 0.5, -1, T * k), slots).int()
    X, Ys, dY = (torch.randn(n, D, generator=g).to(dt) for n in (T, T * k, T))
    if drop:
        Ys[lost] = float("nan")
    gates = torch.rand(T, k, generator=g)
    ldt, lds = D + 8, D + 24
    plan = nk.RoutePlan(T, max(k, 40), k, width=D, dtype=TYPES[kind][0], ld_tokens=ldt, ld_slots=lds)
    dX, dYs_in, ddY, dS, dG = strided(X, ldt), strided(Ys, lds), strided(dY, ldt), slots.cuda(), gates.cuda()
    live = (slots >= 0) & (slots < T * k)
    at = slots.clamp(0, T * k - 1).long()
    # dispatch: bits are copied; a place nobody takes is left alone
    Xs = torch.full((T * k, lds), 7.0, dtype=dt, device="cuda")
    plan.dispatch(dX, dS, Xs, stream=stream())
    want = torch.full((T * k, lds), 7.0, dtype=dt)
    want[at[live], :D] = X.repeat_interleave(k, 0).reshape(T, k, D)[live]
    assert torch.equal(Xs.cpu(), want)
    # combine, weighted and plain: k products and sums of FP32, each off by 2^-24 of the partial sums
    rows = torch.where(live[..., None], Ys.double()[at], 0.0)
    for w, gd in ((gates.double(), dG), (torch.ones(T, k, dtype=torch.float64), None)):
        Y = torch.full((T, ldt), 7.0, dtype=dt, device="cuda")
        plan.combine(dYs_in, dS, Y, gates=gd, stream=stream())
        ref = (rows * w[..., None]).sum(1)
        size = (rows.abs() * w[..., None]).sum(1)
        got = Y.cpu()
        assert (got[:, D:] == 7.0).all()
        assert ((got[:, :D].double() - ref).abs() <= rounding(kind, ref) * (1 + 1e-5) + (k + 1) * 2.0 ** -24 * size).all()
    # its gradient
    dYs = torch.full((T * k, lds), 7.0, dtype=dt, device="cuda")
    dgates = torch.full((T, k), 7.0, device="cuda")
    plan.combine_backward(ddY, dYs_in, dS, dG, dYs, dgates, stream=stream())
    plan.check()
    want = torch.full((T * k, lds), 7.0, dtype=torch.float64)
    prod = gates.double()[..., None] * dY.double()[:, None, :]
    want[at[live], :D] = prod[live]
    got = dYs.cpu()
    # the product is rounded to FP32 before its own rounding: half a unit more in 2^-16 of the cases
    assert ((got.double() - want).abs() <= rounding(kind, want) * (1 + 1e-5) + 2.0 ** -24 * want.abs()).all()
    ref = (rows * dY.double()[:, None, :]).sum(-1)
    size = (rows * dY.double()[:, None, :]).abs().sum(-1)
    got = dgates.cpu().double()
    assert (got[~live] == 0).all()
    assert ((got - ref).abs() <= (D / 32 + 6) * 2.0 ** -24 * size + 1e-30).all()


@pytest.mark.gpu
def test_exchange_gradient_against_differences():
    T, k, D = 5, 2, 16
    g = torch.Generator().manual_seed(3)
    slots = places(T, k, 6, 4)
    Ys, dY, gates = torch.randn(T * k, D, generator=g).bfloat16(), torch.randn(T, D, generator=g).bfloat16(), torch.rand(T, k, generator=g)
    plan = nk.RoutePlan(T, 6, k, width=D)
    dYs, dgates = torch.empty(T * k, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, k, device="cuda")
    plan.combine_backward(dY.cuda(), Ys.cuda(), slots.cuda(), gates.cuda(), dYs, dgates, stream=stream())
    plan.check()
    at = slots.long()
    loss = lambda y, w: float(((y[at] * w[..., None]).sum(1) * dY.double()).sum())   # noqa: E731  (bilinear: differences are exact)
    y, w = Ys.double(), gates.double()
    ey, ew = torch.randn(y.shape, generator=g).double(), torch.randn(w.shape, generator=g).double()
    num = (loss(y + ey, w) - loss(y - ey, w)) / 2
    assert abs(num - float((dYs.cpu().double() * ey).sum())) <= 2.0 ** -8 * float((dYs.cpu().double() * ey).abs().sum())
    num = (loss(y, w + ew) - loss(y, w - ew)) / 2
    assert abs(num - float((dgates.cpu().double() * ew).sum())) <= 1e-5 * float((dgates.cpu().double() * ew).abs().sum())


@pytest.mark.gpu
def test_run_refusals():
    plan = nk.RoutePlan(300, 16, 2, width=64)
    z, f, i = torch.zeros(300, 64, device="cuda"), torch.zeros(4096, device="cuda"), torch.zeros(4096, dtype=torch.int32, device="cuda")
    x = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    assert plan.workspace_bytes > 0
    calls = [(plan.run, (None, f, i, i, i), dict(workspace=ws), 1), (plan.run, (z, f, i, None, i), dict(workspace=ws), 1),
             (plan.run, (z, f, i, i, i), {}, 4), (plan.run, (z, f, i, i, i), dict(workspace=ws, workspace_bytes=ws.numel() - 1), 4),
             (plan.run, (z.data_ptr() + 2, f, i, i, i), dict(workspace=ws), 3),
             (plan.backward, (z, i, None, z), {}, 1), (plan.dispatch, (x, None, x), {}, 1), (plan.dispatch, (x[1:], i, x), {}, 3),
             (plan.combine, (x, i, x[4:]), {}, 3), (plan.combine_backward, (x, x, i, None, x, f), {}, 1)]
    for call, args, kw, status in calls:
        with pytest.raises(nk.NkError) as e:
            call(*args, **kw)
        assert e.value.status == status
    bare = nk.RoutePlan(300, 16, 2)                   # no rows: nothing to exchange
    for call, args in ((bare.dispatch, (x, i, x)), (bare.combine, (x, i, x)), (bare.combine_backward, (x, x, i, f, x, f))):
        with pytest.raises(nk.NkError) as e:
            call(*args)
        assert e.value.status == 1


@pytest.mark.parametrize("kw,status", [
    (dict(tokens=-1), 1), (dict(experts=0), 1), (dict(topk=0), 1), (dict(topk=9), 1), (dict(width=-8), 1), (dict(logits_dtype=11), 1),
    (dict(logits_dtype=nk.S8), 2), (dict(dtype=nk.F32), 2), (dict(dtype=-1), 1), (dict(renormalise=2), 1), (dict(experts=1025), 2),
    (dict(experts=64, topk=33), 2), (dict(width=12), 3), (dict(ld_tokens=68), 3), (dict(ld_tokens=32), 1), (dict(ld_slots=8), 1),
    (dict(ld_logits=7), 1), (dict(tokens=(1 << 24) + 1), 2),
])
def test_descriptor_refusals_need_no_device(kw, status):
    args = dict(tokens=10, experts=8, topk=2, width=64)
    args.update(kw)
    with pytest.raises(nk.NkError) as e:
        nk.RoutePlan(**args)
    assert e.value.status == status
