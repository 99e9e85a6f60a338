"""Cases that time the operators of layers whose weights are chosen row by row: the products grouped by
expert with their gradients, the routing around them, and the low-rank adapters beside a shared projection.

Where `own` is false every operator runs in its plain form (elementary torch operations in 32 bits, rounded
once at the end); where it is true the library's own calls run.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decoding step of a layer of many small experts: a handful of rows, nearly every weight read for one or two of them
        {"name": "experts_step", "op": "experts", "rows": 32, "groups": 64, "K": 1024, "N": 4096, "type": "bf16", "out": "bf16",
         "layout": "row"},
        # a prompt of ordinary length through a few large experts kept as [out][in], loads uneven, an odd number of rows
        {"name": "experts_prompt", "op": "experts", "rows": 4099, "groups": 8, "K": 4096, "N": 1024, "type": "f16", "out": "f16",
         "layout": "transposed"},
        # a training batch, the largest product: the tensor cores' rate counts
        {"name": "experts_batch", "op": "experts", "rows": 32768, "groups": 16, "K": 4096, "N": 4096, "type": "bf16", "out": "bf16",
         "layout": "row"},
        # the backward pass of a training batch: gradients of the rows and, in 32 bits, of the weights
        {"name": "experts_gradient", "op": "experts_gradient", "rows": 8192, "groups": 8, "K": 1024, "N": 4096, "type": "bf16",
         "out": "f32", "layout": "row"},
        # the backward pass where an expert has few rows: ragged sums over rows that end anywhere, outputs larger than inputs
        {"name": "experts_gradient_ragged", "op": "experts_gradient", "rows": 2001, "groups": 61, "K": 1024, "N": 1000, "type": "f16",
         "out": "f16", "layout": "transposed"},
        # one decoding step of a batch of requests, each with an adapter of its own
        {"name": "adapters_step", "op": "adapters", "rows": 16, "requests": 16, "K": 4096, "N": 4096, "rank": 16, "adapters": 32,
         "type": "bf16", "out": "bf16", "layout": "transposed"},
        # decoding requests and a few prompts in one batch
        {"name": "adapters_mixed", "op": "adapters", "rows": 1021, "requests": 29, "K": 4096, "N": 1024, "rank": 32, "adapters": 16,
         "type": "bf16", "out": "bf16", "layout": "row"},
        # long prompts, higher rank
        {"name": "adapters_prompt", "op": "adapters", "rows": 8192, "requests": 5, "K": 4096, "N": 4096, "rank": 64, "adapters": 8,
         "type": "f16", "out": "f16", "layout": "transposed"},
        # routing of one decoding step: latency
        {"name": "route_step", "op": "route", "tokens": 16, "experts": 64, "topk": 2, "type": "f32", "renormalise": True},
        # routing of a training batch with its gradient
        {"name": "route_batch", "op": "route", "tokens": 16384, "experts": 128, "topk": 8, "type": "f32", "renormalise": False},
        # rows out to their experts' order and back, weighted
        {"name": "exchange_prompt", "op": "exchange", "tokens": 8192, "experts": 16, "topk": 2, "width": 4096, "type": "bf16"},
        # the gradient of the weighted sum: of the experts' rows and of the weights
        {"name": "exchange_gradient", "op": "exchange_gradient", "tokens": 4096, "experts": 64, "topk": 8, "width": 1024, "type": "bf16"},
    ]


def _spread(rng, low, high, step=1):
    """A whole multiple of `step` between low and high, spread over the logarithm."""
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + step)))) // step * step))


def draw(rng):
    op = rng.choice(["experts", "experts_gradient", "adapters", "route", "exchange", "exchange_gradient"])
    if op in ("experts", "experts_gradient"):
        while True:
            c = {"op": op, "rows": _spread(rng, 1, 32768), "groups": _spread(rng, 1, 128), "K": _spread(rng, 64, 4096, 8),
                 "N": _spread(rng, 64, 4096, 8), "type": rng.choice(["bf16", "f16"])}
            if c["groups"] * c["K"] * c["N"] <= 1 << 28 and (op == "experts" or c["rows"] <= 16384):
                break
        c["out"] = rng.choice([c["type"], c["type"], "f32"])
        c["layout"] = rng.choice(["row", "transposed"])
        return c
    if op == "adapters":
        rows = _spread(rng, 1, 8192)
        kind = rng.choice(["bf16", "f16"])
        return {"op": op, "rows": rows, "requests": _spread(rng, 1, min(rows, 256)), "K": _spread(rng, 64, 4096, 8),
                "N": _spread(rng, 64, 4096, 8), "rank": _spread(rng, 8, 128, 8), "adapters": _spread(rng, 1, 64), "type": kind,
                "out": rng.choice([kind, kind, "f32"]), "layout": rng.choice(["row", "transposed"])}
    experts = _spread(rng, 2, 256)
    topk = rng.randint(1, min(8, experts))
    if op == "route":
        return {"op": op, "tokens": _spread(rng, 1, 32768), "experts": experts, "topk": topk,
                "type": rng.choice(["f32", "bf16", "f16"]), "renormalise": rng.random() < 0.5}
    while True:
        c = {"op": op, "tokens": _spread(rng, 1, 16384), "experts": experts, "topk": topk, "width": _spread(rng, 64, 4096, 8),
             "type": rng.choice(["bf16", "f16"])}
        if c["tokens"] * c["topk"] * c["width"] <= 1 << 27:
            return c


def _bytes_of(kind):
    return 4 if kind == "f32" else 2


def work(case):
    """What one pass cannot do without.  Weights that no row needs are not counted: which ones those are goes by the rows of the
    case, so the expected number of groups with a row stands for it (the loads are drawn as in prepare)."""
    op = case["op"]
    if op in ("experts", "experts_gradient"):
        rows, G, K, N = case["rows"], case["groups"], case["K"], case["N"]
        b, o = _bytes_of(case["type"]), _bytes_of(case["out"])
        live = sum(1.0 - (1.0 - q) ** rows for q in _loads(G))
        if op == "experts":
            return {"bytes": b * (rows * K + live * K * N) + o * rows * N, "flops": 2.0 * rows * K * N}
        # rows and their gradient read once, the weights read once, both gradients written
        return {"bytes": b * (rows * K + rows * N + live * K * N) + b * rows * K + o * G * K * N, "flops": 4.0 * rows * K * N}
    if op == "adapters":
        rows, K, N, r = case["rows"], case["K"], case["N"], case["rank"]
        b, o = _bytes_of(case["type"]), _bytes_of(case["out"])
        live = case["adapters"] * (1.0 - (1.0 - 0.9 / case["adapters"]) ** case["requests"])
        return {"bytes": b * (rows * K + K * N + live * r * (K + N)) + o * rows * N,
                "flops": 2.0 * rows * K * N + 2.0 * rows * r * (K + N)}
    T, E, k = case["tokens"], case["experts"], case["topk"]
    if op == "route":
        b = _bytes_of(case["type"])
        # logits in, weights + experts + places + offsets out; then the weights' gradient in and the logits' gradient out
        return {"bytes": T * E * b + T * k * 12 + 4 * (E + 1) + T * k * 4 + T * E * 4, "flops": 10.0 * T * E}
    D = case["width"]
    b = _bytes_of(case["type"])
    if op == "exchange":   # rows in, k copies out; k rows in, one out
        return {"bytes": T * D * b * (1 + k) + T * D * b * (k + 1) + T * k * 12, "flops": 2.0 * T * k * D}
    return {"bytes": T * D * b + 2 * T * k * D * b + T * k * 12, "flops": 3.0 * T * k * D}


# ------------------------------------------------------------------------------------------------ inputs
def _loads(groups):
    """Shares of the rows that the experts get: uneven, the last ones almost nothing."""
    w = [1.0 / (1.0 + i) ** 0.6 for i in range(groups)]
    s = sum(w)
    return [x / s for x in w]


def _ragged(rows, groups, g):
    """Row offsets of the groups, whole numbers from the seed; empty groups occur."""
    share = torch.tensor(_loads(groups), dtype=torch.float64)[torch.randperm(groups, generator=g)]
    which = torch.multinomial(share, rows, replacement=True, generator=g)
    return torch.cat([torch.zeros(1, dtype=torch.int64), torch.bincount(which, minlength=groups).cumsum(0)])


def _normal(shape, scale, kind, g):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(TYPES[kind])


def _weights(groups, K, N, kind, g):
    """Weights of a linear layer, by group so that the 32-bit values need little room."""
    w = torch.empty(groups, K, N, dtype=TYPES[kind], device="cuda")
    step = max(1, (1 << 26) // (K * N))
    for i in range(0, groups, step):
        w[i:i + step] = _normal((min(step, groups - i), K, N), K ** -0.5, kind, g)
    return w


def prepare(case, seed):
    host = torch.Generator().manual_seed(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = dict(case)
    if own:
        import paper_2511_13764_b200 as nk
        nk_type = {"bf16": nk.BF16, "f16": nk.F16, "f32": nk.F32}
        nk_layout = {"row": nk.ROW_MAJOR, "transposed": nk.TRANSPOSED}

    def scratch(*plans):
        return torch.empty(max(1, max(p.workspace_bytes for p in plans)), dtype=torch.uint8, device="cuda")

    if op in ("experts", "experts_gradient"):
        rows, G, K, N, kind = case["rows"], case["groups"], case["K"], case["N"], case["type"]
        off = _ragged(rows, G, host)
        s["most"] = int((off[1:] - off[:-1]).max())
        s["offsets"] = off.to(torch.int32).cuda()
        s["x"] = _normal((rows, K), 1.0, kind, g)
        # the weights [G][K][N], or the way a linear layer keeps them: [G][N][K]
        s["w"] = _weights(G, K, N, kind, g) if case["layout"] == "row" else _weights(G, N, K, kind, g).mul_((N / K) ** 0.5)
        if op == "experts_gradient":
            s["dy"] = _normal((rows, N), 1.0, kind, g)
        if own:
            layout = nk_layout[case["layout"]]
            if op == "experts":
                s["plan"] = nk.GroupedPlan(G, rows, N, K, in_dtype=nk_type[kind], out_dtype=nk_type[case["out"]], layout_b=layout)
                s["y"] = torch.empty(rows, N, dtype=TYPES[case["out"]], device="cuda")
                s["scratch"] = scratch(s["plan"])
            else:
                # dX = dY . W^T: the same product with the weights' two layouts exchanged
                back = nk.TRANSPOSED if layout == nk.ROW_MAJOR else nk.ROW_MAJOR
                s["plan_rows"] = nk.GroupedPlan(G, rows, K, N, in_dtype=nk_type[kind], out_dtype=nk_type[kind], layout_b=back)
                # dW = X^T . dY, or its transpose, in the weights' own layout
                a, b = (K, N) if case["layout"] == "row" else (N, K)
                s["plan_weights"] = nk.GroupedPlan(G, rows, b, a, kind=nk.GROUPED_WEIGHTS, in_dtype=nk_type[kind],
                                                   out_dtype=nk_type[case["out"]])
                s["dx"] = torch.empty(rows, K, dtype=TYPES[kind], device="cuda")
                s["dw"] = torch.empty(G, a, b, dtype=TYPES[case["out"]], device="cuda")
                s["scratch"] = scratch(s["plan_rows"], s["plan_weights"])
    elif op == "adapters":
        rows, R, K, N, r, L, kind = (case[n] for n in ("rows", "requests", "K", "N", "rank", "adapters", "type"))
        # most requests bring one row (a decoding step), the rest of the rows are prompts of a few requests
        prompts = max(1, R // 8)
        extra = torch.multinomial(torch.rand(prompts, generator=host) + 0.1, rows - R, replacement=True, generator=host) if rows > R else None
        lens = torch.ones(R, dtype=torch.int64)
        if extra is not None:
            lens[torch.randperm(R, generator=host)[:prompts]] += torch.bincount(extra, minlength=prompts)
        off = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
        which = torch.randint(0, L, (R,), generator=host)
        which[torch.rand(R, generator=host) < 0.1] = -1          # requests without an adapter
        s["most"] = int(lens.max())
        s["offsets"], s["adapter"] = off.to(torch.int32).cuda(), which.to(torch.int32).cuda()
        s["x"] = _normal((rows, K), 1.0, kind, g)
        s["scale"] = (0.5 + 1.5 * torch.rand(L, generator=host)).cuda()
        if case["layout"] == "row":
            s["w"], s["a"], s["b"] = _weights(1, K, N, kind, g)[0], _weights(L, K, r, kind, g), _weights(L, r, N, kind, g)
        else:
            s["w"] = _weights(1, N, K, kind, g)[0].mul_((N / K) ** 0.5)
            s["a"], s["b"] = _weights(L, r, K, kind, g).mul_((r / K) ** 0.5), _weights(L, N, r, kind, g).mul_((N / r) ** 0.5)
        if own:
            s["plan"] = nk.LoraPlan(rows, N, K, r, L, R, in_dtype=nk_type[kind], out_dtype=nk_type[case["out"]],
                                    layout=nk_layout[case["layout"]])
            s["y"] = torch.empty(rows, N, dtype=TYPES[case["out"]], device="cuda")
            s["scratch"] = scratch(s["plan"])
    else:
        T, E, k, kind = case["tokens"], case["experts"], case["topk"], case["type"]
        # logits of a router: some experts are liked by all tokens; 16-bit ones have ties
        logits = torch.randn(T, E, generator=g, device="cuda") * 1.5 + torch.randn(E, generator=g, device="cuda")
        if op == "route":
            s["logits"] = logits.to(TYPES[kind])
            s["dgates"] = torch.randn(T, k, generator=g, device="cuda")
            if own:
                s["plan"] = nk.RoutePlan(T, E, k, logits_dtype=nk_type[kind], renormalise=int(case["renormalise"]))
                s["scratch"] = scratch(s["plan"])
                i32 = {"dtype": torch.int32, "device": "cuda"}
                s["out"] = {"gates": torch.empty(T, k, device="cuda"), "experts": torch.empty(T, k, **i32),
                            "offsets": torch.empty(E + 1, **i32), "slots": torch.empty(T, k, **i32),
                            "dlogits": torch.empty(T, E, device="cuda")}
        else:
            D = case["width"]
            gates, chosen = torch.topk(torch.softmax(logits, 1), k, dim=1)
            s["gates"] = (gates / gates.sum(1, keepdim=True)).contiguous()
            order = torch.argsort(chosen.reshape(-1), stable=True)
            slots = torch.empty_like(order)
            slots[order] = torch.arange(T * k, device="cuda")
            s["slots"] = slots.reshape(T, k).to(torch.int32)
            s["x"] = _normal((T, D), 1.0, kind, g)               # the rows, or the gradient of the summed rows
            s["ys"] = _normal((T * k, D), 1.0, kind, g)          # the experts' rows
            if own:
                s["plan"] = nk.RoutePlan(T, E, k, width=D, dtype=nk_type[kind])
                s["xs"] = torch.empty(T * k, D, dtype=TYPES[kind], device="cuda")
                s["y"] = torch.empty(T, D, dtype=TYPES[kind], device="cuda")
                s["dgates"] = torch.empty(T, k, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    st = torch.cuda.current_stream().cuda_stream
    op = s["op"]
    if op == "experts":
        s["plan"].run(s["x"], s["w"], s["y"], s["offsets"], workspace=s["scratch"], stream=st)
        return s["y"]
    if op == "experts_gradient":
        s["plan_rows"].run(s["dy"], s["w"], s["dx"], s["offsets"], workspace=s["scratch"], stream=st)
        a, b = (s["x"], s["dy"]) if s["layout"] == "row" else (s["dy"], s["x"])
        s["plan_weights"].run(a, b, s["dw"], s["offsets"], workspace=s["scratch"], stream=st)
        return [s["dx"], s["dw"]]
    if op == "adapters":
        s["plan"].run(s["x"], s["w"], s["a"], s["b"], s["scale"], s["offsets"], s["adapter"], s["y"], workspace=s["scratch"], stream=st)
        return s["y"]
    if op == "route":
        o = s["out"]
        s["plan"].run(s["logits"], o["gates"], o["experts"], o["offsets"], o["slots"], workspace=s["scratch"], stream=st)
        s["plan"].backward(s["logits"], o["experts"], s["dgates"], o["dlogits"], stream=st)
        return o
    if op == "exchange":
        s["plan"].dispatch(s["x"], s["slots"], s["xs"], stream=st)
        s["plan"].combine(s["ys"], s["slots"], s["y"], gates=s["gates"], stream=st)
        return [s["xs"], s["y"]]
    s["plan"].combine_backward(s["x"], s["ys"], s["slots"], s["gates"], s["xs"], s["dgates"], stream=st)
    return [s["xs"], s["dgates"]]


def _padded(offsets, most):
    """Row numbers [groups][most] of the groups' rows, and which of them there are."""
    idx = offsets[:-1, None].long() + torch.arange(most, device="cuda")
    return idx, idx < offsets[1:, None]


def _take(x, idx, live):
    return x[idx.clamp(max=x.shape[0] - 1)].float() * live[..., None]


def _run_plain(s):
    op = s["op"]
    if op == "experts":
        idx, live = _padded(s["offsets"], s["most"])
        w = s["w"].float()
        y = torch.bmm(_take(s["x"], idx, live), w if s["layout"] == "row" else w.transpose(1, 2))
        out = torch.empty(s["rows"], s["N"], dtype=TYPES[s["out"]], device="cuda")
        out[idx[live]] = y[live].to(out.dtype)
        return out
    if op == "experts_gradient":
        idx, live = _padded(s["offsets"], s["most"])
        w = s["w"].float()
        dy, x = _take(s["dy"], idx, live), _take(s["x"], idx, live)
        dx = torch.empty_like(s["x"])
        dx[idx[live]] = torch.bmm(dy, w.transpose(1, 2) if s["layout"] == "row" else w)[live].to(dx.dtype)
        a, b = (x, dy) if s["layout"] == "row" else (dy, x)
        return [dx, torch.bmm(a.transpose(1, 2), b).to(TYPES[s["out"]])]
    if op == "adapters":
        idx, live = _padded(s["offsets"], s["most"])
        rows = s["layout"] == "row"
        which = s["adapter"].clamp(min=0).long()
        scale = torch.where(s["adapter"] >= 0, s["scale"][which], torch.zeros((), device="cuda"))
        a, b, w = s["a"][which].float(), s["b"][which].float(), s["w"].float()
        if not rows:
            a, b, w = a.transpose(1, 2), b.transpose(1, 2), w.t()
        h = torch.bmm(_take(s["x"], idx, live), a) * scale[:, None, None]
        y = torch.mm(s["x"].float(), w)
        y[idx[live]] += torch.bmm(h, b)[live]
        return y.to(TYPES[s["out"]])
    if op == "route":
        k = s["topk"]
        z = s["logits"].float()
        T, E = z.shape
        # the largest first, ties by the lower index
        chosen = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
        e = torch.exp(z - z.amax(1, keepdim=True))
        p = e / e.sum(1, keepdim=True)
        top = p.gather(1, chosen)
        gates = top / top.sum(1, keepdim=True) if s["renormalise"] else top
        flat = chosen.reshape(-1)
        order = torch.sort(flat, stable=True).indices
        slots = torch.empty_like(flat)
        slots[order] = torch.arange(T * k, device="cuda")
        counts = torch.zeros(E, dtype=torch.int64, device="cuda").scatter_add_(0, flat, torch.ones_like(flat))
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)])
        # gradient: d gate_j / d logit_i = gate_j (delta_ij - share_i), shares over the selected or over all experts
        dg = s["dgates"]
        inner = (dg * gates).sum(1, keepdim=True)
        if s["renormalise"]:
            dz = torch.zeros_like(z).scatter_(1, chosen, gates * (dg - inner))
        else:
            dz = (-p * inner).scatter_add_(1, chosen, gates * dg)
        return {"gates": gates, "experts": chosen.int(), "offsets": offsets.int(), "slots": slots.reshape(T, k).int(), "dlogits": dz}
    T, k, D = s["tokens"], s["topk"], s["width"]
    at = s["slots"].long()
    if op == "exchange":
        xs = torch.empty(T * k, D, dtype=s["x"].dtype, device="cuda")
        xs[at.reshape(-1)] = s["x"].repeat_interleave(k, 0)
        y = (s["ys"][at].float() * s["gates"][..., None]).sum(1).to(s["ys"].dtype)
        return [xs, y]
    d = s["x"].float()[:, None, :]
    dys = torch.empty(T * k, D, dtype=s["x"].dtype, device="cuda")
    dys[at.reshape(-1)] = (d * s["gates"][..., None]).to(dys.dtype).reshape(T * k, D)
    return [dys, (s["ys"][at].float() * d).sum(-1)]


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    op = case["op"]
    if op in ("experts", "experts_gradient"):
        ends = s["offsets"].tolist()
        of = (lambda m: m.to(f64)) if case["layout"] == "row" else (lambda m: m.to(f64).t())   # noqa: E731
        if op == "experts":
            return torch.cat([s["x"][lo:hi].to(f64) @ of(s["w"][e]) for e, (lo, hi) in enumerate(zip(ends, ends[1:]))])
        dx = torch.cat([s["dy"][lo:hi].to(f64) @ of(s["w"][e]).t() for e, (lo, hi) in enumerate(zip(ends, ends[1:]))])
        dw = torch.empty(s["w"].shape, dtype=f64, device="cuda")
        for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
            g = s["x"][lo:hi].to(f64).t() @ s["dy"][lo:hi].to(f64)
            dw[e] = g if case["layout"] == "row" else g.t()
        return [dx, dw]
    if op == "adapters":
        ends, which = s["offsets"].tolist(), s["adapter"].tolist()
        of = (lambda m: m.to(f64)) if case["layout"] == "row" else (lambda m: m.to(f64).t())   # noqa: E731
        y = s["x"].to(f64) @ of(s["w"])
        for lo, hi, a in zip(ends, ends[1:], which):
            if a >= 0:
                y[lo:hi] += s["scale"][a].to(f64) * (s["x"][lo:hi].to(f64) @ of(s["a"][a]) @ of(s["b"][a]))
        return y
    if op == "route":
        z = s["logits"].to(f64)
        chosen = torch.argsort(-z, dim=1, stable=True)[:, : case["topk"]]
        picked = torch.zeros_like(z, dtype=torch.bool).scatter_(1, chosen, True)
        base = torch.where(picked, z, torch.full_like(z, -math.inf)) if case["renormalise"] else z
        share = torch.softmax(base, 1)
        gates = share.gather(1, chosen)
        up = torch.zeros_like(z).scatter_(1, chosen, s["dgates"].to(f64))
        return {"gates": gates, "experts": None, "offsets": None, "slots": None,
                "dlogits": share * (up - (share * up).sum(1, keepdim=True))}
    at = s["slots"].long()
    g = s["gates"].to(f64)
    if op == "exchange":
        y = torch.zeros(s["x"].shape, dtype=f64, device="cuda")
        xs = torch.zeros(s["ys"].shape, dtype=f64, device="cuda")
        for j in range(case["topk"]):
            y += g[:, j, None] * s["ys"][at[:, j]].to(f64)
            xs[at[:, j]] = s["x"].to(f64)
        return [xs, y]
    d = s["x"].to(f64)
    dys, dg = torch.zeros(s["ys"].shape, dtype=f64, device="cuda"), torch.zeros(g.shape, dtype=f64, device="cuda")
    for j in range(case["topk"]):
        dys[at[:, j]] = g[:, j, None] * d
        dg[:, j] = (s["ys"][at[:, j]].to(f64) * d).sum(1)
    return [dys, dg]
