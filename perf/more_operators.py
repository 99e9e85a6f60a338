"""Cases that time the operators in 4-bit floating point (packing, products, products grouped by expert, a layer's
gradients) and the balance of a router's loads.

A 4-bit element is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; a block of elements that lie side by side along the
contraction has a scale:

    mxf4   32 elements, scale 2^(floor(log2 m) - 2), m the block's largest magnitude
    nvf4   16 elements, scale s = m / (6 t) rounded to E4M3 (at most 448), value of an element: s t e; t is the tensor's own
           scale, its largest magnitude / 2688 rounded up to 8 significant bits

Where `own` is false every operator runs in its plain form (elementary torch operations in 32 bits, rounded once at the
end); where it is true the library's own calls run.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = {"mxf4": 32, "nvf4": 16}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the rows of one decoding step, packed and read back: latency
        {"name": "pack_step", "op": "pack", "rows": 16, "K": 4096, "format": "nvf4", "type": "bf16", "out": "bf16", "along": "rows"},
        # a layer's weights, or the rows of a long batch, with the tensor's own scale taken first: memory
        {"name": "pack_batch", "op": "pack", "rows": 8192, "K": 4096, "format": "nvf4", "type": "bf16", "out": "f32", "along": "rows"},
        # rows packed along their columns, as the gradient of weights contracts them; an odd number of rows, a cut last block
        {"name": "pack_columns", "op": "pack", "rows": 4099, "K": 1032, "format": "mxf4", "type": "f16", "out": "f16", "along": "columns"},
        # one decoding step through a linear layer: 4-bit weights are read, latency
        {"name": "product_step", "op": "product", "rows": 16, "N": 4096, "K": 4096, "format": "nvf4", "out": "bf16", "relu": False},
        # a prompt through a layer with bias and ReLU, odd sizes
        {"name": "product_prompt", "op": "product", "rows": 1021, "N": 4104, "K": 4072, "format": "mxf4", "out": "f16", "relu": True},
        # the largest product: the tensor cores' rate counts
        {"name": "product_batch", "op": "product", "rows": 8192, "N": 8192, "K": 8192, "format": "nvf4", "out": "bf16", "relu": False},
        # a training step of a linear layer whose three products are in 4 bits: result, gradient of the rows and, in 32 bits, of the
        # weights, everything packed on the way
        {"name": "layer_batch", "op": "layer", "rows": 8192, "N": 4096, "K": 1024, "format": "nvf4", "out": "bf16"},
        # the same for a short odd batch through a small layer
        {"name": "layer_small", "op": "layer", "rows": 333, "N": 520, "K": 776, "format": "mxf4", "out": "f16"},
        # one decoding step of a layer of many small experts: rows packed, nearly every weight read for one or two of them
        {"name": "experts_step", "op": "experts", "rows": 32, "groups": 64, "N": 4096, "K": 1024, "format": "nvf4", "out": "bf16"},
        # a prompt through a few large experts, loads uneven
        {"name": "experts_prompt", "op": "experts", "rows": 4099, "groups": 8, "N": 1024, "K": 4096, "format": "mxf4", "out": "f16"},
        # the balance of one small step: latency
        {"name": "balance_step", "op": "balance", "tokens": 16, "experts": 64, "topk": 2, "type": "f32", "padded": False},
        # the balance of a padded training batch, with its gradient
        {"name": "balance_batch", "op": "balance", "tokens": 16384, "experts": 128, "topk": 8, "type": "f32", "padded": True},
    ]


def _spread(rng, low, high, step=1):
    """A whole multiple of `step` between low and high, spread over the logarithm."""
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + step)))) // step * step))


def draw(rng):
    op = rng.choice(["pack", "product", "layer", "experts", "balance"])
    half, form = rng.choice(["bf16", "f16"]), rng.choice(["mxf4", "nvf4"])
    if op == "pack":
        while True:
            c = {"op": op, "rows": _spread(rng, 1, 16384), "K": _spread(rng, 64, 8192, 8), "format": form,
                 "type": rng.choice([half, half, "f32"]), "along": rng.choice(["rows", "columns"])}
            if c["rows"] * c["K"] <= 1 << 25:
                break
        c["out"] = rng.choice(["f32", half])
        return c
    if op == "product":
        return {"op": op, "rows": _spread(rng, 1, 8192), "N": _spread(rng, 64, 8192, 8), "K": _spread(rng, 64, 8192, 8), "format": form,
                "out": rng.choice([half, half, "f32"]), "relu": rng.random() < 0.3}
    if op == "layer":
        return {"op": op, "rows": _spread(rng, 16, 8192), "N": _spread(rng, 64, 4096, 8), "K": _spread(rng, 64, 4096, 8),
                "format": form, "out": half}
    if op == "experts":
        while True:
            c = {"op": op, "rows": _spread(rng, 1, 16384), "groups": _spread(rng, 1, 128), "N": _spread(rng, 64, 4096, 8),
                 "K": _spread(rng, 64, 4096, 8), "format": form, "out": rng.choice([half, half, "f32"])}
            if c["groups"] * c["K"] * c["N"] <= 1 << 28:
                return c
    experts = _spread(rng, 2, 256)
    return {"op": op, "tokens": _spread(rng, 1, 32768), "experts": experts, "topk": rng.randint(1, min(8, experts)),
            "type": rng.choice(["f32", "bf16", "f16"]), "padded": rng.random() < 0.5}


def _bytes_of(kind):
    return 4 if kind == "f32" else 2


def _packed(elements, form):
    return elements * (0.5 + 1.0 / BLOCK[form])


def work(case):
    """What one pass cannot do without."""
    op = case["op"]
    if op == "balance":
        T, E = case["tokens"], case["experts"]
        # logits and choices in, counts and shares out; then the logits' gradient out (the logits are read once)
        return {"bytes": T * E * _bytes_of(case["type"]) + T * case["topk"] * 4 + T * E * 4 + E * 8, "flops": 12.0 * T * E}
    form, rows, K = case["format"], case["rows"], case["K"]
    if op == "pack":
        n = rows * K
        return {"bytes": n * (_bytes_of(case["type"]) + _bytes_of(case["out"])) + 2 * _packed(n, form), "flops": 4.0 * n}
    N, o = case["N"], _bytes_of(case["out"])
    if op == "product":
        return {"bytes": _packed(rows * K + N * K, form) + o * rows * N, "flops": 2.0 * rows * N * K}
    if op == "layer":
        # 16-bit rows, weights and gradient in; result and both gradients out
        return {"bytes": 2 * (rows * K + N * K + rows * N) + 2 * (rows * N + rows * K) + 4 * N * K, "flops": 6.0 * rows * N * K}
    live = sum(1.0 - (1.0 - q) ** rows for q in _loads(case["groups"]))
    return {"bytes": 2 * rows * K + _packed(live * N * K, form) + o * rows * N, "flops": 2.0 * rows * N * K}


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
    """Normal values whose columns differ in size, as the features of rows and weights do."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    x *= scale * torch.exp(0.5 * torch.randn(shape[-1], generator=g, device="cuda"))
    return x.to(TYPES[kind])


def _weights(groups, N, K, kind, g):
    w = torch.empty(groups, N, K, dtype=TYPES[kind], device="cuda")
    step = max(1, (1 << 26) // (K * N))
    for i in range(0, groups, step):
        w[i:i + step] = _normal((min(step, groups - i), N, K), K ** -0.5, kind, g)
    return w


def prepare(case, seed):
    host = torch.Generator().manual_seed(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = dict(case)
    if op == "balance":
        T, E = case["tokens"], case["experts"]
        # logits of a router: some experts are liked by all tokens
        logits = torch.randn(T, E, generator=g, device="cuda") * 1.5 + torch.randn(E, generator=g, device="cuda")
        s["logits"] = logits.to(TYPES[case["type"]])
        s["chosen"] = torch.topk(s["logits"].float(), case["topk"], dim=1).indices.to(torch.int32)
        s["mask"] = (torch.rand(T, generator=g, device="cuda") < 0.8).to(torch.uint8) if case["padded"] else None
        s["dlosses"] = torch.tensor([1e-2, 1e-3], device="cuda")
        if own:
            import paper_2511_13764_b200 as nk
            kind = {"bf16": nk.BF16, "f16": nk.F16, "f32": nk.F32}[case["type"]]
            s["plan"] = nk.RoutePlan(T, E, case["topk"], logits_dtype=kind)
            s["scratch"] = torch.empty(max(1, s["plan"].balance_workspace_bytes), dtype=torch.uint8, device="cuda")
            s["counts"] = torch.empty(E + 1, dtype=torch.int32, device="cuda")
            s["share"], s["losses"] = torch.empty(E, device="cuda"), torch.empty(2, device="cuda")
            s["dlogits"] = torch.empty(T, E, device="cuda")
        return s

    rows, K, form = case["rows"], case["K"], case["format"]
    kind = case["type"] if op == "pack" else case["out"] if case["out"] != "f32" else "bf16"
    x = _normal((rows, K), 1.0, kind, g)
    if op == "pack":
        s["x"] = x
        if own:
            s["pack"] = _Pack(rows, K, form, kind, transposed=case["along"] == "columns", out=case["out"])
            shape = (rows, K) if case["along"] == "rows" else (K, rows)
            s["values"] = torch.empty(shape, dtype=TYPES[case["out"]], device="cuda")
        return s
    N = case["N"]
    G = case.get("groups", 1)
    w = _weights(G, N, K, kind, g)
    if op == "layer":
        s["x"], s["w"], s["dy"] = x, w[0], _normal((rows, N), 1e-3, kind, g)
        if own:
            s["packs"] = {n: _Pack(*s[n].shape, form, kind) for n in ("x", "w", "dy")}
            s["turned"] = {n: _Pack(*s[n].shape, form, kind, transposed=True) for n in ("x", "w", "dy")}
            s["forward"] = _Mul(rows, N, K, form, case["out"])
            s["to_rows"] = _Mul(rows, K, N, form, case["out"])
            s["to_weights"] = _Mul(N, K, rows, form, "f32")
        return s
    if op == "product":
        s["bias"] = torch.randn(N, generator=g, device="cuda") * 0.1 if case["relu"] else None
        if own:
            s["a"], s["b"] = _Pack(rows, K, form, kind), _Pack(N, K, form, kind)
            s["a"](x)
            s["b"](w)
            s["mul"] = _Mul(rows, N, K, form, case["out"], relu=case["relu"])
        else:
            s["a"], s["b"] = _quantise(x, form), _quantise(w[0], form)
        return s
    off = _ragged(rows, G, host)
    s["most"] = int((off[1:] - off[:-1]).max())
    s["offsets"], s["x"] = off.to(torch.int32).cuda(), x
    # the rows' scale is known beforehand, from earlier batches; weights have one each
    s["scale"] = _tensor_scale(x) if form == "nvf4" else None
    if own:
        s["a"], s["b"] = _Pack(rows, K, form, kind, groups=G), _Pack(N, K, form, kind, batch=G)
        s["b"](w)
        s["mul"] = _Mul(rows, N, K, form, case["out"], groups=G)
    else:
        s["b"] = [_quantise(m, form) for m in w]
    return s


# ------------------------------------------------------------------------------------------------ the library's calls
class _Pack:
    """A plan that packs, and the buffers it packs into."""

    def __init__(self, rows, K, form, kind, transposed=False, out="f32", batch=1, groups=0):
        import paper_2511_13764_b200 as nk
        types = {"bf16": nk.BF16, "f16": nk.F16, "f32": nk.F32}
        self.plan = nk.PackPlan(rows, K, format=nk.NVF4 if form == "nvf4" else nk.MXF4, in_dtype=types[kind], value_dtype=types[out],
                                batch=batch, groups=groups, transposed=int(transposed))
        self.data = torch.empty(self.plan.data_bytes, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(self.plan.scales_bytes, dtype=torch.uint8, device="cuda")
        self.scratch = torch.empty(max(1, self.plan.workspace_bytes), dtype=torch.uint8, device="cuda")
        self.scale = torch.empty(batch, device="cuda") if form == "nvf4" else None

    def __call__(self, x, stream=None, scale=None, offsets=None):
        """`scale`: the tensor's, where it is known already."""
        if self.scale is not None and scale is None:
            self.plan.tensor_scale(x, self.scale, workspace=self.scratch, stream=stream)
        self.used = self.scale if scale is None else scale
        self.plan.run(x, self.data, self.scales, scale=self.used, offsets=offsets, stream=stream)
        return self


class _Mul:
    """A plan that multiplies packed operands, its result and workspace."""

    def __init__(self, rows, N, K, form, out, relu=False, groups=0):
        import paper_2511_13764_b200 as nk
        types = {"bf16": nk.BF16, "f16": nk.F16, "f32": nk.F32}
        self.plan = nk.MxPlan(rows, N, K, groups=groups, format=nk.NVF4 if form == "nvf4" else nk.MXF4, out_dtype=types[out],
                              epilogue=nk.EPI_BIAS_RELU if relu else nk.EPI_NONE)
        self.c = torch.empty(rows, N, dtype=TYPES[out], device="cuda")
        self.scratch = torch.empty(max(1, self.plan.workspace_bytes), dtype=torch.uint8, device="cuda")

    def __call__(self, a, b, stream, bias=None, offsets=None):
        self.plan.run(a.data, a.scales, b.data, b.scales, self.c, scale_a=a.used, scale_b=b.used, bias=bias, offsets=offsets,
                      workspace=self.scratch, stream=stream)
        return self.c


def _run_own(s):
    st = torch.cuda.current_stream().cuda_stream
    op = s["op"]
    if op == "balance":
        s["plan"].balance(s["logits"], s["chosen"], s["counts"], s["share"], s["losses"], mask=s["mask"], workspace=s["scratch"], stream=st)
        s["plan"].balance_backward(s["logits"], s["counts"], s["dlosses"], s["dlogits"], mask=s["mask"], stream=st)
        return {n: s[n] for n in ("counts", "share", "losses", "dlogits")}
    if op == "pack":
        p = s["pack"](s["x"], st)
        p.plan.values(p.data, p.scales, s["values"], scale=p.used, stream=st)
        return s["values"]
    if op == "product":
        return s["mul"](s["a"], s["b"], st, bias=s["bias"])
    if op == "experts":
        return s["mul"](s["a"](s["x"], st, scale=s["scale"], offsets=s["offsets"]), s["b"], st, offsets=s["offsets"])
    p, t = s["packs"], s["turned"]
    for n in ("x", "w", "dy"):
        p[n](s[n], st)
        t[n](s[n], st, scale=p[n].used)               # a matrix has one scale whichever way it is packed
    return [s["forward"](p["x"], p["w"], st), s["to_rows"](p["dy"], t["w"], st), s["to_weights"](t["dy"], t["x"], st)]


# ------------------------------------------------------------------------------------------------ plain forms
def _tensor_scale(x):
    """max |x| / 2688 rounded up to 8 significant bits; 2^-60 at least."""
    t = (x.abs().amax().double() / 2688).clamp(min=2.0 ** -60)
    step = _power(torch.frexp(t).exponent - 8)
    return (torch.ceil(t / step) * step).float().reshape(1)


def _power(e):
    """2^e in 64 bits, exactly: the exponent's bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _elements(y):
    """The 4-bit numbers nearest to y, ties to the one with an even last bit."""
    a = y.abs()
    e = ((a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float()) * 0.5
    e = e + (a > 2.5).float() + (a >= 3.5).float() + 2.0 * (a > 5.0).float()
    return torch.copysign(e, y)


def _quantise(x, form, t=None):
    """Elements and scales of the blocks along the rows of x, as 32-bit values [rows][blocks][block] and [rows][blocks], and the
    tensor's scale."""
    b = BLOCK[form]
    rows, K = x.shape
    z = torch.zeros(rows, (K + b - 1) // b * b, device="cuda")
    z[:, :K] = x
    z = z.reshape(rows, -1, b)
    m = z.abs().amax(2)
    if form == "mxf4":
        s = torch.where(m > 0, _power((torch.frexp(m).exponent - 3).clamp(min=-126)).float(), torch.ones_like(m))
        return _elements(z / s[..., None]), s, None, K
    t = _tensor_scale(x) if t is None else t
    s = (m / (6 * t)).clamp(max=448).to(torch.float8_e4m3fn).float()
    d = torch.where(s > 0, s * t, torch.full_like(s, math.inf))
    return _elements(z / d[..., None]), s, t, K


def _values(q):
    e, s, t, K = q
    v = (e * s[..., None]).reshape(e.shape[0], -1)[:, :K]
    return v if t is None else v * t


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_plain(s):
    op = s["op"]
    if op == "balance":
        z, E, k = s["logits"].float(), s["experts"], s["topk"]
        live = torch.ones(z.shape[0], device="cuda") if s["mask"] is None else s["mask"].float()
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        sums = e.sum(1, keepdim=True)
        p, lse = e / sums, (m + torch.log(sums))[:, 0]
        which = s["chosen"].long()
        counts = torch.zeros(E, dtype=torch.int64, device="cuda")
        counts.scatter_add_(0, which.reshape(-1), live.long()[:, None].expand(-1, k).reshape(-1))
        n = live.long().sum()
        d = n.double().clamp(min=1)
        share = (p.double() * live[:, None]).sum(0) / d
        balance = E / (d * k) * (counts * share).sum()
        size = (lse.double() ** 2 * live).sum() / d
        c = counts.double()
        pd = p.double()
        dz = pd * (s["dlosses"][0] * (E / (d * d * k)) * (c - (pd * c).sum(1, keepdim=True)) + s["dlosses"][1] * 2 / d * lse[:, None])
        return {"counts": torch.cat([counts, n[None]]).int(), "share": share.float(), "losses": torch.stack([balance, size]).float(),
                "dlogits": (dz * live[:, None]).float()}
    form = s["format"]
    if op == "pack":
        x = s["x"].float()
        return _values(_quantise(x if s["along"] == "rows" else x.t(), form)).to(TYPES[s["out"]])
    out = TYPES[s["out"]]
    if op == "product":
        y = torch.mm(_values(s["a"]), _values(s["b"]).t())
        return (torch.relu(y + s["bias"]) if s["relu"] else y).to(out)
    if op == "layer":
        x, w, dy = (s[n].float() for n in ("x", "w", "dy"))
        y = torch.mm(_values(_quantise(x, form)), _values(_quantise(w, form)).t())
        dx = torch.mm(_values(_quantise(dy, form)), _values(_quantise(w.t(), form)).t())
        dw = torch.mm(_values(_quantise(dy.t(), form)), _values(_quantise(x.t(), form)).t())
        return [y.to(out), dx.to(out), dw]
    x = _values(_quantise(s["x"].float(), form, s["scale"]))
    idx = s["offsets"][:-1, None].long() + torch.arange(s["most"], device="cuda")
    there = idx < s["offsets"][1:, None]
    xs = x[idx.clamp(max=x.shape[0] - 1)] * there[..., None]
    y = torch.bmm(xs, torch.stack([_values(q) for q in s["b"]]).transpose(1, 2))
    c = torch.empty(s["rows"], s["N"], dtype=out, device="cuda")
    c[idx[there]] = y[there].to(out)
    return c


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_values(x, form, t=None):
    """What the packed rows of x stand for, in 64 bits: the nearest number of a table, of two as near the one with the even place."""
    b = BLOCK[form]
    K = x.shape[1]
    z = torch.nn.functional.pad(x.double(), (0, -K % b)).reshape(x.shape[0], -1, b)
    m = z.abs().amax(2, keepdim=True)
    if form == "mxf4":
        unit = _power((torch.frexp(m).exponent - 3).clamp(min=-127))
    else:
        t = float(_tensor_scale(x) if t is None else t)
        grid = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
        unit = t * _nearest(m / (6 * t), grid)
    e = _nearest(torch.where(unit > 0, z.abs() / unit.clamp(min=1e-300), torch.zeros_like(z)),
                 torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda"))
    return (torch.copysign(e, z) * unit).reshape(x.shape[0], -1)[:, :K]


def _nearest(y, grid):
    hi = torch.searchsorted(grid, y.contiguous()).clamp(max=grid.numel() - 1)
    lo = (hi - 1).clamp(min=0)
    down, up = y - grid[lo], grid[hi] - y
    return grid[torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)]


def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    op = case["op"]
    if op == "balance":
        z, E, k = s["logits"].double(), case["experts"], case["topk"]
        z = z if s["mask"] is None else z[s["mask"] != 0]
        chosen = s["chosen"].long() if s["mask"] is None else s["chosen"].long()[s["mask"] != 0]
        n = z.shape[0]
        if n == 0:
            return {"counts": None, "share": torch.zeros(E).cuda(), "losses": torch.zeros(2).cuda(), "dlogits": torch.zeros(s["logits"].shape).cuda()}
        loads = torch.nn.functional.one_hot(chosen, E).sum((0, 1)).double() / (n * k)
        p, lse = torch.softmax(z, 1), torch.logsumexp(z, 1)
        share = p.mean(0)
        d0, d1 = s["dlosses"].tolist()
        up = d0 * E * loads / n
        part = p * (up - p @ up[:, None]) + p * (2 * d1 / n * lse)[:, None]
        dz = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
        dz[slice(None) if s["mask"] is None else s["mask"] != 0] = part
        return {"counts": None, "share": share, "losses": torch.stack([E * (loads * share).sum(), (lse ** 2).mean()]), "dlogits": dz}
    form = case["format"]
    if op == "pack":
        return _exact_values(s["x"] if case["along"] == "rows" else s["x"].t(), form)
    if op == "layer":
        x, w, dy = s["x"], s["w"], s["dy"]
        return [_exact_values(a, form) @ _exact_values(b, form).t() for a, b in ((x, w), (dy, w.t()), (dy.t(), x.t()))]
    if op == "product":
        g = torch.Generator(device="cuda").manual_seed(seed)
        kind = case["out"] if case["out"] != "f32" else "bf16"
        x = _normal((case["rows"], case["K"]), 1.0, kind, g)
        w = _weights(1, case["N"], case["K"], kind, g)[0]
        y = _exact_values(x, form) @ _exact_values(w, form).t()
        return torch.relu(y + s["bias"].double()) if case["relu"] else y
    x = _exact_values(s["x"], form, s["scale"])
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["out"] if case["out"] != "f32" else "bf16"
    _normal((case["rows"], case["K"]), 1.0, kind, g)
    w = _weights(case["groups"], case["N"], case["K"], kind, g)
    ends = s["offsets"].tolist()
    return torch.cat([x[lo:hi] @ _exact_values(w[e], form).t() for e, (lo, hi) in enumerate(zip(ends, ends[1:]))])
