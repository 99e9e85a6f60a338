"""The expert layer with its experts in 4-bit floating point and the balance of their loads, with the calls of this library (and, backwards, one
elementwise product of torch: where the ReLU was 0).

    z      = h . Wr                                    the router's logits                              (nk_gemm)
    choice = the topk largest of z                     gates, experts' order                            (nk_route)
    loss   = g0 balance + g1 size of the logits        evenly loaded experts, padding left out          (nk_route_balance)
    y_t    = sum_j gate_tj relu(q(h_t) q(U_e)^T) ...   rows and weights in 4 bits, grouped by expert    (nk_pack, nk_mx)

`forward` is what a serving or training step calls; `backward` takes the gradients of the rows in 4 bits, too, with the weights packed along
their other dimension, and those of the weights from 16-bit rows (nk_grouped).
Run it for a comparison with the formulas in 64 bits:  python examples/expert_layer_4bit.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_13764_b200 as nk  # noqa: E402

BF16 = torch.bfloat16


class Packed:
    """A matrix (or one for each expert) in 4 bits: its plan and buffers."""

    def __init__(self, rows, K, format, experts=0, batch=1, transposed=0):
        self.plan = nk.PackPlan(rows, K, format=format, batch=batch, groups=experts, transposed=transposed)
        self.data = torch.empty(max(16, self.plan.data_bytes), dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(max(16, self.plan.scales_bytes), dtype=torch.uint8, device="cuda")
        self.scratch = torch.empty(max(16, self.plan.workspace_bytes), dtype=torch.uint8, device="cuda")
        self.scale = torch.empty(batch, device="cuda") if format == nk.NVF4 else None

    def __call__(self, x, stream, offsets=None, scale=None):
        """`scale`: the tensor's, where it is known."""
        if scale is not None:
            self.scale = scale
        elif self.scale is not None:
            self.plan.tensor_scale(x, self.scale, workspace=self.scratch, stream=stream)
        self.plan.run(x, self.data, self.scales, scale=self.scale, offsets=offsets, stream=stream)
        return self

    def values(self, shape, offsets=None):
        y = torch.zeros(shape, device="cuda")
        self.plan.values(self.data, self.scales, y, scale=self.scale, offsets=offsets, stream=torch.cuda.current_stream().cuda_stream)
        return y


class ExpertLayer4:
    """Plans and buffers for one number of rows; weights up [experts][hidden][width] and down [experts][width][hidden] are packed once."""

    def __init__(self, rows, width, hidden, experts, topk, up, down, format=nk.NVF4):
        self.rows, self.width, self.hidden, self.experts, self.topk = rows, width, hidden, experts, topk
        pairs = rows * topk
        s = torch.cuda.current_stream().cuda_stream
        self.up_w, self.up_t = Packed(hidden, width, format, batch=experts), Packed(hidden, width, format, batch=experts, transposed=1)
        self.down_w, self.down_t = Packed(width, hidden, format, batch=experts), Packed(width, hidden, format, batch=experts, transposed=1)
        self.up_t(up, s, scale=self.up_w(up, s).scale)
        self.down_t(down, s, scale=self.down_w(down, s).scale)
        self.hs4, self.u4 = Packed(pairs, width, format, experts), Packed(pairs, hidden, format, experts)
        self.dys4, self.du4 = Packed(pairs, width, format, experts), Packed(pairs, hidden, format, experts)

        def product(N, K, **more):
            return nk.MxPlan(pairs, N, K, groups=experts, format=format, out_dtype=nk.BF16, **more)

        self.logits = nk.Plan(rows, experts, width, in_dtype=nk.BF16, out_dtype=nk.F32)
        self.route = nk.RoutePlan(rows, experts, topk, width=width)
        self.up, self.down = product(hidden, width, epilogue=nk.EPI_BIAS_RELU), product(width, hidden)
        self.up_rows, self.down_rows = product(width, hidden), product(hidden, width)
        self.up_weights = nk.GroupedPlan(experts, pairs, width, hidden, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32)
        self.down_weights = nk.GroupedPlan(experts, pairs, hidden, width, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32)
        self.plans = (self.logits, self.route, self.up, self.down, self.up_rows, self.down_rows, self.up_weights, self.down_weights)
        # one workspace serves all plans: they run one after the other on one stream
        self.scratch = torch.empty(max(16, self.route.balance_workspace_bytes, max(p.workspace_bytes for p in self.plans)), dtype=torch.uint8, device="cuda")

        def new(*shape, dtype=BF16):
            return torch.empty(*shape, dtype=dtype, device="cuda")

        f32, i32 = torch.float32, torch.int32
        self.z, self.gates, self.chosen = new(rows, experts, dtype=f32), new(rows, topk, dtype=f32), new(rows, topk, dtype=i32)
        self.offsets, self.slots = new(experts + 1, dtype=i32), new(rows, topk, dtype=i32)
        self.counts, self.share, self.losses = new(experts + 1, dtype=i32), new(experts, dtype=f32), new(2, dtype=f32)
        self.hs, self.u, self.ys, self.y = new(pairs, width), new(pairs, hidden), new(pairs, width), new(rows, width)
        self.dys, self.du, self.dhs, self.dh = new(pairs, width), new(pairs, hidden), new(pairs, width), new(rows, width)
        self.dgates, self.dz = new(rows, topk, dtype=f32), new(rows, experts, dtype=f32)
        self.dup, self.ddown = new(experts, hidden, width, dtype=f32), new(experts, width, hidden, dtype=f32)

    def multiply(self, plan, a, b, c, s):
        plan.run(a.data, a.scales, b.data, b.scales, c, scale_a=a.scale, scale_b=b.scale, offsets=self.offsets, workspace=self.scratch, stream=s)

    def forward(self, h, router, mask=None):
        s, ws = torch.cuda.current_stream().cuda_stream, self.scratch
        self.logits.run(h, router, self.z, workspace=ws, stream=s)
        self.route.run(self.z, self.gates, self.chosen, self.offsets, self.slots, workspace=ws, stream=s)
        self.route.balance(self.z, self.chosen, self.counts, self.share, self.losses, mask=mask, workspace=ws, stream=s)
        self.route.dispatch(h, self.slots, self.hs, stream=s)
        self.multiply(self.up, self.hs4(self.hs, s, self.offsets), self.up_w, self.u, s)
        self.multiply(self.down, self.u4(self.u, s, self.offsets), self.down_w, self.ys, s)
        self.route.combine(self.ys, self.slots, self.y, gates=self.gates, stream=s)
        return self.y, self.losses

    def backward(self, h, dy, dlosses, mask=None):
        """Gradients of h through the experts (not through the router), of the logits (the balance's among them) and of the weights."""
        s, ws = torch.cuda.current_stream().cuda_stream, self.scratch
        self.route.combine_backward(dy, self.ys, self.slots, self.gates, self.dys, self.dgates, stream=s)
        self.multiply(self.down_rows, self.dys4(self.dys, s, self.offsets), self.down_t, self.du, s)
        self.du.mul_(self.u > 0)
        self.multiply(self.up_rows, self.du4(self.du, s, self.offsets), self.up_t, self.dhs, s)
        self.down_weights.run(self.dys, self.u, self.ddown, self.offsets, workspace=ws, stream=s)
        self.up_weights.run(self.du, self.hs, self.dup, self.offsets, workspace=ws, stream=s)
        self.route.combine(self.dhs, self.slots, self.dh, stream=s)
        self.route.backward(self.z, self.chosen, self.dgates, self.dz, stream=s)
        self.route.balance_backward(self.z, self.counts, dlosses, self.dz, mask=mask, accumulate=True, stream=s)
        return self.dh, self.dz, self.dup, self.ddown

    def check(self):
        for p in self.plans + tuple(q.plan for q in (self.hs4, self.u4, self.dys4, self.du4, self.up_w, self.up_t, self.down_w, self.down_t)):
            p.check()


def inputs(rows, width, hidden, experts, seed):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g) * scale).to(BF16).cuda()

    mask = (torch.rand(rows, generator=g) < 0.9).to(torch.uint8).cuda()
    return (normal(rows, width), normal(width, experts, scale=width ** -0.5), normal(experts, hidden, width, scale=width ** -0.5),
            normal(experts, width, hidden, scale=hidden ** -0.5), normal(rows, width), mask)


def example(rows=300, width=256, hidden=512, experts=8, topk=2, format=nk.NVF4, seed=0, layer=None):
    """Runs the layer forwards and backwards; returns the relative 2-norm errors against the formulas in 64 bits, each step's from the step's own
    operands as the library packed and rounded them."""
    h, router, up, down, dy, mask = inputs(rows, width, hidden, experts, seed)
    dlosses = torch.tensor([1e-2, 1e-3], device="cuda")
    layer = layer or ExpertLayer4(rows, width, hidden, experts, topk, up, down, format)
    layer.forward(h, router, mask)
    layer.backward(h, dy, dlosses, mask)
    layer.check()
    return errors_of(layer, router, h, dy, dlosses, mask)


def errors_of(layer, router, h, dy, dlosses, mask):
    d, errors = torch.float64, {}
    rows, width, hidden, experts, topk = layer.rows, layer.width, layer.hidden, layer.experts, layer.topk
    pairs = rows * topk

    def off_by(name, got, want):
        size = float(want.norm())
        errors[name] = float((got.to(d) - want).norm()) / (size if size > 1e-12 else 1.0)

    z = layer.z.to(d).requires_grad_(True)
    off_by("logits", layer.z, h.to(d) @ router.to(d))
    top = torch.argsort(-layer.z.to(d), dim=1, stable=True)[:, :topk]
    assert torch.equal(top.int(), layer.chosen)
    live = mask.to(d)
    n = live.sum()
    p = torch.softmax(z, 1)
    counts = torch.zeros(experts, dtype=d, device="cuda").scatter_add_(0, top.reshape(-1), live[:, None].expand(-1, topk).reshape(-1))
    assert torch.equal(counts.int(), layer.counts[:-1]) and int(n) == int(layer.counts[-1])
    balance = experts / (n * n * topk) * (counts * (p * live[:, None]).sum(0)).sum()
    size = (torch.logsumexp(z, 1) ** 2 * live).sum() / n
    off_by("losses", layer.losses, torch.stack([balance, size]).detach())
    gates = torch.softmax(z.gather(1, top), 1)

    # the experts' products, from what the packed operands stand for
    slots = layer.slots.long()
    expert = torch.empty(pairs, dtype=torch.int64, device="cuda")
    expert[slots.reshape(-1)] = top.reshape(-1)
    off = layer.offsets
    hs, u = layer.hs4.values((pairs, width), off).to(d), layer.u4.values((pairs, hidden), off).to(d)
    dys, du = layer.dys4.values((pairs, width), off).to(d), layer.du4.values((pairs, hidden), off).to(d)
    up, down = layer.up_w.values((experts, hidden, width)).to(d), layer.down_w.values((experts, width, hidden)).to(d)
    up_t, down_t = layer.up_t.values((experts, width, hidden)).to(d), layer.down_t.values((experts, hidden, width)).to(d)

    def grouped(x, w):
        y = torch.empty(pairs, w.shape[1], dtype=d, device="cuda")
        for e in range(experts):
            y[expert == e] = x[expert == e] @ w[e].t()
        return y

    off_by("up", layer.u, torch.relu(grouped(hs, up)))
    off_by("down", layer.ys, grouped(u, down))
    off_by("result", layer.y, (gates.detach()[..., None] * layer.ys.to(d)[slots]).sum(1))
    off_by("gradient through down", layer.du, grouped(dys, down_t) * (layer.u > 0))
    off_by("gradient through up", layer.dhs, grouped(du, up_t))
    off_by("gradient of the rows", layer.dh, layer.dhs.to(d)[slots].sum(1))
    ((gates * layer.dgates.to(d)).sum() + dlosses[0].to(d) * balance + dlosses[1].to(d) * size).backward()
    off_by("gradient of the gates", layer.dgates, (dy.to(d)[:, None] * layer.ys.to(d)[slots]).sum(-1))
    off_by("gradient of the logits", layer.dz, z.grad)
    dup = torch.stack([layer.du.to(d)[expert == e].t() @ layer.hs.to(d)[expert == e] for e in range(experts)])
    ddown = torch.stack([layer.dys.to(d)[expert == e].t() @ layer.u.to(d)[expert == e] for e in range(experts)])
    off_by("gradient of up", layer.dup, dup)
    off_by("gradient of down", layer.ddown, ddown)
    return errors


if __name__ == "__main__":
    for form in (nk.NVF4, nk.MXF4):
        print("NVF4" if form == nk.NVF4 else "MXF4")
        for name, error in example(format=form).items():
            print(f"  {name:24s} relative error {error:.2e}")
