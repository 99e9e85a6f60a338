"""A feed-forward layer whose weights are chosen row by row, with the calls of this library only.

    h      = X . W + scale[a] (X . A_a) . B_a       shared projection, one adapter per request       (nk_lora)
    z      = h . Wr                                 the router's logits                              (nk_gemm)
    choice = the topk largest of z                  gates, experts' order                            (nk_route)
    y_t    = sum_j gate_tj relu(h_t U_e) D_e        e the chosen experts                             (nk_route, nk_grouped)

`forward` is what a serving step calls; `backward` returns the gradients of everything after the projection.
Run it for a comparison with the formulas in 64 bits:  python examples/expert_layer.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_13764_b200 as nk  # noqa: E402

BF16 = torch.bfloat16


class ExpertLayer:
    """Plans and buffers for one number of rows; weights are the caller's."""

    def __init__(self, rows, width, hidden, experts, topk, rank, adapters, requests):
        self.rows, self.width, self.hidden, self.experts, self.topk = rows, width, hidden, experts, topk
        pairs = rows * topk
        self.project = nk.LoraPlan(rows, width, width, rank, adapters, requests, out_dtype=nk.BF16)
        self.logits = nk.Plan(rows, experts, width, in_dtype=nk.BF16, out_dtype=nk.F32)
        self.route = nk.RoutePlan(rows, experts, topk, width=width)
        self.up = nk.GroupedPlan(experts, pairs, hidden, width, out_dtype=nk.BF16)
        self.down = nk.GroupedPlan(experts, pairs, width, hidden, out_dtype=nk.BF16)
        # gradients: of the rows (the same products, weights read as their transposes) and of the weights
        self.up_rows = nk.GroupedPlan(experts, pairs, width, hidden, layout_b=nk.TRANSPOSED, out_dtype=nk.BF16)
        self.down_rows = nk.GroupedPlan(experts, pairs, hidden, width, layout_b=nk.TRANSPOSED, out_dtype=nk.BF16)
        self.up_weights = nk.GroupedPlan(experts, pairs, hidden, width, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32)
        self.down_weights = nk.GroupedPlan(experts, pairs, width, hidden, kind=nk.GROUPED_WEIGHTS, out_dtype=nk.F32)
        plans = (self.project, self.logits, self.route, self.up, self.down, self.up_rows, self.down_rows, self.up_weights,
                 self.down_weights)
        # one workspace serves all plans: they run one after the other on one stream
        self.scratch = torch.empty(max(16, max(p.workspace_bytes for p in plans)), dtype=torch.uint8, device="cuda")
        self.plans = plans

        def new(*shape, dtype=BF16):
            return torch.empty(*shape, dtype=dtype, device="cuda")

        f32, i32 = torch.float32, torch.int32
        self.h, self.z = new(rows, width), new(rows, experts, dtype=f32)
        self.gates, self.chosen = new(rows, topk, dtype=f32), new(rows, topk, dtype=i32)
        self.offsets, self.slots = new(experts + 1, dtype=i32), new(rows, topk, dtype=i32)
        self.hs, self.u, self.ys, self.y = new(pairs, width), new(pairs, hidden), new(pairs, width), new(rows, width)
        self.dys, self.du, self.dhs, self.dh = new(pairs, width), new(pairs, hidden), new(pairs, width), new(rows, width)
        self.dgates, self.dz = new(rows, topk, dtype=f32), new(rows, experts, dtype=f32)
        self.dup, self.ddown = new(experts, width, hidden, dtype=f32), new(experts, hidden, width, dtype=f32)

    def forward(self, x, w, a, b, scale, offsets, adapter, router, up, down):
        s, ws = torch.cuda.current_stream().cuda_stream, self.scratch
        self.project.run(x, w, a, b, scale, offsets, adapter, self.h, workspace=ws, stream=s)
        self.logits.run(self.h, router, self.z, workspace=ws, stream=s)
        self.route.run(self.z, self.gates, self.chosen, self.offsets, self.slots, workspace=ws, stream=s)
        self.route.dispatch(self.h, self.slots, self.hs, stream=s)
        self.up.run(self.hs, up, self.u, self.offsets, workspace=ws, stream=s)
        torch.relu_(self.u)
        self.down.run(self.u, down, self.ys, self.offsets, workspace=ws, stream=s)
        self.route.combine(self.ys, self.slots, self.y, gates=self.gates, stream=s)
        return self.y

    def backward(self, dy, up, down):
        """Gradients of h through the experts (not through the router), of the logits and of the experts' weights."""
        s, ws = torch.cuda.current_stream().cuda_stream, self.scratch
        self.route.combine_backward(dy, self.ys, self.slots, self.gates, self.dys, self.dgates, stream=s)
        self.down_weights.run(self.u, self.dys, self.ddown, self.offsets, workspace=ws, stream=s)
        self.down_rows.run(self.dys, down, self.du, self.offsets, workspace=ws, stream=s)
        self.du.mul_(self.u > 0)
        self.up_weights.run(self.hs, self.du, self.dup, self.offsets, workspace=ws, stream=s)
        self.up_rows.run(self.du, up, self.dhs, self.offsets, workspace=ws, stream=s)
        self.route.combine(self.dhs, self.slots, self.dh, stream=s)
        self.route.backward(self.z, self.chosen, self.dgates, self.dz, stream=s)
        return self.dh, self.dz, self.dup, self.ddown

    def check(self):
        for p in self.plans:
            p.check()


def example(rows=300, width=256, hidden=512, experts=8, topk=2, rank=16, adapters=4, seed=0):
    """Runs the layer forwards and backwards; returns the relative 2-norm errors against the formulas in 64 bits, each
    step's from the step's own inputs as the library rounded them."""
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g) * scale).to(BF16).cuda()

    # half of the requests decode one row, the others are prompts
    ends = sorted(torch.randperm(rows - 1, generator=g)[:3].tolist())
    sizes = [b - a for a, b in zip([0] + [e + 1 for e in ends], [e + 1 for e in ends] + [rows])]
    sizes = [n for n in sizes if n] + [0]
    off = torch.tensor([0] + sizes).cumsum(0).to(torch.int32)
    adapter = torch.tensor([(i % (adapters + 1)) - 1 for i in range(len(sizes))], dtype=torch.int32)
    x, w = normal(rows, width), normal(width, width, scale=width ** -0.5)
    a, b = normal(adapters, width, rank, scale=width ** -0.5), normal(adapters, rank, width, scale=rank ** -0.5)
    scale = 0.5 + torch.rand(adapters, generator=g)
    router, up, down = normal(width, experts, scale=width ** -0.5), normal(experts, width, hidden, scale=width ** -0.5), normal(experts, hidden, width, scale=hidden ** -0.5)
    dy = normal(rows, width)

    layer = ExpertLayer(rows, width, hidden, experts, topk, rank, adapters, len(sizes))
    layer.forward(x, w, a, b, scale.cuda(), off.cuda(), adapter.cuda(), router, up, down)
    layer.backward(dy, up, down)
    layer.check()

    def off_by(got, want):
        size = float(want.norm())                 # (zero for the logits' gradient with one renormalised choice: then the error itself)
        return float((got.double() - want).norm()) / (size if size > 1e-12 else 1.0)

    d = torch.float64
    h = x.to(d) @ w.to(d)
    for lo, hi, n in zip(off.tolist(), off[1:].tolist(), adapter.tolist()):
        if n >= 0:
            h[lo:hi] += float(scale[n]) * (x[lo:hi].to(d) @ a[n].to(d) @ b[n].to(d))
    errors = {"projection": off_by(layer.h, h), "logits": off_by(layer.z, layer.h.to(d) @ router.to(d))}
    z = layer.z.to(d)
    top = torch.argsort(-z, dim=1, stable=True)[:, :topk]
    assert torch.equal(top.int(), layer.chosen)
    z.requires_grad_(True)
    gates = torch.softmax(z.gather(1, top), 1)
    errors["gates"] = off_by(layer.gates, gates.detach())
    hh, uu, dd = (t.to(d).requires_grad_(True) for t in (layer.h, up, down))
    y = torch.zeros(rows, width, dtype=d, device="cuda")
    for j in range(topk):
        e = top[:, j]
        y = y + gates[:, j, None] * torch.bmm(torch.relu(torch.bmm(hh[:, None], uu[e])), dd[e])[:, 0]
    errors["result"] = off_by(layer.y, y.detach())
    y.backward(dy.to(d))
    for name, got, want in (("gradient of the rows", layer.dh, hh.grad), ("gradient of the logits", layer.dz, z.grad),
                            ("gradient of up", layer.dup, uu.grad), ("gradient of down", layer.ddown, dd.grad)):
        errors[name] = off_by(got, want)
    return errors


if __name__ == "__main__":
    for name, error in example().items():
        print(f"{name:24s} relative error {error:.2e}")
