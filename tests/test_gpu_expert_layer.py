"""The operators together, as a layer uses them: the example against 64-bit formulas, and a step in a CUDA graph."""
import os
import sys

import pytest
import torch

import paper_2511_13764_b200 as nk

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,experts,topk", [(300, 8, 2), (33, 16, 4), (5, 8, 1)])
def test_layer_against_the_formulas(rows, experts, topk):
    from expert_layer import example
    errors = example(rows=rows, experts=experts, topk=topk)
    # a BF16 value is off by 2^-9 of itself at most, 2^-9 / sqrt(3) on average; the result and the rows' gradient pass
    # through three such roundings one after the other (hidden row, expert's row, result), the weights' through two
    one = 2.0 ** -9
    assert errors["projection"] <= one and errors["logits"] <= 1e-5 and errors["gates"] <= 1e-5
    for name in ("result", "gradient of the rows", "gradient of the logits", "gradient of up", "gradient of down"):
        assert errors[name] <= 3 * one, (name, errors[name])


def test_a_step_in_a_graph():
    """Every launch of a decoding step can be captured; a replay follows new inputs and a new spread of the rows."""
    from expert_layer import ExpertLayer
    rows, width, hidden, experts, topk = 16, 128, 256, 8, 2
    g = torch.Generator().manual_seed(4)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g) * scale).bfloat16().cuda()

    layer = ExpertLayer(rows, width, hidden, experts, topk, 8, 3, rows)
    x, w = normal(rows, width), normal(width, width, scale=0.1)
    a, b, scale = normal(3, width, 8, scale=0.1), normal(3, 8, width, scale=0.3), torch.ones(3, device="cuda")
    off, adapter = torch.arange(rows + 1, dtype=torch.int32).cuda(), torch.randint(-1, 3, (rows,), generator=g, dtype=torch.int32).cuda()
    router, up, down = normal(width, experts, scale=0.1), normal(experts, width, hidden, scale=0.1), normal(experts, hidden, width, scale=0.1)
    args = (x, w, a, b, scale, off, adapter, router, up, down)
    layer.forward(*args)
    layer.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(*args)
    for _ in range(3):
        x.copy_(normal(rows, width))
        adapter.copy_(torch.randint(-1, 3, (rows,), generator=g, dtype=torch.int32))
        layer.forward(*args)
        want = layer.y.clone(), layer.chosen.clone(), layer.offsets.clone()
        layer.y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.y, want[0]) and torch.equal(layer.chosen, want[1]) and torch.equal(layer.offsets, want[2])
    layer.check()


def test_plans_of_one_workspace_after_one_another():
    """Launches overlap at their ends; what one writes the next one reads."""
    rows, width = 64, 256
    g = torch.Generator().manual_seed(5)
    W = (torch.randn(2, width, width, generator=g) * width ** -0.5).bfloat16().cuda()
    off = torch.tensor([0, 20, rows], dtype=torch.int32).cuda()
    plan = nk.GroupedPlan(2, rows, width, width, out_dtype=nk.BF16)
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    for trial in range(20):
        x = torch.randn(rows, width, generator=g).bfloat16().cuda()
        bufs = [x] + [torch.full_like(x, float("nan")) for _ in range(8)]
        for i in range(8):
            plan.run(bufs[i], W, bufs[i + 1], off, workspace=ws, stream=st)
        plan.check()
        for i in range(8):
            y = torch.cat([bufs[i][:20].double() @ W[0].double(), bufs[i][20:].double() @ W[1].double()])
            size = float((bufs[i].double().abs() @ W.double().abs().sum(0)).max())
            assert ((bufs[i + 1].double() - y).abs() <= 2.0 ** -8 * y.abs() + 1e-5 * size).all()
