"""The 4-bit operators and the balance together, as a layer of experts uses them: the example against 64-bit formulas, and steps in a CUDA
graph.

Each step is compared with its formula from the step's own operands, so its error is one rounding of its result: 2^-8 of an element at most (BF16),
and of a 2-norm; results in FP32 are sums of some hundred products in FP32, 1e-5 of their norm (a gradient that is the difference of such sums: 1e-4).
"""
import os
import sys

import pytest
import torch

import paper_2511_13764_b200 as nk

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu

FP32 = {"logits": 1e-5, "losses": 1e-5, "gradient of the gates": 1e-5, "gradient of the logits": 1e-4, "gradient of up": 1e-5, "gradient of down": 1e-5}


@pytest.mark.parametrize("format", [nk.NVF4, nk.MXF4])
@pytest.mark.parametrize("rows,experts,topk,width,hidden", [(300, 8, 2, 256, 512), (33, 16, 4, 136, 264), (5, 8, 1, 64, 128), (1, 8, 2, 72, 8)])
def test_layer_against_the_formulas(format, rows, experts, topk, width, hidden):
    from expert_layer_4bit import example
    errors = example(rows=rows, experts=experts, topk=topk, width=width, hidden=hidden, format=format)
    for name, error in errors.items():
        assert error <= FP32.get(name, 2.0 ** -8), (name, error)


def test_a_training_step_in_a_graph():
    """Every launch can be captured; a replay follows new rows and another spread of them."""
    from expert_layer_4bit import ExpertLayer4, errors_of, inputs
    rows, width, hidden, experts, topk = 100, 128, 256, 8, 2
    h, router, up, down, dy, mask = inputs(rows, width, hidden, experts, 0)
    dlosses = torch.tensor([1e-2, 1e-3], device="cuda")
    layer = ExpertLayer4(rows, width, hidden, experts, topk, up, down)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(h, router, mask)
        layer.backward(h, dy, dlosses, mask)
    for seed in (1, 2, 3):
        new = inputs(rows, width, hidden, experts, seed)
        for old, fresh in zip((h, router, dy, mask), (new[0], new[1], new[4], new[5])):
            old.copy_(fresh)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (layer.y, layer.losses, layer.dh, layer.dz, layer.dup, layer.ddown)]
        for name, error in errors_of(layer, router, h, dy, dlosses, mask).items():
            assert error <= FP32.get(name, 2.0 ** -8), (seed, name, error)
        layer.forward(h, router, mask)
        layer.backward(h, dy, dlosses, mask)
        for a, b in zip(replayed, (layer.y, layer.losses, layer.dh, layer.dz, layer.dup, layer.ddown)):
            assert torch.equal(a, b)
    layer.check()
