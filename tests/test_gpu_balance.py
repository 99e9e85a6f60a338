"""nk_route_balance and its gradient against the formulas in 64 bits.

Tolerances.  A probability is exp(z - m) / sum: the difference is off by 2^-24 of at most 32 here (2^-19 of the exponential), expf by 2 of
its last places (2^-22), the sum and the division by less; a mean adds up to 64 + 32 of them in FP32 (100 x 2^-24).  Together below 2^-16
of the mean.  A row's log-sum-exp is off by the same few 2^-24 of the row's largest size, its square by twice that: 2^-16.  The gradient is
a sum of products of such numbers: 2^-16 of the sum of their sizes.
"""
import pytest
import torch

import paper_2511_13764_b200 as nk

pytestmark = pytest.mark.gpu

TYPES = {"f32": (nk.F32, torch.float32), "bf16": (nk.BF16, torch.bfloat16), "f16": (nk.F16, torch.float16)}
REL = 2.0 ** -16


def stream():
    return torch.cuda.current_stream().cuda_stream


def inputs(tokens, experts, topk, kind="f32", seed=0, even=False):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(tokens, experts, generator=g) * (1e-3 if even else 2.0) + (0.0 if even else 1.0) * torch.randn(experts, generator=g)
    z = z.to(TYPES[kind][1])
    chosen = torch.argsort(-z.float(), dim=1, stable=True)[:, :topk].to(torch.int32)
    return z, chosen


def formulas(z, chosen, mask, d, k):
    """Counts, shares, losses, gradient and the sum of the sizes of what the gradient adds up, in 64 bits."""
    z = z.double()
    E = z.shape[1]
    live = torch.ones(z.shape[0], dtype=torch.bool) if mask is None else mask.cpu() != 0
    ok = (chosen >= 0) & (chosen < E) & live[:, None]
    counts = torch.bincount(chosen[ok].long(), minlength=E)
    n = int(live.sum())
    if n == 0:
        return counts, n, torch.zeros(E).double(), torch.zeros(2).double(), torch.zeros_like(z), torch.zeros_like(z)
    none = (z == -torch.inf).all(1)
    p = torch.where(none[:, None], 0.0, torch.softmax(z, 1))
    lse = torch.where(none, 0.0, torch.logsumexp(z, 1))
    share = (p * live[:, None]).sum(0) / n
    c = counts.double()
    losses = torch.stack([E / (n * k) * (c * share).sum(), (lse ** 2 * live).sum() / n])
    away = c - n * k // E
    up = d[0] * E / (n * n * k)
    grad = p * (up * (c - (p * c).sum(1, keepdim=True)) + d[1] * 2 / n * lse[:, None])
    grad = torch.where(none[:, None], 0.0, grad) * live[:, None]
    size = p * (abs(up) * (away.abs() + (p * away.abs()).sum(1, keepdim=True)) + abs(d[1]) * 2 / n * lse.abs()[:, None]) * live[:, None]
    return counts, n, share, losses, grad, size


def run(z, chosen, mask, d, topk, kind, accumulate=None, ld=0):
    tokens, E = z.shape
    plan = nk.RoutePlan(tokens, E, topk, logits_dtype=TYPES[kind][0], ld_logits=ld)
    dev = torch.empty(tokens, max(ld, E), dtype=z.dtype).fill_(float("nan"))
    dev[:, :E] = z
    dev, ch = dev.cuda(), chosen.cuda()
    counts = torch.full((E + 2,), -7, dtype=torch.int32, device="cuda")
    share, losses = torch.full((E + 1,), -7.0, device="cuda"), torch.full((3,), -7.0, device="cuda")
    ws = torch.full((max(1, plan.balance_workspace_bytes),), 0xFF, dtype=torch.uint8, device="cuda")
    plan.balance(dev, ch, counts, share, losses, mask=mask, workspace=ws, stream=stream())
    dz = torch.full((tokens, E), float("nan"), device="cuda") if accumulate is None else accumulate.clone().cuda()
    plan.balance_backward(dev, counts, torch.tensor(d, device="cuda"), dz, mask=mask, accumulate=accumulate is not None, stream=stream())
    plan.check()
    assert counts[E + 1] == -7 and share[E] == -7 and losses[2] == -7
    return counts[:E + 1].cpu(), share[:E].double().cpu(), losses[:2].double().cpu(), dz.double().cpu()


def check(z, chosen, mask, topk, kind, d=(0.3, 0.02), **more):
    got = run(z, chosen, mask, list(d), topk, kind, **more)
    d = torch.tensor(d).double().tolist()
    counts, n, share, losses, grad, size = formulas(z, chosen, mask, d, topk)
    assert torch.equal(got[0][:-1].long(), counts) and got[0][-1] == n
    assert ((got[1] - share).abs() <= REL * share).all()
    assert ((got[2] - losses).abs() <= REL * losses.abs()).all()
    base = more.get("accumulate")
    if base is None:
        assert ((got[3] - grad).abs() <= REL * size).all()
    else:
        assert ((got[3] - grad - base.double()).abs() <= REL * size + 2.0 ** -24 * (base.double().abs() + size)).all()


@pytest.mark.parametrize("tokens,experts,topk", [(1, 1, 1), (1, 2, 1), (3, 5, 2), (16, 64, 2), (64, 33, 8), (65, 128, 8), (1000, 257, 4),
                                                 (4099, 8, 2), (300, 1024, 32), (20000, 64, 6)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_formulas(tokens, experts, topk, kind):
    z, chosen = inputs(tokens, experts, topk, kind, seed=tokens)
    check(z, chosen, None, topk, kind)


@pytest.mark.parametrize("tokens", [1, 40, 1000])
@pytest.mark.parametrize("live", [0.0, 0.5, 1.0])
def test_padding(tokens, live):
    z, chosen = inputs(tokens, 24, 3, seed=4)
    mask = (torch.rand(tokens, generator=torch.Generator().manual_seed(1)) < live).to(torch.uint8)
    z[mask == 0] = float("nan")                            # padding may hold anything
    chosen[mask == 0] = 1 << 30
    d = [0.3, 0.02]
    got = run(z, chosen, mask.cuda(), d, 3, "f32")
    keep = mask != 0
    counts, n, share, losses, grad, size = formulas(z[keep], chosen[keep], None, d, 3)
    assert torch.equal(got[0][:-1].long(), counts) and got[0][-1] == n
    assert ((got[1] - share).abs() <= REL * share).all() and ((got[2] - losses).abs() <= REL * losses.abs()).all()
    assert ((got[3][keep] - grad).abs() <= REL * size).all() and (got[3][~keep] == 0).all()


@pytest.mark.parametrize("tokens", [50, 3000])
def test_even_loads_keep_their_digits(tokens):
    """Loads next to even: the gradient is the small difference of large counts."""
    z, chosen = inputs(tokens, 16, 2, seed=6, even=True)
    check(z, chosen, None, 2, "f32", d=(1.0, 0.0))


@pytest.mark.parametrize("tokens", [20, 900])
def test_rows_without_experts_and_dropped_pairs(tokens):
    z, chosen = inputs(tokens, 40, 4, seed=8)
    z[::7] = float("-inf")                                # nothing may be chosen
    z[1::7, ::2] = float("-inf")
    chosen[2::5, 1] = -1                                   # dropped
    chosen[3::5, 0] = 40
    check(z, chosen, None, 4, "f32")


def test_a_nan_reaches_the_losses_and_its_own_row():
    z, chosen = inputs(200, 12, 2, seed=2)
    z[77, 3] = float("nan")
    counts, share, losses, dz = run(z, chosen, None, [1.0, 1.0], 2, "f32")
    assert share.isnan().all() and losses.isnan().all() and counts[-1] == 200
    assert dz[77].isnan().all() and not dz[:77].isnan().any() and not dz[78:].isnan().any()


def test_strides_and_accumulation():
    z, chosen = inputs(333, 48, 3, seed=3)
    base = torch.randn(333, 48, generator=torch.Generator().manual_seed(2))
    check(z, chosen, None, 3, "f32", accumulate=base, ld=61)
    mask = (torch.arange(333) % 3 != 0).to(torch.uint8)
    _, _, _, dz = run(z, chosen, mask.cuda(), [1.0, 1.0], 3, "f32", accumulate=base)
    assert torch.equal(dz[::3].float(), base[::3])


def test_gradient_against_differences():
    """The losses' change along a direction, in 64 bits, with the counts held."""
    z, chosen = inputs(90, 20, 2, seed=11)
    d = [0.7, 0.05]
    _, _, _, dz = run(z, chosen, None, d, 2, "f32")
    v = torch.randn(z.shape, generator=torch.Generator().manual_seed(1)).double()
    h = 1e-5

    def loss(w):
        _, _, _, losses, _, _ = formulas(w, chosen, None, d, 2)
        return d[0] * losses[0] + d[1] * losses[1]
    slope = (loss(z.double() + h * v) - loss(z.double() - h * v)) / (2 * h)
    # differences: third derivatives times h^2, rounding 2^-52 / h; the gradient REL of its terms
    _, _, _, _, _, size = formulas(z, chosen, None, d, 2)
    assert abs((dz * v).sum() - slope) <= REL * (size * v.abs()).sum() + 1e-7


def test_repeats_bit_for_bit_and_in_a_graph():
    z, chosen = inputs(5000, 96, 4, seed=1)
    first = run(z, chosen, None, [1.0, 1.0], 4, "f32")
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, run(z, chosen, None, [1.0, 1.0], 4, "f32")))
    plan = nk.RoutePlan(5000, 96, 4)
    zd, ch, d = z.cuda(), chosen.cuda(), torch.ones(2, device="cuda")
    counts, share, losses = torch.empty(97, dtype=torch.int32, device="cuda"), torch.empty(96, device="cuda"), torch.empty(2, device="cuda")
    dz, ws = torch.empty(5000, 96, device="cuda"), torch.empty(plan.balance_workspace_bytes, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        plan.balance(zd, ch, counts, share, losses, workspace=ws, stream=stream())
        plan.balance_backward(zd, counts, d, dz, stream=stream())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(counts.cpu(), first[0]) and torch.equal(losses.double().cpu(), first[2]) and torch.equal(dz.double().cpu(), first[3])


def test_no_tokens_and_refusals():
    plan = nk.RoutePlan(0, 8, 2)
    counts, share, losses = torch.full((9,), 5, dtype=torch.int32, device="cuda"), torch.ones(8, device="cuda"), torch.ones(2, device="cuda")
    plan.balance(None, None, counts, share, losses, stream=stream())
    plan.balance_backward(None, None, None, None, stream=stream())
    plan.check()
    assert not counts.any() and not share.any() and not losses.any()
    plan = nk.RoutePlan(100, 8, 2)
    z, ch = torch.zeros(100, 8, device="cuda"), torch.zeros(100, 2, dtype=torch.int32, device="cuda")
    ws = torch.empty(plan.balance_workspace_bytes, dtype=torch.uint8, device="cuda")
    for status, call in ((1, lambda: plan.balance(None, ch, counts, share, losses, workspace=ws)), (1, lambda: plan.balance(z, ch, None, share, losses, workspace=ws)),
                         (4, lambda: plan.balance(z, ch, counts, share, losses)), (4, lambda: plan.balance(z, ch, counts, share, losses, workspace=ws[:-4])),
                         (3, lambda: plan.balance(z.data_ptr() + 2, ch, counts, share, losses, workspace=ws)),
                         (1, lambda: plan.balance_backward(z, counts, None, z)), (1, lambda: plan.balance_backward(z, counts, losses, z, accumulate=2)),
                         (3, lambda: plan.balance_backward(z, counts, losses, z.data_ptr() + 1))):
        with pytest.raises(nk.NkError) as e:
            call()
        assert e.value.status == status


@pytest.mark.parametrize("tokens,cut,experts,topk", [(64, 20, 24, 3), (5000, 1234, 96, 4), (300, 299, 8, 2), (2000, 0, 40, 1)])
def test_loads_over_several_ranks(tokens, cut, experts, topk):
    """Each rank has its own tokens; with the sum of the ranks' counts the gradients are those of the losses of all tokens, and the losses come from
    shares weighted by the ranks' numbers of tokens."""
    z, chosen = inputs(tokens, experts, topk, seed=tokens)
    mask = (torch.rand(tokens, generator=torch.Generator().manual_seed(1)) < 0.8).to(torch.uint8)
    d = [0.3, 0.02]
    counts, n, share, losses, grad, size = formulas(z, chosen, mask, torch.tensor(d).double().tolist(), topk)
    parts = []
    for lo, hi in ((0, cut), (cut, tokens)):
        plan = nk.RoutePlan(hi - lo, experts, topk)
        c = torch.empty(experts + 1, dtype=torch.int32, device="cuda")
        s, l = torch.empty(experts, device="cuda"), torch.empty(2, device="cuda")
        ws = torch.empty(max(1, plan.balance_workspace_bytes), dtype=torch.uint8, device="cuda")
        zd, ch, m = z[lo:hi].cuda(), chosen[lo:hi].cuda(), mask[lo:hi].cuda()
        plan.balance(zd, ch, c, s, l, mask=m, workspace=ws, stream=stream())
        plan.check()
        parts.append((plan, zd, m, c, s.double().cpu(), l.double().cpu()))
    total = parts[0][3] + parts[1][3]                      # what an all-reduce gives
    assert torch.equal(total[:-1].cpu().long(), counts) and int(total[-1]) == n
    own = [int(p[3][-1]) for p in parts]
    mean = sum(k * p[4] for k, p in zip(own, parts)) / n
    assert ((mean - share).abs() <= REL * share).all()
    assert abs(experts / (n * topk) * (total[:-1].cpu().double() * mean).sum() - losses[0]) <= REL * losses[0]
    assert abs(sum(k * p[5][1] for k, p in zip(own, parts)) / n - losses[1]) <= REL * losses[1]
    got = []
    for plan, zd, m, _, _, _ in parts:
        dz = torch.full(zd.shape, float("nan"), device="cuda")
        plan.balance_backward(zd, total, torch.tensor(d, device="cuda"), dz, mask=m, stream=stream())
        plan.check()
        got.append(dz.double().cpu())
    assert ((torch.cat(got) - grad).abs() <= REL * size).all()
