"""The oracle of routing and of the routed experts (CPU): its gradients against
autograd and against differences, its choices on hand-made rows."""

from __future__ import annotations

import math

import pytest
import torch

import routed_oracle as routed
import sublayer_oracle as oracle

INF = float("inf")


def test_choices_by_hand():
    l = torch.tensor([[1.0, 3.0, 2.0, 3.0], [-INF, 0.0, -INF, -1.0], [-INF] * 4])
    assert routed.choose(l, None, 3, "softmax") == [[1, 3, 2], [1, 3, -1], [-1, -1, -1]]
    bias = torch.tensor([0.0, -1.0, 0.5, -INF])
    assert routed.choose(l[:1], bias, 3, "sigmoid") == [[2, 0, 1]]
    # Groups of two: sums of the best two, or of the best.
    l = torch.tensor([[4.0, -9.0, 3.0, 3.0]])
    assert routed.choose(l, None, 2, "sigmoid", groups=2, kept=1, group_top=2) == [[2, 3]]
    assert routed.choose(l, None, 2, "sigmoid", groups=2, kept=1, group_top=1) == [[0, 1]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_route_gradient(score, renormalise):
    gen = torch.Generator().manual_seed(4)
    l = torch.randn(5, 9, generator=gen).double()
    chosen = torch.tensor(routed.choose(l, None, 4, score))
    dw = torch.randn(5, 4, generator=gen).double()
    want, bound = routed.route_backward(dw, l, chosen, score, renormalise, 1.7)
    v = l.clone().requires_grad_()
    s = torch.softmax(v, 1) if score == "softmax" else torch.sigmoid(v)
    w = s.gather(1, chosen)
    w = 1.7 * (w / w.sum(1, keepdim=True) if renormalise else w)
    assert torch.allclose(w, routed.weights(l, chosen, score, renormalise, 1.7), rtol=1e-12)
    (w * dw).sum().backward()
    assert torch.allclose(v.grad, want, rtol=1e-10, atol=1e-13) and (bound >= 0).all()
    # Against differences (the choice held).
    h = 1e-6
    for e in range(9):
        up, down = l.clone(), l.clone()
        up[:, e] += h
        down[:, e] -= h
        diff = (routed.weights(up, chosen, score, renormalise, 1.7) -
                routed.weights(down, chosen, score, renormalise, 1.7)) / (2 * h)
        assert torch.allclose((diff * dw).sum(1), want[:, e], rtol=1e-6, atol=1e-8)


def test_plan_by_hand():
    assert routed.plan(torch.tensor([[2, 0], [0, -1], [2, 2]]), 3) == ([0, 2, 2, 5], [1, 2, 0, 4, 5], [2, 0, 1, -1, 3, 4])


@pytest.mark.parametrize("act", ["silu", "gelu", "leaky"])
def test_experts_gradient(act):
    gen = torch.Generator().manual_seed(6)
    M, k, E, C, F = 6, 3, 4, 5, 7
    new = lambda *s: torch.randn(*s, generator=gen).double()  # noqa: E731
    x, w, dy = new(M, C), torch.rand(M, k, generator=gen).double(), new(M, C)
    ws = [new(E, F, C) / 2, new(E, F, C) / 2, new(E, C, F) / 2]
    experts = torch.randint(-1, E, (M, k), generator=gen)
    experts[2] = 1  # one expert three times
    plan = routed.plan(experts, E)
    f = routed.experts_forward(x, w, *ws, plan, k, torch.float32, act, 0.1)
    leaves = [v.clone().requires_grad_() for v in (x, w, *ws)]
    rows = []
    for t in range(M):
        terms = [torch.zeros(C).double()]
        for s in range(k):
            e = int(experts[t, s])
            if e >= 0:
                g, u = leaves[2][e] @ leaves[0][t], leaves[3][e] @ leaves[0][t]
                a = {"silu": lambda v: v * torch.sigmoid(v), "gelu": lambda v: v * torch.special.ndtr(v),
                     "leaky": lambda v: torch.where(v >= 0, v, 0.1 * v)}[act](g)
                terms.append(leaves[1][t, s] * (leaves[4][e] @ (a * u)))
        rows.append(sum(terms))
    y = torch.stack(rows)
    assert torch.allclose(y, f["y"][0], rtol=1e-11, atol=1e-12)
    (y * dy).sum().backward()
    b = routed.experts_backward(dy, x, w, f["g"][0], f["u"][0], *ws, plan, k, torch.float32, act, 0.1)
    for name, leaf in zip(("dx", "dweights", "dw_gate", "dw_up", "dw_down"), leaves):
        assert torch.allclose(b[name][0].reshape(leaf.shape), leaf.grad, rtol=1e-10, atol=1e-11), name


def test_a_wrong_value_is_outside_the_bounds():
    """The bounds tell a result that takes one pair's weight or term wrongly."""
    gen = torch.Generator().manual_seed(8)
    M, k, E, C, F = 20, 2, 3, 64, 48
    new = lambda *s, std=1.0: (torch.randn(*s, generator=gen) * std).bfloat16().double()  # noqa: E731
    x, ws = new(M, C), [new(E, F, C, std=C ** -0.5), new(E, F, C, std=C ** -0.5), new(E, C, F, std=F ** -0.5)]
    experts, w = torch.randint(0, E, (M, k), generator=gen), torch.rand(M, k, generator=gen).double()
    plan = routed.plan(experts, E)
    value, bound = routed.experts_forward(x, w, *ws, plan, k, torch.bfloat16, "silu", 0.0)["y"]
    oracle.check("y", value.bfloat16(), value, bound, torch.bfloat16)
    w[3, 1] *= 1.2
    wrong = routed.experts_forward(x, w, *ws, plan, k, torch.bfloat16, "silu", 0.0)["y"][0]
    with pytest.raises(AssertionError):
        oracle.check("y", wrong.bfloat16(), value, bound, torch.bfloat16)
    assert math.isfinite(float(bound.max()))
