"""fp32 experts: what a long sum loses is bounded by parts of 256 terms and their number,
not by its length.  A first term of 2^24 swallows every 1 that is added to it on its
own; sums of 1's are exact."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

M = 100  # (more than the few tokens' kernels take)
BIG = 4096.0


def check(name, got, terms, parts=None):
    """Each of `terms` terms: BIG^2, and ones.  A part of 256 terms rounds 256 times, the
    parts' sum as often as there are parts (two more where a sum is of two products),
    each by half a step of at most the sum."""
    want = BIG * BIG + terms - 1
    allowed = (256 + (parts or -(-terms // 256)) + 2) * 2.0 ** -24 * want
    assert allowed < 0.15 * terms
    off = float((got.double() - want).abs().max())
    assert off <= allowed, (name, off, allowed)


def vector(n):
    v = torch.ones(n)
    v[0] = BIG
    return v


def plan_of_one(rows):
    plan = torch.empty(iabn.iabn_experts_plan_size(rows, 1, 1), dtype=torch.int32, device="cuda")
    return iabn.iabn_experts_plan(torch.zeros(rows, 1, dtype=torch.int32, device="cuda"), plan, 1)


@pytest.mark.parametrize("F", [4096, 4097, 8190])
@pytest.mark.parametrize("C", [64, 5, 3])  # (3: k-strided rows too short to be fetched)
def test_down_and_dx(C, F):
    """y sums over the hidden width; dx too, of the gate's and of the up projection's
    gradients."""
    new = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    x, w_gate, w_up, w_down = new(M, C), new(1, F, C), new(1, F, C), new(1, C, F)
    x[:, 0] = 1.0
    w_gate[:, :, 0], w_up[0, :, 0], w_down[:] = 1.0, vector(F).cuda(), vector(F).cuda()
    plan, w = plan_of_one(M), torch.ones(M, 1, device="cuda")
    y = iabn.iabn_experts_forward(x, plan, w, w_gate, w_up, w_down, torch.empty_like(x), act="leaky", slope=0.0)
    check("y", y, F)
    # dy W_d = (BIG, 1, ...) from the first column; g = u = 1.
    dy = x
    w_down[:, 1:] = 0.0
    for of in ("gate", "up"):
        w_gate[:], w_up[:] = 0.0, 0.0
        (w_gate if of == "gate" else w_up)[0] = vector(F).cuda()[:, None]
        g, dx = torch.ones(M, F, device="cuda"), torch.empty_like(x)
        iabn.iabn_experts_backward(dy, x, plan, w, g, g.clone(), w_gate, w_up, w_down, dx, torch.empty_like(w),
                                   torch.empty_like(g), torch.empty_like(g), *[torch.empty_like(v) for v in
                                                                               (w_gate, w_up, w_down)], act="leaky")
        check("dx of " + of, dx, F)


@pytest.mark.parametrize("C", [4096, 4099])
@pytest.mark.parametrize("F", [64, 7, 3])
def test_projections_and_dh(C, F):
    """g and u sum over the width; dh too, which dg and du are here."""
    new = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    x = vector(C).cuda().expand(M, C).contiguous()
    w_gate, w_up, w_down = (vector(C).cuda().expand(1, F, C).contiguous() for _ in range(3))
    w_down = w_down.transpose(1, 2).contiguous()
    plan, w = plan_of_one(M), torch.ones(M, 1, device="cuda")
    g, u = new(M, F), new(M, F)
    iabn.iabn_experts_forward(x, plan, w, w_gate, w_up, w_down, new(M, C), g, u, act="leaky")
    check("g", g, C)
    check("u", u, C)
    one, dg, du = torch.ones(M, F, device="cuda"), new(M, F), new(M, F)
    iabn.iabn_experts_backward(x, x, plan, w, one, one.clone(), w_gate, w_up, w_down, new(M, C), new(M, 1), dg, du,
                               new(1, F, C), new(1, F, C), new(1, C, F), act="leaky")
    check("dg", dg, C)
    check("du", du, C)


@pytest.mark.parametrize("rows,k,E,N", [(16, 4, 64, 512), (1, 1, 1, 24), (40, 8, 64, 256), (50, 2, 3, 40)])
def test_few_tokens(rows, k, E, N):
    """Few tokens' kernels: a wave adds 256 terms, a block has 8 waves for 2048 (many
    blocks too, whose waves would fill the chip with fewer)."""
    K = 2048
    ones = torch.zeros(rows, K, device="cuda")
    ones[:, 0] = 1.0
    x = vector(K).cuda().expand(rows, K).contiguous()
    w = vector(K).cuda().expand(E, N, K).contiguous()
    chosen = torch.arange(rows * k, dtype=torch.int32, device="cuda").view(rows, k) % E
    plan = torch.empty(iabn.iabn_experts_plan_size(rows, k, E), dtype=torch.int32, device="cuda")
    iabn.iabn_experts_plan(chosen, plan, E)
    weights = torch.zeros(rows, k, device="cuda")
    weights[:, 0] = 1.0
    g, u = (torch.empty(rows * k, N, device="cuda") for _ in range(2))
    iabn.iabn_experts_forward(x, plan, weights, w, w, w.transpose(1, 2).contiguous(), torch.empty_like(x), g, u)
    check("g", g, K, parts=8)
    check("u", u, K, parts=8)
    # y: h = (BIG, 1, ...), the down weights too.
    x, wide = ones[:, :N].contiguous(), torch.zeros(E, K, N, device="cuda")
    wide[:, :, 0] = 1.0
    up = wide.clone()
    up[:, 0, 0] = BIG
    y = iabn.iabn_experts_forward(x, plan, weights, wide, up, w, torch.empty_like(x), act="leaky")
    check("y", y, K, parts=8 + 16)  # (a sum may be split over 16 blocks)
