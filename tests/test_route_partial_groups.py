"""A group with fewer usable experts than group_top has the sum of those that it has:
an expert that is switched off takes nothing from the others of its group.  By hand in
the oracle (CPU), and the kernel against it."""

from __future__ import annotations

import pytest
import torch

import routed_oracle as routed

INF = float("inf")

# Three groups of two; scores are sigmoids: 1/2 of 0, 0.88 of 2, 0.95 of 3, 0.12 of -2.
ROWS = torch.tensor([[3.0, -INF, -2.0, -2.0, 0.0, 0.0],      # 0.95, 0.24, 1.0
                     [3.0, -INF, -2.0, -2.0, -INF, 0.0],     # 0.95, 0.24, 0.5
                     [-INF, -INF, -2.0, -INF, -2.0, -2.0],   # nothing, 0.12, 0.24
                     [-INF, -INF, -INF, -INF, -INF, 2.0]])   # nothing, nothing, 0.88


@pytest.mark.parametrize("biased", [False, True])
def test_by_hand(biased):
    bias = torch.zeros(6) if biased else None
    kw = dict(score="sigmoid", groups=3, group_top=2)
    assert routed.choose(ROWS, bias, 2, kept=1, **kw) == [[4, 5], [0, -1], [4, 5], [5, -1]]
    assert routed.choose(ROWS, bias, 3, kept=2, **kw) == [[0, 4, 5], [0, 5, -1], [2, 4, 5], [5, -1, -1]]
    # Switched off by the bias: the same.
    off = torch.tensor([0.0, -INF, 0.0, 0.0, 0.0, 0.0])
    assert routed.choose(ROWS[:1].clamp(min=-2.0), off, 2, kept=2, **kw) == [[0, 4]]


@pytest.mark.parametrize("M", [7, 1100])  # 64 and 16 lanes a row
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("groups,per,kept", [(3, 2, 1), (3, 2, 2), (8, 4, 3), (4, 64, 2)])
@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")
def test_kernel(M, score, biased, groups, per, kept):
    from test_gpu_route import run

    gen = torch.Generator().manual_seed(groups * per)
    E = groups * per
    if E == 6:
        run(ROWS, 2 * kept, score=score, groups=groups, kept=kept, group_top=2)
    l = torch.randn(M, E, generator=gen) * 1.5
    # Of every group 0, 1, 2 or all experts are left, row by row another number.
    left = torch.randint(0, 4, (M, groups, 1), generator=gen)
    rank = torch.rand(M, groups, per, generator=gen).argsort(2)
    l[((rank >= left) & (left < 3)).view(M, E)] = -INF
    bias = torch.randn(E, generator=gen) * 0.05 if biased else None
    if biased:
        bias[::5] = -INF
    for group_top in (1, 2):
        run(l, min(2 * kept, E), bias=bias, score=score, groups=groups, kept=kept, group_top=group_top)
