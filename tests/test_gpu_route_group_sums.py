"""Groups whose score is a sum of two that cancel, or that leaves fp32's range: the
groups that iabn_route_forward keeps are those of 64-bit sums.

A score plus a bias of B is off by B*2^-24 in fp32, however small the sum of two such
values is; sums that differ by less than that have to be told apart all the same."""

from __future__ import annotations

import pytest
import torch

import routed_oracle as routed
from test_gpu_route import run

INF = float("inf")
pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]


def close_sums(M, groups, per, B, seed):
    """Logits and biases: of every group the two highest have biases of opposite sign
    (B*(g % 3), so that some groups have none), the others lie far below; a row's
    logits are alike but for a few units of 2^-22, those of the others any (they make
    a softmax's scores any numbers)."""
    gen = torch.Generator().manual_seed(seed)
    l = torch.rand(M, 1, 1, generator=gen) * 2 - 1
    l = l + torch.randint(-6, 7, (M, groups, per), generator=gen) * 2.0 ** -22
    l[:, :, 2:] += torch.rand(M, groups, per - 2, generator=gen)
    b = torch.full((groups, per), -4.0 * B)
    for g in range(groups):
        b[g, 0], b[g, 1] = B * (g % 3), -B * (g % 3)
    return l.reshape(M, -1).contiguous(), b.flatten().contiguous()


def told_apart(l, b, score, groups):
    """The rows of which 64-bit sums, however they are formed, say the order of the
    groups.  A score (at most 1) is off by at most 2^-50 (8 units) in either of two
    evaluations, each score plus its bias by 2^-53 of itself more, a sum of two by
    2^-53 of itself: a difference of two sums by less than 2^-48 + 2^-51 of the four
    values' sizes.  (The oracle's own choice is not the exact one in 7 of 1100 softmax
    rows of 4 groups of 3 with B = 1; all of them are closer than that.)"""
    c = (routed.scores(l, score) + b.double()).unflatten(1, (groups, -1))[:, :, :2]
    sums, sizes = c.sum(2), c.abs().sum(2)
    far = (sums[:, :, None] - sums[:, None]).abs() > 2.0 ** -48 + 2.0 ** -51 * (sizes[:, :, None] + sizes[:, None])
    return (far | torch.eye(groups, dtype=torch.bool)).all(2).all(1)


@pytest.mark.parametrize("M", [5, 1100])  # 64 and 16 lanes a row
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("B", [1.0, 16.0, 64.0, 256.0, 4096.0])
@pytest.mark.parametrize("groups,per,kept", [(2, 2, 1), (4, 3, 2), (8, 16, 3)])
def test_sums_that_cancel(M, score, B, groups, per, kept):
    for seed in range(20 if M == 5 else 1):
        l, b = close_sums(8 * M, groups, per, B, seed)
        l = l[told_apart(l, b, score, groups)][:M].contiguous()
        assert l.shape[0] == M or M == 5
        run(l, 2 * kept, bias=b, score=score, groups=groups, kept=kept, group_top=2)


@pytest.mark.parametrize("M", [5, 1100])
@pytest.mark.parametrize("B", [16.0, 64.0, 4096.0])
def test_sums_that_are_equal(M, B):
    """Scores of 1/2 make the sums exact: the lower group, whichever has the biases."""
    for biased in (0, 1):
        b = torch.zeros(4)
        b[2 * biased], b[2 * biased + 1] = B, -B
        got, _ = run(torch.zeros(M, 4), 2, bias=b, score="sigmoid", groups=2, kept=1, group_top=2)
        assert (got == torch.tensor([0, 1])).all()


@pytest.mark.parametrize("M", [5, 1100])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_sums_past_fp32(M, sign):
    """Two biases whose sum is past fp32's range: the groups are still in their order,
    and one below that range is not one with nothing in it."""
    b = sign * torch.tensor([2.5, 2.5, 3.0, 3.0, 2.0, 2.0]) * 1e38
    l = torch.zeros(M, 6)
    for kept in (1, 2):
        got, _ = run(l, 2 * kept, bias=b, score="sigmoid", groups=3, kept=kept, group_top=2)
        assert (got >= 0).all()
    l[:, :2] = -INF
    got, _ = run(l, 4, bias=b, score="sigmoid", groups=3, kept=2, group_top=2)
    assert (got >= 2).all()
