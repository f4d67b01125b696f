"""The example's backward overwrites the two projections that its forward kept.
A second backward through the same graph therefore has to fail, not to compute
from what is left there."""

from __future__ import annotations

import pytest
import torch

from test_gpu_sublayer import example  # noqa: F401  (a fixture)

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]


def test_a_second_backward_is_refused(example):  # noqa: F811
    torch.manual_seed(1)
    model = example.Stack(64, 96, 1, torch.float32)
    x = torch.randn(10, 64, device="cuda")
    loss = model(x).square().sum()
    loss.backward(retain_graph=True)
    first = [p.grad.clone() for p in model.parameters()]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    model.zero_grad()
    model(x).square().sum().backward()
    assert all(torch.equal(p.grad, g) for p, g in zip(model.parameters(), first))
