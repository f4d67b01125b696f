"""iabn_grad_clip at the ends of fp32: an infinite limit and an infinite norm."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

INF, NAN = float("inf"), float("nan")


def clip(grads, norm, max_norm, in_place=False):
    outs = grads if in_place else [torch.full_like(g, 7.0) for g in grads]
    iabn.iabn_grad_clip(grads, outs, torch.tensor([norm], device="cuda"), max_norm)
    torch.cuda.synchronize()
    return outs


def bits(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("in_place", [False, True])
def test_no_limit_leaves_gradients_of_an_infinite_norm(in_place):
    """max_norm = inf clips nothing, whatever the norm; a norm that is NaN shows."""
    for d in (torch.float32, torch.float16, torch.bfloat16):
        g = torch.linspace(-3, 5, 4099).to(d).cuda()
        g[7], g[9] = INF, -INF
        for norm in (INF, 3.0, 0.0):
            got = clip([g.clone()], norm, INF, in_place)[0]
            assert torch.equal(bits(got), bits(g)), (d, norm)
        assert torch.isnan(clip([g.clone()], NAN, INF, in_place)[0]).all()
    # Finite gradients whose norm is past fp32.
    large = torch.full((64,), torch.finfo(torch.float32).max, device="cuda")
    norm = iabn.iabn_grad_norm([large], torch.zeros(1, device="cuda"))
    assert float(norm) == INF
    assert torch.equal(iabn.iabn_grad_clip([large], [torch.empty_like(large)], norm, INF)[0], large)
    assert (iabn.iabn_grad_clip([large], [torch.empty_like(large)], norm, 1.0)[0] == 0).all()
