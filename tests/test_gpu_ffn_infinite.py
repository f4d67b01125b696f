"""Projections that are infinite as stored (fp16 ones overflow at 65520) are at
the activations' limits: a forward that was finite has a finite backward."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
from gpu_helpers import TORCH_DTYPES, say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

INF = float("inf")


@pytest.mark.parametrize("act,slope", [("silu", 0.0), ("gelu", 0.0), ("leaky", 0.0), ("leaky", 0.25)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_limits(act, slope, dtype):
    say("infinite projections: %s %s" % (act, dtype))
    d = TORCH_DTYPES[dtype]
    g = torch.tensor([[-INF], [INF], [float("nan")], [1.0]], dtype=d, device="cuda")
    u = torch.ones_like(g)
    x = torch.ones(4, 2, dtype=d, device="cuda")
    w, wd = torch.ones(1, 2, dtype=d, device="cuda"), torch.tensor([[1.0], [0.0]], dtype=d, device="cuda")
    dy = torch.tensor([[1.0, 0.0]], dtype=d, device="cuda").repeat(4, 1)
    dx, dg, du = torch.empty_like(x), torch.empty_like(g), torch.empty_like(g)
    iabn.iabn_ffn_backward(dy, x, g, u, w, w, wd, dx, dg, du, *[torch.empty_like(t) for t in (w, w, wd)], act=act,
                           slope=slope)
    a, da = du[:, 0].tolist(), dg[:, 0].tolist()
    assert a[0] == (-INF if slope else 0.0) and a[1] == INF and a[2] != a[2]
    assert da[:2] == [slope if act == "leaky" else 0.0, 1.0]
    assert da[2] != da[2] or act == "leaky"


@pytest.mark.parametrize("act", ["silu", "gelu", "leaky"])
def test_an_overflow_below(act):
    """g = -90000 is -inf in fp16: y is 0, and so are the gradients through it."""
    d = torch.float16
    x = torch.tensor([[300.0, 1.0], [1.0, 0.5]], dtype=d, device="cuda")
    wg = torch.tensor([[-300.0, 0.0], [0.5, 0.25]], dtype=d, device="cuda")
    wu = torch.tensor([[0.5, 0.0], [0.25, 0.5]], dtype=d, device="cuda")
    wd = torch.tensor([[1.0, 1.0], [0.5, -1.0]], dtype=d, device="cuda")
    y, g, u = (torch.empty_like(x) for _ in range(3))
    iabn.iabn_ffn_forward(x, wg, wu, wd, y, g, u, act=act, slope=0.0)
    assert g[0, 0].item() == -INF and torch.isfinite(y).all()
    out = [torch.empty_like(x) for _ in range(6)]
    iabn.iabn_ffn_backward(torch.ones_like(x), x, g, u, wg, wu, wd, *out, act=act, slope=0.0)
    assert all(torch.isfinite(t).all() for t in out)
    assert out[1][0, 0].item() == 0.0 and out[2][0, 0].item() == 0.0
