"""The gated block's activations one value at a time: weights that pick the
value v for the gate and 1 for the other projection, so that the block's result
is act(v) and its gradients are act'(v) and act(v).  The values reach into the
tails, where the functions themselves become small: their errors are bounded
relative to them.

U = 2^-24.  A 32-bit evaluation of exp(-v^2/2) is off by U v^2 or so from its
argument's roundings (at most 4 of them), of exp(-v) by U |v|; Phi of 16-bit
values adds its polynomial's 2^-19; the library's functions and divisions for
fp32 values, some units.  Then one rounding to storage.  Values below 2^-118
may be lost to the exponential's range."""

from __future__ import annotations

import math

import pytest
import torch

import paper_1712_02616_amd as iabn
from gpu_helpers import TORCH_DTYPES, say
from sublayer_oracle import TINY, UNIT

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

U = 2.0 ** -24


def exact(v, act):
    """act(v), act'(v) in 64 bits, and the bounds of both before storage."""
    if act == "silu":
        s = torch.sigmoid(v)
        return v * s, s * (1 + v * (1 - s)), (v * s).abs(), s * (1 + v.abs()), lambda f32: (
            16 * U if f32 else (16 + 4 * v.abs()) * U)
    if act == "gelu":
        c, e = 0.5 * torch.special.erfc(-v / math.sqrt(2)), torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
        return v * c, c + v * e, (v * c).abs(), c + v.abs() * e, lambda f32: (
            (32 + 8 * v * v) * U + (0.0 if f32 else 2.0 ** -19))
    a = torch.where(v >= 0, v, 0.125 * v)
    d = torch.where(v >= 0, torch.ones_like(v), torch.full_like(v, 0.125))
    return a, d, a.abs(), d, lambda f32: 0.0


def near(name, got, want, err, dtype):
    off = (got.cpu().double() - want).abs() / (err * (1 + UNIT[dtype]) + UNIT[dtype] * want.abs() + TINY[dtype] + 2.0 ** -118)
    worst = int(off.argmax())
    assert float(off[worst]) <= 1.0, "%s: %.3g of the bound at value %d: %.9g, exact %.9g" % (
        name, float(off[worst]), worst, float(got[worst]), float(want[worst]))


@pytest.mark.parametrize("act", ["silu", "gelu", "leaky"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", [61, 3001])
def test_values(act, dtype, M):
    d = TORCH_DTYPES[dtype]
    for span in (1.0, 6.0, 30.0):
        say("activation %s %s to %g" % (act, dtype, span))
        v = torch.linspace(-span, span, M).to(d)
        x = torch.stack([v, torch.ones_like(v)], 1).cuda()
        wg = torch.tensor([[1.0, 0.0]], dtype=d, device="cuda")
        wu = torch.tensor([[0.0, 1.0]], dtype=d, device="cuda")
        wd = torch.tensor([[1.0], [0.0]], dtype=d, device="cuda")
        y, g, u = (torch.empty(M, n, dtype=d, device="cuda") for n in (2, 1, 1))
        iabn.iabn_ffn_forward(x, wg, wu, wd, y, g, u, act=act, slope=0.125)
        assert torch.equal(g[:, 0].cpu(), v) and (u == 1).all() and (y[:, 1] == 0).all()
        a, da, asize, dsize, rel = exact(v.double(), act)
        rel = rel(dtype == "f32")
        near("y", y[:, 0], a, rel * asize, d)
        dy = torch.tensor([[1.0, 0.0]], dtype=d, device="cuda").repeat(M, 1)
        dx, dg, du = torch.empty_like(x), torch.empty_like(g), torch.empty_like(g)
        iabn.iabn_ffn_backward(dy, x, g, u, wg, wu, wd, dx, dg, du, *[torch.empty_like(w) for w in (wg, wu, wd)],
                               act=act, slope=0.125)
        near("du", du[:, 0], a, rel * asize, d)
        near("dg", dg[:, 0], da, rel * dsize, d)


@pytest.mark.parametrize("act", ["silu", "gelu", "leaky"])
@pytest.mark.parametrize("dtype,large", [("f32", 3e38), ("f16", 6e4), ("bf16", 3e38)])
@pytest.mark.parametrize("M", [8, 80])
def test_large_values(act, dtype, large, M):
    """Far out the activations are v (or v's slope) and 0; a NaN and an infinity
    stay in their rows."""
    say("activation %s %s: large values" % (act, dtype))
    d = TORCH_DTYPES[dtype]
    inf, nan = float("inf"), float("nan")
    v = torch.tensor([large, 100.0, 0.0, -0.0, -150.0, -large, inf, nan]).repeat(M // 8).to(d)
    slope = 0.0
    g, u = v[:, None].cuda(), torch.ones(M, 1, dtype=d, device="cuda")
    low = 0.0 if act == "leaky" else 0.5
    a = torch.tensor([float(v[0]), 100.0, 0.0, 0.0, 0.0, 0.0, inf, nan]).repeat(M // 8)
    da = torch.tensor([1.0, 1.0, low or 1.0, low or 1.0, 0.0, 0.0, 1.0, nan]).repeat(M // 8)
    # The block as a whole: h = act(g), y = h.
    x = torch.stack([v, torch.ones_like(v)], 1)
    x[torch.isinf(v), 0] = large  # (0 * inf would be another value's NaN)
    x[torch.isnan(v), 0] = 1.0
    wg = torch.tensor([[1.0, 0.0]], dtype=d, device="cuda")
    wu = torch.tensor([[0.0, 1.0]], dtype=d, device="cuda")
    wd = torch.tensor([[1.0], [0.0]], dtype=d, device="cuda")
    y = torch.empty(M, 2, dtype=d, device="cuda")
    iabn.iabn_ffn_forward(x.cuda(), wg, wu, wd, y, act=act, slope=slope)
    finite = torch.isfinite(v)
    assert torch.equal(y[:, 0].cpu()[finite] + 0.0, a.to(d)[finite] + 0.0)
    dy = torch.tensor([[1.0, 0.0]], dtype=d, device="cuda").repeat(M, 1)
    dx, dg, du = torch.empty(M, 2, dtype=d, device="cuda"), torch.empty_like(g), torch.empty_like(g)
    iabn.iabn_ffn_backward(dy, x.cuda(), g, u, wg, wu, wd, dx, dg, du, *[torch.empty_like(w) for w in (wg, wu, wd)],
                           act=act, slope=slope)
    rows = ~torch.isnan(v)
    assert torch.equal(du[:, 0].cpu()[rows] + 0.0, a.to(d)[rows] + 0.0)
    assert torch.equal(dg[:, 0].cpu()[finite] + 0.0, da.to(d)[finite] + 0.0)
    if act != "leaky":
        assert torch.isnan(du[:, 0].cpu()[~rows]).all() and torch.isnan(dg[:, 0].cpu()[~rows]).all()
