"""The backward of layer norms on rows whose mean is far larger than their
spread: the normalised row is (v - mean)*rstd, and the subtraction of two
values that are close loses nothing that they held.

Given the stored statistics, v - mean is rounded once and its product with
rstd once, so a normalised value is within 2 * 2^-24 of its own size (not of
mean/spread), whatever the mean."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
from gpu_helpers import say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

U = 2.0 ** -24


def rows(R, C, mean, seed):
    """Rows about `mean` with a spread of one, their statistics as stored (fp32),
    and the normalised rows that these define, in 64 bits."""
    gen = torch.Generator().manual_seed(seed)
    v = torch.randn(R, C, generator=gen) + mean
    d = v.double()
    mu = d.mean(1).float()
    rstd = (1 / (d.var(1, unbiased=False) + 1e-5).sqrt()).float()
    hat = (d - mu.double()[:, None]) * rstd.double()[:, None]
    return v, torch.stack([mu, rstd]), hat


def near(name, got, want, bound):
    off = (got.cpu().double() - want).abs() - bound
    assert float(off.max()) <= 0, "%s is %.3g beyond its bound (of at most %.3g)" % (
        name, float(off.max()), float(bound.max()))


@pytest.mark.parametrize("mean", [300.0, -1e4])
@pytest.mark.parametrize("C", [64, 512, 640, 1501, 2048, 4100, 9000])
def test_gradients(C, mean):
    for R in (1, 7):
        say("large mean: %dx%d about %g" % (R, C, mean))
        r, pre, rhat = rows(R, C, mean, 1)
        h, post, hhat = rows(R, C, -mean, 2)
        gen = torch.Generator().manual_seed(3)
        du, dr, qw, pw = (torch.randn(*s, generator=gen) for s in ((R, C), (R, C), (C,), (C,)))
        dev = {k: t.cuda() for k, t in dict(r=r, h=h, du=du, dr=dr, qw=qw, pw=pw, pre=pre, post=post).items()}
        du, dr, qw, pw = du.double(), dr.double(), qw.double(), pw.double()

        def gradient(d, hat, rstd):
            """The layer norm's, with the sums of its terms' absolute values."""
            value = d - d.mean(1, keepdim=True) - hat * (d * hat).mean(1, keepdim=True)
            size = d.abs() + d.abs().mean(1, keepdim=True) + hat.abs() * (d * hat).abs().mean(1, keepdim=True)
            return value * rstd[:, None], size * rstd[:, None]

        # Roundings in a row: 2 of hat, 16 terms of a thread, 6 steps of a wave, 16
        # waves and 8 of the formula itself.
        ops = 48
        # The norm before the next block.
        dx, w, b = torch.empty_like(dev["r"]), torch.empty_like(dev["qw"]), torch.empty_like(dev["qw"])
        iabn.iabn_resnorm_backward(dev["dr"], dev["du"], dev["r"], None, dx, None, pre_norm="layer",
                                   pre_weight=dev["qw"], pre_stats=dev["pre"], dpre_weight=w, dpre_bias=b)
        v, size = gradient(du * qw, rhat, pre[1].double())
        near("dx", dx, dr + v, ops * U * (dr.abs() + size))
        # A sum over R rows: 2 roundings of hat, one each of the product and of R sums.
        near("dpre_weight", w, (du * rhat).sum(0), (4 + R) * U * (du * rhat).abs().sum(0))
        # The norm after a block (no gate, no dropout: what arrives is dr).
        dh, w = torch.empty_like(dev["h"]), torch.empty_like(dev["pw"])
        iabn.iabn_resnorm_backward(dev["dr"], None, None, dev["h"], None, dh, post_norm="layer",
                                   post_weight=dev["pw"], post_stats=dev["post"], dpost_weight=w)
        v, size = gradient(dr * pw, hhat, post[1].double())
        near("dh", dh, v, ops * U * size)
        near("dpost_weight", w, (dr * hhat).sum(0), (4 + R) * U * (dr * hhat).abs().sum(0))


@pytest.mark.parametrize("C", [128, 777])
def test_gate(C):
    """The gate's gradient takes the normalised row too."""
    R = 5
    h, post, hhat = rows(R, C, 5e3, 4)
    dr, gate = torch.randn(R, C), torch.randn(R, C)
    dgate, dh = torch.empty(R, C, device="cuda"), torch.empty(R, C, device="cuda")
    iabn.iabn_resnorm_backward(dr.cuda(), None, None, h.cuda(), None, dh, gate=gate.cuda(), post_norm="layer",
                               post_stats=post.cuda(), dgate=dgate)
    want = dr.double() * hhat
    near("dgate", dgate, want, 4 * U * want.abs())
