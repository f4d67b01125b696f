"""iabn_grad_clip at the ends of fp32: an infinite limit and an infinite norm, and
factors below fp32's smallest normal number."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
import sublayer_oracle as oracle

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

INF, NAN = float("inf"), float("nan")
U32 = 2.0 ** -24


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


@pytest.mark.parametrize("max_norm", [2.0 ** -149, 1e-40, 1e-30, 1e-10, 1e-3, 1.0])
@pytest.mark.parametrize("norm", [2.0 ** 127, 3e38, 1e33, 1e12])
def test_small_factors_keep_their_digits(norm, max_norm):
    """A factor of less than 2^-126 has fewer digits as an fp32 number; the product
    with a large gradient shows it.  The bound is that of any factor: the factor's
    rounding and the product's, and a rounding of a subnormal result."""
    gen = torch.Generator().manual_seed(5)
    for d in (torch.float32, torch.bfloat16):
        g = (torch.randn(5000, generator=gen) * (norm / 8)).clamp(-2.0 ** 127, 2.0 ** 127).to(d)
        limit = float(torch.tensor(max_norm))  # (as the call takes it)
        v = g.double() * min(1.0, limit / (float(torch.tensor(norm)) + 1e-6))
        for in_place in (False, True):
            got = clip([g.cuda()], norm, max_norm, in_place)[0]
            oracle.check("%s norm %g max %g" % (d, norm, max_norm), got, v, 2 * U32 * v.abs() + 2.0 ** -150, d)


@pytest.mark.parametrize("norm", [float.fromhex("0x1.fffff0p+0"), float.fromhex("0x1.fde722p-13"), 2.0])
def test_a_small_factor_is_no_factor_of_one(norm):
    """Limits of 2^-140 over these norms (and 10^-6) are a power of two to within 2^-25."""
    g = torch.linspace(-norm, norm, 999)
    v = g.double() * (2.0 ** -140 / (norm + 1e-6))
    for in_place in (False, True):
        got = clip([g.cuda()], norm, 2.0 ** -140, in_place)[0]
        oracle.check("norm %g" % norm, got, v, 2 * U32 * v.abs() + 2.0 ** -150, torch.float32)


def test_refuses_outputs_over_what_it_reads():
    x = torch.ones(64, device="cuda")
    a, b, norm = x[:16], x[16:32], torch.full((1,), 3.0, device="cuda")
    for grads, outs, n in (([a, b], [b, a], norm), ([a], [x[1:17]], norm), ([a], [b], x[31:32]), ([a], [a], x[:1]),
                           ([a, x[8:24]], [a, x[40:56]], norm)):
        with pytest.raises(iabn.IabnError) as e:
            iabn.iabn_grad_clip(grads, outs, n, 1.0)
        assert e.value.status == 3
    assert (x == 1).all()
    outs = iabn.iabn_grad_clip([a, b, a], [a.clone(), b, x[32:48]], norm, 1.0)
    assert all(torch.equal(o, outs[0]) for o in outs) and (x[:16] == 1).all() and (x[48:] == 1).all()
