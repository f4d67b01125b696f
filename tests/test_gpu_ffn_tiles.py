"""Every instance of the gated block's matrix kernel, at ragged sizes
(test_sublayer_plan.py: which size takes which), against the definition in 64
bits; and the kernels for few tokens with sums long enough for several batches
of loads in flight.  The bounds are test_gpu_ffn.py's."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
import sublayer_oracle as oracle
from gpu_helpers import TORCH_DTYPES, say
from test_gpu_ffn import U32, activation_error, inputs, run_case, stored
from test_sublayer_plan import SIZES

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]


def product(a, bt, aerr=None):
    """a bt^T in 64 bits on the device, with test_gpu_ffn.product's bound."""
    b = bt.t().contiguous()
    v, k = a @ b, (a.shape[1] + 4) * U32
    babs = b.abs()
    err = k * (a.abs() @ babs)
    return v, err if aerr is None else err + (1 + k) * (aerr @ babs)


def near(name, got, want, err, dtype):
    assert torch.isfinite(got).all(), name
    off = (got.double() - want).abs() / stored(want, err, dtype)
    assert float(off.max()) <= 1.0, "%s is %.2f of its bound off" % (name, float(off.max()))


@pytest.mark.parametrize("number", range(len(SIZES)))
def test_instances(number):
    dtype, M, C, F = SIZES[number]
    act, in_place = ("silu", "gelu", "leaky")[number % 3], number % 2 == 0
    say("tiles: %s M=%d C=%d F=%d %s" % (dtype, M, C, F, act))
    d, slope = TORCH_DTYPES[dtype], 0.1
    dev = {k: v.cuda() for k, v in inputs(M, C, F, dtype).items()}
    f = {k: v.double() for k, v in dev.items()}
    nan = lambda *s: torch.full(s, float("nan"), dtype=d, device="cuda")  # noqa: E731
    ws = torch.full((iabn.iabn_ffn_workspace_size(M, C, F, d) // 2,), float("nan"), dtype=torch.bfloat16, device="cuda")

    def forward():
        y, g, u = nan(M, C), nan(M, F), nan(M, F)
        iabn.iabn_ffn_forward(dev["x"], dev["wg"], dev["wu"], dev["wd"], y, g, u, act=act, slope=slope, workspace=ws)
        return y, g, u

    (y, g, u), again = forward(), forward()
    assert all(torch.equal(a, b) for a, b in zip((y, g, u), again))
    gv, ge = product(f["x"], f["wg"])
    uv, ue = product(f["x"], f["wu"])
    near("g", g, gv, ge, d)
    near("u", u, uv, ue, d)
    av, _ = oracle.act(gv, act, slope)
    ae, _ = activation_error(gv, ge, act, slope)
    h = av * uv
    he = stored(h, ae * uv.abs() + av.abs() * ue + ae * ue + 2 * U32 * h.abs(), d)
    near("y", y, *product(h, f["wd"], he), d)
    del gv, ge, uv, ue, av, ae, h, he, again

    gs, us = g.double(), u.double()

    def backward():
        a, b = g.clone(), u.clone()
        dx, dwg, dwu, dwd = nan(M, C), nan(F, C), nan(F, C), nan(C, F)
        dg, du = (a, b) if in_place else (nan(M, F), nan(M, F))
        iabn.iabn_ffn_backward(dev["dy"], dev["x"], a, b, dev["wg"], dev["wu"], dev["wd"], dx, dg, du, dwg, dwu, dwd,
                               act=act, slope=slope, workspace=ws)
        return dx, dg, du, dwg, dwu, dwd

    out, again = backward(), backward()
    assert all(torch.equal(a, b) for a, b in zip(out, again))
    dx, dg, du, dwg, dwu, dwd = out
    av, dv = oracle.act(gs, act, slope)
    ae, de = activation_error(gs, torch.zeros_like(gs), act, slope)
    dh, dhe = product(f["dy"], f["wd"].t().contiguous())
    dgv, duv, h = dh * us * dv, dh * av, av * us
    dge = dhe * (us * dv).abs() + (dh * us).abs() * de + dhe * us.abs() * de + 3 * U32 * dgv.abs()
    due = dhe * av.abs() + dh.abs() * ae + dhe * ae + 2 * U32 * duv.abs()
    near("dg", dg, dgv, dge, d)
    near("du", du, duv, due, d)
    dge, due = stored(dgv, dge, d), stored(duv, due, d)
    he = stored(h, ae * us.abs() + 2 * U32 * h.abs(), d)
    t = lambda v: v.t().contiguous()  # noqa: E731
    a, ea = product(dgv, t(f["wg"]), dge)
    b, eb = product(duv, t(f["wu"]), due)
    near("dx", dx, a + b, ea + eb + (2 * F + 4) * U32 * (dgv.abs() @ f["wg"].abs() + duv.abs() @ f["wu"].abs()), d)
    near("dw_gate", dwg, *product(t(dgv), t(f["x"]), t(dge)), d)
    near("dw_up", dwu, *product(t(duv), t(f["x"]), t(due)), d)
    v, e = product(t(h), t(f["dy"]), t(he))
    near("dw_down", dwd, t(v), t(e), d)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", [1, 17, 50, 64])
@pytest.mark.parametrize("C,F", [(4104, 640), (2056, 2048), (3100, 2056), (1031, 2011)])
def test_few_tokens_long_sums(M, C, F, dtype):
    run_case(M, C, F, dtype, train=M != 17)
