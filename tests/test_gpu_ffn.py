"""iabn_ffn_forward and iabn_ffn_backward on the GPU against their definition
in 64 bits.  Both sides take the same stored values; where the block rounds
between products (h, dg, du), so does the bound: a stored intermediate is off
by at most its unit roundoff, which the next product carries on."""

from __future__ import annotations

import math

import pytest
import torch

import paper_1712_02616_amd as iabn
import sublayer_oracle as oracle
from gpu_helpers import TORCH_DTYPES, say
from test_gpu_resnorm import guarded, placed

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

U32, UNIT, TINY = oracle.U32, oracle.UNIT, oracle.TINY


def product(a, b, aerr=None):
    """a b^T in 64 bits with a bound: a 32-bit sum of K terms in any order
    (K + 4 roundings of partial sums at most), and a's own error."""
    v, mag = a @ b.T, a.abs() @ b.abs().T
    err = (a.shape[1] + 4) * U32 * mag
    return v, err if aerr is None else err + aerr @ b.abs().T * (1 + (a.shape[1] + 4) * U32)


def activation_error(v, err, act, slope):
    """Bounds of act(v) and act'(v) computed in 32 bits from v off by err.  |act''|
    and |act'| are below 1.2; the functions themselves to 16 units of v's scale
    (their exponentials of up to v^2/2 or v are off by that in relative terms,
    against at most exp(-1)-sized values times v)."""
    if act == "leaky":
        near = v.abs() <= err  # either branch
        return err + 2 * U32 * v.abs(), torch.where(near, torch.ones_like(v), torch.zeros_like(v))
    return 1.2 * err + 16 * U32 * (1 + v.abs()), 1.2 * err + 16 * U32 * (1 + v.abs())


def stored(v, err, dtype):
    """The bound of a value that is rounded to storage."""
    return err * (1 + UNIT[dtype]) + UNIT[dtype] * v.abs() + TINY[dtype]


def inputs(M, C, F, dtype, seed=5):
    gen = torch.Generator().manual_seed(seed)
    d = TORCH_DTYPES[dtype]
    new = lambda a, b, s: (torch.randn(a, b, generator=gen) * s).to(d)  # noqa: E731
    return {"x": new(M, C, 1.0), "wg": new(F, C, 1 / math.sqrt(C)), "wu": new(F, C, 1 / math.sqrt(C)),
            "wd": new(C, F, 1 / math.sqrt(F)), "dy": new(M, C, 0.3)}


def run_case(M, C, F, dtype, act="silu", slope=0.1, shift=0, in_place=False, train=True, stream=None):
    say("ffn M=%d C=%d F=%d %s %s shift=%d in_place=%s" % (M, C, F, dtype, act, shift, in_place))
    d = TORCH_DTYPES[dtype]
    i = inputs(M, C, F, dtype)
    f = {k: v.double() for k, v in i.items()}
    dev = {k: placed(v, shift) for k, v in i.items()}
    checks = []

    def out(name, *shape):
        t, intact = guarded(shape, d, shift)
        checks.append((name, intact))
        return t

    y = out("y", M, C)
    g, u = (out("g", M, F), out("u", M, F)) if train else (None, None)
    torch.cuda.synchronize()
    assert iabn.iabn_ffn_forward(dev["x"], dev["wg"], dev["wu"], dev["wd"], y, g, u, act=act, slope=slope,
                                 stream=stream) is y
    torch.cuda.synchronize()
    gv, ge = product(f["x"], f["wg"])
    uv, ue = product(f["x"], f["wu"])
    av, _ = oracle.act(gv, act, slope)
    ae, _ = activation_error(gv, ge, act, slope)
    h = av * uv
    he = stored(h, ae * uv.abs() + av.abs() * ue + ae * ue + 2 * U32 * h.abs(), d)
    oracle.check("y", y, *product(h, f["wd"], he), d)
    if train:
        oracle.check("g", g, gv, ge, d)
        oracle.check("u", u, uv, ue, d)

        gs, us = g.cpu().double(), u.cpu().double()
        av, dv = oracle.act(gs, act, slope)
        ae, de = activation_error(gs, torch.zeros_like(gs), act, slope)
        dh, dhe = product(f["dy"], f["wd"].T)
        dgv, duv, h = dh * us * dv, dh * av, av * us
        dge = stored(dgv, dhe * (us * dv).abs() + (dh * us).abs() * de + dhe * us.abs() * de + 3 * U32 * dgv.abs(), d)
        due = stored(duv, dhe * av.abs() + dh.abs() * ae + dhe * ae + 2 * U32 * duv.abs(), d)
        he = stored(h, ae * us.abs() + 2 * U32 * h.abs(), d)
        dx, dwg, dwu, dwd = out("dx", M, C), out("dwg", F, C), out("dwu", F, C), out("dwd", C, F)
        dg, du = (g, u) if in_place else (out("dg", M, F), out("du", M, F))
        torch.cuda.synchronize()
        iabn.iabn_ffn_backward(dev["dy"], dev["x"], g, u, dev["wg"], dev["wu"], dev["wd"], dx, dg, du, dwg, dwu, dwd,
                               act=act, slope=slope, stream=stream)
        torch.cuda.synchronize()
        a, ea = product(dgv, f["wg"].T, dge)
        b, eb = product(duv, f["wu"].T, due)
        oracle.check("dx", dx, a + b, ea + eb + (2 * F + 4) * U32 * (dgv.abs() @ f["wg"].abs() + duv.abs() @ f["wu"].abs()),
                     d)
        oracle.check("dw_gate", dwg, *product(dgv.T, f["x"].T, dge.T), d)
        oracle.check("dw_up", dwu, *product(duv.T, f["x"].T, due.T), d)
        v, e = product(h.T, f["dy"].T, he.T)
        oracle.check("dw_down", dwd, v.T, e.T, d)
        # dg and du are stored from what their bounds hold already.
        for name, got, want, err in (("dg", dg, dgv, dge), ("du", du, duv, due)):
            off = (got.cpu().double() - want).abs() - err
            assert float(off.max()) <= 0, "%s is off by %g more than its bound" % (name, float(off.max()))
    for name, intact in checks:
        intact(name)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,C,F", [(1, 1, 1), (1, 64, 128), (2, 8, 24), (3, 7, 5), (16, 128, 256), (17, 96, 64),
                                   (40, 200, 136), (64, 72, 88), (65, 129, 33), (130, 64, 260), (200, 333, 137),
                                   (513, 40, 8)])
def test_shapes(M, C, F, dtype):
    run_case(M, C, F, dtype)


@pytest.mark.parametrize("act", ["silu", "gelu", "leaky"])
@pytest.mark.parametrize("M", [4, 150])
def test_activations(act, M):
    run_case(M, 72, 104, "f32", act=act)
    run_case(M, 72, 104, "f16", act=act, slope=0.0)


@pytest.mark.parametrize("dtype,shift", [("f32", 1), ("f16", 1), ("bf16", 3), ("f16", 4)])
@pytest.mark.parametrize("M", [1, 9, 140])
def test_alignment(dtype, shift, M):
    run_case(M, 136, 200, dtype, shift=shift)


@pytest.mark.parametrize("M", [1, 30, 300])
def test_inference_and_in_place(M):
    run_case(M, 160, 96, "bf16", train=False)
    run_case(M, 160, 96, "f16", in_place=True)


@pytest.mark.parametrize("M,C,F", [(2048, 256, 1536), (1536, 1100, 2056)])
def test_large_tiles(M, C, F):
    """Enough tiles for the larger ones, and ragged edges of them."""
    run_case(M, C, F, "f16")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,C,F", [(1, 40, 4096), (20, 96, 4104), (50, 33, 3001), (100, 64, 4096), (70, 2056, 136),
                                   (3000, 40, 48), (3001, 41, 47)])
def test_long_sums(M, C, F, dtype):
    """Few tiles and a long sum, which is split over blocks."""
    run_case(M, C, F, dtype)


def test_another_stream():
    st = torch.cuda.Stream()
    run_case(100, 96, 128, "bf16", stream=st)
    run_case(5, 96, 128, "f32", stream=st.cuda_stream)


def test_empty():
    d = torch.float16
    new = lambda *s: torch.full(s, 3.0, dtype=d, device="cuda")  # noqa: E731
    w, wd = new(24, 16), new(16, 24)
    y = new(0, 16)
    iabn.iabn_ffn_forward(new(0, 16), w, w, wd, y, new(0, 24), new(0, 24))
    dwg, dwu, dwd = new(24, 16), new(24, 16), new(16, 24)
    iabn.iabn_ffn_backward(new(0, 16), new(0, 16), new(0, 24), new(0, 24), w, w, wd, new(0, 16), new(0, 24), new(0, 24),
                           dwg, dwu, dwd)
    assert all((t == 0).all() for t in (dwg, dwu, dwd))
    y = new(5, 16)
    iabn.iabn_ffn_forward(new(5, 16), new(0, 16), new(0, 16), new(16, 0), y)
    assert (y == 0).all()


@pytest.mark.parametrize("M", [3, 200])
def test_a_bad_row_stays_in_its_row(M):
    i = {k: v.cuda() for k, v in inputs(M, 100, 64, "bf16").items()}
    ys = []
    for bad in (False, True):
        if bad:
            i["x"][1, 7] = float("nan")
        y = torch.empty_like(i["x"])
        ys.append(iabn.iabn_ffn_forward(i["x"], i["wg"], i["wu"], i["wd"], y))
    rows = [r for r in range(M) if r != 1]
    assert torch.equal(ys[0][rows], ys[1][rows]) and torch.isnan(ys[1][1]).all()
