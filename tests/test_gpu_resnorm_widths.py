"""The norms' kernels at the widths whose instances differ (rows of one wave,
of two to four, of up to eight and of up to sixteen, with one chunk of a thread
and with two; filled and partly filled), each with several rows per block; and
the in-place orders of both directions."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
from gpu_helpers import TORCH_DTYPES, say
from test_gpu_resnorm import EPS, inputs, run_case

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("R,C", [(1100, 504), (1100, 1024), (1100, 1536), (1100, 2048), (1100, 1100), (530, 3001), (530, 3584),
                                 (530, 4097), (530, 5000), (530, 8192), (300, 9001)])
def test_widths(R, C, dtype):
    run_case(R, C, dtype, "rms", "layer", 1, 0.1)
    run_case(R, C, dtype, "layer", "rms", 10, 0.0, vectors=C % 2 == 0)


@pytest.mark.parametrize("C", [1536, 2048, 4097, 8192])
def test_parts(C):
    """Only one side of the block at those widths."""
    run_case(520, C, "bf16", None, "rms", 520, 0.25)
    run_case(520, C, "f16", "layer", None, 0, 0.25)
    run_case(520, C, "f16", None, "layer", 0, 0.0, branch=False)


WIDTHS = [3, 96, 505, 512, 777, 1024, 2048, 4100, 9000]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_in_place_forward(C, dtype):
    """r over x or h, u over x or h: the same bits as apart."""
    R = 21
    say("in place: forward %dx%d %s" % (R, C, dtype))
    i = {k: None if v is None else v.cuda() for k, v in inputs(R, C, dtype, 3).items()}
    for post, pre, with_h in (("layer", "rms", True), (None, "layer", True), ("rms", None, True), (None, None, True),
                              (None, "rms", False)):
        def call(x, h, r, u):
            stats = torch.empty(2, R, device="cuda"), torch.empty(2, R, device="cuda")
            iabn.iabn_resnorm_forward(x, h, r, u, gate=i["gate"] if with_h else None, post_norm=post, pre_norm=pre,
                                      post_stats=stats[0] if post else None, pre_stats=stats[1] if pre else None,
                                      alpha=0.5, beta=0.75, eps=EPS, p=0.25 if with_h else 0.0, seed=3)
            return [t for t, on in zip(stats, (post, pre)) if on]

        r, u = torch.empty_like(i["x"]), torch.empty_like(i["x"])
        stats = call(i["x"], i["h"] if with_h else None, r, u if pre else None)
        for r_at, u_at in (("x", None), ("h", None), (None, "x"), (None, "h"), ("x", "h"), ("h", "x")):
            if (not with_h and "h" in (r_at, u_at)) or (not pre and u_at):
                continue
            t = {"x": i["x"].clone(), "h": i["h"].clone() if with_h else None}
            got_r = t[r_at] if r_at else torch.empty_like(r)
            got_u = (t[u_at] if u_at else torch.empty_like(u)) if pre else None
            other = call(t["x"], t["h"], got_r, got_u)
            assert torch.equal(got_r, r), (post, pre, r_at, u_at)
            assert not pre or torch.equal(got_u, u), (post, pre, r_at, u_at)
            assert all(torch.equal(a, b) for a, b in zip(stats, other))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_in_place_backward(C, dtype):
    """dx and dh over dr, du, r or h: the same bits as apart."""
    R = 1100 if C < 1000 else 300
    say("in place: backward %dx%d %s" % (R, C, dtype))
    d = TORCH_DTYPES[dtype]
    i = {k: None if v is None else v.cuda() for k, v in inputs(R, C, dtype, 2).items()}
    i["r"] = i.pop("x")
    stats = torch.rand(2, R, device="cuda") + 0.5
    names = ("dr", "du", "r", "h")
    pairs = [(a, None) for a in names] + [(None, a) for a in names] + [(a, b) for a in names for b in names if a != b]

    def call(t, dx, dh):
        out = [torch.empty(C, device="cuda") for _ in range(4)] + [torch.empty(2, C, dtype=d, device="cuda")]
        iabn.iabn_resnorm_backward(t["dr"], t["du"], t["r"], t["h"], dx, dh, gate=i["gate"], post_norm="layer",
                                   post_weight=w, pre_norm="layer", pre_weight=w, post_stats=stats, pre_stats=stats,
                                   dpost_weight=out[0], dpost_bias=out[1], dpre_weight=out[2], dpre_bias=out[3],
                                   dgate=out[4], alpha=0.5, beta=0.75, p=0.25, seed=3)
        return out

    w = i["pw"]
    dx, dh = torch.empty_like(i["r"]), torch.empty_like(i["r"])
    want = call(i, dx, dh)
    for at_dx, at_dh in pairs:
        t = {k: i[k].clone() for k in names}
        got_dx = t[at_dx] if at_dx else torch.empty_like(dx)
        got_dh = t[at_dh] if at_dh else torch.empty_like(dh)
        got = call(t, got_dx, got_dh)
        assert torch.equal(got_dx, dx) and torch.equal(got_dh, dh), (at_dx, at_dh)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (at_dx, at_dh)
