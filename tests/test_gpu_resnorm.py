"""iabn_dropout, iabn_resnorm_forward and iabn_resnorm_backward on the GPU
against their definitions in 64 bits (sublayer_oracle.py)."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
import sublayer_oracle as oracle
from gpu_helpers import TORCH_DTYPES, say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

EPS = 1e-5


def placed(t, shift):
    """A device copy of t that starts `shift` elements into its allocation."""
    if t is None:
        return None
    buf = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
    out = buf[shift:].view(t.shape)
    out.copy_(t)
    return out


def guarded(shape, dtype, shift=0):
    """An output between guard values: (tensor, check)."""
    n = 1
    for s in shape:
        n *= s
    buf = torch.full((n + shift + 64,), -7.0, dtype=dtype, device="cuda")

    def check(name):
        assert (buf[:shift] == -7).all() and (buf[shift + n:] == -7).all(), "%s: written outside" % name

    return buf[shift:shift + n].view(shape), check


# ------------------------------------------------------------------ dropout

@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 8), (3, 7), (5, 1000), (33, 1025), (257, 64), (0, 16), (4, 0)])
def test_dropout_is_exact(dtype, rows, width):
    say("dropout %s %dx%d" % (dtype, rows, width))
    x = torch.randn(rows, width, dtype=torch.float32).to(TORCH_DTYPES[dtype])
    for p, seed, offset, shift in ((0.1, 1, 0, 0), (0.5, 2 ** 64 - 1, 2 ** 64 - 1, 1), (0.0, 3, 4, 3), (1.0, 5, 6, 0)):
        y, intact = guarded(x.shape, x.dtype, shift)
        assert iabn.iabn_dropout(placed(x, shift), y, p, seed, offset) is y
        # One 32-bit product, rounded to storage: the same on both sides.
        f = oracle.factors(rows, width, p, seed, offset).float()
        want = (x.float() * f).to(x.dtype)
        assert torch.equal(y.cpu() + 0.0, want + 0.0)
        intact("y")


def test_dropout_in_place_and_nonfinite():
    x = torch.full((4, 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[1] = float("inf")
    keep = oracle.factors(4, 24, 0.5, 8, 9) > 0
    iabn.iabn_dropout(x, x, 0.5, 8, 9)
    got = x.cpu().float()
    assert (got[~keep] == 0).all()
    assert torch.isnan(got[keep & (torch.arange(4) != 1)[:, None]]).all() and torch.isinf(got[1][keep[1]]).all()


def test_dropout_group_index_passes_32_bits_of_elements():
    # Elements past 2^32 (groups past 2^29): the place is counted in 64 bits.
    rows, width = (1 << 17) + 3, 1 << 15
    x = torch.ones(rows, width, dtype=torch.float16, device="cuda")
    iabn.iabn_dropout(x, x, 0.5, 77, 1)
    last = x[-1].cpu().double()
    for col in range(0, width, 4099):
        q = (rows - 1) * (width // 8) + col // 8
        w = oracle.philox([q & 0xFFFFFFFF, q >> 32, 1, 0], [77, 0])
        bits = (w[col % 8 // 2] >> (16 * (col % 2))) & 0xFFFF
        assert float(last[col]) == (2.0 if bits >= 32768 else 0.0)


# ------------------------------------------------------------------ norms

def inputs(R, C, dtype, groups, seed=3, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    d = TORCH_DTYPES[dtype]
    new = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return {"x": (new(R, C) * 2 + mean).to(d), "h": (new(R, C) * 1.5 - mean).to(d),
            "dr": (new(R, C) * 0.2).to(d), "du": (new(R, C) * 0.3).to(d),
            "gate": new(groups, C).to(d) if groups else None,
            "pw": new(C) * 0.3 + 1, "pb": new(C) * 0.2, "qw": new(C) * 0.3 - 1, "qb": new(C) * 0.2}


def run_case(R, C, dtype, post, pre, groups, p, vectors=True, branch=True, shift=0, mean=0.0, in_place=False):
    say("resnorm %dx%d %s post=%s pre=%s groups=%d p=%g vectors=%s branch=%s shift=%d"
        % (R, C, dtype, post, pre, groups, p, vectors, branch, shift))
    alpha, beta, seed, offset, d = 0.875, -1.25, 0xABCDEF0123456789, 1 << 33, TORCH_DTYPES[dtype]
    i = inputs(R, C, dtype, groups, mean=mean)
    if not branch:
        post, groups, p = None, 0, 0.0
        i["h"] = i["gate"] = None
    pw, pb = (i["pw"], i["pb"]) if post and vectors else (None, None)
    qw, qb = (i["qw"], i["qb"]) if pre and vectors else (None, None)
    f64 = lambda t: None if t is None else t.double()  # noqa: E731
    keep = oracle.factors(R, C, p, seed, offset)
    want = oracle.forward(f64(i["x"]), f64(i["h"]), f64(i["gate"]), post, f64(pw), f64(pb), pre, f64(qw), f64(qb),
                          alpha, beta, EPS, keep)
    dev = {k: placed(v, shift) for k, v in i.items()}
    vec = {k: None if v is None else v.cuda() for k, v in (("pw", pw), ("pb", pb), ("qw", qw), ("qb", qb))}
    checks = []

    def out(name, shape, dt):
        t, intact = guarded(shape, dt, shift)
        checks.append((name, intact))
        return t

    r = dev["x"].clone() if in_place else out("r", (R, C), d)
    u = None if pre is None else out("u", (R, C), d)
    stats = {"post_stats": out("post_stats", (2, R), torch.float32) if post else None,
             "pre_stats": out("pre_stats", (2, R), torch.float32) if pre else None}
    kw = dict(gate=dev["gate"], post_norm=post, post_weight=vec["pw"], post_bias=vec["pb"], pre_norm=pre,
              pre_weight=vec["qw"], alpha=alpha, beta=beta, p=p, seed=seed, offset=offset)
    iabn.iabn_resnorm_forward(r if in_place else dev["x"], dev["h"], r, u, pre_bias=vec["qb"], eps=EPS, **stats, **kw)
    oracle.check("r", r, *want["r"], d)
    if pre:
        oracle.check("u", u, *want["u"], d)
    for k, t in stats.items():
        if t is not None:
            oracle.check(k, t, *want[k], torch.float32)

    # The backward, of the r and statistics that the forward stored.
    kept = {k: None if t is None else t.cpu().double() for k, t in stats.items()}
    for dr, du in [(i["dr"], i["du"] if pre else None)] + ([(None, i["du"])] if pre else []):
        ref = oracle.backward(f64(dr), f64(du), f64(r.cpu()), f64(i["h"]), f64(i["gate"]), post, f64(pw), f64(pb),
                              pre, f64(qw), kept["post_stats"], kept["pre_stats"], alpha, beta, keep)
        ddr, ddu = placed(dr, shift), placed(du, shift)
        dx = ddr if in_place and ddr is not None else out("dx", (R, C), d)
        dh = out("dh", (R, C), d) if branch else None
        extra = {}
        if i["gate"] is not None:
            extra["dgate"] = out("dgate", i["gate"].shape, d)
        for k, on in (("dpost_weight", post), ("dpost_bias", post), ("dpre_weight", pre), ("dpre_bias", pre)):
            if on:
                extra[k] = out(k, (C,), torch.float32)
        iabn.iabn_resnorm_backward(ddr, ddu, r, dev["h"], dx, dh, **stats, **extra, **kw)
        oracle.check("dx", dx, *ref["dx"], d)
        if branch:
            oracle.check("dh", dh, *ref["dh"], d)
        for k, t in extra.items():
            oracle.check(k, t, *ref[k], t.dtype)
    for name, intact in checks:
        intact(name)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("R,C", [(1, 1), (1, 8), (3, 7), (5, 512), (9, 520), (130, 100), (37, 1501), (12, 4096), (6, 8200),
                                 (2, 16384)])
def test_shapes(R, C, dtype):
    run_case(R, C, dtype, "rms", "layer", 1, 0.1)
    run_case(R, C, dtype, "layer", "rms", 0, 0.0)


@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("pre", [None, "rms", "layer"])
@pytest.mark.parametrize("groups", [0, 1, 4, 60])
def test_stages(post, pre, groups):
    for C in (96, 777):
        run_case(60, C, "f16", post, pre, groups, 0.25)
        run_case(60, C, "f32", post, pre, groups, 0.0, vectors=False)


@pytest.mark.parametrize("R,groups", [(6000, 3000), (6000, 1), (6000, 6000), (5999, 7), (4200, 600)])
def test_many_rows(R, groups):
    """Groups shorter and longer than a block's rows."""
    run_case(R, 72, "bf16", "layer", "rms", groups, 0.1)
    run_case(R, 700, "f32", "rms", None, groups, 0.1)


@pytest.mark.parametrize("C", [64, 100, 1111, 9000])
def test_norm_alone(C):
    """No branch: the norm before the first block."""
    run_case(11, C, "bf16", None, "layer", 0, 0.0, branch=False)
    run_case(11, C, "f32", None, "rms", 0, 0.0, branch=False)


@pytest.mark.parametrize("dtype,shift", [("f32", 1), ("f16", 1), ("bf16", 3), ("f16", 4)])
def test_alignment(dtype, shift):
    run_case(20, 256, dtype, "layer", "rms", 4, 0.1, shift=shift)
    run_case(20, 1001, dtype, "rms", "layer", 1, 0.1, shift=shift)


def test_large_mean():
    """Rows whose mean is 300 times their spread."""
    run_case(17, 640, "f32", "layer", "layer", 1, 0.0, mean=600.0)


@pytest.mark.parametrize("C", [200, 1500])
def test_in_place(C):
    run_case(40, C, "f16", "rms", "rms", 1, 0.1, in_place=True)


def test_empty():
    x = torch.empty(0, 64, dtype=torch.float16, device="cuda")
    st = torch.empty(2, 0, device="cuda")
    w = torch.ones(64, device="cuda")
    iabn.iabn_resnorm_forward(x, x, x, x, post_norm="rms", pre_norm="rms", post_stats=st, pre_stats=st)
    gate = torch.ones(3, 64, dtype=torch.float16, device="cuda")
    outs = [torch.full((64,), 5.0, device="cuda") for _ in range(4)]
    dgate = torch.full_like(gate, 5.0)
    iabn.iabn_resnorm_backward(x, x, x, x, x, x, gate=gate, post_norm="layer", post_weight=w, pre_norm="layer",
                               pre_weight=w, post_stats=st, pre_stats=st, dgate=dgate, dpost_weight=outs[0],
                               dpost_bias=outs[1], dpre_weight=outs[2], dpre_bias=outs[3])
    assert all((t == 0).all() for t in outs) and (dgate == 0).all()


def test_a_bad_row_stays_in_its_row():
    R, C = 12, 600
    x, h = torch.randn(R, C, device="cuda"), torch.randn(R, C, device="cuda")
    outs = []
    for bad in (False, True):
        if bad:
            h[5, 17], x[7, 3] = float("nan"), float("inf")
        r, u = torch.empty_like(x), torch.empty_like(x)
        iabn.iabn_resnorm_forward(x, h, r, u, post_norm="layer", pre_norm="rms")
        outs.append((r, u))
    good = [i for i in range(R) if i not in (5, 7)]
    for a, b in zip(*outs):
        assert torch.equal(a[good], b[good])
    assert torch.isnan(outs[1][0][5]).all() and torch.isinf(outs[1][0][7, 3])


def test_deterministic_and_on_another_stream():
    R, C = 3000, 1000
    i = {k: v.cuda() for k, v in inputs(R, C, "bf16", 1).items()}
    st = torch.cuda.Stream()
    seen = []
    for k in range(3):
        stats = [torch.empty(2, R, device="cuda") for _ in range(2)]
        r, u, dx, dh = (torch.empty_like(i["x"]) for _ in range(4))
        v = [torch.empty(C, device="cuda") for _ in range(4)]
        dg = torch.empty_like(i["gate"])
        kw = dict(gate=i["gate"], post_norm="rms", post_weight=i["pw"], post_bias=i["pb"], pre_norm="layer",
                  pre_weight=i["qw"], p=0.1, seed=4, post_stats=stats[0], pre_stats=stats[1])
        torch.cuda.synchronize()
        s = {0: None, 1: st, 2: st.cuda_stream}[k]
        iabn.iabn_resnorm_forward(i["x"], i["h"], r, u, pre_bias=i["qb"], stream=s, **kw)
        iabn.iabn_resnorm_backward(i["dr"], i["du"], r, i["h"], dx, dh, dgate=dg, dpost_weight=v[0], dpost_bias=v[1],
                                   dpre_weight=v[2], dpre_bias=v[3], stream=s, **kw)
        torch.cuda.synchronize()
        seen.append([r, u, dx, dh, dg] + v + stats)
    for other in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], other))
