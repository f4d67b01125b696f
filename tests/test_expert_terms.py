"""What a pair adds to its token's y and dx keeps 16 digits and fp32's range between the
kernels, in fp16 and bf16: whole numbers of 16 digits, which cancel over the slots
down to a few digits that every type holds, so that results are exact.

Rounded to the storage type, or without their lower byte, such terms give other sums
(on the CPU here); so do fp16 terms past 65504."""

from __future__ import annotations

import pytest
import torch

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
K = 4  # slots; the experts 2j and 2j + 1 cancel


def case(M, C, F, dtype, scale, seed=3):
    """Inputs of both directions and the exact y and dx.

    forward: g = 1 and u = a_j + (t % 50) in column 0, 1 in column 1 (x_t = 1, t % 50,
    0, ...), so h = g*u; the down weights of expert 2j are b in column 0, those of
    2j + 1 are -b there and r in column 1: terms of +-(a + t % 50)*b < 2^16, sum r.
    backward: dy W_d = d_t in every column, dg = d*u and du = d; the gate's weights of
    2j are b in row 0, those of 2j + 1 -b, the up projection's r in row 1."""
    gen = torch.Generator().manual_seed(seed + M + C)
    d = DTYPES[dtype]
    ints = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=gen).double()  # noqa: E731
    t = torch.arange(M)
    f = {"x": torch.zeros(M, C).double()}
    f["x"][:, 0], f["x"][:, 1] = 1.0, (t % 50).double()
    a = 150.0 + 7 * torch.arange(K // 2)
    forward = {n: torch.zeros(s).double() for n, s in (("w_gate", (K, F, C)), ("w_up", (K, F, C)), ("w_down", (K, C, F)))}
    forward["w_gate"][:, :, 0] = 1.0
    forward["w_up"][:, 0, 0], forward["w_up"][:, 0, 1] = a.repeat_interleave(2).double(), 1.0
    forward["w_up"][:, 1, 0] = 1.0
    b, r = ints(150, 255, K // 2, C), ints(-127, 127, K // 2, C)
    forward["w_down"][0::2, :, 0], forward["w_down"][1::2, :, 0], forward["w_down"][1::2, :, 1] = b, -b, r
    backward = {n: torch.zeros_like(v) for n, v in forward.items()}
    dy = torch.zeros(M, C).double()
    dy[:, 0] = 2.0 ** (t % 2)
    backward["w_down"][:, 0, :] = 1.0
    backward["w_gate"][0::2, 0], backward["w_gate"][1::2, 0], backward["w_up"][1::2, 1] = b, -b, r
    experts = torch.stack([torch.randperm(K, generator=gen) for _ in range(M)])
    g, u = torch.ones(M, F).double(), torch.zeros(M, F).double()
    u[:, 0] = 75.0 + (t % 50)  # (d = 2 doubles it)
    weights = torch.full((M, K), float(scale))
    out = {"x": f["x"], "forward": forward, "backward": backward, "dy": dy, "experts": experts, "weights": weights,
           "g": g, "u": u, "a": a.double(), "b": b, "r": r,
           "y": scale * r.sum(0).expand(M, C), "dx": scale * dy[:, :1] * r.sum(0)}
    for n in ("x", "dy", "g", "u", "y", "dx"):  # all of them are of the type
        assert torch.equal(out[n].to(d).double(), out[n]), n
    return out


def terms24(v, low=True):
    """As they are between the kernels: the upper 24 bits of fp32."""
    bits = v.float().view(torch.int32) + 0x80
    return (bits & (-0x100 if low else -0x10000)).view(torch.float32).double()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("scale", [1, 4])
def test_wrong_terms_show(dtype, scale):
    c = case(64, 40, 24, dtype, scale)
    h = c["a"][:, None] + torch.arange(64) % 50  # [K/2, M]
    plus = scale * h[:, :, None] * c["b"][:, None]
    terms = torch.stack([plus, -plus + scale * c["r"][:, None]])
    assert terms.abs().max() < scale * 2.0 ** 16 and (scale == 1 or terms.abs().max() > 65504)
    sums = lambda v: v.sum((0, 1))  # noqa: E731
    assert torch.equal(sums(terms24(terms)), c["y"])
    for wrong in (terms24(terms, low=False), terms.to(DTYPES[dtype]).double()):
        assert (sums(wrong) != c["y"]).any(1).all()
    # The backward's.
    d = c["dy"][:, :1]
    plus = scale * (d * c["u"][:, :1])[None] * c["b"][:, None]
    terms = torch.stack([plus, -plus + scale * d[None] * c["r"][:, None]])
    assert terms.abs().max() < scale * 2.0 ** 16
    assert torch.equal(sums(terms24(terms)), c["dx"])
    for wrong in (terms24(terms, low=False), terms.to(DTYPES[dtype]).double()):
        assert (sums(wrong) != c["dx"]).any(1).all()


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("scale", [1, 4])
@pytest.mark.parametrize("M,C,F", [(7, 40, 24), (57, 40, 24), (64, 41, 23), (700, 264, 136), (901, 301, 201),
                                   (2100, 512, 264), (4096, 1024, 64)])
def test_terms_keep_their_digits(M, C, F, dtype, scale):
    import paper_1712_02616_amd as iabn

    c = case(M, C, F, dtype, scale)
    dev = lambda v: v.to(DTYPES[dtype]).cuda()  # noqa: E731
    plan = torch.empty(iabn.iabn_experts_plan_size(M, K, K), dtype=torch.int32, device="cuda")
    iabn.iabn_experts_plan(c["experts"].int().cuda(), plan, K)
    w, x = c["weights"].cuda(), dev(c["x"])
    ws = [dev(c["forward"][n]) for n in ("w_gate", "w_up", "w_down")]
    y = iabn.iabn_experts_forward(x, plan, w, *ws, torch.empty_like(x), act="leaky", slope=0.0)
    assert torch.equal(y.cpu().double(), c["y"])
    ws = [dev(c["backward"][n]) for n in ("w_gate", "w_up", "w_down")]
    order = plan[K + 1:K + 1 + M * K].long() // K
    g, u = dev(c["g"])[order].contiguous(), dev(c["u"])[order].contiguous()
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    iabn.iabn_experts_backward(dev(c["dy"]), x, plan, w, g, u, *ws, dx, dw, torch.empty_like(g), torch.empty_like(u),
                               *[torch.empty_like(v) for v in ws], act="leaky", slope=0.0)
    assert torch.equal(dx.cpu().double(), c["dx"])
