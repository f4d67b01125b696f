"""The 64-bit definitions of the sublayer's operators (sublayer_oracle.py):
the generator against known answers, the gradients against autograd and
against differences."""

from __future__ import annotations

import pytest
import torch

import sublayer_oracle as oracle


def test_philox_known_answers():
    # The published test vectors of the generator (all zeros; all ones; digits of pi).
    assert oracle.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert oracle.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert oracle.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_factors_take_the_generators_bits():
    seed, offset, p = 0x123456789ABCDEF0, 0xFEDCBA9876543210, 0.3
    f = oracle.factors(5, 19, p, seed, offset)
    cut = int(0.3 * 65536 + 0.5)
    for row, col in ((0, 0), (0, 7), (2, 8), (4, 18), (3, 13)):
        w = oracle.philox([row * 3 + col // 8, 0, offset & 0xFFFFFFFF, offset >> 32],
                          [seed & 0xFFFFFFFF, seed >> 32])
        bits = (w[col % 8 // 2] >> (16 * (col % 2))) & 0xFFFF
        assert float(f[row, col]) == (65536 / (65536 - cut) if bits >= cut else 0.0)


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_factors_keep_the_right_share(p):
    f = oracle.factors(512, 512, p, 99, 3)
    kept = float((f > 0).double().mean())
    # Five standard deviations of a mean of 2^18 independent choices.
    assert abs(kept - (1 - p)) < 5 * (p * (1 - p) / 2 ** 18) ** 0.5 + 2 ** -17
    assert abs(float(f.mean()) - 1.0) < 5 * (p / (1 - p) / 2 ** 18) ** 0.5
    assert oracle.factors(4, 9, 1.0, 5, 6).abs().sum() == 0
    assert (oracle.factors(4, 9, 0.0, 5, 6) == 1).all()


@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("pre", [None, "rms", "layer"])
@pytest.mark.parametrize("groups", [0, 1, 2, 6])
def test_gradients(post, pre, groups):
    torch.manual_seed(5)
    R, C, d = 6, 5, torch.float64
    new = lambda *s: torch.randn(*s, dtype=d)  # noqa: E731
    keep = oracle.factors(R, C, 0.25, 11, 12)
    p = {"x": new(R, C), "h": new(R, C)}
    if groups:
        p["gate"] = new(groups, C)
    if post:
        p["pw"], p["pb"] = new(C), new(C)
    if pre:
        p["qw"], p["qb"] = new(C), new(C)
    dr, du = new(R, C), new(R, C) if pre else None
    alpha, beta, eps = 0.75, 1.5, 1e-3

    def run(q):
        return oracle.forward(q["x"], q["h"], q.get("gate"), post, q.get("pw"), q.get("pb"), pre, q.get("qw"),
                              q.get("qb"), alpha, beta, eps, keep)

    def loss(q):
        out = run(q)
        v = (dr * out["r"][0]).sum()
        return v + (du * out["u"][0]).sum() if pre else v

    out = run(p)
    stats = {k: out[k][0] if k in out else None for k in ("post_stats", "pre_stats")}
    got = oracle.backward(dr, du, out["r"][0], p["h"], p.get("gate"), post, p.get("pw"), p.get("pb"), pre, p.get("qw"),
                          stats["post_stats"], stats["pre_stats"], alpha, beta, keep)
    names = {"x": "dx", "h": "dh", "gate": "dgate", "pw": "dpost_weight", "pb": "dpost_bias",
             "qw": "dpre_weight", "qb": "dpre_bias"}
    leaves = {k: v.clone().requires_grad_(True) for k, v in p.items()}
    grads = dict(zip(leaves, torch.autograd.grad(loss(leaves), list(leaves.values()))))
    step = 1e-6
    for k, v in p.items():
        value = got[names[k]][0]
        torch.testing.assert_close(value, grads[k], rtol=1e-9, atol=1e-10)
        flat = v.reshape(-1)
        for i in range(0, flat.numel(), 3):
            keep_i = float(flat[i])
            flat[i] = keep_i + step
            up = float(loss(p))
            flat[i] = keep_i - step
            down = float(loss(p))
            flat[i] = keep_i
            # Central differences: O(step^2) and the loss's rounding / step.
            assert abs((up - down) / (2 * step) - float(value.reshape(-1)[i])) < 1e-6


@pytest.mark.parametrize("kind", ["silu", "gelu", "leaky"])
def test_activations(kind):
    v = torch.linspace(-6, 6, 1001, dtype=torch.float64, requires_grad=True)
    a, da = oracle.act(v, kind, 0.2)
    (grad,) = torch.autograd.grad(a.sum(), v)
    torch.testing.assert_close(da, grad, rtol=1e-9, atol=1e-12)
    library = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
               "leaky": lambda t: torch.nn.functional.leaky_relu(t, 0.2)}[kind]
    torch.testing.assert_close(a, library(v), rtol=1e-9, atol=1e-12)
