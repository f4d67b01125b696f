"""Columns' sums of the norms' backward over very many rows.  A block adds its
rows in fp32, one after the other, at most 1024 of them in a row (a wave's);
the blocks' sums are joined in double.  So a sum is within (1024 + 76) * 2^-24
of its terms' absolute values, however many rows there are: 1024 additions, a
handful in the join of a block's waves, and the roundings of the terms."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
from gpu_helpers import say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

BOUND = 1100 * 2.0 ** -24


def test_small_terms_after_a_large_one():
    """Each 2^-24 is half a unit of the 1 before it: a chain loses what it adds
    to it, so a chain of 8192 would lose 4.9e-4."""
    R, C = 1 << 24, 8
    say("long sums: %d rows" % R)
    du = torch.full((R, C), 2.0 ** -24, device="cuda")
    du[0] = 1.0
    ones = torch.ones(R, C, device="cuda")
    stats = torch.ones(2, R, device="cuda")
    stats[0] = 0.0
    w, b = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    iabn.iabn_resnorm_backward(None, du, ones, None, None, None, pre_norm="rms", pre_stats=stats, dpre_weight=w,
                               dpre_bias=b)
    want = 1 + (R - 1) * 2.0 ** -24
    assert float((w.double() - want).abs().max()) <= BOUND * want
    assert float((b.double() - want).abs().max()) <= BOUND * want
    # The same sums of the norm after a block, and of the gates of 512 groups.
    G = 512
    du.view(G, R // G, C)[:, 0] = 1.0
    gate, dgate = torch.ones(G, C, device="cuda"), torch.empty(G, C, device="cuda")
    iabn.iabn_resnorm_backward(du, None, None, ones, None, None, gate=gate, post_norm="rms", post_stats=stats,
                               dgate=dgate, dpost_weight=w, dpost_bias=b)
    of_group = 1 + (R // G - 1) * 2.0 ** -24
    assert float((dgate.double() - of_group).abs().max()) <= BOUND * of_group
    for v in (w, b):
        assert float((v.double() - G * of_group).abs().max()) <= BOUND * G * of_group


@pytest.mark.parametrize("rows,width,groups,dtype", [
    (3_000_017, 8, 0, torch.float32), (600 * 7001, 8, 600, torch.float32), (3000 * 1501, 16, 3000, torch.bfloat16),
    (66_000 * 41, 8, 66_000, torch.float32), (1100 * 1100, 520, 1100, torch.bfloat16),
    (33_000 * 4100, 1, 33_000, torch.bfloat16)])
def test_many_rows(rows, width, groups, dtype):
    say("long sums: %dx%d, %d groups" % (rows, width, groups))
    gen = torch.Generator(device="cuda").manual_seed(8)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    dr, h = new(rows, width).to(dtype), (new(rows, width) + 1).to(dtype)
    stats = torch.stack([torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")])
    gate = torch.ones(groups, width, dtype=dtype, device="cuda") if groups else None
    dgate = torch.empty_like(gate) if groups else None
    w, b = torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
    iabn.iabn_resnorm_backward(dr, None, None, h, None, None, gate=gate, post_norm="rms", post_stats=stats,
                               dgate=dgate, dpost_weight=w, dpost_bias=b)

    def near(got, terms, unit=0.0):
        for i in range(0, width, 8):
            t = terms(slice(i, i + 8))
            want, size = t.sum(-2), t.abs().sum(-2)
            off = (got[..., i:i + 8].double() - want).abs() - BOUND * size - unit * want.abs()
            assert float(off.max()) <= 0

    near(w, lambda c: dr[:, c].double() * h[:, c].double())
    near(b, lambda c: dr[:, c].double())
    if groups:
        near(dgate, lambda c: (dr[:, c].double() * h[:, c].double()).view(groups, rows // groups, -1),
             2.0 ** -8 if dtype is torch.bfloat16 else 0.0)
