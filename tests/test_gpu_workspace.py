"""A workspace that the binding takes for a call on another stream: its first
use does not meet the work that torch's current stream still has on blocks of
the same size."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
from gpu_helpers import say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]


def _release_a_block_in_use(nbytes):
    """Leaves a block of the current stream free in the allocator, with a kernel
    that will write to it queued behind a long one."""
    block = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    torch.cuda._sleep(4_000_000)
    block.fill_(0x7F)


@pytest.mark.parametrize("raw", [False, True])
def test_gated_block(raw):
    M, C, F, d = 300, 264, 1000, torch.bfloat16
    say("workspace: gated block")
    gen = torch.Generator(device="cuda").manual_seed(2)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(d)  # noqa: E731
    x, dy, wg, wu, wd = new(M, C), new(M, C), new(F, C) / 16, new(F, C) / 16, new(C, F) / 32
    nbytes = iabn.iabn_ffn_workspace_size(M, C, F, d)

    def run(stream, before):
        y, g, u, dx, dg, du = (torch.empty(M, n, dtype=d, device="cuda") for n in (C, F, F, C, F, F))
        dw = [torch.empty_like(w) for w in (wg, wu, wd)]
        torch.cuda.synchronize()
        before()
        iabn.iabn_ffn_forward(x, wg, wu, wd, y, g, u, stream=stream)
        before()
        iabn.iabn_ffn_backward(dy, x, g, u, wg, wu, wd, dx, dg, du, *dw, stream=stream)
        torch.cuda.synchronize()
        return [y, g, u, dx, dg, du] + dw

    want = run(None, lambda: None)
    side = torch.cuda.Stream()
    for _ in range(3):
        got = run(side.cuda_stream if raw else side, lambda: _release_a_block_in_use(nbytes))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_norms():
    R, C = 2000, 500
    say("workspace: norms")
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    dr, du, r, h, w = new(R, C), new(R, C), new(R, C), new(R, C), new(C)
    stats = torch.rand(2, R, device="cuda") + 0.5
    nbytes = iabn.iabn_resnorm_workspace_size(R, C)

    def run(stream, before):
        out = [torch.empty_like(r), torch.empty_like(r)] + [torch.empty_like(w) for _ in range(4)]
        torch.cuda.synchronize()
        before()
        iabn.iabn_resnorm_backward(dr, du, r, h, out[0], out[1], post_norm="layer", post_weight=w, pre_norm="layer",
                                   pre_weight=w, post_stats=stats, pre_stats=stats, dpost_weight=out[2],
                                   dpost_bias=out[3], dpre_weight=out[4], dpre_bias=out[5], stream=stream)
        torch.cuda.synchronize()
        return out

    want = run(None, lambda: None)
    side = torch.cuda.Stream()
    for _ in range(3):
        got = run(side, lambda: _release_a_block_in_use(nbytes))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_normalisation_layer():
    """The streaming kernels, which use the workspace."""
    shape = (4, 24, 20008)
    say("workspace: normalisation layer")
    gen = torch.Generator(device="cuda").manual_seed(4)
    x0, dz0 = (torch.randn(shape, generator=gen, device="cuda") for _ in range(2))
    g = torch.rand(24, generator=gen, device="cuda") + 0.5
    nbytes = iabn.iabn_workspace_size(*shape, torch.float32)

    def run(stream, before):
        x, dz = x0.clone(), dz0.clone()
        c = [torch.ones_like(g) for _ in range(6)]
        torch.cuda.synchronize()
        before()
        iabn.iabn_forward_train(x, g, g, c[0], c[1], c[2], c[3], stream=stream)
        before()
        iabn.iabn_backward(x, dz, g, g, c[3], c[4], c[5], stream=stream)
        torch.cuda.synchronize()
        return [x, dz] + c

    want = run(None, lambda: None)
    side = torch.cuda.Stream()
    for _ in range(3):
        got = run(side, lambda: _release_a_block_in_use(nbytes))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_default_stream_by_its_handle():
    """stream=0 with another stream current: the workspace is the default stream's."""
    M, C, F, d = 100, 96, 128, torch.float32
    gen = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, wg, wu, wd = new(M, C), new(F, C), new(F, C), new(C, F)
    want, got = torch.empty_like(x), torch.empty_like(x)
    iabn.iabn_ffn_forward(x, wg, wu, wd, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _release_a_block_in_use(iabn.iabn_ffn_workspace_size(M, C, F, d))
        iabn.iabn_ffn_forward(x, wg, wu, wd, got, stream=0)
        assert torch.cuda.current_stream() == side
    torch.cuda.synchronize()
    assert torch.equal(got, want)
