"""The sublayer's operators together: the example's stack against the same
model in plain float64 autograd, serving, graph capture, and sizes whose
offsets pass 32 bits."""

from __future__ import annotations

import importlib.util
import os

import pytest
import torch

import paper_1712_02616_amd as iabn
import sublayer_oracle as oracle
from gpu_helpers import say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "ffn_sublayer.py")
    spec = importlib.util.spec_from_file_location("ffn_sublayer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def rms(v, w, eps):
    return v * (v.square().mean(1, keepdim=True) + eps).rsqrt() * w


def test_stack_against_plain_autograd(example):
    """fp32, two layers: a chain of some 30 operations whose sums have up to 160
    terms; errors of single operations (at most 200 * 2^-24 of a term's scale)
    grow by the layers' gains, which are of order one: 1e-4 of the largest."""
    torch.manual_seed(3)
    width, hidden, rows = 96, 160, 50
    model = example.Stack(width, hidden, 2, torch.float32, p=0.25)
    x = torch.randn(rows, width, device="cuda", requires_grad=True)
    weight = torch.randn(rows, width, device="cuda")
    (model(x, step=5) * weight).sum().backward()

    leaves = {k: v.detach().cpu().double().requires_grad_(True) for k, v in model.named_parameters()}
    x64 = x.detach().cpu().double().requires_grad_(True)
    stream, u = x64, rms(x64, leaves["norms.0"], example.EPS)
    for i in range(2):
        p = lambda n: leaves["blocks.%d.%s" % (i, n)]  # noqa: E731, B023
        g = u @ p("w_gate").T
        h = (g * torch.sigmoid(g) * (u @ p("w_up").T)) @ p("w_down").T
        keep = oracle.factors(rows, width, 0.25, 5 * 2 + i, 0)
        stream = stream + p("gate") * keep * rms(h, p("post"), example.EPS)
        u = rms(stream, leaves["norms.%d" % (i + 1)], example.EPS)
    (u * weight.cpu().double()).sum().backward()

    def near(name, got, want):
        off = float((got.cpu().double() - want).abs().max() / want.abs().max())
        assert off < 1e-4, (name, off)

    near("x", x.grad, x64.grad)
    for k, v in model.named_parameters():
        near(k, v.grad, leaves[k].grad)


def test_training_learns_and_serving_agrees(example):
    torch.manual_seed(0)
    model = example.Stack(256, 512, 2, torch.bfloat16, p=0.05)
    losses = example.train(model, 1024, 256, 60, 0.5, torch.bfloat16, say)
    assert losses[-1] < 0.8 * losses[0], losses
    tokens = torch.randn(20, 256, device="cuda").bfloat16()
    together = model.serve(tokens).float()
    single = torch.cat([model.serve(t[None]) for t in tokens]).float()
    # bf16 values of order one to four that were rounded in another order.
    assert float((together - single).abs().max()) < 0.15
    assert float((together - single).square().mean().sqrt()) < 0.02


def test_graph_replay_matches_eager():
    """A training step of one sublayer in a graph, with eager work and
    synchronizations between its replays."""
    M, C, F, d = 200, 264, 520, torch.bfloat16
    new = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    x, u, dr, du = (new(M, C).to(d) for _ in range(4))
    wg, wu, wd = (new(F, C) * C ** -0.5).to(d), (new(F, C) * C ** -0.5).to(d), (new(C, F) * F ** -0.5).to(d)
    gate, pw, qw = new(1, C).to(d), new(C), new(C)
    ws = torch.empty(max(iabn.iabn_ffn_workspace_size(M, C, F, d), iabn.iabn_resnorm_workspace_size(M, C, 1)),
                     dtype=torch.uint8, device="cuda")
    e = lambda *s, t=d: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    out = {"h": e(M, C), "g": e(M, F), "up": e(M, F), "r": e(M, C), "un": e(M, C), "dx": e(M, C), "dh": e(M, C),
           "dgate": e(1, C), "du": e(M, C), "dwg": e(F, C), "dwu": e(F, C), "dwd": e(C, F), "drop": e(M, C)}
    vec = {k: e(2, M, t=torch.float32) for k in ("ps", "qs")} | {k: e(C, t=torch.float32) for k in ("dpw", "dqw")}

    def step():
        o, v = out, vec
        iabn.iabn_ffn_forward(u, wg, wu, wd, o["h"], o["g"], o["up"], workspace=ws)
        kw = dict(gate=gate, post_norm="layer", post_weight=pw, pre_norm="rms", pre_weight=qw, p=0.1, seed=7,
                  post_stats=v["ps"], pre_stats=v["qs"])
        iabn.iabn_resnorm_forward(x, o["h"], o["r"], o["un"], **kw)
        iabn.iabn_resnorm_backward(dr, du, o["r"], o["h"], o["dx"], o["dh"], dgate=o["dgate"], dpost_weight=v["dpw"],
                                   dpre_weight=v["dqw"], workspace=ws, **kw)
        iabn.iabn_ffn_backward(o["dh"], u, o["g"], o["up"], wg, wu, wd, o["du"], o["g"], o["up"], o["dwg"], o["dwu"],
                               o["dwd"], workspace=ws)
        iabn.iabn_dropout(o["r"], o["drop"], 0.3, 11)
        # No rows: the zeros are a kernel's too.
        iabn.iabn_resnorm_backward(dr[:0], du[:0], o["r"][:0], o["h"][:0], o["dx"][:0], o["dh"][:0], post_norm="rms",
                                   post_weight=pw, pre_norm="rms", post_stats=v["ps"][:, :0].contiguous(),
                                   pre_stats=v["qs"][:, :0].contiguous(), workspace=ws)

    step()
    torch.cuda.synchronize()
    eager = {k: t.clone() for k, t in (out | vec).items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    for rep in range(4):
        say("sublayer graph: replay %d" % rep)
        for t in (out | vec).values():
            t.fill_(float("nan"))
        torch.randn(1 << 18, device="cuda").mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        for k, want in eager.items():
            assert torch.equal((out | vec)[k], want), "replay %d: %s" % (rep, k)


def test_offsets_past_32_bits():
    """The last rows of tensors of more than 2^31 elements (and 2^32 bytes)."""
    say("offsets: norms")
    R, C = (1 << 21) + 5, 1024
    x = torch.ones(R, C, dtype=torch.float16, device="cuda")
    h = torch.ones(R, C, dtype=torch.float16, device="cuda")
    tail = torch.randn(5, C, device="cuda").half()
    x[-5:], h[-5:] = tail, tail.flip(0)
    u = torch.empty_like(x)
    stats = torch.empty(2, R, device="cuda")
    iabn.iabn_resnorm_forward(x, h, x, u, pre_norm="rms", pre_stats=stats, p=0.5, seed=9)
    small = [torch.empty(5, C, dtype=torch.float16, device="cuda") for _ in range(2)]
    # The same rows alone, with the mask of their place in the large tensor.
    kept = torch.zeros(5, C, dtype=torch.float64)
    for i in range(5):
        for col in range(0, C, 8):
            q = (R - 5 + i) * (C // 8) + col // 8
            w = oracle.philox([q & 0xFFFFFFFF, q >> 32, 0, 0], [9, 0])
            bits = [(w[j // 2] >> (16 * (j % 2))) & 0xFFFF for j in range(8)]
            kept[i, col:col + 8] = torch.tensor([2.0 * (b >= 32768) for b in bits], dtype=torch.float64)
    want = tail.cpu().double() + kept * tail.flip(0).cpu().double()
    oracle.check("r", x[-5:], want, 4 * oracle.U32 * want.abs(), torch.float16)
    iabn.iabn_resnorm_forward(want.half().cuda(), None, None, small[1], pre_norm="rms")
    assert float((u[-5:].float() - small[1].float()).abs().max()) < 1e-2
    dx = x  # in place over r
    iabn.iabn_resnorm_backward(u, u, x, None, dx, None, pre_norm="rms", pre_stats=stats)
    rhat = want.half().double() * stats[1, -5:].cpu().double()[:, None]
    d = u[-5:].cpu().double()
    g = d + stats[1, -5:].cpu().double()[:, None] * (d - rhat * (d * rhat).mean(1, keepdim=True))
    assert float((dx[-5:].cpu().double() - g).abs().max()) < 2 ** -9 * float(g.abs().max())
    del x, h, u, dx, stats

    say("offsets: gated block")
    M, C, F = 140_001, 64, 16_384
    x = torch.zeros(M, C, dtype=torch.float16, device="cuda")
    x[-3:] = torch.randn(3, C, device="cuda").half()
    wg, wu = ((torch.randn(F, C, device="cuda") / 8).half() for _ in range(2))
    wd = (torch.randn(C, F, device="cuda") / 128).half()
    g, up = (torch.empty(M, F, dtype=torch.float16, device="cuda") for _ in range(2))
    y = torch.empty_like(x)
    iabn.iabn_ffn_forward(x, wg, wu, wd, y, g, up)
    few = [torch.empty(3, n, dtype=torch.float16, device="cuda") for n in (C, F, F)]
    iabn.iabn_ffn_forward(x[-3:].contiguous(), wg, wu, wd, *few)
    for name, got, want in (("y", y, few[0]), ("g", g, few[1]), ("u", up, few[2])):
        assert float((got[-3:].float() - want.float()).abs().max()) <= 4e-3 * float(want.abs().max()), name
        assert float(got[:-3].abs().max()) == 0.0, name
    dw = [torch.empty_like(t) for t in (wg, wu, wd)]
    dx = torch.empty_like(x)
    dy = torch.zeros_like(x)
    dy[-3:] = torch.randn(3, C, device="cuda").half()
    iabn.iabn_ffn_backward(dy, x, g, up, wg, wu, wd, dx, g, up, *dw)
    sw = [torch.empty_like(t) for t in (wg, wu, wd)]
    sdx, sg, su = (torch.empty_like(t) for t in few)
    iabn.iabn_ffn_backward(dy[-3:].contiguous(), x[-3:].contiguous(), few[1], few[2], wg, wu, wd, sdx, sg, su, *sw)
    for a, b in list(zip(dw, sw)) + [(dx[-3:], sdx), (g[-3:], sg), (up[-3:], su)]:
        assert float((a.float() - b.float()).abs().max()) <= 8e-3 * float(b.abs().max())


def test_a_workspace_that_is_too_small_is_refused():
    x = torch.zeros(4, 64, dtype=torch.float16, device="cuda")
    w, wd = torch.zeros(128, 64, dtype=torch.float16, device="cuda"), torch.zeros(64, 128, dtype=torch.float16, device="cuda")
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(iabn.IabnError) as e:
        iabn.iabn_ffn_forward(x, w, w, wd, torch.empty_like(x), workspace=small)
    assert e.value.status == 5
    for bad in (x.t(), x.float(), x.cpu(), x[:, :32]):
        with pytest.raises((ValueError, TypeError)):
            iabn.iabn_ffn_forward(x, w, w, wd, bad)
        with pytest.raises((ValueError, TypeError)):
            iabn.iabn_resnorm_forward(x, bad, x, x, pre_norm="rms")
    with pytest.raises(ValueError, match="2\\^64"):
        iabn.iabn_dropout(x, x, 0.1, -1)
