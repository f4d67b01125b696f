"""Routing, the experts and the clipping together: the example's stack against the
same model in plain float64 autograd, graph capture, several streams, infinities,
and sizes whose offsets pass 32 bits."""

from __future__ import annotations

import importlib.util
import os

import pytest
import torch

import paper_1712_02616_amd as iabn
import sublayer_oracle as oracle
from gpu_helpers import say
from test_gpu_sublayer import rms

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "routed_sublayer.py")
    spec = importlib.util.spec_from_file_location("routed_sublayer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def new_(*s, std=1.0, t=torch.float32):
    return (torch.randn(*s, device="cuda") * std).to(t)


@pytest.mark.parametrize("rows", [40, 150])
def test_stack_against_plain_autograd(example, rows):
    """fp32, two layers, the choice taken from the GPU's own logits: a chain of some 30
    operations whose sums have up to 96 * 3 terms (at most 300 * 2^-24 of a term's
    scale each), which grow by the layers' gains, of order one, and by those of the
    renormalised weights (up to 1 over the least chosen sum of scores): 1e-4 of the
    largest."""
    torch.manual_seed(5)
    width, hidden, E, top = 64, 96, 6, 3
    model = example.Stack(width, hidden, E, top, 2, torch.float32)
    x = torch.randn(rows, width, device="cuda", requires_grad=True)
    weight = torch.randn(rows, width, device="cuda")
    chosen = []
    real = example.route

    def route(logits, k, bias=None):
        out = real(logits, k, bias)
        chosen.append(out[0].cpu().long())
        return out

    example.route = route
    try:
        (model(x) * weight).sum().backward()
    finally:
        example.route = real

    leaves = {k: v.detach().cpu().double().requires_grad_(True) for k, v in model.named_parameters()}
    x64 = x.detach().cpu().double().requires_grad_(True)
    stream, u = x64, rms(x64, leaves["norms.0"], example.EPS)
    for i in range(2):
        p = lambda n: leaves["blocks.%d.%s" % (i, n)]  # noqa: E731, B023
        s = torch.softmax(u @ p("router").T, 1).gather(1, chosen[i])
        w = s / s.sum(1, keepdim=True)
        every = []
        for e in range(E):
            g = u @ p("w_gate")[e].T
            every.append((g * torch.sigmoid(g) * (u @ p("w_up")[e].T)) @ p("w_down")[e].T)
        of = torch.stack(every, 1)
        h = (of.gather(1, chosen[i][:, :, None].expand(-1, -1, width)) * w[:, :, None]).sum(1)
        stream = stream + rms(h, p("post"), example.EPS)
        u = rms(stream, leaves["norms.%d" % (i + 1)], example.EPS)
    (u * weight.cpu().double()).sum().backward()
    for k, v in [("x", x)] + list(model.named_parameters()):
        want = x64.grad if k == "x" else leaves[k].grad
        off = float((v.grad.cpu().double() - want).abs().max() / want.abs().max())
        assert off < 1e-4, (k, off)
    # And the step's end.
    grads = [v.grad for v in model.parameters()]
    want = float(torch.stack([g.double().square().sum() for g in grads]).sum().sqrt())
    norm = iabn.iabn_grad_norm(grads, torch.empty((), device="cuda"))
    assert abs(float(norm) - want) <= 2 * oracle.U32 * want
    iabn.iabn_grad_clip(grads, grads, norm, 0.5 * want)
    after = float(torch.stack([g.double().square().sum() for g in grads]).sum().sqrt())
    assert abs(after / want - 0.5) < 1e-5


def test_example_runs_and_serves(example):
    torch.manual_seed(0)
    model = example.Stack(128, 64, 8, 2, 2, torch.bfloat16)
    losses, norms = example.train(model, 512, 128, 5, 0.1, torch.bfloat16, say=say)
    assert all(0 < v < INF for v in losses + norms)
    for p in model.parameters():
        p.grad = None
    out = model(torch.randn(40, 128, device="cuda").bfloat16())
    out.sum().backward(retain_graph=True)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    tokens = torch.randn(12, 128, device="cuda").bfloat16()
    together = model.serve(tokens).float()
    assert torch.equal(together, model.serve(tokens).float()) and torch.isfinite(together).all()


class Step:
    """One training step's calls of a routed sublayer on tensors that stay."""

    def __init__(self, M=300, k=4, E=12, C=264, F=136, d=torch.bfloat16, seed=1, ws=None):
        torch.manual_seed(seed)
        self.shape = (M, k, E, C, F, d)
        e = lambda *s, t=d: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        self.x, self.dy, self.logits = new_(M, C, t=d), new_(M, C, t=d), new_(M, E, t=d)
        self.bias = new_(E, std=0.1)
        self.w = [new_(E, F, C, std=C ** -0.5, t=d), new_(E, F, C, std=C ** -0.5, t=d), new_(E, C, F, std=F ** -0.5, t=d)]
        need = max(iabn.iabn_experts_workspace_size(M, k, E, C, F, d),
                   iabn.iabn_grad_norm_workspace_size([t.numel() for t in self.w]))
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda") if ws is None else ws
        f32 = torch.float32
        self.out = {"experts": e(M, k, t=torch.int32), "weights": e(M, k, t=f32), "y": e(M, C),
                    "g": e(M * k, F), "u": e(M * k, F), "dx": e(M, C), "dweights": e(M, k, t=f32),
                    "dlogits": e(M, E), "dwg": e(E, F, C), "dwu": e(E, F, C), "dwd": e(E, C, F), "norm": e(1, t=f32)}
        self.plan = torch.zeros(iabn.iabn_experts_plan_size(M, k, E), dtype=torch.int32, device="cuda")

    def run(self):
        o = self.out
        kw = dict(score="sigmoid", renormalise=True)
        iabn.iabn_route_forward(self.logits, o["experts"], o["weights"], bias=self.bias, groups=4, groups_kept=2,
                                group_top=2, **kw)
        iabn.iabn_experts_plan(o["experts"], self.plan, self.shape[2])
        iabn.iabn_experts_forward(self.x, self.plan, o["weights"], *self.w, o["y"], o["g"], o["u"], workspace=self.ws)
        iabn.iabn_experts_backward(self.dy, self.x, self.plan, o["weights"], o["g"], o["u"], *self.w, o["dx"],
                                   o["dweights"], o["g"], o["u"], o["dwg"], o["dwu"], o["dwd"], workspace=self.ws)
        iabn.iabn_route_backward(o["dweights"], self.logits, o["experts"], o["dlogits"], **kw)
        grads = [o["dwg"], o["dwu"], o["dwd"]]
        iabn.iabn_grad_norm(grads, o["norm"], workspace=self.ws)
        iabn.iabn_grad_clip(grads, grads, o["norm"], 1.0)
        # No tokens: the zeros are a kernel's.
        iabn.iabn_route_backward(o["dweights"][:0], self.logits[:0], o["experts"][:0], o["dlogits"][:0], **kw)

    def copies(self):
        return {k: t.clone() for k, t in self.out.items()}

    def spoil(self):
        for t in self.out.values():
            t.fill_(-5 if t.dtype == torch.int32 else NAN)


def same(step, want):
    for k, t in step.out.items():
        assert torch.equal(t, want[k]), k


@pytest.mark.parametrize("M", [9, 300])
def test_graph_replay_matches_eager(M):
    step = Step(M=M)
    step.run()
    torch.cuda.synchronize()
    eager = step.copies()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    for rep in range(4):
        say("routed graph: replay %d" % rep)
        step.spoil()
        torch.randn(1 << 18, device="cuda").mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        same(step, eager)
    # Another choice at replay: the launches do not depend on it.
    step.logits.copy_(new_(*step.logits.shape, t=step.logits.dtype))
    step.logits[:, :5] = -INF
    step.run()
    torch.cuda.synchronize()
    other = step.copies()
    step.spoil()
    graph.replay()
    torch.cuda.synchronize()
    same(step, other)


def test_two_graphs_share_a_workspace():
    """One after the other on one stream."""
    a = Step(seed=1)
    b = Step(seed=2, ws=a.ws)
    wants, graphs = [], []
    for s in (a, b):
        s.run()
        torch.cuda.synchronize()
        wants.append(s.copies())
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run()
        graphs.append(g)
    for _ in range(3):
        for s in (a, b):
            s.spoil()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, want in zip((a, b), wants):
            same(s, want)


def test_two_streams_at_once():
    steps, wants = [Step(seed=s, M=500) for s in (3, 4)], []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        wants.append(s.copies())
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for s in steps:
            s.spoil()
        torch.cuda.synchronize()
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
        torch.cuda.synchronize()
        for s, want in zip(steps, wants):
            same(s, want)


def test_the_native_path_is_taken(monkeypatch):
    """Plain calls do not go through the Python code."""
    step = Step()
    step.run()
    torch.cuda.synchronize()
    want = step.copies()
    monkeypatch.setattr(iabn, "_enqueue", None)
    step.spoil()
    iabn_ws, step.ws = step.ws, None  # (and the library takes its own workspace)
    step.run()
    torch.cuda.synchronize()
    same(step, want)
    step.ws = iabn_ws


@pytest.mark.parametrize("M", [5, 300])
def test_infinite_projections_give_the_limits(M):
    """fp16 projections that overflow: the activations' limits, in both directions."""
    k, E, C, F = 2, 3, 64, 32
    d = torch.float16
    x = torch.full((M, C), 200.0, dtype=d, device="cuda")
    w = torch.zeros(E, F, C, dtype=d, device="cuda")
    w[:, 0], w[:, 1] = 20.0, -20.0  # g = +-256000: infinite as stored
    up = torch.zeros(E, F, C, dtype=d, device="cuda")
    up[:, :2] = 1e-4
    down = torch.full((E, C, F), 1e-3, dtype=d, device="cuda")
    experts = (torch.arange(M * k, device="cuda") % E).view(M, k).int()
    plan = torch.empty(iabn.iabn_experts_plan_size(M, k, E), dtype=torch.int32, device="cuda")
    iabn.iabn_experts_plan(experts, plan, E)
    weights = torch.full((M, k), 1e-4, device="cuda")
    y = torch.empty_like(x)
    g, u = (torch.empty(M * k, F, dtype=d, device="cuda") for _ in range(2))
    iabn.iabn_experts_forward(x, plan, weights, w, up, down, y, g, u)
    assert (g[:, 0] == INF).all() and (g[:, 1] == -INF).all() and not torch.isnan(y).any()
    g[:, 0] = 1000.0
    g[:, 1] = -INF
    dx, dw = torch.empty_like(x), torch.empty_like(weights)
    dws = [torch.empty_like(t) for t in (w, up, down)]
    iabn.iabn_experts_backward(torch.full_like(x, 1e-3), x, plan, weights, g, u, w, up, down, dx, dw, g, u, *dws)
    for t in (dx, dw, *dws):
        assert torch.isfinite(t).all()


def test_offsets_past_32_bits():
    """The last tokens of tensors of more than 2^31 elements; a matrix past the 2^32
    bytes that a gathered row's offset reaches."""
    M, C, F, E, d = 140_001, 64, 16_384, 2, torch.float16
    say("offsets: wide hidden rows")
    x = torch.zeros(M, C, dtype=d, device="cuda")
    x[-3:] = new_(3, C, t=d)
    wg, wu = new_(E, F, C, std=1 / 8, t=d), new_(E, F, C, std=1 / 8, t=d)
    wd = new_(E, C, F, std=1 / 128, t=d)
    experts = (torch.arange(M, device="cuda") % 2)[:, None].int()
    weights = torch.rand(M, 1, device="cuda") + 0.5
    dy = torch.zeros(M, C, dtype=d, device="cuda")
    dy[-3:] = new_(3, C, t=d)

    def run(rows):
        n = x[rows].shape[0]
        plan = torch.empty(iabn.iabn_experts_plan_size(n, 1, E), dtype=torch.int32, device="cuda")
        iabn.iabn_experts_plan(experts[rows].contiguous(), plan, E)
        xs, ws, dys = (t[rows].contiguous() for t in (x, weights, dy))
        y, g, u = torch.empty_like(xs), torch.empty(n, F, dtype=d, device="cuda"), torch.empty(n, F, dtype=d, device="cuda")
        iabn.iabn_experts_forward(xs, plan, ws, wg, wu, wd, y, g, u)
        outs = [torch.empty_like(xs), torch.empty_like(ws)] + [torch.empty_like(t) for t in (wg, wu, wd)]
        iabn.iabn_experts_backward(dys, xs, plan, ws, g, u, wg, wu, wd, *outs[:2], g, u, *outs[2:])
        return y, outs

    y, outs = run(slice(0, M))
    few_y, few = run(slice(M - 3, M))
    assert float((y[-3:].float() - few_y.float()).abs().max()) <= 4e-3 * float(few_y.abs().max())
    assert float(y[:-3].abs().max()) == 0.0 and float(outs[0][:-3].abs().max()) == 0.0
    for a, b in zip([outs[0][-3:], outs[1][-3:]] + outs[2:], few):
        assert float((a.float() - b.float()).abs().max()) <= 8e-3 * float(b.abs().max())
    del x, dy, y, outs

    say("offsets: many tokens")
    M, C, F, E = (1 << 20) + 77, 2056, 8, 3  # 4.3 GB of tokens: gathered through registers
    x = torch.zeros(M, C, dtype=d, device="cuda")
    x[-2:] = new_(2, C, t=d)
    wg, wu, wd = new_(E, F, C, std=1 / 45, t=d), new_(E, F, C, std=1 / 45, t=d), new_(E, C, F, std=1 / 3, t=d)
    experts = (torch.arange(M, device="cuda") % 3)[:, None].int()
    weights = torch.ones(M, 1, device="cuda")
    plan = torch.empty(iabn.iabn_experts_plan_size(M, 1, E), dtype=torch.int32, device="cuda")
    iabn.iabn_experts_plan(experts, plan, E)
    y = torch.empty_like(x)
    iabn.iabn_experts_forward(x, plan, weights, wg, wu, wd, y)
    for t in (M - 2, M - 1):
        e = t % 3
        v = x[t].double()
        g = wg[e].double() @ v
        want = wd[e].double() @ (g * torch.sigmoid(g) * (wu[e].double() @ v))
        assert float((y[t].double() - want).abs().max()) <= 4e-3 * float(want.abs().max())
    assert float(y[:-2].abs().max()) == 0.0


def test_many_rows_of_routing():
    """2^21 rows: logits past 2^32 bytes, rows past one launch's worth of blocks."""
    M, E, k = (1 << 21) + 3, 1024, 2
    l = torch.zeros(M, E, dtype=torch.bfloat16, device="cuda")
    l[:, 5], l[-1, 1000], l[-1, 7] = 1.0, 3.0, 2.0
    experts, weights = torch.empty(M, k, dtype=torch.int32, device="cuda"), torch.empty(M, k, device="cuda")
    iabn.iabn_route_forward(l, experts, weights, renormalise=True)
    assert (experts[:-1] == torch.tensor([5, 0], device="cuda")).all() and experts[-1].tolist() == [1000, 7]
    want = torch.softmax(torch.tensor([3.0, 2.0], dtype=torch.float64), 0)
    assert float((weights[-1].cpu().double() - want).abs().max()) < 1e-6
    # Equal gradients of renormalised weights, which add up to 1: none of the logits'
    # (1 - sum p is within two units of 32 bits).
    dl = iabn.iabn_route_backward(torch.ones_like(weights), l, experts, l, renormalise=True)
    assert float(dl.abs().max()) < 1e-6


def test_refusals_on_the_gpu():
    x = torch.zeros(4, 64, dtype=torch.float16, device="cuda")
    w, wd = torch.zeros(3, 128, 64, dtype=torch.float16, device="cuda"), torch.zeros(3, 64, 128, dtype=torch.float16,
                                                                                  device="cuda")
    experts, weights = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    plan = torch.empty(iabn.iabn_experts_plan_size(4, 2, 3), dtype=torch.int32, device="cuda")
    iabn.iabn_experts_plan(experts, plan, 3)
    with pytest.raises(iabn.IabnError) as e:
        iabn.iabn_experts_forward(x, plan, weights, w, w, wd, torch.empty_like(x),
                                  workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 5
    with pytest.raises(iabn.IabnError) as e:
        iabn.iabn_grad_norm([x] * 3, torch.empty(1, device="cuda"), workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 5
    for bad in (x.t(), x.float(), x.cpu(), x[:, :32], x[:2]):
        with pytest.raises((ValueError, TypeError)):
            iabn.iabn_experts_forward(x, plan, weights, w, w, wd, bad)
        with pytest.raises((ValueError, TypeError)):
            iabn.iabn_route_backward(weights, x, experts, bad)
    for bad in (weights.double(), weights[:2], weights.cpu(), weights.t().contiguous().t()):
        with pytest.raises((ValueError, TypeError)):
            iabn.iabn_route_forward(x, experts, bad)
        with pytest.raises((ValueError, TypeError)):
            iabn.iabn_experts_forward(x, plan, bad, w, w, wd, torch.empty_like(x))
    with pytest.raises(iabn.IabnError):
        iabn.iabn_route_forward(x, experts, weights, groups=7)
    with pytest.raises(iabn.IabnError):
        iabn.iabn_grad_clip([x], [x], torch.zeros(1, device="cuda"), -1.0)
    with pytest.raises(ValueError):
        iabn.iabn_grad_clip([x], [x.float()], torch.zeros(1, device="cuda"), 1.0)
