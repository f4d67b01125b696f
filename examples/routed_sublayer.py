"""A stack of sublayers of routed experts on libiabn: trained for some steps with
clipped gradients, then serving token by token.

    python examples/routed_sublayer.py [--rows 4096 --width 1024 --hidden 512 --experts 32 --top 4 --layers 2]

One sublayer takes the residual stream x and its normalised values u:

    experts, weights = route(u Wr^T)               iabn_route_forward
    h = experts' gated blocks of u                 iabn_experts_plan, iabn_experts_forward
    x = x + norm(h), u = norm(x)                   iabn_resnorm_forward, one pass

and a training step ends with iabn_grad_norm and iabn_grad_clip over all
gradients.  What is kept for the backward is what ffn_sublayer.py keeps, the
projections once for each of a token's experts, and the choice: the scores, the
experts' outputs and their weighted sum are not.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from ffn_sublayer import EPS, InputNorm, iabn  # noqa: E402


def route(logits, top, bias=None):
    """The experts of each token, their weights, and the plan of the products."""
    rows, E = logits.shape
    experts = torch.empty(rows, top, dtype=torch.int32, device=logits.device)
    weights = torch.empty(rows, top, device=logits.device)
    iabn.iabn_route_forward(logits, experts, weights, bias=bias, renormalise=True)
    plan = torch.empty(iabn.iabn_experts_plan_size(rows, top, E), dtype=torch.int32, device=logits.device)
    return experts, weights, iabn.iabn_experts_plan(experts, plan, E)


class RoutedBlock(torch.autograd.Function):
    """(u, logits) -> the weighted sum of the chosen experts' blocks."""

    @staticmethod
    def forward(ctx, u, logits, w_gate, w_up, w_down, top):
        experts, weights, plan = route(logits, top)
        h = torch.empty_like(u)
        g = torch.empty(u.shape[0] * top, w_gate.shape[1], dtype=u.dtype, device=u.device)
        up = torch.empty_like(g)
        iabn.iabn_experts_forward(u, plan, weights, w_gate, w_up, w_down, h, g, up)
        ctx.save_for_backward(u, logits, w_gate, w_up, w_down, experts, weights, plan, g, up)
        return h

    @staticmethod
    def backward(ctx, dh):
        u, logits, w_gate, w_up, w_down, experts, weights, plan, g, up = ctx.saved_tensors
        du, dlogits, dweights = torch.empty_like(u), torch.empty_like(logits), torch.empty_like(weights)
        dws = [torch.empty_like(w) for w in (w_gate, w_up, w_down)]
        # The projections' gradients overwrite the projections, which autograd is
        # told: a second backward through this graph fails.
        torch.autograd.graph.increment_version((g, up))
        iabn.iabn_experts_backward(dh.contiguous(), u, plan, weights, g, up, w_gate, w_up, w_down, du, dweights, g, up,
                                   *dws)
        iabn.iabn_route_backward(dweights, logits, experts, dlogits, renormalise=True)
        return (du, dlogits, *dws, None)


class AddNorm(torch.autograd.Function):
    """(x, h) -> (x + norm(h), its norm)."""

    @staticmethod
    def forward(ctx, x, h, post_weight, pre_weight):
        r, u = torch.empty_like(x), torch.empty_like(x)
        post_stats, pre_stats = (torch.empty(2, x.shape[0], device=x.device) for _ in range(2))
        iabn.iabn_resnorm_forward(x, h, r, u, post_norm="rms", post_weight=post_weight, pre_norm="rms",
                                  pre_weight=pre_weight, post_stats=post_stats, pre_stats=pre_stats, eps=EPS)
        ctx.save_for_backward(r, h, post_weight, pre_weight, post_stats, pre_stats)
        return r, u

    @staticmethod
    def backward(ctx, dr, du):
        r, h, post_weight, pre_weight, post_stats, pre_stats = ctx.saved_tensors
        dx, dh, dpost, dpre = (torch.empty_like(t) for t in (r, h, post_weight, pre_weight))
        iabn.iabn_resnorm_backward(dr.contiguous(), du.contiguous(), r, h, dx, dh, post_norm="rms",
                                   post_weight=post_weight, pre_norm="rms", pre_weight=pre_weight,
                                   post_stats=post_stats, pre_stats=pre_stats, dpost_weight=dpost, dpre_weight=dpre)
        return dx, dh, dpost, dpre


class Stack(torch.nn.Module):
    def __init__(self, width, hidden, experts, top, layers, dtype, device="cuda"):
        super().__init__()
        self.top = top
        param = lambda t, d=dtype: torch.nn.Parameter(t.to(device=device, dtype=d))  # noqa: E731
        self.norms = torch.nn.ParameterList(
            [param(torch.ones(width), torch.float32) for _ in range(layers + 1)])
        self.blocks = torch.nn.ModuleList()
        for _ in range(layers):
            b = torch.nn.Module()
            b.router = param(torch.randn(experts, width) * width ** -0.5)
            b.w_gate = param(torch.randn(experts, hidden, width) * width ** -0.5)
            b.w_up = param(torch.randn(experts, hidden, width) * width ** -0.5)
            b.w_down = param(torch.randn(experts, width, hidden) * hidden ** -0.5)
            b.post = param(torch.ones(width), torch.float32)
            self.blocks.append(b)

    def forward(self, x):
        u = InputNorm.apply(x, self.norms[0])
        for i, b in enumerate(self.blocks):
            h = RoutedBlock.apply(u, u @ b.router.t(), b.w_gate, b.w_up, b.w_down, self.top)
            x, u = AddNorm.apply(x, h, b.post, self.norms[i + 1])
        return u

    @torch.no_grad()
    def serve(self, x):
        """Inference: nothing is kept, the stream is updated in place."""
        x = x.clone()
        u, h = torch.empty_like(x), torch.empty_like(x)
        iabn.iabn_resnorm_forward(x, None, None, u, pre_norm="rms", pre_weight=self.norms[0], eps=EPS)
        for i, b in enumerate(self.blocks):
            _, weights, plan = route(u @ b.router.t(), self.top)
            iabn.iabn_experts_forward(u, plan, weights, b.w_gate, b.w_up, b.w_down, h)
            iabn.iabn_resnorm_forward(x, h, x, u, post_norm="rms", post_weight=b.post, pre_norm="rms",
                                      pre_weight=self.norms[i + 1], eps=EPS)
        return u


def train(model, rows, width, steps, lr, dtype, max_norm=1.0, say=print):
    """Fits a random linear map of the input; returns the losses and gradient norms."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    teach = torch.randn(width, width, generator=gen, device="cuda") * width ** -0.5
    opt = torch.optim.SGD(model.parameters(), lr=lr, momentum=0.9)
    losses, norms = [], []
    for _ in range(steps):
        x = torch.randn(rows, width, generator=gen, device="cuda")
        loss = (model(x.to(dtype)).float() - x @ teach).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        grads = [p.grad for p in model.parameters()]
        norm = iabn.iabn_grad_norm(grads, torch.empty((), device="cuda"))
        iabn.iabn_grad_clip(grads, grads, norm, max_norm)
        opt.step()
        losses.append(loss.detach())
        norms.append(norm)
    losses, norms = [float(v) for v in losses], [float(v) for v in norms]
    say("loss %.4f -> %.4f over %d steps, gradient norm %.3f -> %.3f"
        % (losses[0], losses[-1], steps, norms[0], norms[-1]))
    return losses, norms


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=4096)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--experts", type=int, default=32)
    ap.add_argument("--top", type=int, default=4)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=30)
    args = ap.parse_args()
    torch.manual_seed(0)
    model = Stack(args.width, args.hidden, args.experts, args.top, args.layers, torch.bfloat16)
    train(model, args.rows, args.width, args.steps, 0.5, torch.bfloat16)
    print("peak memory %.2f GB" % (torch.cuda.max_memory_allocated() / 1e9))
    tokens = torch.randn(8, args.width, device="cuda").bfloat16()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for n in (1, 8):
        model.serve(tokens[:n])
        start.record()
        for _ in range(50):
            model.serve(tokens[:n])
        end.record()
        torch.cuda.synchronize()
        print("%d tokens: %.1f us for %d sublayers" % (n, start.elapsed_time(end) / 50 * 1e3, args.layers))


if __name__ == "__main__":
    main()
