"""A stack of feed-forward sublayers on libiabn: trained for some steps, then
serving token by token.

    python examples/ffn_sublayer.py [--rows 4096 --width 1024 --hidden 4096 --layers 4]

One sublayer takes the residual stream x and its normalised values u:

    h = feed-forward(u)                        iabn_ffn_forward
    x = x + gate * dropout(norm(h)), u = norm(x)   iabn_resnorm_forward, one pass

Its backward recomputes instead of storing: the activation's product from the
two projections (which its gradients then overwrite), the normalised rows from
the statistics, and the dropout's mask from its seed.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_1712_02616_amd as iabn  # noqa: E402

EPS = 1e-5


class InputNorm(torch.autograd.Function):
    """u = norm(x): the norm before the first block."""

    @staticmethod
    def forward(ctx, x, weight):
        u = torch.empty_like(x)
        stats = torch.empty(2, x.shape[0], device=x.device)
        iabn.iabn_resnorm_forward(x, None, None, u, pre_norm="rms", pre_weight=weight,
                                  pre_stats=stats, eps=EPS)
        ctx.save_for_backward(x, weight, stats)
        return u

    @staticmethod
    def backward(ctx, du):
        x, weight, stats = ctx.saved_tensors
        dx, dweight = torch.empty_like(x), torch.empty_like(weight)
        iabn.iabn_resnorm_backward(None, du.contiguous(), x, None, dx, None, pre_norm="rms",
                                   pre_weight=weight, pre_stats=stats, dpre_weight=dweight)
        return dx, dweight


class Sublayer(torch.autograd.Function):
    """(x, u) -> (x + gate*dropout(norm(feed-forward(u))), its norm)."""

    @staticmethod
    def forward(ctx, x, u, w_gate, w_up, w_down, gate, post_weight, pre_weight, p, seed):
        rows, hidden = x.shape[0], w_gate.shape[0]
        h = torch.empty_like(x)
        g = torch.empty(rows, hidden, dtype=x.dtype, device=x.device)
        up = torch.empty_like(g)
        iabn.iabn_ffn_forward(u, w_gate, w_up, w_down, h, g, up)
        r, out = torch.empty_like(x), torch.empty_like(x)
        post_stats = torch.empty(2, rows, device=x.device)
        pre_stats = torch.empty(2, rows, device=x.device)
        iabn.iabn_resnorm_forward(x, h, r, out, gate=gate, post_norm="rms", post_weight=post_weight,
                                  pre_norm="rms", pre_weight=pre_weight, post_stats=post_stats,
                                  pre_stats=pre_stats, eps=EPS, p=p, seed=seed)
        ctx.save_for_backward(u, g, up, h, r, w_gate, w_up, w_down, gate, post_weight, pre_weight,
                              post_stats, pre_stats)
        ctx.p, ctx.seed = p, seed
        return r, out

    @staticmethod
    def backward(ctx, dr, dout):
        u, g, up, h, r, w_gate, w_up, w_down, gate, post_weight, pre_weight, post_stats, pre_stats = \
            ctx.saved_tensors
        dx, dh = torch.empty_like(r), torch.empty_like(r)
        dgate, dpost, dpre = (torch.empty_like(t) for t in (gate, post_weight, pre_weight))
        iabn.iabn_resnorm_backward(dr.contiguous(), dout.contiguous(), r, h, dx, dh, gate=gate,
                                   post_norm="rms", post_weight=post_weight, pre_norm="rms",
                                   pre_weight=pre_weight, post_stats=post_stats, pre_stats=pre_stats,
                                   dgate=dgate, dpost_weight=dpost, dpre_weight=dpre, p=ctx.p,
                                   seed=ctx.seed)
        du = torch.empty_like(u)
        dws = [torch.empty_like(w) for w in (w_gate, w_up, w_down)]
        # The projections' gradients overwrite the projections, which autograd is
        # told: a second backward through this graph fails.
        torch.autograd.graph.increment_version((g, up))
        iabn.iabn_ffn_backward(dh, u, g, up, w_gate, w_up, w_down, du, g, up, *dws)
        return (dx, du, *dws, dgate, dpost, dpre, None, None)


class Stack(torch.nn.Module):
    def __init__(self, width, hidden, layers, dtype, device="cuda", p=0.1):
        super().__init__()
        self.p = p
        param = lambda t, d=dtype: torch.nn.Parameter(t.to(device=device, dtype=d))  # noqa: E731
        self.norms = torch.nn.ParameterList(
            [param(torch.ones(width), torch.float32) for _ in range(layers + 1)])
        self.blocks = torch.nn.ModuleList()
        for _ in range(layers):
            b = torch.nn.Module()
            b.w_gate = param(torch.randn(hidden, width) * width ** -0.5)
            b.w_up = param(torch.randn(hidden, width) * width ** -0.5)
            b.w_down = param(torch.randn(width, hidden) * hidden ** -0.5)
            b.gate = param(torch.full((1, width), 0.5))
            b.post = param(torch.ones(width), torch.float32)
            self.blocks.append(b)

    def forward(self, x, step=0):
        """Training: a mask per layer and step."""
        u = InputNorm.apply(x, self.norms[0])
        for i, b in enumerate(self.blocks):
            x, u = Sublayer.apply(x, u, b.w_gate, b.w_up, b.w_down, b.gate, b.post,
                                  self.norms[i + 1], self.p, step * len(self.blocks) + i)
        return u

    @torch.no_grad()
    def serve(self, x):
        """Inference: nothing is kept, the stream is updated in place."""
        x = x.clone()
        u, h = torch.empty_like(x), torch.empty_like(x)
        iabn.iabn_resnorm_forward(x, None, None, u, pre_norm="rms", pre_weight=self.norms[0], eps=EPS)
        for i, b in enumerate(self.blocks):
            iabn.iabn_ffn_forward(u, b.w_gate, b.w_up, b.w_down, h)
            iabn.iabn_resnorm_forward(x, h, x, u, gate=b.gate, post_norm="rms", post_weight=b.post,
                                      pre_norm="rms", pre_weight=self.norms[i + 1], eps=EPS)
        return u


def train(model, rows, width, steps, lr, dtype, say=print):
    """Fits a random linear map of the input; returns the losses."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    teach = torch.randn(width, width, generator=gen, device="cuda") * width ** -0.5
    opt = torch.optim.SGD(model.parameters(), lr=lr, momentum=0.9)
    losses = []
    for step in range(steps):
        x = torch.randn(rows, width, generator=gen, device="cuda")
        want = x @ teach
        loss = (model(x.to(dtype), step).float() - want).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    losses = [float(v) for v in losses]
    say("loss %.4f -> %.4f over %d steps" % (losses[0], losses[-1], steps))
    return losses


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--rows", type=int, default=4096)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=30)
    args = ap.parse_args()
    torch.manual_seed(0)
    model = Stack(args.width, args.hidden, args.layers, torch.bfloat16)
    train(model, args.rows, args.width, args.steps, 0.5, torch.bfloat16)
    print("peak memory %.2f GB" % (torch.cuda.max_memory_allocated() / 1e9))

    tokens = torch.randn(8, args.width, device="cuda").bfloat16()
    together = model.serve(tokens)
    one_by_one = torch.cat([model.serve(t[None]) for t in tokens])
    print("one token at a time against 8 at once: largest difference %.3g"
          % float((together.float() - one_by_one.float()).abs().max()))
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(50):
        model.serve(tokens[:1])
    end.record()
    torch.cuda.synchronize()
    print("a token: %.1f us for %d sublayers" % (start.elapsed_time(end) / 50 * 1e3, args.layers))


if __name__ == "__main__":
    main()
