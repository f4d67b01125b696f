"""Routing, the plan and the routed experts in 64 bits on the CPU (not a test
module), with bounds of a 32-bit evaluation (see sublayer_oracle)."""

from __future__ import annotations

import math

import torch

import sublayer_oracle as oracle

U32 = oracle.U32
INF = float("inf")


def scores(logits, score):
    """[M, E] float64; a row of nothing but -inf has zeros."""
    l = logits.double()
    if score == "sigmoid":
        return torch.sigmoid(l)
    e = torch.exp(l - l.amax(1, keepdim=True))
    return torch.where((l == -INF).all(1, keepdim=True), torch.zeros_like(l), e / e.sum(1, keepdim=True))


def choose(logits, bias, k, score, groups=1, kept=None, group_top=1):
    """The choices of every row, as lists in Python: [M][k], -1 where nothing is left."""
    s, l = scores(logits, score), logits.double()
    M, E = l.shape
    kept = groups if kept is None else kept
    per = E // groups
    b = torch.zeros(E, dtype=torch.float64) if bias is None else bias.double()
    nan_first = lambda v: (0, 0.0) if math.isnan(v) else (1, -v)  # noqa: E731
    rows = []
    for m in range(M):
        may = [e for e in range(E) if float(l[m, e]) != -INF and float(b[e]) != -INF]
        c = {e: float(l[m, e]) if bias is None else float(s[m, e] + b[e]) for e in may}
        if kept < groups:
            of = {e: float(s[m, e] + b[e]) for e in may}
            tops = {}
            for e in may:
                tops.setdefault(e // per, []).append(of[e])
            totals = {}
            for g, vs in tops.items():
                vs = sorted(vs, key=nan_first)[:group_top]
                totals[g] = sum(vs[1:], vs[0])
            best = sorted(totals, key=lambda g: (nan_first(totals[g]), g))[:kept]
            may = [e for e in may if e // per in best]
        got = sorted(may, key=lambda e: (nan_first(c[e]), e))[:k]
        rows.append(got + [-1] * (k - len(got)))
    return rows


def weights(logits, chosen, score, renormalise, scale):
    """The weights of the choices [M, k] (int64), float64."""
    s = scores(logits, score)
    there = chosen >= 0
    w = torch.where(there, s.gather(1, chosen.clamp(min=0)), torch.zeros(()).double())
    if renormalise:
        w = torch.where(there, w / w.sum(1, keepdim=True), w)
    return scale * w


# A weight's relative error in 32 bits: two functions of 2 units each, a sum of the
# row's terms (16 of a lane, 6 steps between lanes; each term off by 3), two
# divisions and the scale.
WEIGHT_ERROR = 36 * U32


def route_backward(dw, logits, chosen, score, renormalise, scale):
    """(value, bound) of the logits' gradient."""
    s, l = scores(logits, score), logits.double()
    M, E = l.shape
    there = (chosen >= 0) & (chosen < E)
    at = torch.where(there, chosen, torch.zeros_like(chosen))
    there = there & (l.gather(1, at) != -INF)
    d = torch.where(there, scale * dw.double(), torch.zeros(()).double())
    p = torch.where(there, s.gather(1, at), torch.zeros(()).double())
    zero = torch.zeros_like(s)
    if renormalise:
        p = torch.where(there, p / p.sum(1, keepdim=True), p)
        q = p * (d - (p * d).sum(1, keepdim=True))
        m = p * (d.abs() + (p * d.abs()).sum(1, keepdim=True))
        if score == "sigmoid":
            keep = torch.sigmoid(-l).gather(1, at)
            q, m = q * keep, m * keep
        # (p and the sum's p are each off by WEIGHT_ERROR.)
        return zero.scatter_add(1, at, q), zero.scatter_add(1, at, m) * 4 * WEIGHT_ERROR
    ds, dm = zero.scatter_add(1, at, d), zero.scatter_add(1, at, d.abs())
    if score == "sigmoid":
        f = s * torch.sigmoid(-l)
        return ds * f, dm * f * 2 * WEIGHT_ERROR
    dot, mag = (p * d).sum(1, keepdim=True), (p * d.abs()).sum(1, keepdim=True)
    return s * (ds - dot), s * (dm + mag) * 4 * WEIGHT_ERROR


def plan(experts, E):
    """offsets, order, place of a [M, k] choice, in Python."""
    flat = experts.flatten().tolist()
    order, offsets = [], [0]
    for e in range(E):
        order += [i for i, v in enumerate(flat) if v == e]
        offsets.append(len(order))
    place = [-1] * len(flat)
    for p, i in enumerate(order):
        place[i] = p
    return offsets, order, place


def product(a, b, aerr=None):
    """a b^T with a bound: a sum of K terms in any order (K + 4 roundings), and a's
    own error."""
    v, mag = a @ b.T, a.abs() @ b.abs().T
    err = (a.shape[1] + 4) * U32 * mag
    return v, err if aerr is None else err + aerr @ b.abs().T * (1 + (a.shape[1] + 4) * U32)


def stored(v, err, dtype):
    return err * (1 + oracle.UNIT[dtype]) + oracle.UNIT[dtype] * v.abs() + oracle.TINY[dtype]


def activation_error(v, err, act):
    """Bounds of act(v) and act'(v) in 32 bits of v off by err (|act''|, |act'| < 1.2;
    the functions to 16 units)."""
    if act == "leaky":
        near = v.abs() <= err
        return err + 2 * U32 * v.abs(), torch.where(near, torch.ones_like(v), torch.zeros_like(v))
    return 1.2 * err + 16 * U32 * (1 + v.abs()), 1.2 * err + 16 * U32 * (1 + v.abs())


def experts_forward(x, weights, w_gate, w_up, w_down, sorted_plan, k, dtype, act, slope):
    """{name: (value, bound)} of y, and of g, u up to the plan's last row.  h and each
    weighted term are rounded to the storage type in between."""
    offsets, order, _ = sorted_plan
    M, C = x.shape
    F = w_gate.shape[1]
    rows = offsets[-1]
    g, ge = torch.zeros(rows, F).double(), torch.zeros(rows, F).double()
    u, ue = g.clone(), g.clone()
    y, ye = torch.zeros(M, C).double(), torch.zeros(M, C).double()
    mag = torch.zeros(M, C).double()
    for e in range(w_gate.shape[0]):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        pairs = torch.tensor(order[lo:hi])
        xe, w = x[pairs // k], weights.flatten()[pairs][:, None]
        gv, gerr = product(xe, w_gate[e])
        uv, uerr = product(xe, w_up[e])
        g[lo:hi], ge[lo:hi], u[lo:hi], ue[lo:hi] = gv, gerr, uv, uerr
        av, _ = oracle.act(gv, act, slope)
        ae, _ = activation_error(gv, gerr, act)
        h = av * uv
        he = stored(h, ae * uv.abs() + av.abs() * uerr + ae * uerr + 2 * U32 * h.abs(), dtype)
        o, oe = product(h, w_down[e], he)
        t, te = w * o, w.abs() * oe + 2 * U32 * (w * o).abs()
        te = stored(t, te, dtype)
        y.index_add_(0, pairs // k, t)
        ye.index_add_(0, pairs // k, te)
        mag.index_add_(0, pairs // k, t.abs())
    return {"y": (y, ye + (k + 1) * U32 * mag), "g": (g, ge), "u": (u, ue)}


def experts_backward(dy, x, weights, g, u, w_gate, w_up, w_down, sorted_plan, k, dtype, act, slope):
    """{name: (value, bound)} of every gradient, from the kept g, u (sorted rows)."""
    offsets, order, _ = sorted_plan
    M, C = x.shape
    E, F = w_gate.shape[:2]
    zero = lambda *s: torch.zeros(*s).double()  # noqa: E731
    out = {n: [zero(E, F, C), zero(E, F, C)] for n in ("dw_gate", "dw_up")}
    out["dw_down"] = [zero(E, C, F), zero(E, C, F)]
    out["dx"], out["dweights"] = [zero(M, C), zero(M, C)], [zero(M * k), zero(M * k)]
    out["dg"], out["du"] = [zero(offsets[-1], F), zero(offsets[-1], F)], [zero(offsets[-1], F), zero(offsets[-1], F)]
    mag = zero(M, C)
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if lo == hi:
            continue
        pairs = torch.tensor(order[lo:hi])
        xe, dye, w = x[pairs // k], dy[pairs // k], weights.flatten()[pairs][:, None]
        gs, us = g[lo:hi], u[lo:hi]
        av, dv = oracle.act(gs, act, slope)
        ae, de = activation_error(gs, torch.zeros_like(gs), act)
        dh, dhe = product(dye, w_down[e].T)
        h = av * us
        herr = ae * us.abs() + 2 * U32 * h.abs()
        out["dweights"][0][pairs] = (h * dh).sum(1)
        out["dweights"][1][pairs] = (herr * dh.abs() + h.abs() * dhe + herr * dhe + (F + 8) * U32 * (h * dh).abs()).sum(1)
        dgv, duv = w * dh * us * dv, w * dh * av
        dge = w.abs() * (dhe * (us * dv).abs() + (dh * us).abs() * de + dhe * us.abs() * de) + 4 * U32 * dgv.abs()
        due = w.abs() * (dhe * av.abs() + dh.abs() * ae + dhe * ae) + 3 * U32 * duv.abs()
        dge, due = stored(dgv, dge, dtype), stored(duv, due, dtype)
        hw = w * h
        hwe = stored(hw, w.abs() * herr + 2 * U32 * hw.abs(), dtype)
        out["dg"][0][lo:hi], out["dg"][1][lo:hi] = dgv, dge
        out["du"][0][lo:hi], out["du"][1][lo:hi] = duv, due
        out["dw_gate"][0][e], out["dw_gate"][1][e] = product(dgv.T, xe.T, dge.T)
        out["dw_up"][0][e], out["dw_up"][1][e] = product(duv.T, xe.T, due.T)
        v, err = product(hw.T, dye.T, hwe.T)
        out["dw_down"][0][e], out["dw_down"][1][e] = v.T, err.T
        a, ea = product(dgv, w_gate[e].T, dge)
        b, eb = product(duv, w_up[e].T, due)
        t = a + b
        te = ea + eb + (2 * F + 4) * U32 * (dgv.abs() @ w_gate[e].abs() + duv.abs() @ w_up[e].abs())
        te = stored(t, te, dtype)
        out["dx"][0].index_add_(0, pairs // k, t)
        out["dx"][1].index_add_(0, pairs // k, te)
        mag.index_add_(0, pairs // k, t.abs())
    out["dx"][1] += (k + 1) * U32 * mag
    return {n: tuple(v) for n, v in out.items()}
