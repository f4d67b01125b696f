"""The feed-forward sublayer's operators in 64 bits on the CPU (not a test
module), with the magnitudes that bound a 32-bit evaluation's error: `mag`
values are the same formulas with every term replaced by its absolute value,
so that |computed - exact| <= k * 2^-24 * mag for k operations in a row."""

from __future__ import annotations

import math

import numpy as np
import torch

U32 = 2.0 ** -24
# Unit roundoff of a stored value.
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# The smallest step of a stored value (subnormal values round to multiples of it).
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def philox(counter, key):
    """Philox4x32-10 of one 4-word counter and 2-word key, in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def factors(rows, width, p, seed, offset):
    """The dropout's factor of every element, [rows, width] float64."""
    cut = int(float(np.float32(p)) * 65536.0 + 0.5)
    if cut == 0:
        return torch.ones(rows, width, dtype=torch.float64)
    per = -(-width // 8)
    ctr = [np.arange(rows * per, dtype=np.uint64)]
    ctr = [ctr[0] & np.uint64(0xFFFFFFFF), ctr[0] >> np.uint64(32),
           np.full(rows * per, offset & 0xFFFFFFFF, np.uint64), np.full(rows * per, offset >> 32, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        hi, lo, m = (lambda v: v >> np.uint64(32)), (lambda v: v & np.uint64(0xFFFFFFFF)), np.uint64
        ctr = [hi(b) ^ ctr[1] ^ m(k0), lo(b), hi(a) ^ ctr[3] ^ m(k1), lo(a)]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    lanes = np.stack([v & np.uint64(0xFFFF) if half == 0 else v >> np.uint64(16)
                      for v in ctr for half in (0, 1)], axis=1).reshape(rows, per * 8)[:, :width]
    scale = 65536.0 / (65536 - cut) if cut < 65536 else 0.0
    return torch.from_numpy((lanes >= cut).astype(np.float64) * scale)


def _norm(v, kind, w, b, eps, verr, ops):
    """hat*w + b, statistics, hat, and a bound of the 32-bit error given the
    input's (verr): `ops` roundings in a sum over the row."""
    if kind is None:
        z = torch.zeros(v.shape[0], dtype=torch.float64)
        return v, None, v, verr, None
    mu = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    rstd = ((v - mu).square().mean(1, keepdim=True) + eps).rsqrt()
    hat = (v - mu) * rstd
    mag = v.abs() + (v.abs().mean(1, keepdim=True) if kind == "layer" else 0.0)
    cerr = verr + (verr.mean(1, keepdim=True) if kind == "layer" else 0.0) + ops * U32 * mag
    # d(rstd)/rstd = -rstd^2 mean(c dc): at most rstd * rms(cerr), and the sum's own roundings.
    rerr = rstd * cerr.square().mean(1, keepdim=True).sqrt() + ops * U32
    herr = cerr * rstd + (hat.abs() + cerr * rstd) * rerr
    w = torch.ones(v.shape[1], dtype=torch.float64) if w is None else w
    out = hat * w + (0.0 if b is None else b)
    err = herr * w.abs() + 4 * U32 * (hat.abs() * w.abs() + (0.0 if b is None else b.abs()))
    merr = (verr.mean(1) + ops * U32 * v.abs().mean(1)) if kind == "layer" else torch.zeros(v.shape[0])
    return out, torch.stack([mu[:, 0], rstd[:, 0]]), hat, err, torch.stack([merr, rstd[:, 0] * rerr[:, 0]])


def forward(x, h, gate, post, pw, pb, pre, qw, qb, alpha, beta, eps, keep):
    """All [R, C] float64 (vectors [C], gate [G, C] or None); returns a dict of
    (value, bound) for r, u and the statistics."""
    R, C = x.shape
    # Additions in a row: 16 of a thread, 6 steps of a wave, 16 waves, and the
    # handful of the formula.
    ops = 48
    zero = torch.zeros_like(x)
    out = {}
    r, rerr = alpha * x, 2 * U32 * (alpha * x).abs()
    if h is not None:
        n, stats, _, nerr, serr = _norm(h, post, pw, pb, eps, zero, ops)
        if stats is not None:
            out["post_stats"] = (stats, serr)
        g = torch.ones_like(x) if gate is None else gate.repeat_interleave(R // gate.shape[0], 0)
        f = beta * g * keep
        r = r + f * n
        rerr = rerr + f.abs() * nerr + 6 * U32 * ((alpha * x).abs() + (f * n).abs())
    out["r"] = (r, rerr)
    if pre is not None:
        u, stats, _, uerr, serr = _norm(r, pre, qw, qb, eps, rerr, ops)
        out["u"], out["pre_stats"] = (u, uerr), (stats, serr)
    return out


def backward(dr, du, r, h, gate, post, pw, pb, pre, qw, post_stats, pre_stats, alpha, beta, keep):
    """(value, bound) of every gradient."""
    like = dr if dr is not None else du
    R, C = like.shape
    ops, rows = 48, 64 + R  # a column's sum: one addition a row
    out = {}
    g = torch.zeros_like(like) if dr is None else dr
    gm = g.abs()

    def back(d, dm, hat, rstd, kind):
        v = d - hat * (d * hat).mean(1, keepdim=True)
        m = dm + hat.abs() * (dm * hat.abs()).mean(1, keepdim=True)
        if kind == "layer":
            v, m = v - d.mean(1, keepdim=True), m + dm.mean(1, keepdim=True)
        return v * rstd, m * rstd

    def hat_of(v, stats):
        # hat's own error: the subtraction's operands, relative to what is left.
        mu, rstd = stats[0][:, None], stats[1][:, None]
        return (v - mu) * rstd, (v.abs() + mu.abs()) * rstd

    if pre is not None:
        rhat, rmag = hat_of(r, pre_stats)
        out["dpre_weight"] = ((du * rhat).sum(0), (du.abs() * rmag).sum(0) * rows * U32)
        out["dpre_bias"] = (du.sum(0), du.abs().sum(0) * rows * U32)
        a = du * (1.0 if qw is None else qw)
        v, _ = back(a, a.abs(), rhat, pre_stats[1][:, None], pre)
        _, m = back(a, a.abs(), rmag, pre_stats[1][:, None], pre)
        g, gm = g + v, gm + m
    out["dx"] = (alpha * g, abs(alpha) * gm * ops * U32)
    if h is None and post is None and gate is None:
        gr = torch.ones_like(like)
        out["dh"] = (beta * g * keep, abs(beta) * gm * keep * ops * U32)
        return out
    e, em = beta * g * keep, abs(beta) * gm * keep
    hhat, hmag = (h, h.abs()) if post is None else hat_of(h, post_stats)
    n, nm = hhat, hmag
    if post is not None:
        n = hhat * (1.0 if pw is None else pw) + (0.0 if pb is None else pb)
        nm = hmag * (1.0 if pw is None else pw.abs()) + (0.0 if pb is None else pb.abs())
    gr = torch.ones_like(like)
    if gate is not None:
        G = gate.shape[0]
        gr = gate.repeat_interleave(R // G, 0)
        out["dgate"] = ((e * n).reshape(G, R // G, C).sum(1),
                        (em * nm).reshape(G, R // G, C).sum(1) * (rows + ops) * U32)
    dn, dm = e * gr, em * gr.abs()
    if post is None:
        out["dh"] = (dn, dm * ops * U32)
        return out
    out["dpost_weight"] = ((dn * hhat).sum(0), (dm * hmag).sum(0) * (rows + ops) * U32)
    out["dpost_bias"] = (dn.sum(0), dm.sum(0) * (rows + ops) * U32)
    w = torch.ones(C, dtype=torch.float64) if pw is None else pw
    v, _ = back(dn * w, dm, hhat, post_stats[1][:, None], post)
    _, m = back(dn * w, dm * w.abs(), hmag, post_stats[1][:, None], post)
    out["dh"] = (v, m * 2 * ops * U32)
    return out


def act(v, kind, slope=0.01):
    """The activation and its derivative."""
    if kind == "silu":
        s = torch.sigmoid(v)
        return v * s, s + v * s * (1 - s)
    if kind == "gelu":
        c = torch.special.ndtr(v)
        return v * c, c + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    return torch.where(v >= 0, v, slope * v), torch.where(v >= 0, torch.ones_like(v), torch.full_like(v, slope))


def check(name, got, want, bound, dtype):
    """`got` (a device tensor of `dtype`) against the exact value, where the
    32-bit value is within `bound` and is then rounded to the stored type."""
    got = got.detach().cpu().double().reshape(want.shape)
    u = UNIT[dtype]
    allowed = bound * (1 + 2 * u) + u * want.abs() + TINY[dtype]
    off = (got - want).abs() / allowed
    assert torch.isfinite(got).all(), "%s has non-finite values" % name
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 1.0, "%s is %.2f of its bound off (largest difference %.3g)" % (
        name, worst, float((got - want).abs().max()))
