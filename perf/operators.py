"""The work that a program training or serving a transformer's feed-forward
sublayer has this library do, as measurable cases.

The sublayer: a residual stream x [rows, width], a gated feed-forward block,
and the norms before and after it, fused with the gate, the residual scale and
the dropout of the sublayer.

- norm_forward:   r = alpha*x + beta*gate*dropout(post(h)), u = pre(r)
- norm_backward:  its gradients from dr and du
- dropout:        the counter-based dropout alone
- ffn_forward:    y = (act(x Wg^T) * (x Wu^T)) Wd^T
- ffn_backward:   its gradients from dy
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
# The residual scale and the branch's scale of the norm cases.
ALPHA, BETA = 0.875, 0.5


def _norm(name, direction, dtype, rows, width, post, pre, groups, p, train=True):
    """groups: rows of the gate (0: no gate); row i of the stream takes gate
    row i // (rows // groups).  train: the statistics are kept."""
    return {"name": name, "op": "norm_" + direction, "dtype": dtype, "rows": rows, "width": width,
            "post": post, "pre": pre, "groups": groups, "p": p, "train": train}


def _dropout(name, dtype, rows, width, p):
    return {"name": name, "op": "dropout", "dtype": dtype, "rows": rows, "width": width, "p": p}


def _ffn(name, direction, dtype, rows, width, hidden, act, train=True):
    """train: the forward gives the two projections too, which its backward
    takes."""
    return {"name": name, "op": "ffn_" + direction, "dtype": dtype, "rows": rows, "width": width,
            "hidden": hidden, "act": act, "train": train}


def listed():
    return [
        # Serving: one token between two sublayers; the cost of a call.
        _norm("norm_token_bf16", "forward", "bf16", 1, 2048, "rms", "rms", 0, 0.0, train=False),
        # Training: 8 samples of 64x64 positions and 1024 channels, a gate per sample.
        _norm("norm_forward_f16", "forward", "f16", 32768, 1024, "layer", "layer", 8, 0.1),
        # The backward of a wide stream with a gate shared by every token.
        _norm("norm_backward_bf16", "backward", "bf16", 16384, 2048, "rms", "rms", 1, 0.1),
        # A prime number of tokens, rows that are no whole number of 16-byte accesses.
        _norm("norm_backward_odd_f32", "backward", "f32", 1031, 1501, "layer", "layer", 1, 0.0),
        # Dropout on a small batch's embeddings: the cost of a call.
        _dropout("dropout_small_f16", "f16", 64, 1024, 0.25),
        # And on a training batch's.
        _dropout("dropout_bf16", "bf16", 32768, 2048, 0.1),
        # Serving: the next token of one sequence; every weight is read once.
        _ffn("ffn_token_bf16", "forward", "bf16", 1, 4096, 10240, "silu", train=False),
        # Serving: the next tokens of a batch of sequences.
        _ffn("ffn_batch_f16", "forward", "f16", 24, 2048, 8192, "silu", train=False),
        # A prompt of odd length through a block of odd sizes.
        _ffn("ffn_odd_f32", "forward", "f32", 333, 1000, 2731, "gelu", train=False),
        # Training's forward.
        _ffn("ffn_forward_bf16", "forward", "bf16", 4096, 2048, 8192, "silu"),
        # Training's backward: a ragged number of tokens.
        _ffn("ffn_backward_f16", "backward", "f16", 2085, 1024, 4096, "gelu"),
        # The largest: the backward of a wide block.
        _ffn("ffn_backward_bf16", "backward", "bf16", 8192, 4096, 10240, "silu"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm_forward", "norm_backward", "dropout", "ffn_forward", "ffn_backward"])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    if kind.startswith("ffn"):
        width, hidden = _spread(rng, 256, 4096), _spread(rng, 512, 10240)
        if rng.random() < 0.75:  # most blocks' sizes are whole numbers of 16-byte accesses
            width, hidden = (width + 7) // 8 * 8, (hidden + 7) // 8 * 8
        rows = _spread(rng, 1, 8192)
        if dtype == "f32":  # 32-bit blocks are the smaller ones
            rows = min(rows, 2048)
        return _drop_name(_ffn("", kind[4:], dtype, rows, width, hidden, rng.choice(["silu", "gelu"]),
                               train=rng.random() < 0.5 or kind == "ffn_backward"))
    width = _spread(rng, 64, 8192)
    if rng.random() < 0.5:
        width = (width + 7) // 8 * 8
    rows = _spread(rng, 1, max(1, (1 << 26) // width))
    p = rng.choice([0.0, 0.1, 0.5])
    if kind == "dropout":
        return _drop_name(_dropout("", dtype, rows, width, p or 0.25))
    groups = rng.choice([0, 1, 4])
    if groups:
        rows = max(1, rows // groups) * groups
    return _drop_name(_norm("", kind[5:], dtype, rows, width, rng.choice(["rms", "layer", "none"]),
                            rng.choice(["rms", "layer"]), groups, p))


def _drop_name(case):
    return {k: v for k, v in case.items() if k != "name"}


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 13)
    dtype = DTYPES[case["dtype"]]
    rows, width = case["rows"], case["width"]

    def normal(*shape, std=1.0, to=dtype):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(to)

    def uniform(*shape, lo, hi):
        return torch.rand(*shape, generator=gen, device="cuda") * (hi - lo) + lo

    state = {"case": case}
    if case["op"].startswith("ffn"):
        hidden = case["hidden"]
        state["x"] = normal(rows, width)
        state["w_gate"] = normal(hidden, width, std=1.0 / math.sqrt(width))
        state["w_up"] = normal(hidden, width, std=1.0 / math.sqrt(width))
        state["w_down"] = normal(width, hidden, std=1.0 / math.sqrt(hidden))
        if case["op"] == "ffn_backward":
            # What the forward kept, and the gradient that arrives.
            x = state["x"].float()
            state["g"] = (x @ state["w_gate"].float().t()).to(dtype)
            state["u"] = (x @ state["w_up"].float().t()).to(dtype)
            state["dy"] = normal(rows, width, std=0.1)
        return state

    # A residual stream whose channels differ in scale, and a block's output.
    scale = uniform(width, lo=0.5, hi=3.0)
    state["x"] = (torch.randn(rows, width, generator=gen, device="cuda") * scale).to(dtype)
    state["p"] = case["p"]
    state["seed"] = int(torch.randint(1 << 62, (1,), generator=gen, device="cuda").item())
    state["offset"] = int(torch.randint(1 << 40, (1,), generator=gen, device="cuda").item())
    if case["op"] == "dropout":
        return state
    state["h"] = normal(rows, width, std=1.5)
    state["gate"] = normal(case["groups"], width, std=0.5) if case["groups"] else None
    for stage in ("post", "pre"):
        affine, bias = case[stage] != "none", case[stage] == "layer"
        state[stage + "_weight"] = uniform(width, lo=0.5, hi=1.5) if affine else None
        state[stage + "_bias"] = normal(width, std=0.1, to=torch.float32) if bias else None
    if case["op"] == "norm_backward":
        # What the forward kept, and the gradients that arrive.
        r, _, state["post_stats"], state["pre_stats"] = _norm_forward(state)
        state["r"] = r.to(dtype)
        state["dr"] = normal(rows, width, std=0.1)
        state["du"] = normal(rows, width, std=0.1)
    return state


# ------------------------------------------------------------------ plain forms


def _keep(rows, width, p, seed, offset):
    """The dropout's factor of every element: 0, or 1/(1 - p) with p to 16
    bits.  Philox4x32-10 with the key `seed` on the counter (row * ceil(width
    / 8) + column // 8, offset); its 128 bits are 16 for each of 8 columns."""
    per_row = (width + 7) // 8
    q = torch.arange(rows * per_row, device="cuda", dtype=torch.int64)
    low = 0xFFFFFFFF
    c0, c1 = q & low, q >> 32
    c2, c3 = torch.full_like(q, offset & low), torch.full_like(q, (offset >> 32) & low)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):  # the rounds of the generator
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64-bit products (the sign bit is a bit as any)
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    bits = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16,
                        c3 & 0xFFFF, c3 >> 16], dim=1)
    threshold = int(math.floor(p * 65536 + 0.5))
    kept = (bits >= threshold).reshape(rows, per_row * 8)[:, :width]
    return kept.float() * (65536.0 / (65536 - threshold) if threshold < 65536 else 0.0)


def _normalise(v, kind):
    """The normalised rows and their [2, rows] statistics (mean, 1/deviation)."""
    mean = v.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    centred = v - mean
    rstd = 1.0 / torch.sqrt((centred * centred).mean(dim=1, keepdim=True) + EPS)
    return centred * rstd, torch.stack([mean[:, 0], rstd[:, 0]])


def _affine(v, weight, bias):
    v = v * weight if weight is not None else v
    return v + bias if bias is not None else v


def _gate_rows(s):
    if s["gate"] is None:
        return 1.0
    return s["gate"].float().repeat_interleave(s["case"]["rows"] // s["case"]["groups"], dim=0)


def _factor(s):
    if s["p"] == 0.0:
        return 1.0
    return _keep(s["case"]["rows"], s["case"]["width"], s["p"], s["seed"], s["offset"])


def _norm_forward(s):
    """r, u and the statistics of both norms, in 32 bits."""
    case = s["case"]
    n, post_stats = s["h"].float(), None
    if case["post"] != "none":
        n, post_stats = _normalise(n, case["post"])
        n = _affine(n, s["post_weight"], s["post_bias"])
    r = ALPHA * s["x"].float() + BETA * _gate_rows(s) * (_factor(s) * n)
    u, pre_stats = _normalise(r, case["pre"])
    return r, _affine(u, s["pre_weight"], s["pre_bias"]), post_stats, pre_stats


def _norm_gradient(d, hat, rstd, kind):
    """The gradient of the normalised rows, back through the norm."""
    mean = d.mean(dim=1, keepdim=True) if kind == "layer" else 0.0
    return rstd * (d - mean - hat * (d * hat).mean(dim=1, keepdim=True))


def _plain_norm_backward(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    out = {}
    du = s["du"].float()
    mean, rstd = s["pre_stats"][0][:, None], s["pre_stats"][1][:, None]
    rhat = (s["r"].float() - mean) * rstd
    out["dpre_weight"] = (du * rhat).sum(dim=0)
    if s["pre_bias"] is not None:
        out["dpre_bias"] = du.sum(dim=0)
    g = s["dr"].float() + _norm_gradient(du * s["pre_weight"], rhat, rstd, case["pre"])
    out["dx"] = (ALPHA * g).to(dtype)
    e = BETA * g * _factor(s)
    hat = s["h"].float()
    if case["post"] != "none":
        mean, rstd = s["post_stats"][0][:, None], s["post_stats"][1][:, None]
        hat = (hat - mean) * rstd
    if s["gate"] is not None:
        n = _affine(hat, s["post_weight"], s["post_bias"])
        out["dgate"] = (e * n).reshape(case["groups"], -1, case["width"]).sum(dim=1).to(dtype)
    dn = e * _gate_rows(s)
    if case["post"] == "none":
        out["dh"] = dn.to(dtype)
        return out
    out["dpost_weight"] = (dn * hat).sum(dim=0)
    if s["post_bias"] is not None:
        out["dpost_bias"] = dn.sum(dim=0)
    out["dh"] = _norm_gradient(dn * s["post_weight"], hat, rstd, case["post"]).to(dtype)
    return out


def _activation(v, act):
    """The activation and its derivative."""
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-v))
        return v * s, s * (1.0 + v * (1.0 - s))
    c = 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5)))
    return v * c, c + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_ffn_forward(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    x = s["x"].float()
    g, u = x @ s["w_gate"].float().t(), x @ s["w_up"].float().t()
    y = (_activation(g, case["act"])[0] * u) @ s["w_down"].float().t()
    out = {"y": y.to(dtype)}
    if case["train"]:
        out.update(g=g.to(dtype), u=u.to(dtype))
    return out


def _plain_ffn_backward(s):
    dtype = DTYPES[s["case"]["dtype"]]
    x, g, u, dy = (s[k].float() for k in ("x", "g", "u", "dy"))
    a, da = _activation(g, s["case"]["act"])
    dh = dy @ s["w_down"].float()
    dg, du = dh * u * da, dh * a
    return {"dx": (dg @ s["w_gate"].float() + du @ s["w_up"].float()).to(dtype),
            "dw_gate": (dg.t() @ x).to(dtype), "dw_up": (du.t() @ x).to(dtype),
            "dw_down": (dy.t() @ (a * u)).to(dtype)}


# ------------------------------------------------------------------ the pass


def run(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    op = case["op"]
    if own:
        return _own(s)
    if op == "norm_forward":
        r, u, post_stats, pre_stats = _norm_forward(s)
        out = {"r": r.to(dtype), "u": u.to(dtype)}
        if case["train"]:
            out["pre_stats"] = pre_stats
            if post_stats is not None:
                out["post_stats"] = post_stats
        return out
    if op == "norm_backward":
        return _plain_norm_backward(s)
    if op == "dropout":
        return (s["x"].float() * _keep(case["rows"], case["width"], s["p"], s["seed"],
                                       s["offset"])).to(dtype)
    return _plain_ffn_forward(s) if op == "ffn_forward" else _plain_ffn_backward(s)


def _own(s):
    import paper_1712_02616_amd as iabn

    case = s["case"]
    op, rows, width = case["op"], case["rows"], case["width"]

    def vector(*shape):
        return torch.empty(shape, dtype=torch.float32, device="cuda")

    if op == "dropout":
        return iabn.iabn_dropout(s["x"], torch.empty_like(s["x"]), s["p"], s["seed"], s["offset"])
    if op == "ffn_forward":
        out = {"y": torch.empty_like(s["x"])}
        if case["train"]:
            out["g"] = torch.empty(rows, case["hidden"], dtype=s["x"].dtype, device="cuda")
            out["u"] = torch.empty_like(out["g"])
        iabn.iabn_ffn_forward(s["x"], s["w_gate"], s["w_up"], s["w_down"], out["y"], out.get("g"),
                              out.get("u"), act=case["act"])
        return out
    if op == "ffn_backward":
        out = {"dx": torch.empty_like(s["x"]), "dw_gate": torch.empty_like(s["w_gate"]),
               "dw_up": torch.empty_like(s["w_up"]), "dw_down": torch.empty_like(s["w_down"])}
        iabn.iabn_ffn_backward(s["dy"], s["x"], s["g"], s["u"], s["w_gate"], s["w_up"], s["w_down"],
                               out["dx"], torch.empty_like(s["g"]), torch.empty_like(s["u"]),
                               out["dw_gate"], out["dw_up"], out["dw_down"], act=case["act"])
        return out
    kinds = {"post_norm": case["post"], "pre_norm": case["pre"]}
    if op == "norm_forward":
        out = {"r": torch.empty_like(s["x"]), "u": torch.empty_like(s["x"])}
        if case["train"]:
            out["pre_stats"] = vector(2, rows)
            if case["post"] != "none":
                out["post_stats"] = vector(2, rows)
        iabn.iabn_resnorm_forward(
            s["x"], s["h"], out["r"], out["u"], gate=s["gate"], post_weight=s["post_weight"],
            post_bias=s["post_bias"], pre_weight=s["pre_weight"], pre_bias=s["pre_bias"],
            post_stats=out.get("post_stats"), pre_stats=out.get("pre_stats"), alpha=ALPHA, beta=BETA,
            eps=EPS, p=s["p"], seed=s["seed"], offset=s["offset"], **kinds)
        return out
    out = {"dpre_weight": vector(width)}
    if s["pre_bias"] is not None:
        out["dpre_bias"] = vector(width)
    out["dx"] = torch.empty_like(s["dr"])
    if s["gate"] is not None:
        out["dgate"] = torch.empty_like(s["gate"])
    if s["post_weight"] is not None:
        out["dpost_weight"] = vector(width)
    if s["post_bias"] is not None:
        out["dpost_bias"] = vector(width)
    out["dh"] = torch.empty_like(s["h"])
    iabn.iabn_resnorm_backward(
        s["dr"], s["du"], s["r"], s["h"], out["dx"], out["dh"], gate=s["gate"],
        post_weight=s["post_weight"], post_bias=s["post_bias"], pre_weight=s["pre_weight"],
        post_stats=s["post_stats"], pre_stats=s["pre_stats"], dgate=out.get("dgate"),
        dpost_weight=out.get("dpost_weight"), dpost_bias=out.get("dpost_bias"),
        dpre_weight=out["dpre_weight"], dpre_bias=out.get("dpre_bias"), alpha=ALPHA, beta=BETA,
        p=s["p"], seed=s["seed"], offset=s["offset"], **kinds)
    return out


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    b, rows, width = BYTES[case["dtype"]], case["rows"], case["width"]
    cells = rows * width
    if case["op"] == "dropout":
        # x in, y out; the generator's integer work per element counts as 12.
        return {"bytes": 2 * cells * b, "flops": 13 * cells}
    if case["op"].startswith("ffn"):
        hidden = case["hidden"]
        weights = 3 * width * hidden * b
        if case["op"] == "ffn_forward":
            kept = 2 * rows * hidden * b if case["train"] else 0
            return {"bytes": weights + 2 * cells * b + kept,
                    "flops": 6 * rows * width * hidden + 10 * rows * hidden}
        # x, dy, g, u and the weights in, dx and the weights' gradients out.
        return {"bytes": 2 * weights + 3 * cells * b + 2 * rows * hidden * b,
                "flops": 12 * rows * width * hidden + 20 * rows * hidden}
    vectors = 4 * width * ((case["post"] != "none") + (case["post"] == "layer") + 1 +
                           (case["pre"] == "layer")) + case["groups"] * width * b
    stats = 8 * rows * (1 + (case["post"] != "none"))
    if case["op"] == "norm_forward":
        # x and h in, r and u out.
        return {"bytes": 4 * cells * b + vectors + (stats if case["train"] else 0), "flops": 20 * cells}
    # dr, du, r and h in, dx and dh out, and the vectors' gradients.
    return {"bytes": 6 * cells * b + 2 * vectors + stats, "flops": 40 * cells}


# ------------------------------------------------------------------ the definition, in 64 bits


def _exact_keep(rows, width, p, seed, offset):
    """The dropout's factors from the generator's definition, on the host, in
    numpy's unsigned arithmetic."""
    cut = int(p * 65536 + 0.5)
    if cut == 0:
        return 1.0
    u64, mask = np.uint64, np.uint64(0xFFFFFFFF)
    groups = -(-width // 8)
    index = np.arange(rows * groups, dtype=u64)
    ctr = [index & mask, index >> u64(32),
           np.full(index.shape, offset & 0xFFFFFFFF, u64), np.full(index.shape, offset >> 32, u64)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for step in range(10):
        first, second = ctr[0] * u64(0xD2511F53), ctr[2] * u64(0xCD9E8D57)
        ctr = [(second >> u64(32)) ^ ctr[1] ^ u64((key[0] + step * 0x9E3779B9) & 0xFFFFFFFF),
               second & mask,
               (first >> u64(32)) ^ ctr[3] ^ u64((key[1] + step * 0xBB67AE85) & 0xFFFFFFFF),
               first & mask]
    words = np.stack([c.astype(np.uint32) for c in ctr], axis=1)
    lanes = words.view(np.uint16).reshape(rows, groups * 8)[:, :width]  # little endian: low half first
    keep = torch.from_numpy(np.ascontiguousarray(lanes >= cut)).to("cuda")
    return keep.double() / (1.0 - cut / 65536.0)


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    op, act = case["op"], case.get("act")

    if op == "dropout":
        return d["x"] * _exact_keep(case["rows"], case["width"], s["p"], s["seed"], s["offset"])

    if op.startswith("ffn"):
        def phi(v):
            return torch.sigmoid(v) if act == "silu" else torch.special.ndtr(v)

        if op == "ffn_forward":
            g, u = d["x"].matmul(d["w_gate"].T), d["x"].matmul(d["w_up"].T)
            y = (g * phi(g) * u).matmul(d["w_down"].T)
            return {"y": y, "g": g, "u": u} if case["train"] else {"y": y}
        g, u, c = d["g"], d["u"], phi(d["g"])
        slope = c + g * c * (1 - c) if act == "silu" else \
            c + g * torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)
        dh = d["dy"].matmul(d["w_down"])
        dg, du = dh * u * slope, dh * g * c
        return {"dx": dg.matmul(d["w_gate"]) + du.matmul(d["w_up"]),
                "dw_gate": dg.T.matmul(d["x"]), "dw_up": du.T.matmul(d["x"]),
                "dw_down": d["dy"].T.matmul(g * c * u)}

    keep = _exact_keep(case["rows"], case["width"], s["p"], s["seed"], s["offset"]) if s["p"] else 1.0
    per = case["rows"] // case["groups"] if case["groups"] else 1
    gate = d["gate"][torch.arange(case["rows"], device="cuda") // per] if case["groups"] else 1.0

    def scale_shift(v, stage):
        w, b = d[stage + "_weight"], d[stage + "_bias"]
        return v * (1.0 if w is None else w) + (0.0 if b is None else b)

    if op == "norm_forward":
        out = {}

        def stage_of(v, stage):
            if case[stage] == "none":
                return v
            mu = v.mean(1) if case[stage] == "layer" else torch.zeros_like(v[:, 0])
            inv = ((v - mu[:, None]).square().mean(1) + EPS).rsqrt()
            if case["train"]:
                out[stage + "_stats"] = torch.stack([mu, inv])
            return scale_shift((v - mu[:, None]) * inv[:, None], stage)

        n = stage_of(d["h"], "post")
        r = ALPHA * d["x"] + BETA * gate * keep * n
        u = stage_of(r, "pre")
        return {"r": r, "u": u, **{k: out[k] for k in ("pre_stats", "post_stats") if k in out}}

    def hat_of(v, stage):
        return (v - d[stage + "_stats"][0, :, None]) * d[stage + "_stats"][1, :, None]

    def back(dn, hat, stage):
        """Through scale and norm: the row's projections on 1 (layer) and on
        hat are taken out."""
        a = dn * d[stage + "_weight"]
        along = hat * (a * hat).mean(1, keepdim=True)
        a = a - along - (a.mean(1, keepdim=True) if case[stage] == "layer" else 0.0)
        return a * d[stage + "_stats"][1, :, None]

    rhat = hat_of(d["r"], "pre")
    g = d["dr"] + back(d["du"], rhat, "pre")
    hhat = d["h"] if case["post"] == "none" else hat_of(d["h"], "post")
    e = BETA * g * keep
    dn = e * gate
    out = {"dpre_weight": (d["du"] * rhat).sum(0)}
    if d["pre_bias"] is not None:
        out["dpre_bias"] = d["du"].sum(0)
    out["dx"] = ALPHA * g
    if case["groups"]:
        n = hhat if case["post"] == "none" else scale_shift(hhat, "post")
        out["dgate"] = (e * n).unflatten(0, (case["groups"], per)).sum(1)
    if case["post"] != "none":
        out["dpost_weight"] = (dn * hhat).sum(0)
        if d["post_bias"] is not None:
            out["dpost_bias"] = dn.sum(0)
    out["dh"] = dn if case["post"] == "none" else back(dn, hhat, "post")
    return out
