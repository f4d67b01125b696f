"""The work that a program training or serving a feed-forward sublayer of routed
experts has this library do, as measurable cases.

The sublayer: a router gives every token the `top` of `experts` gated
feed-forward blocks, whose outputs are added up with the router's weights; a
training step ends by clipping all gradients to a global norm.

- route_forward:    logits [rows, experts] -> experts and weights [rows, top]
- route_backward:   the logits' gradient from the weights'
- experts_forward:  y_t = sum over slots of w (act(x Wg_e^T) * (x Wu_e^T)) Wd_e^T,
                    with the sorting of the tokens by expert
- experts_backward: its gradients from dy
- clip:             the norm over a list of gradients, and the clipped ones
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
INF = float("inf")


def _route(name, direction, dtype, rows, experts, top, score, bias, groups, groups_kept, group_top,
           renormalise, scale, masked=0):
    """bias: added to the scores for the choice alone.  groups: the experts'
    groups, of which each token keeps groups_kept, by the sum of their group_top
    highest.  masked: experts that are switched off (logits of -inf)."""
    return {"name": name, "op": "route_" + direction, "dtype": dtype, "rows": rows, "experts": experts,
            "top": top, "score": score, "bias": bias, "groups": groups, "groups_kept": groups_kept,
            "group_top": group_top, "renormalise": renormalise, "scale": scale, "masked": masked}


def _experts(name, direction, dtype, rows, experts, top, width, hidden, act, skew, train=True):
    """skew: how far apart the experts' popularity is (the deviation of their
    mean logits).  train: the forward gives the projections too."""
    return {"name": name, "op": "experts_" + direction, "dtype": dtype, "rows": rows, "experts": experts,
            "top": top, "width": width, "hidden": hidden, "act": act, "skew": skew, "train": train}


def _clip(name, dtype, layers, width, hidden, max_norm):
    """The gradients of `layers` gated blocks and their norms' fp32 weights."""
    return {"name": name, "op": "clip", "dtype": dtype, "layers": layers, "width": width, "hidden": hidden,
            "max_norm": max_norm}


def listed():
    return [
        # Serving: the next token of one sequence; the cost of a call.
        _route("route_token_bf16", "forward", "bf16", 1, 64, 8, "softmax", False, 1, 1, 1, True, 1.0),
        # Training with balancing biases and groups of experts.
        _route("route_forward_bf16", "forward", "bf16", 16384, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.0),
        # A prime number of tokens, odd numbers of experts and choices, one expert switched off.
        _route("route_odd_f32", "forward", "f32", 4099, 61, 5, "softmax", False, 1, 1, 1, False, 1.0, 1),
        # The router's backward: softmax scores that are not renormalised reach every logit.
        _route("route_backward_bf16", "backward", "bf16", 16384, 256, 8, "softmax", False, 1, 1, 1, False, 1.0),
        # Serving: the next token of one sequence; the chosen experts' weights are read once.
        _experts("experts_token_bf16", "forward", "bf16", 1, 64, 8, 2048, 1024, "silu", 0.5, train=False),
        # Serving: the next tokens of a batch of sequences; almost every expert has some.
        _experts("experts_batch_f16", "forward", "f16", 24, 32, 4, 2048, 1200, "silu", 0.5, train=False),
        # A prompt of odd length through few experts of odd sizes.
        _experts("experts_odd_f32", "forward", "f32", 333, 7, 2, 1000, 731, "gelu", 0.5, train=False),
        # Training's forward: many small experts.
        _experts("experts_forward_bf16", "forward", "bf16", 4096, 64, 8, 2048, 1024, "silu", 0.5),
        # Training's backward: a ragged number of tokens, few large experts.
        _experts("experts_backward_f16", "backward", "f16", 2085, 8, 2, 1024, 4096, "gelu", 0.3),
        # The largest: the backward of many small experts.
        _experts("experts_backward_bf16", "backward", "bf16", 8192, 64, 8, 2048, 1024, "silu", 0.5),
        # A small model's gradients: the cost of the calls.
        _clip("clip_small_f32", "f32", 4, 64, 256, 1.0),
        # A stack of eight blocks, (2048, 8192): 403 million gradients.
        _clip("clip_bf16", "bf16", 8, 2048, 8192, 1.0),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["route_forward", "route_backward", "experts_forward", "experts_forward",
                       "experts_backward", "clip"])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    if kind == "clip":
        width, hidden = _spread(rng, 32, 4096), _spread(rng, 64, 8192)
        layers = min(_spread(rng, 1, 24), max(1, (1 << 28) // (3 * width * hidden)))
        return _drop_name(_clip("", dtype, layers, width, hidden, rng.choice([1.0, 1.0, 1e6])))
    if kind.startswith("route"):
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = _spread(rng, 2, 512 // groups) * groups
        kept = rng.randint(1, groups)
        group_top = rng.choice([1, 2])
        top = _spread(rng, 1, min(16, experts // groups * kept))
        masked = rng.choice([0, 0, 1]) if groups == 1 and experts > top else 0
        rows = _spread(rng, 1, min(65536, (1 << 22) // experts))
        return _drop_name(_route("", kind[6:], dtype, rows, experts, top, rng.choice(["softmax", "sigmoid"]),
                                 rng.random() < 0.5, groups, kept, group_top, rng.random() < 0.5,
                                 rng.choice([1.0, 2.0]), masked))
    experts = _spread(rng, 2, 128)
    top = _spread(rng, 1, min(8, experts))
    width, hidden = _spread(rng, 256, 4096), _spread(rng, 256, 4096)
    while experts * width * hidden > 1 << 27:
        width, hidden = width * 3 // 4, hidden * 3 // 4
    if rng.random() < 0.75:  # most blocks' sizes are whole numbers of 16-byte accesses
        width, hidden = (width + 7) // 8 * 8, (hidden + 7) // 8 * 8
    most = (1 << 34 if dtype == "f32" else 1 << 37) // (top * width * hidden)
    rows = _spread(rng, 1, max(1, min(8192, most)))
    train = kind == "experts_backward" or rng.random() < 0.5
    return _drop_name(_experts("", kind[8:], dtype, rows, experts, top, width, hidden,
                               rng.choice(["silu", "gelu"]), rng.choice([0.0, 0.5, 1.5]), train))


def _drop_name(case):
    return {k: v for k, v in case.items() if k != "name"}


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 6361 + 29)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, to=dtype):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(to)

    state = {"case": case}
    if case["op"] == "clip":
        width, hidden = case["width"], case["hidden"]
        state["grads"] = []
        for _ in range(case["layers"]):
            state["grads"] += [normal(hidden, width, std=0.01), normal(hidden, width, std=0.01),
                               normal(width, hidden, std=0.01), normal(width, std=0.1, to=torch.float32),
                               normal(width, std=0.1, to=torch.float32)]
        # The clipped gradients' place, which a program keeps.
        state["outs"] = [torch.empty_like(g) for g in state["grads"]]
        return state

    rows, experts, top = case["rows"], case["experts"], case["top"]
    if case["op"].startswith("route"):
        # Experts differ in popularity.
        popular = normal(experts, std=0.5, to=torch.float32)
        logits = normal(rows, experts, std=1.5, to=torch.float32) + popular
        if case["masked"]:
            off = torch.randperm(experts, generator=gen, device="cuda")[:case["masked"]]
            logits[:, off] = -INF
        state["logits"] = logits.to(dtype)
        state["bias"] = normal(experts, std=0.05, to=torch.float32) if case["bias"] else None
        if case["op"] == "route_backward":
            state["chosen"] = _choose(state)[0].int()
            state["dweights"] = normal(rows, top, std=0.1, to=torch.float32)
        return state

    width, hidden = case["width"], case["hidden"]
    logits = normal(rows, experts, to=torch.float32) + normal(experts, std=case["skew"], to=torch.float32)
    noise = torch.rand(rows, experts, generator=gen, device="cuda").clamp_min(1e-9)
    state["chosen"] = torch.topk(logits - torch.log(-torch.log(noise)), top, dim=1).indices.int()
    weights = torch.exp(torch.gather(logits, 1, state["chosen"].long()))
    state["weights"] = weights / weights.sum(dim=1, keepdim=True)
    state["x"] = normal(rows, width)
    state["w_gate"] = normal(experts, hidden, width, std=1.0 / math.sqrt(width))
    state["w_up"] = normal(experts, hidden, width, std=1.0 / math.sqrt(width))
    state["w_down"] = normal(experts, width, hidden, std=1.0 / math.sqrt(hidden))
    # (Where each expert's rows end, on the host, as the loop of the plain form needs it.)
    state["counts"] = torch.bincount(state["chosen"].flatten().long(), minlength=experts).tolist()
    if case["op"] == "experts_backward":
        # What the forward kept, sorted by expert, and the gradient that arrives.
        state["g"] = torch.empty(rows * top, hidden, dtype=dtype, device="cuda")
        state["u"] = torch.empty_like(state["g"])
        for e, at, pairs in _by_expert(state):
            x = state["x"][pairs // top].float()
            state["g"][at] = (x @ state["w_gate"][e].float().t()).to(dtype)
            state["u"][at] = (x @ state["w_up"][e].float().t()).to(dtype)
        state["dy"] = normal(rows, width, std=0.1)
        if own:
            import paper_1712_02616_amd as iabn

            # The plan that the forward made.
            state["plan"] = torch.empty(iabn.iabn_experts_plan_size(rows, top, experts), dtype=torch.int32,
                                        device="cuda")
            iabn.iabn_experts_plan(state["chosen"], state["plan"], experts)
    return state


# ------------------------------------------------------------------ plain forms


def _choose(s):
    """The chosen experts and all scores, in 64 bits: scores next to each other
    decide which expert a token goes to."""
    case = s["case"]
    logits = s["logits"].double()
    if case["score"] == "softmax":
        scores = torch.exp(logits - logits.amax(dim=1, keepdim=True))
        scores = scores / scores.sum(dim=1, keepdim=True)
    else:
        scores = 1.0 / (1.0 + torch.exp(-logits))
    # Without a bias, the order of the scores is that of the logits.
    choice = scores + s["bias"].double() if s["bias"] is not None else logits
    choice = torch.where(logits == -INF, logits, choice)
    if case["groups_kept"] < case["groups"]:
        by_group = (scores if s["bias"] is None else choice).unflatten(1, (case["groups"], -1))
        per = by_group.shape[2]
        group = torch.sort(by_group, dim=2, descending=True).values[:, :, :min(case["group_top"], per)].sum(dim=2)
        best = torch.sort(group, dim=1, descending=True, stable=True).indices[:, :case["groups_kept"]]
        kept = torch.zeros_like(group, dtype=torch.bool).scatter_(1, best, True)
        choice = torch.where(kept.repeat_interleave(per, dim=1), choice, torch.full_like(choice, -INF))
    # (A stable sort: the lower index of two equal ones comes first.)
    chosen = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :case["top"]]
    return chosen, scores


def _plain_route_forward(s):
    case = s["case"]
    chosen, scores = _choose(s)
    weights = torch.gather(scores, 1, chosen)
    if case["renormalise"]:
        weights = weights / weights.sum(dim=1, keepdim=True)
    return {"experts": chosen.int(), "weights": (case["scale"] * weights).float()}


def _plain_route_backward(s):
    case = s["case"]
    logits, chosen, d = s["logits"].float(), s["chosen"].long(), case["scale"] * s["dweights"]
    if case["score"] == "softmax":
        scores = torch.exp(logits - logits.amax(dim=1, keepdim=True))
        scores = scores / scores.sum(dim=1, keepdim=True)
    else:
        scores = 1.0 / (1.0 + torch.exp(-logits))
    picked = torch.gather(scores, 1, chosen)
    if case["renormalise"]:
        total = picked.sum(dim=1, keepdim=True)
        d = (d - (d * picked).sum(dim=1, keepdim=True) / total) / total
    dscores = torch.zeros_like(scores).scatter_(1, chosen, d)
    if case["score"] == "softmax":
        dlogits = scores * (dscores - (scores * dscores).sum(dim=1, keepdim=True))
    else:
        dlogits = dscores * scores * (1.0 - scores)
    return {"dlogits": dlogits.to(s["logits"].dtype)}


def _by_expert(s):
    """For each expert that has any: its number, the span of its rows among the
    sorted pairs, and the pairs (token * top + slot) themselves."""
    pairs = torch.sort(s["chosen"].flatten(), stable=True).indices
    start = 0
    for e, n in enumerate(s["counts"]):
        if n:
            yield e, slice(start, start + n), pairs[start:start + n]
        start += n


def _activation(v, act):
    """The activation and its derivative."""
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-v))
        return v * s, s * (1.0 + v * (1.0 - s))
    c = 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5)))
    return v * c, c + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_experts_forward(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    rows, top = case["rows"], case["top"]
    slots = torch.empty(rows * top, case["width"], device="cuda")
    out = {}
    if case["train"]:
        out["g"] = torch.empty(rows * top, case["hidden"], dtype=dtype, device="cuda")
        out["u"] = torch.empty_like(out["g"])
    weights = s["weights"].flatten()
    for e, at, pairs in _by_expert(s):
        x = s["x"][pairs // top].float()
        g, u = x @ s["w_gate"][e].float().t(), x @ s["w_up"][e].float().t()
        if case["train"]:
            out["g"][at], out["u"][at] = g.to(dtype), u.to(dtype)
        h = _activation(g, case["act"])[0] * u
        slots[pairs] = weights[pairs, None] * (h @ s["w_down"][e].float().t())
    out["y"] = slots.unflatten(0, (rows, top)).sum(dim=1).to(dtype)
    return out


def _plain_experts_backward(s):
    case, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    rows, top = case["rows"], case["top"]
    slots = torch.empty(rows * top, case["width"], device="cuda")
    dweights = torch.empty(rows * top, device="cuda")
    # (An expert without tokens has a gradient of zeros.)
    out = {"dw_gate": torch.zeros_like(s["w_gate"]), "dw_up": torch.zeros_like(s["w_up"]),
           "dw_down": torch.zeros_like(s["w_down"])}
    weights = s["weights"].flatten()
    for e, at, pairs in _by_expert(s):
        x, dy = s["x"][pairs // top].float(), s["dy"][pairs // top].float()
        g, u, w = s["g"][at].float(), s["u"][at].float(), weights[pairs, None]
        a, da = _activation(g, case["act"])
        dh = dy @ s["w_down"][e].float()
        dweights[pairs] = (dh * (a * u)).sum(dim=1)
        dg, du = w * dh * u * da, w * dh * a
        slots[pairs] = dg @ s["w_gate"][e].float() + du @ s["w_up"][e].float()
        out["dw_gate"][e], out["dw_up"][e] = (dg.t() @ x).to(dtype), (du.t() @ x).to(dtype)
        out["dw_down"][e] = (dy.t() @ (w * a * u)).to(dtype)
    out["dx"] = slots.unflatten(0, (rows, top)).sum(dim=1).to(dtype)
    out["dweights"] = dweights.unflatten(0, (rows, top))
    return out


def _plain_clip(s):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["grads"]:
        v = g.float()
        total = total + (v * v).sum(dtype=torch.float64)
    norm = torch.sqrt(total)
    factor = (s["case"]["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
    return {"norm": norm.float(), "outs": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


# ------------------------------------------------------------------ the pass


def run(s):
    if own:
        return _own(s)
    return {"route_forward": _plain_route_forward, "route_backward": _plain_route_backward,
            "experts_forward": _plain_experts_forward, "experts_backward": _plain_experts_backward,
            "clip": _plain_clip}[s["case"]["op"]](s)


def _own(s):
    import paper_1712_02616_amd as iabn

    case = s["case"]
    op = case["op"]
    if op == "clip":
        norm = torch.empty((), device="cuda")
        iabn.iabn_grad_norm(s["grads"], norm)
        iabn.iabn_grad_clip(s["grads"], s["outs"], norm, case["max_norm"])
        return {"norm": norm, "outs": s["outs"]}
    rows, experts, top = case["rows"], case["experts"], case["top"]
    if op == "route_forward":
        out = {"experts": torch.empty(rows, top, dtype=torch.int32, device="cuda"),
               "weights": torch.empty(rows, top, device="cuda")}
        iabn.iabn_route_forward(s["logits"], out["experts"], out["weights"], bias=s["bias"], score=case["score"],
                                groups=case["groups"], groups_kept=case["groups_kept"],
                                group_top=case["group_top"], renormalise=case["renormalise"],
                                scale=case["scale"])
        return out
    if op == "route_backward":
        out = {"dlogits": torch.empty_like(s["logits"])}
        iabn.iabn_route_backward(s["dweights"], s["logits"], s["chosen"], out["dlogits"], score=case["score"],
                                 renormalise=case["renormalise"], scale=case["scale"])
        return out
    if op == "experts_forward":
        plan = torch.empty(iabn.iabn_experts_plan_size(rows, top, experts), dtype=torch.int32, device="cuda")
        iabn.iabn_experts_plan(s["chosen"], plan, experts)
        out = {}
        if case["train"]:
            out["g"] = torch.empty(rows * top, case["hidden"], dtype=s["x"].dtype, device="cuda")
            out["u"] = torch.empty_like(out["g"])
        out["y"] = torch.empty_like(s["x"])
        iabn.iabn_experts_forward(s["x"], plan, s["weights"], s["w_gate"], s["w_up"], s["w_down"], out["y"],
                                  out.get("g"), out.get("u"), act=case["act"])
        return out
    out = {k: torch.empty_like(s["w" + k[2:]]) for k in ("dw_gate", "dw_up", "dw_down")}
    out["dx"], out["dweights"] = torch.empty_like(s["x"]), torch.empty_like(s["weights"])
    iabn.iabn_experts_backward(s["dy"], s["x"], s["plan"], s["weights"], s["g"], s["u"], s["w_gate"], s["w_up"],
                               s["w_down"], out["dx"], out["dweights"], torch.empty_like(s["g"]),
                               torch.empty_like(s["u"]), out["dw_gate"], out["dw_up"], out["dw_down"],
                               act=case["act"])
    return out


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    b = BYTES[case["dtype"]]
    if case["op"] == "clip":
        matrices = 3 * case["layers"] * case["width"] * case["hidden"]
        vectors = 2 * case["layers"] * case["width"]
        # The norm has to be known before the first product: in twice, out once; of
        # "each input once, each output once" that is 2 of 3.
        return {"bytes": 2 * (matrices * b + vectors * 4), "flops": 3 * (matrices + vectors)}
    rows, experts, top = case["rows"], case["experts"], case["top"]
    if case["op"].startswith("route"):
        cells = rows * experts
        if case["op"] == "route_forward":
            # Logits in, an index and a weight per slot out; a score per logit (15)
            # and a comparison per logit and slot.
            return {"bytes": cells * b + 8 * rows * top + (4 * experts if case["bias"] else 0),
                    "flops": cells * (15 + top)}
        return {"bytes": 2 * cells * b + 8 * rows * top, "flops": 20 * cells}
    width, hidden, pairs = case["width"], case["hidden"], rows * top
    # Experts that have a token, were all alike.
    busy = experts * (1.0 - (1.0 - top / experts) ** rows)
    weights = int(3 * busy * width * hidden * b)
    if case["op"] == "experts_forward":
        kept = 2 * pairs * hidden * b if case["train"] else 0
        return {"bytes": weights + 2 * rows * width * b + 8 * pairs + kept,
                "flops": 6 * pairs * width * hidden + 10 * pairs * hidden + 2 * pairs * width}
    return {"bytes": weights + 3 * experts * width * hidden * b + 3 * rows * width * b + 12 * pairs +
            2 * pairs * hidden * b,
            "flops": 12 * pairs * width * hidden + 24 * pairs * hidden + pairs * width}


# ------------------------------------------------------------------ the definition, in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "clip":
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in s["grads"]))
        ratio = min(1.0, case["max_norm"] / (norm + 1e-6))
        return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"),
                "outs": [g.double() * ratio for g in s["grads"]]}
    rows, experts, top = case["rows"], case["experts"], case["top"]
    if op.startswith("route"):
        l = s["logits"].double()
        p = torch.softmax(l, dim=1) if case["score"] == "softmax" else torch.sigmoid(l)
        if op == "route_forward":
            # One choice after the other: the highest, of equal ones the first.
            index = torch.arange(experts, device="cuda")
            c = l.clone() if s["bias"] is None else p + s["bias"].double()
            c[l == -INF] = -INF

            def first_of_highest(v):
                at = torch.arange(v.shape[1], device="cuda").expand_as(v)
                high = v == v.max(dim=1, keepdim=True).values
                return torch.where(high, at, v.shape[1]).min(dim=1).values

            if case["groups_kept"] < case["groups"]:
                per = experts // case["groups"]
                of = (p if s["bias"] is None else c).reshape(rows, case["groups"], per)
                sums = torch.topk(of, min(case["group_top"], per), dim=2).values.sum(dim=2)
                allowed = torch.zeros(rows, experts, dtype=torch.bool, device="cuda")
                for _ in range(case["groups_kept"]):
                    best = first_of_highest(sums)
                    allowed |= (index // per)[None] == best[:, None]
                    sums[torch.arange(rows, device="cuda"), best] = -INF
                c[~allowed] = -INF
            picks = []
            for _ in range(top):
                picks.append(first_of_highest(c))
                c[torch.arange(rows, device="cuda"), picks[-1]] = -INF
            chosen = torch.stack(picks, dim=1)
            w = p.gather(1, chosen)
            if case["renormalise"]:
                w = w / w.sum(1, keepdim=True)
            return {"experts": chosen.int(), "weights": case["scale"] * w}
        # The scores' Jacobian row by row: d log(w_j) = d log(p_j) - sum_i q_i d log(p_i).
        chosen = s["chosen"].long()
        w = p.gather(1, chosen)
        if case["renormalise"]:
            w = w / w.sum(1, keepdim=True)
        dlog = case["scale"] * w * s["dweights"].double()
        if case["renormalise"]:
            dlog = dlog - w * dlog.sum(1, keepdim=True)
        spread = torch.zeros_like(p).scatter_add_(1, chosen, dlog)
        if case["score"] == "softmax":
            return {"dlogits": spread - p * dlog.sum(1, keepdim=True)}
        return {"dlogits": spread * torch.sigmoid(-l)}

    def phi(v):
        return torch.sigmoid(v) if case["act"] == "silu" else torch.special.ndtr(v)

    hidden, width = case["hidden"], case["width"]
    token = torch.arange(rows, device="cuda").repeat_interleave(top)
    flat, weight = s["chosen"].flatten().long(), s["weights"].flatten().double()
    sorted_from = 0
    if op == "experts_forward":
        terms = torch.zeros(rows * top, width, dtype=torch.float64, device="cuda")
        kept = [torch.zeros(rows * top, hidden, dtype=torch.float64, device="cuda") for _ in range(2)] \
            if case["train"] else None
        for e in range(experts):
            mine = (flat == e).nonzero()[:, 0]
            x = s["x"][token[mine]].double()
            g, u = x.matmul(s["w_gate"][e].double().T), x.matmul(s["w_up"][e].double().T)
            if kept:
                for t, v in zip(kept, (g, u)):
                    t[sorted_from:sorted_from + len(mine)] = v
            sorted_from += len(mine)
            terms[mine] = weight[mine, None] * (g * phi(g) * u).matmul(s["w_down"][e].double().T)
        y = terms.reshape(rows, top, width).sum(1)
        return {"g": kept[0], "u": kept[1], "y": y} if kept else {"y": y}
    terms = torch.zeros(rows * top, width, dtype=torch.float64, device="cuda")
    dweights = torch.zeros(rows * top, dtype=torch.float64, device="cuda")
    out = {k: torch.zeros(s["w" + k[2:]].shape, dtype=torch.float64, device="cuda")
           for k in ("dw_gate", "dw_up", "dw_down")}
    for e in range(experts):
        mine = (flat == e).nonzero()[:, 0]
        span = slice(sorted_from, sorted_from + len(mine))
        sorted_from += len(mine)
        if not len(mine):
            continue
        x, dy, w = s["x"][token[mine]].double(), s["dy"][token[mine]].double(), weight[mine, None]
        g, u = s["g"][span].double(), s["u"][span].double()
        c = phi(g)
        slope = c + g * c * (1 - c) if case["act"] == "silu" else \
            c + g * torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)
        back = dy.matmul(s["w_down"][e].double())
        dweights[mine] = (back * g * c * u).sum(1)
        dg, du = w * back * u * slope, w * back * g * c
        terms[mine] = dg.matmul(s["w_gate"][e].double()) + du.matmul(s["w_up"][e].double())
        out["dw_gate"][e], out["dw_up"][e] = dg.T.matmul(x), du.T.matmul(x)
        out["dw_down"][e] = dy.T.matmul(w * g * c * u)
    out["dx"] = terms.reshape(rows, top, width).sum(1)
    out["dweights"] = dweights.reshape(rows, top)
    return out
