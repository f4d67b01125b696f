"""The plan and the routed experts on the GPU against their definition in 64 bits;
both sides take the same stored values, and bounds count every rounding."""

from __future__ import annotations

import math

import pytest
import torch

import paper_1712_02616_amd as iabn
import routed_oracle as routed
import sublayer_oracle as oracle
from gpu_helpers import TORCH_DTYPES, say
from test_gpu_resnorm import guarded, placed

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

NAN = float("nan")


def make_plan(experts, E, stream=None):
    M, k = experts.shape
    plan = torch.full((iabn.iabn_experts_plan_size(M, k, E) + 8,), -99, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    iabn.iabn_experts_plan(experts.int().cuda(), plan[:-8], E, stream=stream)
    torch.cuda.synchronize()
    assert (plan[-8:] == -99).all()
    return plan[:-8]


def check_plan(experts, E):
    offsets, order, place = routed.plan(experts, E)
    plan = make_plan(experts, E).tolist()
    P = experts.numel()
    assert plan[:E + 1] == offsets
    assert plan[E + 1:E + 1 + len(order)] == order
    assert all(v == -99 for v in plan[E + 1 + len(order):E + 1 + P])  # left as it was
    assert plan[E + 1 + P:E + 1 + 2 * P] == place
    sizes = [offsets[e + 1] - offsets[e] for e in range(E)]
    by_size = sorted(range(E), key=lambda e: (-sizes[e], e)) if P > 2048 else list(range(E))
    assert plan[E + 1 + 2 * P:2 * E + 1 + 2 * P] == by_size


@pytest.mark.parametrize("M,k,E", [(1, 1, 1), (1, 8, 64), (3, 2, 5), (100, 3, 7), (255, 8, 64), (256, 8, 64), (257, 8, 64),
                                   (513, 4, 1024), (5000, 2, 8), (3001, 7, 100), (70000, 8, 33), (90001, 1, 1000)])
def test_plan(M, k, E):
    gen = torch.Generator().manual_seed(M + E)
    check_plan(torch.randint(0, E, (M, k), generator=gen), E)


@pytest.mark.parametrize("M", [1, 40, 700, 6000])
def test_plan_leaves_out(M):
    """Pairs without an expert, numbers that are no expert's, one expert for all."""
    gen = torch.Generator().manual_seed(M)
    e = torch.randint(-2, 11, (M, 5), generator=gen)
    e[0, 0], e[-1, -1] = 1 << 30, -(1 << 31)
    check_plan(e, 9)
    check_plan(torch.full((M, 5), -1), 9)
    check_plan(torch.full((M, 5), 8), 9)


def test_plan_of_nothing():
    check_plan(torch.zeros(0, 3, dtype=torch.long), 4)
    check_plan(torch.zeros(6, 0, dtype=torch.long), 4)


def inputs(M, k, E, C, F, dtype, seed=5, choice="random"):
    gen = torch.Generator().manual_seed(seed + M)
    d = TORCH_DTYPES[dtype]
    new = lambda *s, std: (torch.randn(*s, generator=gen) * std).to(d)  # noqa: E731
    i = {"x": new(M, C, std=1.0), "w_gate": new(E, F, C, std=1 / math.sqrt(C)),
         "w_up": new(E, F, C, std=1 / math.sqrt(C)), "w_down": new(E, C, F, std=1 / math.sqrt(F)),
         "dy": new(M, C, std=0.3)}
    if choice == "random":  # distinct, of different popularity
        noise = torch.rand(M, E, generator=gen) + 0.3 * torch.rand(E, generator=gen)
        experts = noise.argsort(1)[:, :k] if k <= E else torch.randint(0, E, (M, k), generator=gen)
    elif choice == "holes":  # some left out, some tokens without any, some twice
        experts = torch.randint(-1, E, (M, k), generator=gen)
        experts[::3] = -1
    else:
        experts = torch.full((M, k), int(choice))
    weights = torch.rand(M, k, generator=gen)
    return i, experts, weights


def run_case(M, k, E, C, F, dtype, act="silu", slope=0.1, shift=0, in_place=False, train=True, choice="random",
             stream=None):
    say("experts M=%d k=%d E=%d C=%d F=%d %s %s shift=%d %s" % (M, k, E, C, F, dtype, act, shift, choice))
    d = TORCH_DTYPES[dtype]
    i, experts, weights = inputs(M, k, E, C, F, dtype, choice=choice)
    f = {n: v.double() for n, v in i.items()}
    dev = {n: placed(v.reshape(-1, v.shape[-1]), shift).view(v.shape) for n, v in i.items()}
    sorted_plan = routed.plan(experts, E)
    rows = sorted_plan[0][-1]
    plan, w = make_plan(experts, E), weights.cuda()
    checks = []

    def out(name, *shape, dtype=d):
        t, intact = guarded((math.prod(shape[:-1]), shape[-1]), dtype, shift)
        checks.append((name, intact))
        return t.view(shape)

    y = out("y", M, C)
    g, u = (out("g", M * k, F), out("u", M * k, F)) if train else (None, None)
    before = [t[rows:].clone() for t in (g, u)] if train else []
    torch.cuda.synchronize()
    assert iabn.iabn_experts_forward(dev["x"], plan, w, dev["w_gate"], dev["w_up"], dev["w_down"], y, g, u, act=act,
                                     slope=slope, stream=stream) is y
    torch.cuda.synchronize()
    want = routed.experts_forward(f["x"], weights.double(), f["w_gate"], f["w_up"], f["w_down"], sorted_plan, k, d,
                                  act, slope)
    oracle.check("y", y, *want["y"], d)
    if train:
        for name, t, kept in zip("gu", (g, u), before):
            oracle.check(name, t[:rows], *want[name], d)
            assert torch.equal(t[rows:].view(torch.uint8), kept.view(torch.uint8))  # left as they were
        want = routed.experts_backward(f["dy"], f["x"], weights.double(), g.cpu().double()[:rows],
                                       u.cpu().double()[:rows], f["w_gate"], f["w_up"], f["w_down"], sorted_plan, k,
                                       d, act, slope)
        outs = {"dx": out("dx", M, C), "dw_gate": out("dw_gate", E, F, C), "dw_up": out("dw_up", E, F, C),
                "dw_down": out("dw_down", E, C, F)}
        dweights = torch.full((M, k), NAN, device="cuda")
        dg, du = (g, u) if in_place else (out("dg", M * k, F), out("du", M * k, F))
        before = [t[rows:].clone() for t in (dg, du)]
        torch.cuda.synchronize()
        iabn.iabn_experts_backward(dev["dy"], dev["x"], plan, w, g, u, dev["w_gate"], dev["w_up"], dev["w_down"],
                                   outs["dx"], dweights, dg, du, outs["dw_gate"], outs["dw_up"], outs["dw_down"],
                                   act=act, slope=slope, stream=stream)
        torch.cuda.synchronize()
        for name in outs:
            oracle.check(name, outs[name], *want[name], d)
        oracle.check("dweights", dweights.flatten(), *want["dweights"], torch.float32)
        for name, t, kept in zip(("dg", "du"), (dg, du), before):
            v, err = want[name]
            off = (t[:rows].cpu().double() - v).abs() - err  # (stored from what the bound holds already)
            assert rows == 0 or float(off.max()) <= 0, "%s is off by %g more than its bound" % (name, float(off.max()))
            assert torch.equal(t[rows:].view(torch.uint8), kept.view(torch.uint8))
    for name, intact in checks:
        intact(name)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,k,E,C,F", [(1, 1, 1, 1, 1), (1, 2, 4, 64, 128), (2, 1, 3, 8, 24), (5, 3, 3, 7, 5),
                                       (24, 4, 16, 128, 64), (64, 2, 5, 96, 136), (65, 2, 5, 96, 136),
                                       (100, 3, 7, 72, 88), (130, 4, 6, 129, 33), (300, 2, 2, 64, 260),
                                       (200, 8, 40, 40, 56)])
def test_shapes(M, k, E, C, F, dtype):
    run_case(M, k, E, C, F, dtype)


@pytest.mark.parametrize("act", ["silu", "gelu", "leaky"])
@pytest.mark.parametrize("M", [4, 150])
def test_activations(act, M):
    run_case(M, 2, 4, 72, 104, "f32", act=act)
    run_case(M, 2, 4, 72, 104, "f16", act=act, slope=0.0)


@pytest.mark.parametrize("dtype,shift", [("f32", 1), ("f16", 1), ("bf16", 3), ("f16", 4)])
@pytest.mark.parametrize("M", [1, 9, 140])
def test_alignment(dtype, shift, M):
    run_case(M, 2, 3, 136, 200, dtype, shift=shift)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M", [1, 30, 300])
def test_inference_and_in_place(M, dtype):
    run_case(M, 2, 4, 160, 96, dtype, train=False)
    run_case(M, 2, 4, 160, 96, dtype, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [3, 50, 200])
@pytest.mark.parametrize("choice", ["holes", "-1", "0", "5"])
def test_choices(M, choice, dtype):
    """Pairs left out, tokens and experts without any, all pairs with one expert
    (which a token then has twice)."""
    run_case(M, 3, 6, 80, 72, dtype, choice=choice)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,k,E,C,F", [(600, 2, 3, 512, 264), (1000, 1, 2, 264, 520), (2500, 2, 4, 300, 200),
                                       (901, 2, 2, 301, 201), (300, 4, 1, 256, 256)])
def test_long_groups(M, k, E, C, F, dtype):
    """Several tiles of an expert's rows, and long sums over them."""
    run_case(M, k, E, C, F, dtype)


def test_more_choices_than_experts():
    run_case(20, 5, 2, 40, 48, "f16")
    run_case(90, 64, 3, 40, 48, "bf16")


def test_another_stream():
    st = torch.cuda.Stream()
    run_case(100, 2, 4, 96, 128, "bf16", stream=st)
    run_case(5, 2, 4, 96, 128, "f32", stream=st.cuda_stream)


def test_many_experts():
    run_case(40, 4, 1024, 24, 16, "f16")
    run_case(300, 6, 777, 17, 24, "f32")


def test_empty():
    d = torch.float16
    new = lambda *s: torch.full(s, 3.0, dtype=d, device="cuda")  # noqa: E731
    E, F, C = 3, 24, 16
    w, wd = new(E, F, C), new(E, C, F)
    none = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    plan = make_plan(none, E)
    weights = torch.zeros(0, 2, device="cuda")
    iabn.iabn_experts_forward(new(0, C), plan, weights, w, w, wd, new(0, C), new(0, F), new(0, F))
    dws = [new(E, F, C), new(E, F, C), new(E, C, F)]
    iabn.iabn_experts_backward(new(0, C), new(0, C), plan, weights, new(0, F), new(0, F), w, w, wd, new(0, C),
                               weights, new(0, F), new(0, F), *dws)
    assert all((t == 0).all() for t in dws)
    chosen = torch.zeros(5, 2, dtype=torch.int32, device="cuda")
    plan, weights, y, dw = make_plan(chosen, E), torch.ones(5, 2, device="cuda"), new(5, C), torch.ones(5, 2, device="cuda")
    iabn.iabn_experts_forward(new(5, C), plan, weights, new(E, 0, C), new(E, 0, C), new(E, C, 0), y)
    assert (y == 0).all()
    dx, z = new(5, C), new(10, 0)
    iabn.iabn_experts_backward(new(5, C), new(5, C), plan, weights, z, z, new(E, 0, C), new(E, 0, C), new(E, C, 0), dx, dw,
                               z, z, new(E, 0, C), new(E, 0, C), new(E, C, 0))
    assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("M", [6, 200])
def test_a_bad_token_stays_in_its_rows(M):
    i, experts, weights = inputs(M, 2, 5, 100, 64, "bf16")
    dev = {n: v.cuda() for n, v in i.items()}
    plan, w = make_plan(experts, 5), weights.cuda()
    ys = []
    for bad in (False, True):
        if bad:
            dev["x"][1, 7] = NAN
        y = torch.empty_like(dev["x"])
        ys.append(iabn.iabn_experts_forward(dev["x"], plan, w, dev["w_gate"], dev["w_up"], dev["w_down"], y))
    rows = [r for r in range(M) if r != 1]
    assert torch.equal(ys[0][rows], ys[1][rows]) and torch.isnan(ys[1][1]).all()


@pytest.mark.parametrize("M", [6, 300])
def test_what_is_left_out_is_not_read(M):
    """NaN in the rows of padding tokens and the weights of slots without an expert
    touch nothing; their own results are 0."""
    i, experts, weights = inputs(M, 2, 5, 96, 64, "f16")
    experts[2] = -1
    experts[0, 1] = -1
    outs = []
    for bad in (False, True):
        dev = {n: v.cuda() for n, v in i.items()}
        w = weights.cuda()
        if bad:
            dev["x"][2] = NAN
            dev["dy"][2] = NAN
            w[2] = NAN
            w[0, 1] = NAN
        plan = make_plan(experts, 5)
        y = torch.empty_like(dev["x"])
        g, u = (torch.zeros(M * 2, 64, dtype=torch.float16, device="cuda") for _ in range(2))
        iabn.iabn_experts_forward(dev["x"], plan, w, dev["w_gate"], dev["w_up"], dev["w_down"], y, g, u)
        dx, dw = torch.empty_like(y), torch.empty_like(w)
        dws = [torch.empty_like(dev[n]) for n in ("w_gate", "w_up", "w_down")]
        iabn.iabn_experts_backward(dev["dy"], dev["x"], plan, w, g, u, dev["w_gate"], dev["w_up"], dev["w_down"], dx, dw,
                                   g, u, *dws)
        outs.append([y, dx, dw, *dws])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    y, dx, dw = outs[1][:3]
    assert (y[2] == 0).all() and (dx[2] == 0).all() and (dw[2] == 0).all() and dw[0, 1] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_twice(dtype):
    """Bit by bit the same, whatever the workspace held."""
    i, experts, weights = inputs(700, 4, 8, 264, 136, dtype)
    dev = {n: v.cuda() for n, v in i.items()}
    plan, w = make_plan(experts, 8), weights.cuda()
    need = iabn.iabn_experts_workspace_size(700, 4, 8, 264, 136, TORCH_DTYPES[dtype])
    runs = []
    for fill in (0, 255):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        y = torch.empty_like(dev["x"])
        g, u = (torch.empty(2800, 136, dtype=TORCH_DTYPES[dtype], device="cuda") for _ in range(2))
        iabn.iabn_experts_forward(dev["x"], plan, w, dev["w_gate"], dev["w_up"], dev["w_down"], y, g, u, workspace=ws)
        outs = [torch.empty_like(dev["x"]), torch.empty_like(w), torch.empty_like(g), torch.empty_like(g)]
        outs += [torch.empty_like(dev[n]) for n in ("w_gate", "w_up", "w_down")]
        ws.fill_(fill)
        iabn.iabn_experts_backward(dev["dy"], dev["x"], plan, w, g, u, dev["w_gate"], dev["w_up"], dev["w_down"], *outs,
                                   workspace=ws)
        runs.append([y, g, u] + outs)
    for a, b in zip(*runs):
        assert torch.equal(a, b)


def test_a_wrong_plan_stays_inside():
    """A plan with numbers out of their ranges gives wrong values, and nothing else."""
    M, k, E, C, F = 200, 2, 4, 64, 72
    i, experts, weights = inputs(M, k, E, C, F, "bf16")
    dev = {n: v.cuda() for n, v in i.items()}
    w = weights.cuda()
    for rows in (M, 20):
        for wrong in (1 << 30, -(1 << 30), M * k, -1):
            plan = make_plan(experts[:rows], E)
            plan[E + 1:E + 1 + 2 * rows * k:7] = wrong
            y, intact = guarded((rows, C), torch.bfloat16, 0)
            x = dev["x"][:rows].contiguous()
            iabn.iabn_experts_forward(x, plan, w[:rows].contiguous(), dev["w_gate"], dev["w_up"], dev["w_down"], y)
            torch.cuda.synchronize()
            intact("y")
            outs = [torch.empty_like(x), torch.empty_like(w[:rows])]
            dws = [guarded((E * F, C), torch.bfloat16, 0) for _ in range(3)]
            gu = [torch.zeros(rows * k, F, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
            for by_size in (wrong, 0):  # (the experts by size)
                plan[E + 1 + 2 * rows * k:2 * E + 1 + 2 * rows * k] = by_size
                iabn.iabn_experts_backward(x, x, plan, w[:rows].contiguous(), *gu[:2], dev["w_gate"], dev["w_up"],
                                           dev["w_down"], *outs, *gu[2:], dws[0][0].view(E, F, C), dws[1][0].view(E, F, C),
                                           dws[2][0].view(E, C, F))
                torch.cuda.synchronize()
                for _, ok in dws:
                    ok("dw")
            plan[:E + 1] = torch.tensor([wrong, 3, -7, 1 << 29, M * k + 5], dtype=torch.int32)
            iabn.iabn_experts_forward(x, plan, w[:rows].contiguous(), dev["w_gate"], dev["w_up"], dev["w_down"], y)
            torch.cuda.synchronize()
            intact("y")
