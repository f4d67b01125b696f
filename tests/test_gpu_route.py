"""iabn_route_forward and iabn_route_backward on the GPU against their definition
in 64 bits: the choices are equal, the weights and gradients within the bounds of a
32-bit evaluation."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
import routed_oracle as routed
import sublayer_oracle as oracle
from gpu_helpers import TORCH_DTYPES, say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

INF, NAN = float("inf"), float("nan")


def run(logits, k, bias=None, score="softmax", groups=1, kept=None, group_top=1, renormalise=False, scale=1.0,
        stream=None, check_weights=True):
    """Both directions of one call on the GPU, checked; returns (experts, weights)."""
    M, E = logits.shape
    say("route M=%d E=%d k=%d %s %s groups=%d kept=%s top=%d renormalise=%s bias=%s" % (
        M, E, k, logits.dtype, score, groups, kept, group_top, renormalise, bias is not None))
    d = logits.cuda()
    b = None if bias is None else bias.cuda()
    experts = torch.full((M + 1, k), -77, dtype=torch.int32, device="cuda")
    weights = torch.full((M + 1, k), -77.0, device="cuda")
    torch.cuda.synchronize()
    iabn.iabn_route_forward(d, experts[:M], weights[:M], bias=b, score=score, groups=groups, groups_kept=kept,
                            group_top=group_top, renormalise=renormalise, scale=scale, stream=stream)
    torch.cuda.synchronize()
    assert (experts[M:] == -77).all() and (weights[M:] == -77).all()
    want = torch.tensor(routed.choose(logits, bias, k, score, groups, kept, group_top)).reshape(M, k)
    got = experts[:M].cpu().long()
    assert torch.equal(got, want), (got[(got != want).any(1)][:4], want[(got != want).any(1)][:4])
    if not check_weights:
        return got, weights[:M].cpu()
    w = routed.weights(logits, want, score, renormalise, scale)
    oracle.check("weights", weights[:M], w, routed.WEIGHT_ERROR * w.abs(), torch.float32)
    gen = torch.Generator().manual_seed(M * 131 + E)
    dw = torch.randn(M, k, generator=gen)
    back = torch.full((M * E + 16,), -77.0, dtype=logits.dtype, device="cuda")
    dl = back[:M * E].view(M, E)
    torch.cuda.synchronize()
    iabn.iabn_route_backward(dw.cuda(), d, experts[:M], dl, score=score, renormalise=renormalise, scale=scale,
                             stream=stream)
    torch.cuda.synchronize()
    assert (back[M * E:] == -77).all()
    v, err = routed.route_backward(dw, logits, want, score, renormalise, scale)
    oracle.check("dlogits", dl, v, err, logits.dtype)
    return got, weights[:M].cpu()


def normal(M, E, dtype="f32", seed=3, std=1.5):
    gen = torch.Generator().manual_seed(seed + 1000 * M + E)
    return (torch.randn(M, E, generator=gen) * std).to(TORCH_DTYPES[dtype])


SIZES = [(1, 1, 1), (1, 64, 8), (3, 2, 2), (5, 7, 7), (64, 16, 4), (70, 17, 3), (33, 61, 5), (20, 65, 9), (9, 100, 16),
         (11, 128, 16), (13, 200, 17), (17, 256, 8), (7, 257, 8), (4, 1000, 64), (3, 1024, 64), (2, 64, 64)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,E,k", SIZES)
def test_sizes(M, E, k, dtype):
    l = normal(M, E, dtype)
    run(l, k)
    run(l, k, score="sigmoid", renormalise=True, scale=2.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,k", [(3, 2), (16, 4), (17, 3), (61, 5), (64, 8), (100, 16), (128, 1), (250, 8), (256, 16)])
def test_many_rows(E, k, dtype):
    """More rows than one wave each: 16 lanes a row."""
    l = normal(1031, E, dtype)
    run(l, k, renormalise=True)
    gen = torch.Generator().manual_seed(E)
    run(l, k, bias=torch.randn(E, generator=gen) * 0.1, score="sigmoid")


@pytest.mark.parametrize("M", [5, 1100])
@pytest.mark.parametrize("E,groups,kept,k", [(8, 2, 1, 3), (64, 8, 3, 6), (256, 8, 4, 8), (60, 4, 2, 5), (63, 9, 4, 7),
                                             (16, 16, 5, 4), (64, 64, 9, 8), (48, 3, 2, 20), (192, 6, 6, 4)])
def test_groups(M, E, groups, kept, k):
    l = normal(M, E, "f32")
    gen = torch.Generator().manual_seed(E)
    b = torch.randn(E, generator=gen) * 0.05
    for group_top in (1, 2):
        run(l, k, bias=b, score="sigmoid", groups=groups, kept=kept, group_top=group_top, renormalise=True)
        run(l, k, groups=groups, kept=kept, group_top=group_top)


@pytest.mark.parametrize("M", [6, 1030])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_forms(M, score, renormalise, biased):
    bias = torch.linspace(-0.2, 0.2, 48)[torch.randperm(48, generator=torch.Generator().manual_seed(1))]
    run(normal(M, 48, "f16"), 6, bias=bias if biased else None, score=score, renormalise=renormalise, scale=0.5)


@pytest.mark.parametrize("M", [4, 1025])
def test_ties_go_to_the_lowest_index(M):
    l = torch.zeros(M, 40)
    l[:, 7::5] = 1.0
    l[:, 3] = -0.0  # equal to 0
    got, _ = run(l, 12)
    assert got[0].tolist() == [7, 12, 17, 22, 27, 32, 37, 0, 1, 2, 3, 4]
    run(l, 12, bias=torch.zeros(40), score="sigmoid")
    run(torch.zeros(M, 40), 9, groups=8, kept=2, group_top=2)


@pytest.mark.parametrize("M", [3, 1027])
def test_close_scores_are_told_apart(M):
    """Scores that differ by less than 2^-24 of themselves (a bias of 1 is added to
    each): a comparison in 32 bits would take the lower index."""
    E = 32
    l = torch.full((M, E), -20.0)
    l += torch.arange(E) * 0.01  # sigmoids of 2e-9 and more, in rising order
    got, _ = run(l, 5, bias=torch.ones(E), score="sigmoid")
    assert got[0].tolist() == [31, 30, 29, 28, 27]


@pytest.mark.parametrize("M", [5, 1029])
@pytest.mark.parametrize("E", [24, 200])
def test_switched_off(M, E):
    """Logits of -inf: rows that have fewer experts than choices, and none."""
    l = normal(M, E, "bf16")
    l[0] = -INF
    l[1, 2:] = -INF
    l[2, 1::2] = -INF
    l[M - 1] = -INF
    for kw in (dict(), dict(renormalise=True), dict(score="sigmoid", renormalise=True), dict(score="sigmoid"),
               dict(groups=4, kept=2, group_top=2, renormalise=True), dict(groups=2, kept=1, score="sigmoid")):
        got, w = run(l, 8, **kw)
        assert (got[0] == -1).all() and (w[0] == 0).all() and (got[1, 2:] == -1).all()
    bias = torch.zeros(E)
    bias[:E - 4] = -INF
    got, _ = run(l, 8, bias=bias, score="sigmoid")
    assert (got[:, 4:] == -1).all() and (got < 0).logical_or(got >= E - 4).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_masks_of_the_lowest_value(dtype):
    l = normal(1026, 20, dtype)
    low = torch.finfo(l.dtype).min
    l[:, ::3] = low
    l[5] = low  # all alike: a plain softmax of equal ones
    for kw in (dict(), dict(renormalise=True)):
        run(l, 8, **kw)
        run(l[:9], 8, **kw)
    for rows in (l, l[:9]):
        got, w = run(rows[:, 1:3].contiguous(), 2, renormalise=True)
        assert torch.isfinite(w).all()


@pytest.mark.parametrize("M", [4, 1025])
def test_underflowing_scores(M):
    """Renormalised weights keep their digits where every score underflows."""
    l = normal(M, 16, "f32")
    l[:2] -= 200.0
    got, w = run(l, 4, score="sigmoid", renormalise=True)
    assert ((w.sum(1) - 1).abs() < 1e-5).all()
    l[:2] += 400.0
    run(l, 4, score="sigmoid", renormalise=True)


@pytest.mark.parametrize("M", [4, 1025])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_nonfinite_logits_show(M, score):
    """A NaN is chosen and shows in its row alone."""
    l = normal(M, 30, "f32")
    clean = run(l, 4, score=score)
    l[1, 9] = NAN
    got, w = run(l, 4, score=score, check_weights=False)
    assert got[1, 0] == 9 and torch.isnan(w[1, 0])
    others = [m for m in range(M) if m != 1]
    assert torch.equal(got[others], clean[0][others]) and torch.equal(w[others], clean[1][others])
    _, w = run(l, 4, score=score, renormalise=True, check_weights=False)
    assert torch.isnan(w[1]).all() and torch.isfinite(w[others]).all()


def test_other_numbers_add_nothing_to_the_gradient():
    """-1 and numbers that are no expert's; an expert twice adds up."""
    l = normal(6, 12)
    chosen = torch.tensor([[0, 5, -1], [3, 3, 7], [12, 1, 2], [-5, -1, -1], [1 << 30, 4, 11], [0, 1, 2]])
    gen = torch.Generator().manual_seed(2)
    dw = torch.randn(6, 3, generator=gen)
    dw[0, 2] = NAN
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            dl = torch.empty(6, 12, device="cuda")
            iabn.iabn_route_backward(dw.cuda(), l.cuda(), chosen.int().cuda(), dl, score=score,
                                     renormalise=renormalise)
            v, err = routed.route_backward(dw, l, chosen, score, renormalise, 1.0)
            oracle.check("dlogits", dl, v, err, torch.float32)
            assert (dl[3] == 0).all()


@pytest.mark.parametrize("M,E", [(5, 33), (2000, 64), (1500, 255)])
def test_gradient_over_the_logits(M, E):
    """dlogits may be logits."""
    l = normal(M, E, "bf16")
    experts = torch.empty(M, 4, dtype=torch.int32, device="cuda")
    w = torch.empty(M, 4, device="cuda")
    d = l.cuda()
    iabn.iabn_route_forward(d, experts, w)
    dw = torch.randn(M, 4, device="cuda")
    apart = iabn.iabn_route_backward(dw, d, experts, torch.empty_like(d))
    assert torch.equal(iabn.iabn_route_backward(dw, d, experts, d), apart)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [7, 1100])
def test_unaligned_and_on_another_stream(dtype, M):
    E = 63
    flat = torch.zeros(M * E + 1, dtype=TORCH_DTYPES[dtype])
    flat[1:] = normal(M, E, dtype).flatten()
    d = flat.cuda()[1:].view(M, E)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    outs = []
    for stream in (None, st, st.cuda_stream):
        e, w = torch.empty(M, 5, dtype=torch.int32, device="cuda"), torch.empty(M, 5, device="cuda")
        torch.cuda.synchronize()
        iabn.iabn_route_forward(d, e, w, renormalise=True, stream=stream)
        torch.cuda.synchronize()
        outs.append((e, w))
    want = torch.tensor(routed.choose(flat[1:].view(M, E), None, 5, "softmax"))
    for e, w in outs:
        assert torch.equal(e.cpu().long(), want) and torch.equal(w, outs[0][1])


def test_no_rows_and_no_choices():
    z = lambda *s, t=torch.float32: torch.full(s, 7, dtype=t, device="cuda")  # noqa: E731
    iabn.iabn_route_forward(z(0, 8), z(0, 2, t=torch.int32), z(0, 2))
    iabn.iabn_route_backward(z(0, 2), z(0, 8), z(0, 2, t=torch.int32), z(0, 8))
    dl = z(3, 8)
    iabn.iabn_route_backward(z(3, 0), z(3, 8), z(3, 0, t=torch.int32), dl)
    assert (dl == 0).all()


def test_leading_dims():
    l = normal(24, 32)
    e, w = torch.empty(2, 3, 4, 5, dtype=torch.int32, device="cuda"), torch.empty(2, 3, 4, 5, device="cuda")
    iabn.iabn_route_forward(l.cuda().view(2, 3, 4, 32), e, w)
    assert torch.equal(e.cpu().long().view(24, 5), torch.tensor(routed.choose(l, None, 5, "softmax")))
