"""The routed experts' and the clipping's entry points on the host: what they
refuse, and their sizes (CPU only; skipped where a GPU is visible, as test_abi.py)."""

from __future__ import annotations

import ctypes

import pytest
import torch

import paper_1712_02616_amd as iabn
from test_sublayer_abi import (BF16, ERR_DTYPE, ERR_NULL, ERR_PARAM, ERR_SHAPE, ERR_WORKSPACE, F16, F32, INF, NAN, OK,
                               P, lib, no_gpu, refused)  # noqa: F401

SOFTMAX, SIGMOID = 0, 1


def route(lib, **kw):
    a = dict(logits=P, dtype=F16, bias=None, experts=P, weights=P, score=SOFTMAX, groups=1, kept=1, top=1, norm=0,
             scale=1.0, M=4, E=16, k=2)
    a.update(kw)
    return lib.iabn_route_forward(*a.values(), None)


def route_backward(lib, **kw):
    a = dict(dw=P, logits=P, experts=P, dlogits=P, dtype=F16, score=SIGMOID, norm=1, scale=1.0, M=4, E=16, k=2)
    a.update(kw)
    return lib.iabn_route_backward(*a.values(), None)


@no_gpu
def test_route_refuses(lib):  # noqa: F811
    both = ((ERR_DTYPE, dict(dtype=3)), (ERR_SHAPE, dict(M=-1)), (ERR_SHAPE, dict(M=(1 << 25) + 1)),
            (ERR_SHAPE, dict(E=0)), (ERR_SHAPE, dict(E=1025)), (ERR_SHAPE, dict(k=-1)), (ERR_SHAPE, dict(k=17)),
            (ERR_SHAPE, dict(E=1024, k=65)), (ERR_SHAPE, dict(M=1 << 25, E=64, k=33)), (ERR_PARAM, dict(score=2)),
            (ERR_PARAM, dict(scale=INF)), (ERR_PARAM, dict(scale=NAN)), (ERR_NULL, dict(logits=None)),
            (ERR_NULL, dict(experts=None)))
    for status, kw in both:
        refused(lib, status, route(lib, **kw))
        refused(lib, status, route_backward(lib, **kw))
    for status, kw in ((ERR_SHAPE, dict(groups=0)), (ERR_SHAPE, dict(groups=3)), (ERR_SHAPE, dict(E=256, groups=128)),
                       (ERR_PARAM, dict(groups=4, kept=0)), (ERR_PARAM, dict(groups=4, kept=5)),
                       (ERR_PARAM, dict(top=0)), (ERR_PARAM, dict(top=3)), (ERR_NULL, dict(weights=None))):
        refused(lib, status, route(lib, **kw))
    refused(lib, ERR_NULL, route_backward(lib, dw=None))
    refused(lib, ERR_NULL, route_backward(lib, dlogits=None))
    assert route(lib, M=0, logits=None, experts=None, weights=None) == OK
    assert route(lib, k=0, logits=None, experts=None, weights=None) == OK
    assert route_backward(lib, M=0, dw=None, logits=None, experts=None, dlogits=None) == OK


@no_gpu
def test_plan_refuses(lib):  # noqa: F811
    plan = lib.iabn_experts_plan
    for status, args in ((ERR_SHAPE, (P, P, -1, 2, 4)), (ERR_SHAPE, (P, P, 4, 65, 4)), (ERR_SHAPE, (P, P, 4, 2, 0)),
                         (ERR_SHAPE, (P, P, 4, 2, 1025)), (ERR_SHAPE, (P, P, 1 << 25, 64, 8)),
                         (ERR_NULL, (None, P, 4, 2, 4)), (ERR_NULL, (P, None, 4, 2, 4)), (ERR_NULL, (None, None, 0, 2, 4))):
        refused(lib, status, plan(*args, None))


def test_plan_size(lib):  # noqa: F811
    size = lib.iabn_experts_plan_size
    assert size(0, 2, 4) == 5 + 4 and size(6, 0, 4) == 5 + 4
    assert size(4, 2, 16) == 17 + 16 + 16
    for M, k, E in ((1, 8, 64), (4096, 8, 64), (100000, 8, 1000), (1 << 25, 32, 1024)):
        assert 2 * E + 1 + 2 * M * k <= size(M, k, E) <= 2 * E + 1 + 2 * M * k + 256 * E
    assert size(-1, 2, 4) == size(4, 65, 4) == size(4, 2, 0) == size(4, 2, 1025) == size(1 << 25, 64, 8) == 0


def forward(lib, **kw):
    a = dict(x=P, plan=P, weights=P, wg=P, wu=P, wd=P, y=P, g=P, u=P, dtype=F16, act=0, slope=0.0, M=4, k=2, E=8, C=16,
             F=24, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.iabn_experts_forward(*a.values(), None)


def backward(lib, **kw):
    a = dict(dy=P, x=P, plan=P, weights=P, g=P, u=P, wg=P, wu=P, wd=P, dx=P, dw=P, dg=P, du=P, dwg=P, dwu=P, dwd=P,
             dtype=F16, act=0, slope=0.0, M=4, k=2, E=8, C=16, F=24, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.iabn_experts_backward(*a.values(), None)


@no_gpu
def test_experts_refuse(lib):  # noqa: F811
    need = lib.iabn_experts_workspace_size(4, 2, 8, 16, 24, F16)
    assert need >= 8 * 24 * 2 + 8 * 16 * 4
    both = ((ERR_DTYPE, dict(dtype=3)), (ERR_SHAPE, dict(M=-1)), (ERR_SHAPE, dict(k=65)), (ERR_SHAPE, dict(E=0)),
            (ERR_SHAPE, dict(E=1025)), (ERR_SHAPE, dict(C=-1)), (ERR_SHAPE, dict(F=(1 << 17) + 1)),
            (ERR_SHAPE, dict(M=1 << 20, k=64, C=1 << 10)), (ERR_SHAPE, dict(E=1024, C=1 << 13, F=1 << 13)),
            (ERR_PARAM, dict(act=3)), (ERR_PARAM, dict(act=2, slope=-0.1)), (ERR_PARAM, dict(act=2, slope=NAN)),
            (ERR_NULL, dict(ws=None)), (ERR_WORKSPACE, dict(ws_bytes=need - 1)),
            (ERR_WORKSPACE, dict(ws=ctypes.c_void_p(4096 + 8))), (ERR_NULL, dict(x=None)), (ERR_NULL, dict(plan=None)),
            (ERR_NULL, dict(weights=None)), (ERR_NULL, dict(wg=None)), (ERR_NULL, dict(wu=None)),
            (ERR_NULL, dict(wd=None)), (ERR_NULL, dict(g=None)), (ERR_NULL, dict(u=None)))
    for status, kw in both:
        refused(lib, status, forward(lib, **kw))
        refused(lib, status, backward(lib, **kw))
    refused(lib, ERR_NULL, forward(lib, y=None))
    refused(lib, ERR_NULL, forward(lib, y=None, F=0))
    for k in ("dy", "dx", "dw", "dg", "du", "dwg", "dwu", "dwd"):
        refused(lib, ERR_NULL, backward(lib, **{k: None}))
    refused(lib, ERR_NULL, backward(lib, M=0, dwg=None))
    assert forward(lib, M=0, x=None, y=None, ws=None) == OK


@no_gpu
def test_experts_refuse_more_pairs_than_a_launch_has_tiles_for(lib):  # noqa: F811
    # 2^30 pairs in tiles of 64 rows, 256 threads each, would be 2^32 threads.
    for M, k in (((1 << 23) + 1, 64), (1 << 25, 17), (1 << 25, 32)):
        many = dict(M=M, k=k, E=64, C=1, F=1, ws_bytes=1 << 45)
        refused(lib, ERR_SHAPE, forward(lib, **many))
        refused(lib, ERR_SHAPE, backward(lib, **many))
        assert lib.iabn_experts_workspace_size(M, k, 64, 1, 1, F16) == 0
    assert lib.iabn_experts_workspace_size(1 << 23, 64, 64, 1, 1, F16) > 0


def test_experts_workspace(lib):  # noqa: F811
    size = lib.iabn_experts_workspace_size
    assert size(-1, 2, 8, 16, 24, F16) == size(4, 2, 8, 16, 24, 9) == size(4, 2, 8, 1 << 18, 24, F16) == 0
    assert size(0, 2, 8, 16, 24, F16) == size(4, 0, 8, 16, 24, F16) == size(4, 2, 8, 0, 24, F16) == 0
    # h, the pairs' terms and the weights' partial gradients, and no more than padding.
    for M, k, E, C, F, dtype, b in ((4096, 8, 64, 2048, 1024, BF16, 2), (333, 2, 7, 1000, 731, F32, 4)):
        pairs = M * k
        least = pairs * (F * b + C * (3 if b == 2 else 4) + -(-F // 64) * 4)
        assert least <= size(M, k, E, C, F, dtype) <= least + 4 * 256
    # Few tokens: fp32 terms, of at most 16 splits.
    assert 8 * 2048 * 4 <= size(1, 8, 64, 2048, 1024, BF16) <= 8 * 2048 * 4 * 16 + 8 * 1024 * 8


def grads(n=2, dtypes=(F32, BF16), sizes=(5, 9), at=4096):
    return ((ctypes.c_void_p * n)(*[at] * n), (ctypes.c_int * n)(*dtypes), (ctypes.c_int64 * n)(*sizes))


@no_gpu
def test_grads_refuse(lib):  # noqa: F811
    p, d, s = grads()
    norm, clip = lib.iabn_grad_norm, lib.iabn_grad_clip
    need = lib.iabn_grad_norm_workspace_size(s, 2)
    assert need == 16
    for args, status in (((p, d, s, -1, P, P, 64), ERR_SHAPE), ((p, d, s, (1 << 20) + 1, P, P, 64), ERR_SHAPE),
                         ((p, d, None, 2, P, P, 64), ERR_NULL), ((None, d, s, 2, P, P, 64), ERR_NULL),
                         ((p, None, s, 2, P, P, 64), ERR_NULL), ((p, d, s, 2, None, P, 64), ERR_NULL),
                         ((p, d, s, 2, P, None, 64), ERR_NULL), ((p, d, s, 2, P, P, 15), ERR_WORKSPACE),
                         ((p, d, s, 2, P, ctypes.c_void_p(4100), 64), ERR_WORKSPACE),
                         (grads(dtypes=(F32, 3)) + (2, P, P, 64), ERR_DTYPE),
                         (grads(sizes=(5, -1)) + (2, P, P, 64), ERR_SHAPE),
                         (grads(sizes=(1 << 42, 1)) + (2, P, P, 1 << 30), ERR_SHAPE),
                         (grads(at=None) + (2, P, P, 64), ERR_NULL)):
        refused(lib, status, norm(*args, None))
    for args, status in (((p, p, d, s, -1, P, 1.0), ERR_SHAPE), ((p, None, d, s, 2, P, 1.0), ERR_NULL),
                         ((None, p, d, s, 2, P, 1.0), ERR_NULL), ((p, p, d, s, 2, None, 1.0), ERR_NULL),
                         ((p, p, d, s, 2, P, -1.0), ERR_PARAM), ((p, p, d, s, 2, P, NAN), ERR_PARAM),
                         ((p, grads(at=None)[0], d, s, 2, P, 1.0), ERR_NULL)):
        refused(lib, status, clip(*args, None))
    # Nothing to clip: empty lists and empty tensors.
    assert clip(None, None, None, None, 0, None, 1.0, None) == OK
    p0, d0, s0 = grads(sizes=(0, 0), at=None)
    assert clip(p0, p0, d0, s0, 2, None, INF, None) == OK


@no_gpu
def test_clip_refuses_an_output_twice(lib):  # noqa: F811
    # Elements that two tensors write would be scaled once or twice, by chance.
    def outs(pairs, dtype=F32):
        n = len(pairs)
        at = (ctypes.c_void_p * n)(*[p for p, _ in pairs])
        return at, at, (ctypes.c_int * n)(*[dtype] * n), (ctypes.c_int64 * n)(*[c for _, c in pairs]), n, P, 1.0

    apart = [(1 << 20, 8), (1 << 12, 8)]
    for wrong in (apart + [(1 << 20, 8)], apart + [((1 << 20) + 28, 4)], apart + [((1 << 20) - 4, 2)],
                  [((1 << 20) + 64 * i, 16) for i in range(300)] + [((1 << 20) + 64 * 17, 1)],
                  [(1 << 20, 16), ((1 << 20) + 8, 1), ((1 << 20) + 32, 1)]):
        refused(lib, ERR_PARAM, lib.iabn_grad_clip(*outs(wrong), None))
    # (Empty ones lie nowhere.)
    assert lib.iabn_grad_clip(*outs([(1 << 20, 0)] * 3), None) == OK


def test_grads_workspace(lib):  # noqa: F811
    size = lambda *n: lib.iabn_grad_norm_workspace_size((ctypes.c_int64 * len(n))(*n), len(n))  # noqa: E731
    assert size() == 0 and size(0, 0) == 0 and size(1) == 8 and size(4096) == 8 and size(4097) == 16
    assert size(-1) == 0 and size(1 << 43) == 0
    for n in (1 << 20, 1 << 30, 1 << 42):
        assert size(n) <= 8 * 8192 and size(n, 1, 0, 1) <= 8 * 8194


def test_python_refuses():
    x = torch.zeros(4, 8)
    e, w = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    with pytest.raises(ValueError, match="HIP device"):
        iabn.iabn_route_forward(x, e, w)
    with pytest.raises(ValueError, match="score"):
        iabn.iabn_route_forward(x, e, w, score="relu")
    with pytest.raises(ValueError, match="HIP device"):
        iabn.iabn_route_backward(w, x, e, x)
    with pytest.raises(ValueError, match="HIP device"):
        iabn.iabn_experts_plan(e, e, 4)
    with pytest.raises(ValueError, match="int32"):
        iabn.iabn_experts_plan(e.long(), e, 4)
    with pytest.raises(TypeError, match="torch.Tensor"):
        iabn.iabn_experts_plan(None, e, 4)
    with pytest.raises(ValueError, match="act"):
        iabn.iabn_experts_forward(x, e, w, x, x, x, x, act="tanh")
    with pytest.raises(ValueError, match="HIP device"):
        iabn.iabn_grad_norm([x], w)
    with pytest.raises(TypeError, match="torch.Tensors"):
        iabn.iabn_grad_clip([None], [x], w, 1.0)
    with pytest.raises(ValueError, match="one float32"):
        iabn.iabn_grad_norm([], torch.zeros(2))


def test_every_name_is_the_packages_too():
    from paper_1712_02616_amd import routed

    for name in routed.__all__:
        assert getattr(iabn, name) is getattr(routed, name)
