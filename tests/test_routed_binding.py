"""The routed experts' binding from the host (no GPU): where it takes its workspace
and enqueues its kernels, and what shapes it refuses (see test_binding_streams)."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
from test_binding_streams import DEVICE, Stream, seen, t  # noqa: F401

M, K, E, C, F = 4, 2, 3, 16, 24
INT = torch.int32


def experts(M=M, k=K):
    return t(M, k, dtype=INT)


def plan():
    return t(iabn.iabn_experts_plan_size(M, K, E), dtype=INT)


def ws():
    return [t(E, F, C), t(E, F, C), t(E, C, F)]


def forward(x=None, **kw):
    return iabn.iabn_experts_forward(t(M, C) if x is None else x, kw.pop("plan", plan()), kw.pop("weights", t(M, K)),
                                     *kw.pop("ws", ws()), t(M, C), **kw)


def backward(**kw):
    gu = kw.pop("gu", t(M * K, F))
    return iabn.iabn_experts_backward(t(M, C), t(M, C), plan(), t(M, K), gu, gu, *ws(), t(M, C), kw.pop("dw", t(M, K)), gu,
                                      gu, *kw.pop("dws", ws()), **kw)


WITH_SPACE = {"experts_forward": forward, "experts_backward": backward,
              "grad_norm": lambda **kw: iabn.iabn_grad_norm([t(5), t(3, 2)], t(1), **kw)}
ALL = dict(WITH_SPACE)
ALL.update({
    "route_forward": lambda **kw: iabn.iabn_route_forward(t(M, E), experts(), t(M, K), **kw),
    "route_backward": lambda **kw: iabn.iabn_route_backward(t(M, K), t(M, E), experts(), t(M, E), **kw),
    "experts_plan": lambda **kw: iabn.iabn_experts_plan(experts(), plan(), E, **kw),
    "grad_clip": lambda **kw: iabn.iabn_grad_clip([t(5)], [t(5)], t(1), 1.0, **kw),
})


@pytest.mark.parametrize("call", WITH_SPACE)
@pytest.mark.parametrize("handle", ["stream", "integer"])
def test_a_new_workspace_belongs_to_the_calls_stream(seen, call, handle):  # noqa: F811
    WITH_SPACE[call](stream=Stream(99) if handle == "stream" else 99)
    assert seen.allocated == [99]
    assert seen.called == [("iabn_" + call, seen.called[0][1], 99)]


@pytest.mark.parametrize("call", WITH_SPACE)
def test_the_callers_workspace_is_taken_as_it_is(seen, call):  # noqa: F811
    WITH_SPACE[call](stream=Stream(99), workspace=t(1 << 16, dtype=torch.uint8))
    assert seen.allocated == [] and seen.called[0][2] == 99


def test_every_entry_point_is_here():
    from paper_1712_02616_amd import routed

    assert {n[len("iabn_"):] for n in routed.__all__ if n.startswith("iabn_") and not n.endswith("_size")} == set(ALL)


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("stream", [None, 0, 99])
def test_the_tensors_device_is_current(seen, call, stream):  # noqa: F811
    ALL[call](stream=stream)
    assert seen.called == [("iabn_" + call, DEVICE, {None: 7, 0: None, 99: 99}[stream])]
    assert seen.device is None


def test_wrong_shapes(seen):  # noqa: F811
    for match, call in (
            ("experts must be", lambda: iabn.iabn_route_forward(t(M, E), t(M, K), t(M, K))),
            ("experts must be", lambda: iabn.iabn_route_forward(t(M, E), experts(M + 1), t(M, K))),
            ("weights must be", lambda: iabn.iabn_route_forward(t(M, E), experts(), t(M, K + 1))),
            ("bias must hold", lambda: iabn.iabn_route_forward(t(M, E), experts(), t(M, K), bias=t(E + 1))),
            ("dlogits must match", lambda: iabn.iabn_route_backward(t(M, K), t(M, E), experts(), t(M, E + 1))),
            ("dweights must be", lambda: iabn.iabn_route_backward(t(M, K + 1), t(M, E), experts(), t(M, E))),
            ("plan must hold", lambda: iabn.iabn_experts_plan(experts(), plan()[:-1], E)),
            ("plan must hold", lambda: forward(plan=plan()[:-1])),
            ("plan must be", lambda: forward(plan=plan().float())),
            ("weights must be", lambda: forward(weights=t(M + 1, K))),
            ("w_gate must be", lambda: forward(ws=[t(E, F, C + 1), t(E, F, C), t(E, C, F)])),
            ("w_gate must be", lambda: forward(ws=[t(F, C), t(E, F, C), t(E, C, F)])),
            ("w_up must be", lambda: forward(ws=[t(E, F, C), t(E + 1, F, C), t(E, C, F)])),
            ("w_down must be", lambda: forward(ws=[t(E, F, C), t(E, F, C), t(E, F, C)])),
            ("g must be", lambda: forward(g=t(M, F), u=t(M, F))),
            ("g must be", lambda: backward(gu=t(M * K, F + 1))),
            ("dweights must be", lambda: backward(dw=t(M * K))),
            ("dw_down must be", lambda: backward(dws=[t(E, F, C)] * 3)),
            ("outs must match", lambda: iabn.iabn_grad_clip([t(5)], [t(6)], t(1), 1.0)),
            ("outs must match", lambda: iabn.iabn_grad_clip([t(5)], [], t(1), 1.0)),
            ("outs must match", lambda: iabn.iabn_grad_clip([t(5)], [t(5).half()], t(1), 1.0)),
            ("contiguous", lambda: iabn.iabn_grad_norm([t(4, 4).t()], t(1))),
            ("norm must be", lambda: iabn.iabn_grad_norm([t(4)], t(2)))):
        with pytest.raises(ValueError, match=match):
            call()
    assert seen.called == []
