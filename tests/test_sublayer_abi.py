"""The sublayer's entry points on the host: what they refuse, and their
workspaces (CPU only; skipped where a GPU is visible, as test_abi.py)."""

from __future__ import annotations

import ctypes

import pytest
import torch

import paper_1712_02616_amd as iabn

OK, ERR_NULL, ERR_SHAPE, ERR_PARAM, ERR_DTYPE, ERR_WORKSPACE = 0, 1, 2, 3, 4, 5
F32, F16, BF16 = 0, 1, 2
NONE, RMS, LAYER = 0, 1, 2
NAN, INF = float("nan"), float("inf")

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="placeholder pointers are only safe without a GPU")
P = ctypes.c_void_p(4096)  # a pointer that nothing may follow


@pytest.fixture(scope="module")
def lib():
    return iabn.load()


def refused(lib, status, rc):
    assert rc == status, (rc, lib.iabn_last_error())
    assert lib.iabn_last_error()


@no_gpu
def test_dropout_refuses(lib):
    call = lib.iabn_dropout
    refused(lib, ERR_DTYPE, call(P, P, 7, 0.1, 0, 0, 4, 8, None))
    refused(lib, ERR_SHAPE, call(P, P, F16, 0.1, 0, 0, -1, 8, None))
    refused(lib, ERR_SHAPE, call(P, P, F16, 0.1, 0, 0, 4, 1 << 31, None))
    refused(lib, ERR_SHAPE, call(P, P, F16, 0.1, 0, 0, 1 << 40, 1 << 20, None))
    for p in (-0.1, 1.5, NAN):
        refused(lib, ERR_PARAM, call(P, P, F16, p, 0, 0, 4, 8, None))
    refused(lib, ERR_NULL, call(None, P, F16, 0.1, 0, 0, 4, 8, None))
    refused(lib, ERR_NULL, call(P, None, F16, 0.1, 0, 0, 4, 8, None))
    assert call(None, None, F16, 0.1, 0, 0, 0, 8, None) == OK
    assert call(None, None, F16, 0.1, 0, 0, 8, 0, None) == OK


def forward(lib, **kw):
    a = dict(x=P, h=P, r=P, u=P, dtype=F16, gate=None, groups=0, post=RMS, post_w=P, post_b=P, pre=LAYER, pre_w=P,
             pre_b=P, post_stats=None, pre_stats=None, alpha=1.0, beta=1.0, eps=1e-5, p=0.0, seed=0, offset=0, R=4,
             C=64)
    a.update(kw)
    return lib.iabn_resnorm_forward(*a.values(), None)


@no_gpu
def test_resnorm_forward_refuses(lib):
    for status, kw in ((ERR_DTYPE, dict(dtype=3)), (ERR_SHAPE, dict(R=-1)), (ERR_SHAPE, dict(C=-2)),
                       (ERR_SHAPE, dict(C=16385)), (ERR_SHAPE, dict(R=1 << 45)), (ERR_PARAM, dict(post=3)),
                       (ERR_PARAM, dict(pre=-1)), (ERR_PARAM, dict(post=NONE)),
                       (ERR_PARAM, dict(pre=NONE, u=None)), (ERR_PARAM, dict(pre=NONE, pre_w=None, pre_b=None)),
                       (ERR_NULL, dict(u=None)), (ERR_NULL, dict(x=None)), (ERR_NULL, dict(h=None)),
                       (ERR_NULL, dict(h=None, post=NONE, post_w=None, post_b=None, gate=P, groups=1)),
                       (ERR_NULL, dict(r=None, u=None, pre=NONE, pre_w=None, pre_b=None)),
                       (ERR_SHAPE, dict(gate=P, groups=0)), (ERR_SHAPE, dict(gate=P, groups=3)),
                       (ERR_PARAM, dict(eps=0.0)), (ERR_PARAM, dict(eps=NAN)), (ERR_PARAM, dict(alpha=INF)),
                       (ERR_PARAM, dict(beta=NAN)), (ERR_PARAM, dict(p=1.0001)), (ERR_PARAM, dict(p=NAN))):
        refused(lib, status, forward(lib, **kw))
    assert forward(lib, R=0, x=None, h=None, r=None, u=None) == OK
    assert forward(lib, C=0, x=None, h=None, r=None, u=None) == OK


def backward(lib, **kw):
    a = dict(dr=P, du=P, r=P, h=P, dx=P, dh=ctypes.c_void_p(8192), dtype=F16, gate=None, groups=0, post=RMS,
             post_w=P, post_b=P, pre=LAYER, pre_w=P, post_stats=P, pre_stats=P, dgate=None, dpost_w=P, dpost_b=P,
             dpre_w=P, dpre_b=P, alpha=1.0, beta=1.0, p=0.0, seed=0, offset=0, R=4, C=64, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.iabn_resnorm_backward(*a.values(), None)


@no_gpu
def test_resnorm_backward_refuses(lib):
    need = lib.iabn_resnorm_workspace_size(4, 64, 0)
    assert need > 0
    for status, kw in ((ERR_DTYPE, dict(dtype=-1)), (ERR_SHAPE, dict(C=16385)), (ERR_SHAPE, dict(R=-4)),
                       (ERR_PARAM, dict(post=9)), (ERR_PARAM, dict(pre=NONE, pre_w=None)),
                       (ERR_PARAM, dict(post=NONE, post_w=None, post_b=None)), (ERR_NULL, dict(du=None)),
                       (ERR_PARAM, dict(pre=NONE, pre_w=None, dpre_w=None, dpre_b=None)),
                       (ERR_NULL, dict(dr=None, du=None, pre=NONE, pre_w=None, dpre_w=None, dpre_b=None)),
                       (ERR_NULL, dict(r=None)), (ERR_NULL, dict(pre_stats=None)), (ERR_NULL, dict(post_stats=None)),
                       (ERR_NULL, dict(h=None)), (ERR_PARAM, dict(dgate=P)), (ERR_SHAPE, dict(gate=P, groups=3)),
                       (ERR_PARAM, dict(dh=P)), (ERR_PARAM, dict(p=-1.0)), (ERR_PARAM, dict(alpha=NAN)),
                       (ERR_NULL, dict(ws=None)), (ERR_WORKSPACE, dict(ws_bytes=need - 1)),
                       (ERR_WORKSPACE, dict(ws=ctypes.c_void_p(4096 + 4)))):
        refused(lib, status, backward(lib, **kw))
    assert backward(lib, C=0, ws=None) == OK


def test_resnorm_workspace(lib):
    size = lib.iabn_resnorm_workspace_size
    assert size(0, 64, 0) == 0 and size(8, 0, 1) == 0
    assert size(-1, 64, 0) == 0 and size(8, 16385, 0) == 0
    for R, C, groups in ((1, 1, 0), (1, 16384, 1), (1 << 20, 1024, 0), (1 << 20, 1024, 1 << 19), (1 << 20, 16384, 7)):
        # A few vectors of every block, whatever the number of rows.
        assert 0 < size(R, C, groups) <= 5 * 4 * C * 2048


def test_python_refuses():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="HIP device"):
        iabn.iabn_dropout(x, x, 0.1, 1)
    with pytest.raises(TypeError, match="torch.Tensor"):
        iabn.iabn_dropout(None, x, 0.1, 1)
    with pytest.raises(ValueError, match="post_norm"):
        iabn.iabn_resnorm_forward(x, x, x, x, post_norm="batch")
    with pytest.raises(ValueError, match="both None"):
        iabn.iabn_resnorm_backward(None, None, None, None, None, None)


def ffn_forward(lib, **kw):
    a = dict(x=P, wg=P, wu=P, wd=P, y=P, g=P, u=P, dtype=F16, act=0, slope=0.0, M=4, C=16, F=24, ws=P,
             ws_bytes=1 << 30)
    a.update(kw)
    return lib.iabn_ffn_forward(*a.values(), None)


def ffn_backward(lib, **kw):
    a = dict(dy=P, x=P, g=P, u=P, wg=P, wu=P, wd=P, dx=P, dg=P, du=P, dwg=P, dwu=P, dwd=P, dtype=F16, act=0,
             slope=0.0, M=4, C=16, F=24, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.iabn_ffn_backward(*a.values(), None)


@no_gpu
def test_ffn_refuses(lib):
    need = lib.iabn_ffn_workspace_size(4, 16, 24, F16)
    assert need >= 4 * 24 * 2
    both = ((ERR_DTYPE, dict(dtype=3)), (ERR_SHAPE, dict(M=-1)), (ERR_SHAPE, dict(C=(1 << 24) + 1)),
            (ERR_SHAPE, dict(F=-8)), (ERR_SHAPE, dict(M=(1 << 26) + 1)), (ERR_SHAPE, dict(M=1 << 26, F=1 << 20)), (ERR_PARAM, dict(act=3)),
            (ERR_PARAM, dict(act=2, slope=-0.1)), (ERR_PARAM, dict(act=2, slope=NAN)),
            (ERR_NULL, dict(ws=None)), (ERR_WORKSPACE, dict(ws_bytes=need - 1)),
            (ERR_WORKSPACE, dict(ws=ctypes.c_void_p(4096 + 8))))
    for status, kw in both:
        refused(lib, status, ffn_forward(lib, **kw))
        refused(lib, status, ffn_backward(lib, **kw))
    for k in ("x", "wg", "wu", "wd", "y"):
        refused(lib, ERR_NULL, ffn_forward(lib, **{k: None}))
    refused(lib, ERR_NULL, ffn_forward(lib, g=None))
    refused(lib, ERR_NULL, ffn_forward(lib, u=None))
    for k in ("dy", "x", "g", "u", "wg", "wu", "wd", "dx", "dg", "du", "dwg", "dwu", "dwd"):
        refused(lib, ERR_NULL, ffn_backward(lib, **{k: None}))
    refused(lib, ERR_NULL, ffn_backward(lib, M=0, dwg=None))
    assert ffn_forward(lib, M=0, x=None, y=None, ws=None) == OK
    assert lib.iabn_ffn_workspace_size(-1, 16, 24, F16) == 0 and lib.iabn_ffn_workspace_size(4, 16, 24, 9) == 0
