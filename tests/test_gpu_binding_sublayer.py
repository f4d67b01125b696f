"""The sublayer's plain calls are the native fast path's: the Python code,
which takes whatever that refuses, is not reached; and both give the same bits."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]

R, C, F = 6, 40, 24


def state(dtype):
    gen = torch.Generator(device="cuda").manual_seed(6)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    t = {k: new(R, C).to(dtype) for k in ("x", "h", "r", "u", "dr", "du", "dx", "dh", "y")}
    t.update({k: new(C) for k in ("pw", "pb", "qw", "qb", "dpw", "dpb", "dqw", "dqb")})
    t.update({k: new(2, R).abs() + 0.5 for k in ("ps", "qs")})
    t.update({k: new(2, C).to(dtype) for k in ("gate", "dgate")})
    t.update({k: new(R, F).to(dtype) for k in ("g", "up", "dg", "dup")})
    t.update({k: new(F, C).to(dtype) for k in ("wg", "wu", "dwg", "dwu")})
    t.update({k: new(C, F).to(dtype) for k in ("wd", "dwd")})
    return t


def norms(t, back, gate=True, **k):
    kw = dict(post_norm="layer", post_weight=t["pw"], post_bias=t["pb"], pre_norm="rms", pre_weight=t["qw"],
              post_stats=t["ps"], pre_stats=t["qs"], alpha=0.5, beta=2, p=0.25, seed=2 ** 64 - 1, offset=5, **k)
    if gate:
        kw["gate"] = t["gate"]
    if not back:
        return iabn.iabn_resnorm_forward(t["x"], t["h"], t["r"], t["u"], pre_bias=t["qb"], eps=1e-3, **kw)
    if gate:
        kw["dgate"] = t["dgate"]
    return iabn.iabn_resnorm_backward(t["dr"], t["du"], t["r"], t["h"], t["dx"], t["dh"], dpost_weight=t["dpw"],
                                      dpost_bias=t["dpb"], dpre_weight=t["dqw"], dpre_bias=t["dqb"], **kw)


def block_backward(t, **k):
    return iabn.iabn_ffn_backward(t["dr"], t["x"], t["g"], t["up"], t["wg"], t["wu"], t["wd"], t["dx"], t["dg"],
                                  t["dup"], t["dwg"], t["dwu"], t["dwd"], act="gelu", **k)


def room():
    return torch.empty(1 << 20, dtype=torch.uint8, device="cuda")


CALLS = {
    "dropout": lambda t, **k: iabn.iabn_dropout(t["x"], t["y"], 0.5, 3, 4, **k),
    "resnorm_forward": lambda t, **k: norms(t, False, **k),
    "resnorm_forward, parts": lambda t, **k: iabn.iabn_resnorm_forward(t["x"], None, None, t["u"], pre_norm="layer", **k),
    "resnorm_backward": lambda t, **k: norms(t, True, **k),
    "resnorm_backward, no gate": lambda t, **k: norms(t, True, gate=False, **k),
    "resnorm_backward, workspace": lambda t, **k: norms(t, True, workspace=room(), **k),
    "resnorm_backward, parts": lambda t, **k: iabn.iabn_resnorm_backward(
        None, t["du"], t["r"], None, t["dx"], None, pre_norm="rms", pre_stats=t["qs"], **k),
    "ffn_forward": lambda t, **k: iabn.iabn_ffn_forward(t["x"], t["wg"], t["wu"], t["wd"], t["y"], t["g"], t["up"], **k),
    "ffn_forward, inference": lambda t, **k: iabn.iabn_ffn_forward(t["x"], t["wg"], t["wu"], t["wd"], t["y"],
                                                                   act="leaky", slope=0.2, workspace=room(), **k),
    "ffn_backward": block_backward,
    "ffn_backward, workspace": lambda t, **k: block_backward(t, workspace=room(), **k),
}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_plain_calls_are_native(call, dtype, monkeypatch):
    python, native = state(dtype), state(dtype)
    CALLS[call](python, stream=torch.cuda.current_stream())

    def not_native(name, *args):
        raise AssertionError("%s went to the Python path" % name)

    monkeypatch.setattr(iabn, "_enqueue", not_native)
    CALLS[call](native)
    torch.cuda.synchronize()
    for k, v in python.items():
        assert torch.equal(native[k], v), k
