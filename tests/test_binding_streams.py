"""Where the Python binding takes its workspace and enqueues its kernels, seen
from the host (no GPU): tensors that say they are on a HIP device, and a
library that records what is current when it is called."""

from __future__ import annotations

import contextlib

import pytest
import torch

import paper_1712_02616_amd as iabn

DEVICE = torch.device("cuda", 1)


class OnDevice(torch.Tensor):
    """A host tensor that says it is on DEVICE (a subclass: the native fast
    path leaves it to the Python code)."""

    device = property(lambda self: DEVICE)


def t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


class Stream:
    """A stream's handle."""

    def __init__(self, handle):
        self.cuda_stream = handle


class Recorder:
    def __init__(self):
        self.stream = self.device = None
        self.allocated, self.called = [], []

    @contextlib.contextmanager
    def on_stream(self, stream):
        before, self.stream = self.stream, stream.cuda_stream
        yield
        self.stream = before

    @contextlib.contextmanager
    def on_device(self, device):
        before, self.device = self.device, device
        yield
        self.device = before


class Library:
    """libiabn whose entry points with a stream only record the call."""

    def __init__(self, lib, seen):
        self.lib, self.seen = lib, seen

    def __getattr__(self, name):
        fn = getattr(self.lib, name)
        if not name.startswith("iabn_") or name.endswith(("_size", "_string", "_error", "version")):
            return fn

        def call(*args):
            self.seen.called.append((name, self.seen.device, args[-1].value))
            return 0

        return call


@pytest.fixture
def seen(monkeypatch):
    seen, lib, empty = Recorder(), iabn.load(), torch.empty
    monkeypatch.setattr(iabn, "_lib", Library(lib, seen))
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", seen.on_stream)
    monkeypatch.setattr(torch.cuda, "device", seen.on_device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream(handle))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(7))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: None)

    def allocate(*shape, **kw):
        seen.allocated.append(seen.stream)
        kw.pop("device", None)
        return empty(*shape, **kw).as_subclass(OnDevice)

    monkeypatch.setattr(torch, "empty", allocate)
    return seen


def _norms(x, **kw):
    return iabn.iabn_resnorm_backward(x, x, x, x, x, t(4, 16), post_norm="rms", pre_norm="rms",
                                      post_stats=t(2, 4), pre_stats=t(2, 4), **kw)


def _block(x, **kw):
    return iabn.iabn_ffn_forward(x, t(24, 16), t(24, 16), t(16, 24), t(4, 16), **kw)


def _block_backward(x, **kw):
    h, w, wd = t(4, 24), t(24, 16), t(16, 24)
    return iabn.iabn_ffn_backward(x, x, h, h, w, w, wd, x, h, h, w, w, wd, **kw)


def _layer(**kw):
    x, c = t(2, 3, 4), t(3)
    iabn.iabn_forward_train(x, c, c, c, c, c, c, **kw)


def _layer_backward(**kw):
    x, c = t(2, 3, 4), t(3)
    iabn.iabn_backward(x, x, c, c, c, c, c, **kw)


CALLS = {"resnorm_backward": lambda **kw: _norms(t(4, 16), **kw), "ffn_forward": lambda **kw: _block(t(4, 16), **kw),
         "ffn_backward": lambda **kw: _block_backward(t(4, 16), **kw), "forward_train": _layer,
         "backward": _layer_backward}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("handle", ["stream", "integer"])
def test_a_new_workspace_belongs_to_the_calls_stream(seen, call, handle):
    """A block that the allocator hands out on another stream may still be in
    use there: only the stream of the kernels orders its first use too."""
    CALLS[call](stream=Stream(99) if handle == "stream" else 99)
    assert seen.allocated == [99]
    assert seen.called == [("iabn_" + call, seen.called[0][1], 99)]


@pytest.mark.parametrize("call", CALLS)
def test_the_callers_workspace_is_taken_as_it_is(seen, call):
    CALLS[call](stream=Stream(99), workspace=t(1 << 16, dtype=torch.uint8))
    assert seen.allocated == [] and seen.called[0][2] == 99


ALL = dict(CALLS)
ALL.update({
    "dropout": lambda **kw: iabn.iabn_dropout(t(4, 16), t(4, 16), 0.1, 1, **kw),
    "resnorm_forward": lambda **kw: iabn.iabn_resnorm_forward(t(4, 16), None, t(4, 16), None, **kw),
    "forward_train_noalloc": lambda **kw: iabn.iabn_forward_train_noalloc(t(2, 3, 4), *[t(3)] * 6, **kw),
    "forward_eval": lambda **kw: iabn.iabn_forward_eval(t(2, 3, 4), *[t(3)] * 4, **kw),
    "backward_ii": lambda **kw: iabn.iabn_backward_ii(t(2, 3, 4), t(2, 3, 4), *[t(3)] * 5, **kw),
    "std_forward_train": lambda **kw: iabn.iabn_std_forward_train(t(2, 3, 4), t(2, 3, 4), *[t(3)] * 6, **kw),
    "std_backward": lambda **kw: iabn.iabn_std_backward(*[t(2, 3, 4)] * 3, *[t(3)] * 6, **kw),
    "ckpt_forward_train": lambda **kw: iabn.iabn_ckpt_forward_train(t(2, 3, 4), t(2, 3, 4), *[t(3)] * 6, **kw),
    "ckpt_recompute": lambda **kw: iabn.iabn_ckpt_recompute(t(2, 3, 4), t(2, 3, 4), t(3), t(3), **kw),
    "ckpt_backward": lambda **kw: iabn.iabn_ckpt_backward(t(2, 3, 4), t(2, 3, 4), *[t(3)] * 5, **kw),
    "forward_stats": lambda **kw: iabn.iabn_forward_stats(t(2, 3, 4), t(4096), **kw),
    "forward_apply": lambda **kw: iabn.iabn_forward_apply(t(2, 3, 4), *[t(3)] * 6, 1e-5, 0.1, 0.01, t(4096), **kw),
    "backward_reduce": lambda **kw: iabn.iabn_backward_reduce(*[t(2, 3, 4)] * 2, t(3), t(3), 0.01, t(4096), **kw),
    "backward_apply": lambda **kw: iabn.iabn_backward_apply(*[t(2, 3, 4)] * 2, *[t(3)] * 5, 1e-5, 0.01, t(4096), **kw),
})


def test_every_entry_point_is_here():
    on_a_stream = {n[len("iabn_"):] for n in iabn.__all__
                   if n.startswith("iabn_") and not n.endswith(("_size", "_string", "version", "plan"))}
    assert on_a_stream == set(ALL)


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("stream", [None, 0, 99])
def test_the_tensors_device_is_current(seen, call, stream):
    """The default stream has one handle for every device (NULL), which means
    the current one's."""
    ALL[call](stream=stream)
    assert seen.called == [("iabn_" + call, DEVICE, {None: 7, 0: None, 99: 99}[stream])]
    assert seen.device is None


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("stream", [None, 7])
def test_the_current_stream_is_not_changed_for_itself(seen, call, stream, monkeypatch):
    monkeypatch.setattr(torch.cuda, "stream", None)
    CALLS[call](stream=stream)
    assert len(seen.allocated) == 1 and seen.called[0][2] == 7


def test_a_device_that_is_current_is_not_set(seen, monkeypatch):
    monkeypatch.setattr(torch.cuda, "device", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: DEVICE.index)
    for name, call in ALL.items():
        seen.called.clear()
        call(stream=99)
        assert seen.called == [("iabn_" + name, None, 99)]
