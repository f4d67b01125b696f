"""iabn_grad_clip refuses an output that overlaps what the call reads: elements would be
scaled twice, or be another tensor's, by which block runs first (CPU only; skipped
where a GPU is visible, as test_abi.py)."""

from __future__ import annotations

import ctypes

import pytest

from test_sublayer_abi import BF16, ERR_PARAM, F32, OK, P, lib, no_gpu, refused  # noqa: F401

AT = 1 << 20


def clip(lib, tensors, norm=P, dtype=F32):  # noqa: F811
    """tensors: (gradient, output, elements)."""
    n = len(tensors)
    ins, outs = ((ctypes.c_void_p * n)(*[t[q] for t in tensors]) for q in (0, 1))
    return lib.iabn_grad_clip(ins, outs, (ctypes.c_int * n)(*[dtype] * n), (ctypes.c_int64 * n)(*[t[2] for t in tensors]),
                              n, norm, 1.0, None)


# Tensors that do not overlap, more than a launch takes.
MANY = [(AT * 64 + 256 * i, AT * 128 + 256 * i, 32) for i in range(300)]


@no_gpu
@pytest.mark.parametrize("tensors", [
    [(AT, 2 * AT, 8), (2 * AT, AT, 8)],                         # two that swap places
    [(AT, AT + 4, 8)], [(AT + 4, AT, 8)],                       # its own, an element on
    [(AT, AT + 28, 8)], [(AT + 28, AT, 8)],                     # by one element
    [(AT, AT, 8), (AT + 16, 2 * AT, 4)],                        # read by one, in place in another
    [(AT, 3 * AT, 8), (AT + 64, AT + 31, 1)],
    MANY + [(AT * 128 + 256 * 17 + 124, AT, 1)], MANY + [(AT, AT * 64 + 256 * 299 + 124, 1)],
    [(AT, 2 * AT, 0), (3 * AT, 4 * AT, 8), (4 * AT - 4, 5 * AT, 2)]])
def test_refuses_an_output_over_a_gradient(lib, tensors):  # noqa: F811
    refused(lib, ERR_PARAM, clip(lib, tensors))


@no_gpu
def test_refuses_the_norm_among_the_outputs(lib):  # noqa: F811
    for at in (AT, AT + 28, AT - 2):
        refused(lib, ERR_PARAM, clip(lib, [(2 * AT, AT, 8)], norm=ctypes.c_void_p(at)))
        refused(lib, ERR_PARAM, clip(lib, [(AT, AT, 8)], norm=ctypes.c_void_p(at)))


@no_gpu
def test_takes_what_does_not_overlap(lib):  # noqa: F811
    """These pass the checks (their launch then fails, as there is no GPU)."""
    for tensors in ([(AT, AT, 8), (AT + 32, AT + 32, 8)], [(AT, AT + 32, 8)], [(AT + 32, AT, 8)],
                    [(AT, 2 * AT, 8), (AT, 3 * AT, 8)], MANY, [(AT, 2 * AT, 0), (2 * AT, AT, 0)]):
        assert clip(lib, tensors) != ERR_PARAM
        assert clip(lib, tensors, norm=ctypes.c_void_p(AT * 4 - 4)) != ERR_PARAM
    # (16-bit types: half the bytes.)
    assert clip(lib, [(AT, AT + 16, 8)], dtype=BF16) != ERR_PARAM
    refused(lib, ERR_PARAM, clip(lib, [(AT, AT + 14, 8)], dtype=BF16))
    assert clip(lib, [(AT, AT + 4, 0)]) == OK
