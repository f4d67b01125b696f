"""The sublayer's entry points on the host at the ends of their ranges (CPU)."""

from __future__ import annotations

import ctypes

import pytest
import torch

import paper_1712_02616_amd as iabn


@pytest.fixture(scope="module")
def lib():
    return iabn.load()


def test_resnorm_workspace_grows_with_very_many_rows(lib):
    """A block adds at most 1024 rows (4096 of those that are one wave's), and the
    sizes stay whole at the largest number of rows."""
    size = lib.iabn_resnorm_workspace_size
    for R, C, rows in ((1 << 24, 8, 4096), (1 << 22, 512, 4096), (1 << 22, 520, 1024), (1 << 22, 16384, 1024)):
        assert size(R, C, 0) >= 5 * 4 * C * (R // rows)
        assert size(R, C, 1 << 10) >= 5 * 4 * C * (R // rows)
    for groups in (0, 1, 1 << 20, 1 << 45, 1 << 46):
        assert 0 < size(1 << 46, 1, groups) <= 5 * 4 * (1 << 22)


NO_GPU = pytest.mark.skipif(torch.cuda.is_available(), reason="placeholder pointers are only safe without a GPU")
P = ctypes.c_void_p(4096)  # a pointer that nothing may follow


@NO_GPU
def test_no_rows_with_a_gate_per_row(lib):
    """A gate of R rows has none where R is 0; any other number of rows divides 0."""
    for groups in (0, 1, 7):
        assert lib.iabn_resnorm_forward(P, P, P, P, 1, P, groups, 1, None, None, 1, None, None, None, None, 1.0, 1.0,
                                        1e-5, 0.0, 0, 0, 0, 64, None) == 0, lib.iabn_last_error()
    # (It goes on to its launches, of which there are none here, and finds no device: 6.)
    assert lib.iabn_resnorm_backward(P, P, P, P, None, None, 1, P, 0, 1, None, None, 1, None, P, P, P, None, None, None,
                                     None, 1.0, 1.0, 0.0, 0, 0, 0, 64, None, 0, None) in (0, 6), lib.iabn_last_error()
    for groups in (-1, 0, 3):
        assert lib.iabn_resnorm_forward(P, P, P, P, 1, P, groups, 1, None, None, 1, None, None, None, None, 1.0, 1.0,
                                        1e-5, 0.0, 0, 0, 4, 64, None) == 2
    assert lib.iabn_resnorm_forward(P, P, P, P, 1, P, -1, 1, None, None, 1, None, None, None, None, 1.0, 1.0,
                                    1e-5, 0.0, 0, 0, 0, 64, None) == 2
