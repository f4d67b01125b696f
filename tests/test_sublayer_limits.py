"""The sublayer's entry points on the host at the ends of their ranges (CPU)."""

from __future__ import annotations

import pytest

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
