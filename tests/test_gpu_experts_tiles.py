"""Every instance of the matrix kernel over groups, against the definition in 64
bits: the sizes that test_routed_plan.py counts, and few tokens at every number of
rows that its kernels tell apart."""

from __future__ import annotations

import pytest
import torch

from test_gpu_experts import run_case
from test_routed_plan import SIZES

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]


@pytest.mark.parametrize("dtype,M,k,E,C,F", SIZES)
def test_every_instance(dtype, M, k, E, C, F):
    run_case(M, min(k, E), E, C, F, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,k,E", [(56, 1, 7), (56, 2, 7), (56, 2, 2), (56, 8, 8), (55, 3, 64), (17, 1, 1), (33, 2, 2)])
def test_few_tokens(M, k, E, dtype):
    """One, two and four tiles of 16 rows; more rows than a block takes (one expert
    for every slot)."""
    run_case(M, k, E, 264, 136, dtype)
    run_case(M, k, E, 200, 520, dtype, choice="0")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,F", [(1, 40, 4104), (7, 33, 3001), (30, 64, 8192)])
def test_few_tokens_long_sums(M, C, F, dtype):
    """Few columns and a long sum, which is split over blocks."""
    run_case(M, 2, 3, C, F, dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows", [1, 64, 127, 128, 129, 255, 256, 257, 384, 385, 513])
def test_rows_about_a_tile(rows, dtype):
    """One expert of as many rows: the largest tile's halves, by a long list of others."""
    M = 4096
    experts = torch.arange(M) % 16 + 1
    experts[:rows] = 0
    import test_gpu_experts as t

    real = t.inputs

    def inputs(*a, **kw):
        i, _, w = real(*a, **kw)
        return i, experts[torch.randperm(M, generator=torch.Generator().manual_seed(rows))][:, None], w

    t.inputs = inputs
    try:
        run_case(M, 1, 17, 520, 264, dtype)
    finally:
        t.inputs = real
