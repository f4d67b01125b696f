"""The widest rows that iabn_dropout takes."""

from __future__ import annotations

import pytest
import torch

import paper_1712_02616_amd as iabn
import sublayer_oracle as oracle
from gpu_helpers import say

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a HIP GPU")]


@pytest.mark.parametrize("width", [2 ** 31 - 1, 2 ** 31 - 7, 2 ** 31 - 8])
def test_widest_rows(width):
    say("dropout 1 x %d" % width)
    x = torch.ones(1, width, dtype=torch.float16, device="cuda")
    iabn.iabn_dropout(x, x, 0.5, 77, 3)
    for lo in (0, 2 ** 30 - 9, width - 40):
        got = x[0, lo:lo + 40].cpu()
        for i, v in enumerate(got.tolist()):
            col = lo + i
            w = oracle.philox([col // 8, 0, 3, 0], [77, 0])
            bits = (w[col % 8 // 2] >> (16 * (col % 2))) & 0xFFFF
            assert v == (2.0 if bits >= 32768 else 0.0), col
    # Every element was written: kept or dropped, near half of each.
    kept = float((x == 2.0).sum(dtype=torch.int64)) / width
    assert float((x == 1.0).sum(dtype=torch.int64)) == 0 and abs(kept - 0.5) < 1e-3
