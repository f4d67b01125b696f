"""How the gated block's products are cut, on the host: every tile that the
library has an instance of is one that some product takes, and every tile that a
product takes has its instance."""

from __future__ import annotations

import ctypes
import random
import re
import shutil
import subprocess

import pytest

import paper_1712_02616_amd as iabn

DTYPES = {"f32": 0, "f16": 1, "bf16": 2}
KINDS = ("up", "down", "dh", "dx", "dw")  # GemmKind
TILES = ((256, 256), (128, 128), (64, 128), (32, 128))  # TileSize


def planner():
    """(dtype, kind, direct, M, N, K, products) -> (tile, splits); the library's
    own function, which its C interface does not name."""
    fn = getattr(iabn.load(), "_ZN9iabn_impl9plan_gemmEiNS_8GemmKindEbllli")
    fn.restype = ctypes.c_uint64  # two 32-bit values
    fn.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_bool] + [ctypes.c_int64] * 3 + [ctypes.c_int]

    def plan(dtype, kind, direct, M, N, K, products=1):
        v = fn(DTYPES[dtype], KINDS.index(kind), direct, M, N, K, products)
        return TILES[v & 0xFFFFFFFF], v >> 32

    return plan


def fetchable(dtype, ld, row):
    """Whether an operand goes straight to LDS (of tensors at their allocation's start)."""
    size = 4 if dtype == "f32" else 2
    return row >= 16 // size and ld * size % 4 == 0 and ld * size * 256 < 1 << 31


def products(plan, dtype, M, C, F):
    """What a forward and a backward of [M, C] and [F, C] run on the tiles:
    (kind, direct, tile, split) of each product."""
    out = []
    for kind, (m, n, k), count, rows in (("up", (M, F, C), 1, (C, C)), ("down", (M, C, F), 1, (F, F)),
                                         ("dh", (M, F, C), 1, (C, F)), ("dw", (C, F, M), 1, (C, F)),
                                         ("dw", (F, C, M), 2, (F, C)), ("dx", (M, C, F), 1, (F, C))):
        if M <= 64 and kind in ("up", "down"):
            continue  # a kernel of its own
        direct = all(fetchable(dtype, r, r) for r in rows)
        tile, splits = plan(dtype, kind, direct, m, n, k, count)
        out.append((kind, direct, tile, splits > 1))
    return out


def scan():
    plan, rnd = planner(), random.Random(5)
    seen = set()
    for _ in range(60000):
        dtype, kind, direct = rnd.choice(["f32", "f16", "bf16"]), rnd.choice(KINDS), rnd.random() < 0.5
        top = rnd.choice([8, 13, 20])
        M, N, K = (int(2 ** rnd.uniform(0, top)) for _ in range(3))
        seen.add((dtype, kind, direct, plan(dtype, kind, direct, M, N, K)[0]))
    return seen


@pytest.mark.skipif(shutil.which("nm") is None, reason="needs nm")
def test_instances_are_the_tiles_that_are_chosen():
    names = subprocess.run(["nm", "-C", iabn.library_path()], capture_output=True, text=True, check=True).stdout
    have = set()
    for m in re.finditer(r"__device_stub__gemm_kernel<(\d), (\d), (\d+), (\d+), \d, \d, (true|false)>", names):
        dt, kind, tm, tn = (int(m.group(i)) for i in range(1, 5))
        have.add((list(DTYPES)[dt], KINDS[kind], m.group(5) == "true", (tm, tn)))
    assert have == scan()


# Ragged sizes whose products take every instance of the tiles, with split sums
# and without where both occur (test_gpu_ffn_tiles.py runs them).
SIZES = [
    ("bf16", 65, 1, 1), ("bf16", 65, 2, 4236), ("bf16", 65, 7, 341), ("bf16", 65, 10, 386), ("bf16", 235, 646, 4824),
    ("bf16", 891, 78, 88), ("bf16", 1748, 2352, 8956), ("bf16", 2101, 4, 729), ("bf16", 2712, 770, 5674),
    ("bf16", 5384, 1170, 12), ("bf16", 7063, 152, 1544), ("bf16", 8239, 1524, 796), ("bf16", 9614, 2, 2),
    ("f16", 65, 1, 1), ("f16", 65, 1, 335), ("f16", 65, 8, 454), ("f16", 249, 2, 1040), ("f16", 321, 226, 3955),
    ("f16", 510, 442, 6692), ("f16", 836, 76, 66), ("f16", 1745, 3068, 2328), ("f16", 4258, 10, 5700),
    ("f16", 4629, 2662, 2896), ("f16", 8618, 1, 2), ("f16", 9372, 324, 704), ("f32", 65, 2, 4232),
    ("f32", 219, 134, 94), ("f32", 612, 640, 5830), ("f32", 709, 1, 734), ("f32", 1338, 516, 2), ("f32", 5657, 10, 7762),
    ("f32", 7247, 30, 9706), ("f32", 7928, 398, 1004), ("f32", 8720, 798, 188), ("f32", 9431, 2, 2)]


def test_sizes_take_every_instance():
    plan = planner()
    taken = {(size[0],) + p for size in SIZES for p in products(plan, *size)}
    assert {t[:4] for t in taken} == scan()
    # The products that may split their sum do both, where their tiles do at all.
    for dtype in DTYPES:
        for kind in ("down", "dx", "dw"):
            for direct, tile in ((True, (128, 128)), (True, (64, 128)), (True, (32, 128))):
                assert {t[4] for t in taken if t[:4] == (dtype, kind, direct, tile)} == {False, True}
