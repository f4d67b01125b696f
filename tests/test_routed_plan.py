"""How the routed experts' products are cut, on the host: every instance of the
matrix kernel over groups is one that some product takes, and the sizes that
test_gpu_experts_tiles.py runs take them all."""

from __future__ import annotations

import ctypes
import random
import re
import shutil
import subprocess

import pytest

import paper_1712_02616_amd as iabn

DTYPES = {"f32": 0, "f16": 1, "bf16": 2}
# GemmKind over groups, dW by the operand that is gathered: x (dy, of the down
# projection's) or y (x, of the gate's and the up projection's).
KINDS = {10: "up", 11: "down", 12: "dh", 13: "dx", 14: "dw_x", 15: "dw_y"}
TILES = ((256, 256), (128, 128), (64, 128), (32, 128))  # TileSize
FEW_TOKENS = 56


def planner():
    fn = getattr(iabn.load(), "_ZN9iabn_impl12plan_groupedEiNS_8GemmKindEbllllli")
    fn.restype = ctypes.c_int
    fn.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_bool] + [ctypes.c_int64] * 5 + [ctypes.c_int]
    return lambda dtype, kind, direct, P, E, M, N, K, products: TILES[
        fn(DTYPES[dtype], min(kind - 10, 4), direct, P, E, M, N, K, products)]


def fetchable(dtype, row, strided=False, tokens=0):
    """Whether an operand of rows of `row` goes straight to LDS (of tensors at their
    allocation's start; tokens: it is gathered)."""
    size = 4 if dtype == "f32" else 2
    whole = row % (16 // size) == 0
    return row >= 16 // size and row * size % 4 == 0 and (not tokens or not strided or whole)


def products(plan, dtype, M, k, E, C, F):
    """(kind, direct, tile) of each product of a forward and a backward."""
    P, out = M * k, []
    for kind, x, y, (m, n, kk), count in (
            (10, fetchable(dtype, C, False, M), fetchable(dtype, C), (P, F, C), 1),
            (11, fetchable(dtype, F), fetchable(dtype, F), (P, C, F), 1),
            (12, fetchable(dtype, C, False, M), fetchable(dtype, F, True), (P, F, C), 1),
            (13, fetchable(dtype, F), fetchable(dtype, C, True), (P, C, F), 1),
            (14, fetchable(dtype, C, True, M), fetchable(dtype, F, True), (C, F, P), 1),
            (15, fetchable(dtype, F, True), fetchable(dtype, C, True, M), (F, C, P), 2)):
        if M <= FEW_TOKENS and kind in (10, 11):
            continue  # a kernel of its own
        out.append((KINDS[kind], x and y, plan(dtype, kind, x and y, P, E, m, n, kk, count)))
    return out


def scan():
    plan, rnd = planner(), random.Random(7)
    seen = set()
    for _ in range(60000):
        kind, dtype, direct = rnd.choice(list(KINDS)), rnd.choice(list(DTYPES)), rnd.random() < 0.5
        E, k = int(2 ** rnd.uniform(0, 10)), int(2 ** rnd.uniform(0, 4))
        M, C, F = int(2 ** rnd.uniform(0, 17)), int(2 ** rnd.uniform(0, 13)), int(2 ** rnd.uniform(0, 13))
        P = M * k
        m, n, kk, count = {10: (P, F, C, 1), 11: (P, C, F, 1), 12: (P, F, C, 1), 13: (P, C, F, 1), 14: (C, F, P, 1),
                           15: (F, C, P, 2)}[kind]
        seen.add((dtype, KINDS[kind], direct, plan(dtype, kind, direct, P, E, m, n, kk, count)))
    return seen


@pytest.mark.skipif(shutil.which("nm") is None, reason="needs nm")
def test_instances_are_the_tiles_that_are_chosen():
    names = subprocess.run(["nm", "-C", iabn.library_path()], capture_output=True, text=True, check=True).stdout
    have = set()
    for m in re.finditer(r"__device_stub__gemm_kernel<(\d), (1\d), (\d+), (\d+), \d, \d, (true|false)>", names):
        have.add((list(DTYPES)[int(m.group(1))], KINDS[int(m.group(2))], m.group(5) == "true",
                  (int(m.group(3)), int(m.group(4)))))
    assert have == scan()


# Ragged sizes (type, M, k, E, C, F) whose products take every instance.
SIZES = [
    ("bf16", 1, 6, 35, 1400, 8), ("bf16", 2, 1, 50, 40, 504), ("bf16", 59, 1, 1, 1, 2), ("bf16", 61, 1, 1, 8, 8),
    ("bf16", 1441, 4, 3, 2808, 8), ("bf16", 1686, 6, 13, 1, 344), ("bf16", 3654, 7, 3, 386, 218),
    ("bf16", 3715, 2, 50, 1112, 224), ("bf16", 3892, 3, 31, 268, 2), ("bf16", 6972, 4, 62, 8, 72),
    ("bf16", 7092, 7, 5, 80, 8), ("bf16", 4067, 1, 3, 184, 4008), ("f16", 17, 2, 17, 72, 3456), ("f16", 57, 1, 1, 8, 8),
    ("f16", 141, 1, 1, 1, 1), ("f16", 161, 2, 5, 2481, 1), ("f16", 682, 4, 14, 392, 2088), ("f16", 1373, 6, 15, 648, 8),
    ("f16", 1505, 3, 24, 2784, 8), ("f16", 3777, 4, 38, 1, 154), ("f16", 3919, 2, 39, 8, 348),
    ("f16", 6777, 4, 28, 405, 198), ("f16", 7341, 7, 19, 72, 8), ("f16", 4067, 1, 3, 184, 4008),
    ("f32", 5, 2, 30, 856, 40), ("f32", 60, 2, 3, 1, 1), ("f32", 66, 1, 14, 4, 2234), ("f32", 69, 2, 3, 4, 4),
    ("f32", 313, 3, 55, 1132, 4), ("f32", 2299, 7, 1, 4, 512), ("f32", 2639, 3, 23, 1, 1), ("f32", 6702, 4, 5, 6, 4),
    ("f32", 6914, 6, 34, 3, 125), ("f32", 7035, 2, 33, 401, 6)]


def test_sizes_take_every_instance():
    plan = planner()
    taken = {(size[0],) + p for size in SIZES for p in products(plan, *size)}
    assert taken == scan(), (scan() - taken, taken - scan())
