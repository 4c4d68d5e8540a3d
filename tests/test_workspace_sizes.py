"""A workspace for the largest call does for the smaller ones: its size never falls as a call grows, also where a larger call is
computed in another way that needs none."""
import ctypes as C
import random

import pytest

from paper_2206_07882_amd import qrnnt


def rising(sizes):
    return all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("W,V,n", [(32, 1000, 32), (25, 513, 1), (64, 2048, 64), (24, 2048, 24), (25, 2049, 5), (1, 131072, 8), (64, 512, 64)])
def test_beam_select_over_batches(W, V, n):
    sizes = [qrnnt.beam_select_workspace(B, W, V, n) for B in range(0, 130)]
    assert sizes[0] > 0 and rising(sizes)


def test_beam_select_over_every_size():
    rng = random.Random(1)
    largest = (1 << 21, 64, 1 << 30, 64)
    for _ in range(300):
        sizes = [rng.choice([1, 2, 33, 1000]), rng.randint(1, 64), rng.choice([1, 500, 512, 513, 1000, 2048, 2049, 16384, 16385, 1 << 20, 33558528]), rng.randint(1, 64)]
        at = rng.randrange(4)
        values = sorted({min(largest[at], max(1, int(sizes[at] * f))) for f in (0.5, 0.9, 0.999, 1, 1.0001, 1.001, 1.1, 2, 7)})
        got = []
        for v in values:
            sizes[at] = v
            if sizes[1] * sizes[2] < 1 << 31:
                got.append(qrnnt.beam_select_workspace(*sizes))
        assert all(got) and rising(got), sizes


def linear(rows, cols, M):
    w = qrnnt.CQMat(0x1000, 0x2000, rows, cols, qrnnt.LAYOUT_TILED, 8)
    return qrnnt.load().qrnnt_linear_tokens_workspace(C.byref(w), M)


@pytest.mark.parametrize("rows,cols", [(1024, 4096), (8192, 8192), (4096, 4096), (1024, 8192), (64, 131071), (32000, 1024), (1000, 1283), (5000, 2048)])
def test_linear_tokens_over_tokens(rows, cols):
    sizes = [linear(rows, cols, M) for M in list(range(1, 1200)) + list(range(1200, 60000, 97)) + [1 << 20, 1 << 28]]
    assert rising(sizes) and sizes[0] == 0
    assert all(size <= 512 * 128 * 4 * ((cols + 127) // 128) for size in sizes)


def test_linear_tokens_over_every_size():
    rng = random.Random(2)
    for _ in range(2000):
        sizes = [int(16 * 2000 ** rng.random()), int(40 * 200 ** rng.random()), int(17 * 2000 ** rng.random())]
        got = []
        for f in (0.3, 0.5, 0.9, 0.99, 1, 1.01, 1.1, 2, 10):
            got.append(linear(sizes[0], sizes[1], max(1, int(sizes[2] * f))))
        assert rising(got), sizes
