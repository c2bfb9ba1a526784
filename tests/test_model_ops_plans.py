"""CPU models of two splits that the kernels around the linear layers make on the host: who
fills which rows of a gradient table with zeros, and the order of the group norm's tiles by
XCD. Each follows the source step by step."""

import random

import numpy as np
import pytest


def ceil_div(a, b):
    return -(-a // b)


def fill_split(V, d, N):
    """launch_embedding_sum without accumulate: (first row that the sort's launch fills,
    entries that it fills, workgroups of the rows that the sum's launch looks through)."""
    fill_rows = ((30 << 20) + 1800 * N) // (4 * d)
    filled = ceil_div(V - fill_rows, 4) * 4 if fill_rows < V else 0
    if filled >= V:
        return V, 0, ceil_div(V, 64)
    return filled, (V - filled) * d, ceil_div(filled, 64)


def test_every_row_is_filled_by_one_launch():
    rng = random.Random(3)
    sizes = [(50257, 768, 32768), (50257, 257, 55), (200003, 90, 55), (1, 1, 1), (7, 1 << 20, 1),
             (8, 1 << 20, 1), (9, 1 << 20, 1), (131100, 16, 270)]
    for _ in range(3000):
        d = int(2 ** rng.uniform(0, 20))
        edge = ((30 << 20) + 1800) // (4 * d)     # tables around what one launch fills
        V = max(1, rng.choice([edge + rng.randint(-9, 9), int(2 ** rng.uniform(0, 22))]))
        sizes.append((V, d, rng.choice([1, int(2 ** rng.uniform(0, 16))])))
    both = 0
    for V, d, N in sizes:
        filled, n_zeros, row_wgs = fill_split(V, d, N)
        assert 0 <= filled <= V and n_zeros == (V - filled) * d
        assert filled * d % 4 == 0 or n_zeros == 0       # 16-byte stores from there on
        assert row_wgs * 64 >= filled > (row_wgs - 1) * 64 or filled == row_wgs == 0
        both += 0 < filled < V
    assert both > 100


@pytest.mark.parametrize("n_zeros", [1, 3, 4, 5, 1024 * 16 - 1, 1024 * 16 + 1, 1024 * 64 + 7, 300000])
def test_the_sorts_workgroups_fill_every_entry_once(n_zeros):
    buckets, threads = 4, 1024
    fill = min(ceil_div(n_zeros, 16 * threads), 256)
    seen = np.zeros(n_zeros, dtype=int)
    for wg in range(buckets, buckets + fill):
        first = (wg - buckets) * threads + np.arange(threads)
        for start in range(0, ceil_div(n_zeros >> 2, fill * threads) * fill * threads, fill * threads):
            k = first + start
            k = k[k < n_zeros >> 2]
            for c in range(4):
                seen[4 * k + c] += 1
        tail = first[first < n_zeros & 3]
        seen[(n_zeros & ~3) + tail] += 1
    assert np.all(seen == 1)


@pytest.mark.parametrize("B", [64, 65, 67, 71, 72, 100, 256])
@pytest.mark.parametrize("blocks", [2, 3, 4, 16])
def test_tiles_by_xcd_are_every_tile_once(B, blocks):
    grid, seen = ceil_div(B, 8) * 8 * blocks, {}
    for w in range(grid):
        i = w // 8
        b, rest = i // blocks * 8 + w % 8, i % blocks
        if b >= B:
            continue   # the whole workgroup ends
        assert (b, rest) not in seen
        seen[b, rest] = w % 8
    assert len(seen) == B * blocks
    for b in range(B):   # the tiles of an example, which share lines, on one XCD
        assert len({seen[b, k] for k in range(blocks)}) == 1
