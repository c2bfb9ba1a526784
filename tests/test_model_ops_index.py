"""CPU models of the index arithmetic around the linear layers' kernels: the buckets of
the token sort, the parts of an example's sorted tokens and how they are joined, the
chunks of the sorted list and theirs, and the tiles of the group norm. Each model follows
the kernel step by step with small sizes in place of the kernel's constants."""

import random

import numpy as np
import pytest


def ceil_div(a, b):
    return -(-a // b)


def buckets(n, most_wgs=256, most_keys=512):
    log = 0
    while (1 << log) < n and ((1 << log) < most_wgs or n > most_keys << log):
        log += 1
    return log, ceil_div(n, 1 << log)


@pytest.mark.parametrize("n", [1, 2, 3, 255, 256, 257, 1000, 50257, 131072, 131073, 200003])
def test_every_key_has_a_slot_of_its_own(n):
    log, R = buckets(n)
    keys = np.arange(n)
    slot = (keys & ((1 << log) - 1)) * R + (keys >> log)
    assert R <= 512 and len(np.unique(slot)) == n and slot.max() < R << log


def test_waves_of_the_sort_cover_the_list():
    for N in list(range(1, 300)) + [1024, 24504, 32768, 65537]:
        groups = (N >> 6) + ((N & 63) != 0)
        per = ceil_div(groups, 16)
        seen = 0
        for wave in range(16):
            first = min(per * wave, groups)
            last = min(first + per, groups)
            end = N if last == groups else last << 6
            assert first << 6 == seen or first == last
            seen = max(seen, end) if first < last else seen
        assert seen == N


def squares_of_groups(ids, n_rows, G, wgs, parts):
    """norm_kernel: shares of a list by workgroup (cut at groups), parts of a share (cut
    anywhere), edges joined."""
    order = sorted((v, t) for t, v in enumerate(ids) if 0 <= v < n_rows)
    tok, n, d = [v for v, _ in order], len(order), G.shape[1]

    def start(s):
        if s <= 0 or s >= n:
            return 0 if s <= 0 else n
        if tok[s] != tok[s - 1]:
            return s
        lo, hi = s, n
        while hi - lo > 1:
            mid = lo + (hi - lo) // 2
            lo, hi = (mid, hi) if tok[mid] == tok[s - 1] else (lo, mid)
        return hi

    of_wg, total, seen = ceil_div(n, wgs), 0.0, 0
    for wg in range(wgs):
        S = 0 if wgs == 1 else start(min(of_wg * wg, n))
        E = n if wgs == 1 or n - of_wg * wg <= of_wg else start(of_wg * (wg + 1))
        assert S == seen
        seen = E
        of_part = ceil_div(E - S, parts)

        def cut(q):
            return E if E - S - q * of_part < 0 else S + q * of_part

        heads, tails = [None] * parts, [None] * parts
        for q in range(parts):
            s, e, acc, first = cut(q), cut(q + 1), np.zeros(d), True
            for k in range(s, e):
                if k > s and tok[k] != tok[k - 1]:
                    if first:
                        heads[q], first = acc, False
                    else:
                        total += acc @ acc
                    acc = np.zeros(d)
                acc = acc + G[order[k][1]]
            if first:
                heads[q] = acc
            else:
                tails[q] = acc
        acc = np.zeros(d)
        for q in range(parts):
            s, e = cut(q), cut(q + 1)
            if s >= e:
                assert all(cut(r) >= cut(r + 1) for r in range(q, parts))
                break
            if not (s > S and tok[s] == tok[s - 1]):
                total += acc @ acc
                acc = np.zeros(d)
            acc = acc + heads[q]
            if tok[s] != tok[e - 1]:
                total += acc @ acc
                acc = tails[q]
        total += acc @ acc
    assert seen == n
    return total


@pytest.mark.parametrize("seed", range(30))
def test_parts_of_an_example_join_to_whole_groups(seed):
    rng = np.random.default_rng(seed)
    T, V = int(rng.integers(1, 90)), int(rng.choice([1, 2, 5, 40]))
    ids, G = rng.integers(-1, V + 1, T), rng.standard_normal((T, 3))
    ref = sum(float(np.sum(np.sum(G[ids == v], axis=0) ** 2)) for v in range(V))
    for wgs in (1, 2, 5, 9):
        for parts in (1, 2, 7, 16):
            assert abs(squares_of_groups(list(ids), V, G, wgs, parts) - ref) < 1e-9


def sums_by_chunks(toks, G, N, V, chunk):
    """sum_kernel and join_kernel over a sorted list of tokens (of N positions)."""
    total = len(toks)
    offsets = np.concatenate([[0], np.cumsum([toks.count(v) for v in range(V)])])
    grad, partial = [None if offsets[v] < offsets[v + 1] else 0.0 for v in range(V)], {}
    n_chunks = ceil_div(N, chunk)

    def write(v, x):
        assert grad[v] is None   # each row exactly once
        grad[v] = x

    for q in range(n_chunks):
        s = q * chunk
        if s >= total:
            continue
        n = min(chunk, total - s)
        lane = [toks[s - 1 + l] if l <= n + 1 and 0 <= s - 1 + l < total else -1 for l in range(chunk + 2)]
        starts = [l == 0 or lane[l] != lane[l - 1] for l in range(chunk + 2)]
        opened, acc = not starts[1], 0.0
        for j in range(1, n + 1):
            if j > 1 and starts[j]:
                if opened:
                    partial[q, 0] = acc
                else:
                    write(lane[j - 1], acc)
                opened, acc = False, 0.0
            acc += G[s + j - 1]
        if not opened and starts[n + 1]:
            write(lane[n], acc)
        else:
            partial[q, 0 if opened else 1] = acc
    if n_chunks > 1:
        for q in range(n_chunks):
            s = q * chunk
            if total - s <= chunk:
                continue
            v = toks[s + chunk - 1]
            if offsets[v] < s or offsets[v + 1] <= s + chunk:
                continue
            n = (offsets[v + 1] - 1) // chunk - q + 1
            write(v, sum(partial[q + k, 1 if k == 0 else 0] for k in range(n)))
    return grad


@pytest.mark.parametrize("seed", range(40))
def test_chunks_join_to_whole_rows(seed):
    rng = random.Random(seed)
    for _ in range(40):
        V, N = rng.choice([1, 2, 3, 10, 50]), rng.randint(1, 120)
        toks = sorted(rng.randrange(V) for _ in range(rng.randint(0, N)))
        G = [rng.random() for _ in toks]
        got = sums_by_chunks(toks, G, N, V, 8)
        for v in range(V):
            assert abs(got[v] - sum(g for g, t in zip(G, toks) if t == v)) < 1e-9


def tile_plan(B, S, C, groups, elem, rows):
    """plan_of: (whole, vector, units, lanes, blocks, threads, chunks, rows, segs)."""
    V = next(v for v in (4, 2, 1) if C % v == 0)
    width = C // groups
    for row_bytes in (128, 64):
        least = width
        while least % V:
            least += width
        cb = min(C, least * ceil_div(row_bytes, least * elem))
        units = ceil_div(cb, V)
        if units > 1024:
            continue
        lanes = 1 << (units - 1).bit_length()
        if ceil_div(S, 1024 // lanes) > rows:
            continue
        threads = min(1024, ceil_div(lanes * S, 64) * 64)
        return True, V, units, lanes, ceil_div(C, cb), threads, 1, S, cb // width
    total = C // V
    most = (128 if C * elem % 128 == 0 else 256) // (V * elem)
    while most * S < 256:
        most *= 2
    units = min(total, most)
    blocks = ceil_div(total, units)
    lanes = 1 << (units - 1).bit_length()
    assert lanes <= 256
    of_tile = min(S, rows * (256 // lanes))
    return False, V, units, lanes, blocks, 256, ceil_div(S, of_tile), of_tile, units * V // width + 2


@pytest.mark.parametrize("elem,rows", [(4, 8), (2, 16), (2, 8)])
def test_group_norm_tiles_cover_every_value_once(elem, rows):
    rng = random.Random(5)
    cases = [(1, 1, 64, 1), (2, 1024, 64, 16), (1, 3000, 16, 16), (5, 7, 33, 11), (1, 17, 1032, 8),
             (1, 2048, 320, 32), (2, 3, 4100, 1), (1, 9, 2051, 1), (1, 40, 6200, 2), (1, 100, 8197, 7),
             (2, 16384, 320, 32), (1, 70000, 4, 2), (1, 1, 8200, 1), (3, 2, 5001, 1), (2, 2100, 324, 27)]
    for _ in range(300):
        width, groups = rng.choice([1, 2, 3, 4, 9, 10, 32, 77]), rng.choice([1, 2, 5, 16])
        cases.append((1, rng.randint(1, 3000), width * groups, groups))
    for B, S, C, groups in cases:
        whole, V, units, lanes, blocks, threads, chunks, of_tile, segs = tile_plan(B, S, C, groups, elem, rows)
        width, step = C // groups, threads // lanes
        assert units <= lanes <= 1024 and threads % 64 == 0 and step * lanes == threads
        assert ceil_div(of_tile, step) <= rows            # a thread's rows fit its registers
        assert (chunks - 1) * of_tile < S <= chunks * of_tile
        slots = threads >> 6 if lanes < 64 else step
        assert (2 * slots * units * V + 2 * units * V + 2 * segs) * 4 < 100000   # LDS
        covered = 0
        for blk in range(blocks):
            c0, c1 = blk * units * V, min(C, (blk + 1) * units * V)
            first, here = c0 // width, (c1 - 1) // width - c0 // width + 1
            assert c0 < C and here <= segs
            if whole:
                assert c0 % width == 0 and c1 % width == 0
            covered += c1 - c0
        assert covered == C
