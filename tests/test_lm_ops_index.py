"""CPU models of the index arithmetic of the kernels between and behind the blocks: every
entry is read, and written, by exactly one thread, and nothing past a row's end is."""

import numpy as np
import pytest


def ceil_div(a, b):
    return -(-a // b)


# ------------------------------------------- rows of logits in a team's registers


def held(start, n, ve, nt, nvec):
    """Places (in the row) that each thread of a team has: vectors, and the one beside them.
    start: the row's first entry, counted from a 16-byte boundary."""
    head = min(-start % ve, n)
    vecs = (n - head) // ve
    tail = n - head - vecs * ve
    vectors, edges = [], []
    for tid in range(nt):
        for j in range(nvec):
            if tid < vecs - j * nt:
                at = head + j * nt * ve + tid * ve
                assert (start + at) % ve == 0          # on a boundary
                vectors.append(at)
        edge = tid if tid < head else (n - tail + tid - head if tid - head < tail else -1)
        if edge >= 0:
            edges.append(edge)
    return head, vecs, vectors, edges


@pytest.mark.parametrize("ve", [4, 8])
@pytest.mark.parametrize("nt,nvec", [(64, 4), (256, 4)])
def test_held_rows_are_covered_once(ve, nt, nvec):
    most = nt * nvec * ve
    rng = np.random.default_rng(ve + nt)
    sizes = list(range(1, 3 * ve)) + [most, most - 1, most - ve + 1] + rng.integers(1, most, 40).tolist()
    for n in sizes:
        for start in range(ve):
            _, vecs, vectors, edges = held(start, n, ve, nt, nvec)
            assert vecs <= nt * nvec
            seen = np.zeros(n, int)
            for at in vectors:
                assert 0 <= at and at + ve <= n
                seen[at:at + ve] += 1
            for at in edges:
                seen[at] += 1
            assert (seen == 1).all(), (n, start)


@pytest.mark.parametrize("ve", [4, 8])
def test_the_target_has_one_owner(ve):
    """Which thread and vector (or edge) adds the target's term."""
    nt, nvec, n = 64, 4, 777
    for start in range(ve):
        head, vecs, vectors, edges = held(start, n, ve, nt, nvec)
        for target in list(range(-3, 20)) + list(range(n - 20, n + 3)) + [333]:
            rel = target - head
            vec = rel // ve if 0 <= rel < vecs * ve else -1
            hits = [(tid, j) for tid in range(nt) for j in range(nvec)
                    if vec >= 0 and vec % nt == tid and vec // nt == j and tid < vecs - j * nt]
            in_vectors = any(at <= target < at + ve for at in vectors)
            assert len(hits) == (1 if in_vectors else 0)
            if hits:
                tid, j = hits[0]
                assert head + j * nt * ve + tid * ve + rel % ve == target
            assert (target in edges) == (0 <= target < n and not in_vectors)


@pytest.mark.parametrize("ve", [4, 8])
def test_one_pass_rows_are_covered_once(ve):
    """The pass that holds no entries: batches of four vectors, then single ones, then edges."""
    nt, batch = 64, 4
    for n in [1, 7, 100, 64 * ve * 4, 64 * ve * 4 + 5, 3001, 9999]:
        for start in range(ve):
            head = min(-start % ve, n)
            vecs = (n - head) // ve
            seen = np.zeros(vecs, int)
            for tid in range(nt):
                j = tid
                while j + (batch - 1) * nt < vecs:
                    for b in range(batch):
                        seen[j + b * nt] += 1
                    j += batch * nt
                while j < vecs:
                    seen[j] += 1
                    j += nt
            assert (seen == 1).all()


@pytest.mark.parametrize("most", [4096, 8192])
def test_parts_cover_a_row(most):
    for V in [most * 2 + 1, 32003, 50257, 131073, 300001, 1 << 24, (1 << 24) - 1]:
        n = ceil_div(V, most)
        size = ceil_div(ceil_div(V, n), 64) * 64
        parts = ceil_div(V, size)
        assert size <= most and parts * size >= V and (parts - 1) * size < V
        for target in (0, V - 1, V // 2, size - 1, size):
            p = target // size
            assert p < parts and p * size <= target < min(V, (p + 1) * size)


def test_joined_keys_are_read_once():
    """The order in which the parts' keys are taken: all best ones, all second ones, ..."""
    for n, k in [(7, 5), (32, 64), (1, 3), (300, 2)]:
        seen = np.zeros(n * k, int)
        ranks = []
        for i in range(n * k):
            r = i // n
            seen[(i - r * n) * k + r] += 1
            ranks.append(r)
        assert (seen == 1).all() and ranks == sorted(ranks)


def bound_of_groups(bits, k):
    """The kernel's bound, from the highest bit down to bit 16."""
    least = 0
    for bit in range(31, 15, -1):
        t = least | 1 << bit
        if (bits >= t).sum() >= k:
            least = t
    return least


def test_the_bound_keeps_the_k_largest():
    rng = np.random.default_rng(1)
    for k in (1, 5, 20, 64):
        for ties in (False, True):
            x = rng.standard_normal(4096).astype(np.float32)
            x = np.round(x * 4) / 4 if ties else x
            u = (x.astype(np.float32) + 0).view(np.uint32)
            order = np.where(u & 0x80000000, ~u, u | 0x80000000).astype(np.uint64)
            groups = order.reshape(256, 16).max(1)
            least = bound_of_groups(groups, k)
            assert (order >= least).sum() >= k
            if not ties:   # about 256 ln(256 / (256 - k)), and what 16 bits cannot tell apart
                assert (order >= least).sum() <= 256 * np.log(256 / (256 - k)) * 1.5 + 20


# ------------------------------------------------------------------ residual norms


def plan_rows(C, bf16, elements):
    V = next(v for v in ((8, 4, 2, 1) if bf16 else (4, 2, 1)) if C % v == 0)
    units = C // V
    nv = min(4, elements // V)
    while nv > 1 and units <= 64 * (nv // 2):
        nv //= 2
    while units > nv * 1024:
        nv *= 2
    log = 0
    while nv << log < units:
        log += 1
    threads = 256 if log <= 8 else 1 << log
    return V, nv, log, threads, threads >> log


CHANNELS = [1, 2, 3, 8, 30, 63, 64, 100, 250, 513, 768, 1024, 1032, 2051, 4096, 4100, 8192, 8200, 8191, 12289, 16382, 16383, 16384]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("elements", [8, 16])
def test_channels_of_a_row_are_covered_once(bf16, elements):
    for C in CHANNELS:
        V, nv, log, threads, groups = plan_rows(C, bf16, elements)
        assert threads <= 1024 and groups >= 1 and nv * V <= 16 and nv in (1, 2, 4, 8, 16)
        assert nv <= {8: 2, 4: 4, 2: 8, 1: 16}[V]          # kernels that there are
        if nv * V > elements:
            assert nv * V == 16 and threads == 1024         # sums in LDS: 16 places a thread
        if log < 6:
            assert nv == 1                                  # rows of less than a wave
        seen = np.zeros(C, int)
        for lane in range(1 << log):
            for j in range(nv):
                at = lane * V + j * (V << log)
                if at < C:
                    assert at + V <= C
                    seen[at:at + V] += 1
        assert (seen == 1).all(), C
        assert groups == 1 or groups * C * 4 <= 16384       # a group's sums in LDS


@pytest.mark.parametrize("bf16", [False, True])
def test_rows_are_covered_once(bf16):
    for C in (1, 64, 768, 4096, 16384):
        for B, S in [(1, 1), (8, 1), (3, 5), (37, 61), (1, 2100), (600, 2), (2, 4099), (5000, 1)]:
            _, _, log, threads, groups = plan_rows(C, bf16, 16)
            batches = ceil_div(B * S, groups)
            iters = ceil_div(batches, 4096)
            wgs = ceil_div(batches, iters)
            rows = (np.arange(wgs)[:, None, None] * iters + np.arange(iters)[:, None]) * groups + np.arange(groups)
            rows = rows.reshape(-1)
            assert wgs <= 4096 and sorted(rows[rows < B * S]) == list(range(B * S))
            # Backward: rows of one example a workgroup.
            _, _, log, threads, groups = plan_rows(C, bf16, 8)
            while threads > 64 and groups > 1 and groups // 2 >= S:
                threads, groups = threads // 2, groups // 2
            assert threads >> log == groups and threads % 64 == 0
            batches = ceil_div(S, groups)
            most = min(ceil_div(256 if threads > 512 else 512, B),
                       max(ceil_div(batches, 2), ceil_div(128, B)))
            iters = ceil_div(batches, min(most, batches))
            chunks = ceil_div(batches, iters)
            s = (np.arange(chunks)[:, None, None] * iters + np.arange(iters)[:, None]) * groups + np.arange(groups)
            s = s.reshape(-1)
            assert sorted(s[s < S]) == list(range(S))
            assert chunks == 1 or B < 512


# ------------------------------------------------------------------ 8-bit moments


@pytest.mark.parametrize("per_wave", [1, 4])
def test_blocks_are_covered_once(per_wave):
    for n in (1, 255, 256, 257, 4096, 4097, 100_003):
        wgs = ceil_div(ceil_div(n, 256), per_wave * 4)
        seen = np.zeros(n, int)
        blocks = []
        for wg in range(wgs):
            for wave in range(4):
                for u in range(per_wave):
                    block = (wg * 4 + wave) * per_wave + u
                    if block * 256 >= n:
                        continue
                    blocks.append(block)
                    e = block * 256 + np.arange(256)
                    seen[e[e < n]] += 1
        assert (seen == 1).all() and blocks == list(range(ceil_div(n, 256)))
