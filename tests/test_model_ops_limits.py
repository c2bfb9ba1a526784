"""Calls whose launches would have 2^32 threads or more are refused before anything is
enqueued (CPU only: the refusal comes before the first launch)."""

import ctypes

import pytest

from paper_2609_20532_amd import dpsgd

INVALID = -1
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    return dpsgd.load()


@pytest.mark.parametrize("B,T,n_rows,d", [
    (1 << 22, 1, 100, 8),               # 2^22 workgroups of 1024 threads, one an example
    (1 << 29, 2, 100, 1),
    (1 << 21, 1, 100, (1 << 13) + 1),   # nine blocks of columns an example
    (1, 5000, (1 << 30) + 1, 1),        # the sort's buckets
    (7, 4097, (1 << 31) - 1, 2),
])
@pytest.mark.parametrize("dtype", [dpsgd.DPSGD_F32, dpsgd.DPSGD_BF16])
def test_embedding_norms(lib, B, T, n_rows, d, dtype):
    e = dpsgd.dpsgd_embedding(64, B, T, n_rows, d, dpsgd.DPSGD_I32, 1.0)
    for accumulate in (0, 1):
        assert lib.dpsgd_embedding_norms(ctypes.byref(e), P(16), dtype, P(32), accumulate, P(64),
                                         1 << 60, None) == INVALID


@pytest.mark.parametrize("B,T,n_rows,d", [
    (1 << 14, 1 << 14, 100, 1),             # 2^23 chunks, joined by 512 threads each
    (1 << 30, 1, 100, 1),
    (3, 5, (1 << 31) - 1, 1),               # the sort's buckets
    (3, 5, (1 << 30) + 1, 1),
    (1 << 10, 1 << 10, 3, (1 << 19) + 1),   # chunks by blocks of columns
])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_embedding_sum(lib, B, T, n_rows, d, accumulate):
    e = dpsgd.dpsgd_embedding(64, B, T, n_rows, d, dpsgd.DPSGD_I32, 1.0)
    # Addresses far apart: it is not an overlap that is refused.
    for nsq, fac in ((P(1 << 50), None), (P(1 << 50), P(1 << 52)), (None, None)):
        assert lib.dpsgd_embedding_clip_accumulate(
            ctypes.byref(e), P(16), dpsgd.DPSGD_F32, nsq, 1.0, P(1 << 44), accumulate, fac, None,
            P(64), 1 << 60, None) == INVALID


@pytest.mark.parametrize("B,S,C,groups", [
    (1 << 26, 1, 4, 1),             # 64 threads an example
    ((1 << 31) - 1, 1, 1, 1),
    (1 << 22, 511, 8, 1),           # 1024 threads an example
    (1 << 13, 1 << 17, 512, 512),   # tiles of a part of the rows
    (1 << 12, 3000, 4096, 4096),    # a workgroup a group, where the tiles are joined
    (1 << 17, 9000, 128, 128),
])
@pytest.mark.parametrize("dtype", [dpsgd.DPSGD_F32, dpsgd.DPSGD_BF16])
def test_group_norm(lib, B, S, C, groups, dtype):
    n = dpsgd.dpsgd_group_norm(B, S, C, groups, None, None, dtype, 0, 1e-5)
    a = [P(k << 44) for k in range(1, 10)]
    assert lib.dpsgd_group_norm_forward(ctypes.byref(n), a[0], a[1], None, None, a[2], 1 << 60,
                                        None) == INVALID
    assert lib.dpsgd_group_norm_backward(ctypes.byref(n), *a[:7], a[7], 1 << 60, None) == INVALID


@pytest.mark.parametrize("shapes", [
    [(1 << 18, 1 << 19)],                        # 2^24 blocks of 8192 entries
    [(1, 1)] * 49 + [(1 << 19, 1 << 20)],        # in the second launch
    [(1 << 17, 1 << 18)] * 4,
])
def test_global_clip(lib, shapes):
    layers = (dpsgd.dpsgd_layer * len(shapes))(*[dpsgd.shape_layer(1, 1, b, a) for a, b in shapes])
    g = (P * len(shapes))(*[(k + 1) << 44 for k in range(len(shapes))])
    for outs in (g, (P * len(shapes))(*[(k + 100) << 44 for k in range(len(shapes))])):
        assert lib.dpsgd_global_clip_multi(layers, len(shapes), g, outs, 1.0, None, None, P(64),
                                           1 << 60, None) == INVALID
