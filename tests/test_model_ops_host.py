"""Host-side checks of the calls around the linear layers (CPU only: every call here is
refused before anything is enqueued)."""

import ctypes

import pytest

from paper_2609_20532_amd import dpsgd

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    return dpsgd.load()


def _emb(**kw):
    d = dict(ids=64, B=4, T=8, n_rows=100, d=32, index_dtype=0, scale=1.0)
    d.update(kw)
    return dpsgd.dpsgd_embedding(**d)


def _gn(**kw):
    d = dict(B=2, S=9, C=12, groups=3, gamma=None, beta=None, dtype=0, act=1, eps=1e-5)
    d.update(kw)
    return dpsgd.dpsgd_group_norm(**d)


BAD_EMB = [
    (dict(B=0), INVALID), (dict(T=0), INVALID), (dict(n_rows=0), INVALID), (dict(d=0), INVALID),
    (dict(B=1 << 20, T=1 << 12), INVALID), (dict(n_rows=1 << 31), INVALID),
    (dict(d=(1 << 20) + 1), INVALID), (dict(B=1 << 15, T=(1 << 15) + 1), INVALID), (dict(n_rows=1 << 30, d=1 << 20), INVALID),
    (dict(ids=None), INVALID), (dict(ids=66), INVALID), (dict(ids=68, index_dtype=1), INVALID),
    (dict(index_dtype=2), UNSUPPORTED), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID),
]


@pytest.mark.parametrize("kw,status", BAD_EMB)
def test_embedding_refuses_bad_descriptors(lib, kw, status):
    e = _emb(**kw)
    assert lib.dpsgd_embedding_lookup(ctypes.byref(e), P(16), 0, P(32), 0, None) == status
    assert lib.dpsgd_embedding_norms(ctypes.byref(e), P(16), 0, P(32), 0, P(64), 1 << 40,
                                     None) == status
    assert lib.dpsgd_embedding_clip_accumulate(ctypes.byref(e), P(16), 0, P(32), 1.0, P(48), 0,
                                               None, None, P(64), 1 << 40, None) == status
    if "ids" not in kw:   # the size query does not look at the ids
        assert lib.dpsgd_embedding_workspace_bytes(ctypes.byref(e)) == 0


def test_embedding_refuses_bad_arguments(lib):
    e = _emb()
    r = ctypes.byref(e)
    need = lib.dpsgd_embedding_workspace_bytes(r)
    assert need > 0
    look = lib.dpsgd_embedding_lookup
    assert look(None, P(16), 0, P(32), 0, None) == INVALID
    assert look(r, None, 0, P(32), 0, None) == INVALID
    assert look(r, P(24), 0, P(32), 0, None) == INVALID     # not 16-byte aligned
    assert look(r, P(16), 0, P(40), 0, None) == INVALID
    assert look(r, P(16), 2, P(32), 0, None) == UNSUPPORTED
    assert look(r, P(16), 0, P(32), -1, None) == UNSUPPORTED
    norms = lib.dpsgd_embedding_norms
    assert norms(r, None, 0, P(32), 0, P(64), need, None) == INVALID
    assert norms(r, P(16), 3, P(32), 0, P(64), need, None) == UNSUPPORTED
    assert norms(r, P(16), 0, None, 0, P(64), need, None) == INVALID
    assert norms(r, P(16), 0, P(32), 0, None, need, None) == WORKSPACE
    assert norms(r, P(16), 0, P(32), 0, P(64), need - 1, None) == WORKSPACE
    assert norms(r, P(16), 0, P(32), 0, P(72), need, None) == INVALID
    clip = lib.dpsgd_embedding_clip_accumulate
    for C in (0.0, -1.0, float("nan")):
        assert clip(r, P(16), 0, P(32), C, P(48), 0, None, None, P(64), need, None) == INVALID
    assert clip(r, P(16), 0, P(32), 1.0, P(52), 0, None, None, P(64), need, None) == INVALID
    assert clip(r, P(16), 0, P(32), 1.0, None, 0, None, None, P(64), need, None) == INVALID
    assert clip(r, P(16), 0, None, 1.0, P(48), 0, P(80), None, P(64), need, None) == INVALID
    assert clip(r, P(16), 0, None, 1.0, P(48), 0, None, P(80), P(64), need, None) == INVALID
    assert clip(r, P(16), 0, P(32), 1.0, P(48), 0, None, None, P(64), need - 1, None) == WORKSPACE


BAD_GN = [
    (dict(B=0), INVALID), (dict(S=0), INVALID), (dict(C=0), INVALID), (dict(groups=0), INVALID),
    (dict(groups=5), INVALID), (dict(groups=24), INVALID), (dict(B=1 << 16, S=1 << 16), INVALID),
    (dict(C=1 << 32, groups=1), INVALID), (dict(C=(1 << 20) + 1, groups=1), INVALID), (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(act=4), UNSUPPORTED), (dict(act=-1), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BAD_GN)
def test_group_norm_refuses_bad_descriptors(lib, kw, status):
    n = _gn(**kw)
    assert lib.dpsgd_group_norm_workspace_bytes(ctypes.byref(n)) == 0
    assert lib.dpsgd_group_norm_forward(ctypes.byref(n), P(16), P(32), None, None, P(64), 1 << 40,
                                        None) == status
    assert lib.dpsgd_group_norm_backward(ctypes.byref(n), P(16), P(32), P(48), P(64), P(80), P(96),
                                         P(112), P(128), 1 << 40, None) == status


def test_group_norm_refuses_bad_arguments(lib):
    n = _gn()
    r = ctypes.byref(n)
    need = lib.dpsgd_group_norm_workspace_bytes(r)
    assert need > 0
    f, b = lib.dpsgd_group_norm_forward, lib.dpsgd_group_norm_backward
    assert f(None, P(16), P(32), None, None, P(64), need, None) == INVALID
    assert f(r, None, P(32), None, None, P(64), need, None) == INVALID
    assert f(r, P(20), P(32), None, None, P(64), need, None) == INVALID
    assert f(r, P(16), None, None, None, P(64), need, None) == INVALID
    assert f(r, P(16), P(32), P(3), None, P(64), need, None) == INVALID
    assert f(r, P(16), P(32), None, None, None, need, None) == WORKSPACE
    assert f(r, P(16), P(32), None, None, P(64), need - 1, None) == WORKSPACE
    assert f(ctypes.byref(_gn(gamma=6)), P(16), P(32), None, None, P(64), need, None) == INVALID
    good = [r, P(16), P(32), P(48), P(64), P(80), P(96), P(112), P(128), need, None]
    for at in range(1, 8):   # every tensor is required
        bad = list(good)
        bad[at] = None
        assert b(*bad) == INVALID
    bad = list(good)
    bad[5] = P(16)           # dx over x
    assert b(*bad) == INVALID
    bad = list(good)
    bad[9] = need - 1
    assert b(*bad) == WORKSPACE


def test_global_clip_refuses_bad_arguments(lib):
    arr = (dpsgd.dpsgd_layer * 2)(dpsgd.shape_layer(1, 1, 3, 5), dpsgd.shape_layer(1, 1, 1, 7))
    need = lib.dpsgd_global_norm_workspace_bytes(arr, 2)
    assert need > 0
    g, o = (P * 2)(16, 32), (P * 2)(48, 64)
    clip, norm = lib.dpsgd_global_clip_multi, lib.dpsgd_global_norm_multi
    assert lib.dpsgd_global_norm_workspace_bytes(arr, 0) == 0
    assert clip(None, 2, g, o, 1.0, None, None, P(128), need, None) == INVALID
    assert clip(arr, 0, g, o, 1.0, None, None, P(128), need, None) == INVALID
    assert clip(arr, 2, None, o, 1.0, None, None, P(128), need, None) == INVALID
    assert clip(arr, 2, g, None, 1.0, None, None, P(128), need, None) == INVALID
    for m in (0.0, -2.0, float("nan")):
        assert clip(arr, 2, g, o, m, None, None, P(128), need, None) == INVALID
    assert clip(arr, 2, (P * 2)(16, None), o, 1.0, None, None, P(128), need, None) == INVALID
    assert clip(arr, 2, g, (P * 2)(48, 72), 1.0, None, None, P(128), need, None) == INVALID
    assert clip(arr, 2, g, o, 1.0, P(2), None, P(128), need, None) == INVALID
    assert clip(arr, 2, g, o, 1.0, None, None, P(128), need - 1, None) == WORKSPACE
    assert clip(arr, 2, g, o, 1.0, None, None, P(136), need, None) == INVALID
    assert norm(arr, 2, g, None, P(128), need, None) == INVALID
    assert norm(arr, 2, g, P(80), None, need, None) == WORKSPACE
    bad = (dpsgd.dpsgd_layer * 1)(dpsgd.shape_layer(1, 1, 0, 5))
    assert lib.dpsgd_global_norm_workspace_bytes(bad, 1) == 0
    assert norm(bad, 1, g, P(80), P(128), need, None) == INVALID


def test_binding_refuses_what_the_library_cannot_see():
    import torch
    ids = torch.zeros(2, 3, dtype=torch.int64)
    with pytest.raises(ValueError):
        dpsgd.make_embedding(ids, (4, 8))                      # not on the device
    with pytest.raises(ValueError):
        dpsgd.make_embedding(ids.float(), (4, 8))
    with pytest.raises(ValueError):
        dpsgd.make_embedding(ids.view(6), (4, 8))
    x = torch.zeros(2, 5, 6)
    with pytest.raises(ValueError):
        dpsgd.make_group_norm(x, 3, act="tanh")
    with pytest.raises(ValueError):
        dpsgd.make_group_norm(x.double(), 3)
    with pytest.raises(ValueError):
        dpsgd.make_group_norm(x, 3, gamma=torch.ones(6))       # not on the device
    with pytest.raises(ValueError):
        dpsgd.make_group_norm(torch.zeros(2, 0, 6), 3)
