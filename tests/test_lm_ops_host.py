"""Host-side checks of the calls between and behind the blocks (CPU only: every call here
is refused before anything is enqueued)."""

import ctypes

import pytest

from paper_2609_20532_amd import dpsgd

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
P = ctypes.c_void_p
BIG = 1 << 60


def at(k):
    """Made-up addresses far from each other."""
    return P(1 << 44 | k << 38)


@pytest.fixture(scope="module")
def lib():
    return dpsgd.load()


def test_struct_layouts():
    assert ctypes.sizeof(dpsgd.dpsgd_logits) == 56 and dpsgd.dpsgd_logits.index_dtype.offset == 40
    assert ctypes.sizeof(dpsgd.dpsgd_residual_norm) == 88
    assert dpsgd.dpsgd_residual_norm.gate_per_example.offset == 64
    assert dpsgd.dpsgd_residual_norm.eps.offset == 84


# ------------------------------------------------------------------------- tokens


def _logits(**kw):
    d = dict(targets=1 << 43, B=4, T=8, V=100, stride=100, index_dtype=1, dtype=0, scale=1.0)
    d.update(kw)
    return dpsgd.dpsgd_logits(**d)


BAD_LOGITS = [
    (dict(B=0), INVALID), (dict(T=0), INVALID), (dict(V=0), INVALID), (dict(V=(1 << 24) + 1, stride=1 << 25), INVALID),
    (dict(B=1 << 20, T=1 << 11), INVALID), (dict(stride=99), INVALID), (dict(stride=(1 << 31) + 1), INVALID),
    (dict(B=1 << 15, T=1 << 14, stride=1 << 12), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(targets=(1 << 43) + 4), INVALID),
    (dict(targets=(1 << 43) + 2, index_dtype=0), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(index_dtype=2), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BAD_LOGITS)
def test_token_calls_refuse_bad_descriptors(lib, kw, status):
    d = ctypes.byref(_logits(**kw))
    if "targets" not in kw:
        assert lib.dpsgd_token_workspace_bytes(d, 0) == 0
    assert lib.dpsgd_token_logprobs(d, at(1), at(2), None, None, 0, None, None, at(3), BIG, None) == status
    assert lib.dpsgd_token_logprobs_backward(d, at(1), at(2), None, at(3), None, None, at(4), 100, None) == status
    assert lib.dpsgd_token_loss(d, at(1), None, at(2), None, at(4), 100, at(3), BIG, None) == status


def test_token_logprobs_refuses_bad_arguments(lib):
    d = ctypes.byref(_logits())
    need = lib.dpsgd_token_workspace_bytes(d, 5)
    assert need >= 4 * 8 * 4
    assert lib.dpsgd_token_workspace_bytes(d, 65) == 0 and lib.dpsgd_token_workspace_bytes(d, -1) == 0
    good = [d, at(1), at(2), at(3), at(4), 5, at(5), at(6), at(7), need, None]

    def call(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.dpsgd_token_logprobs(*a)

    assert call(_0=None) == INVALID
    assert call(_1=None) == INVALID and call(_1=P(at(1).value + 2)) == INVALID
    for k in (2, 3, 4, 6):
        assert call(**{f"_{k}": P(at(k).value + 2)}) == INVALID
    assert call(_5=65) == INVALID and call(_5=-1) == INVALID
    assert call(_5=0) == INVALID                                       # alternatives without k
    assert call(_6=None, _7=None) == INVALID                           # k without alternatives
    assert call(_2=None, _3=None, _4=None, _5=0, _6=None, _7=None) == INVALID   # nothing asked for
    assert call(_0=ctypes.byref(_logits(targets=None))) == INVALID     # log probabilities of no token
    assert call(_8=None) == WORKSPACE and call(_9=need - 1) == WORKSPACE
    assert call(_8=P(at(7).value + 8)) == INVALID
    assert call(_3=at(2)) == INVALID                                   # two outputs in one place
    assert call(_2=at(1)) == INVALID and call(_8=at(1)) == INVALID     # over the logits
    assert call(_4=P(1 << 43)) == INVALID                              # over the targets


def test_token_gradients_refuse_bad_arguments(lib):
    d = ctypes.byref(_logits())
    need = lib.dpsgd_token_workspace_bytes(d, 0)
    good = [d, at(1), at(2), at(3), at(4), at(5), at(6), at(7), 100, None]

    def back(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.dpsgd_token_logprobs_backward(*a)

    assert back(_0=None) == INVALID and back(_1=None) == INVALID and back(_2=None) == INVALID
    assert back(_7=None) == INVALID and back(_7=P(at(7).value + 2)) == INVALID
    assert back(_4=None, _5=None, _6=None) == INVALID
    assert back(_3=None) == INVALID                                    # the entropy's gradient needs it
    assert back(_0=ctypes.byref(_logits(targets=None))) == INVALID
    assert back(_8=99) == INVALID and back(_8=(1 << 31) + 1) == INVALID
    assert back(_7=at(1), _8=101) == INVALID                           # in place with another stride
    assert back(_7=P(at(1).value + 4)) == INVALID                      # over a part of the logits
    assert back(_7=at(2)) == INVALID and back(_7=P(1 << 43)) == INVALID
    good2 = [d, at(1), at(2), at(3), at(4), at(5), 100, at(6), need, None]

    def loss(**kw):
        a = list(good2)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.dpsgd_token_loss(*a)

    assert loss(_0=None) == INVALID and loss(_1=None) == INVALID and loss(_5=None) == INVALID
    assert loss(_0=ctypes.byref(_logits(targets=None))) == INVALID
    for k in (2, 3, 4):
        assert loss(**{f"_{k}": P(at(k).value + 1)}) == INVALID
    assert loss(_6=99) == INVALID and loss(_5=at(1), _6=128) == INVALID
    assert loss(_7=None) == WORKSPACE and loss(_8=need - 1) == WORKSPACE
    assert loss(_4=at(2)) == INVALID and loss(_3=at(4)) == INVALID and loss(_5=at(6)) == INVALID


# ------------------------------------------------------------------- residual norms


def _norm(**kw):
    d = dict(B=4, S=8, C=32, gamma=None, beta=None, post_gamma=None, post_beta=None, gate=None,
             gate_per_example=0, post=0, kind=0, dtype=0, residual_scale=1.0, eps=1e-5)
    d.update(kw)
    return dpsgd.dpsgd_residual_norm(**d)


BAD_NORM = [
    (dict(B=0), INVALID), (dict(S=0), INVALID), (dict(C=0), INVALID), (dict(C=16385), INVALID),
    (dict(B=1 << 16, S=1 << 15), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(eps=float("inf")), INVALID), (dict(residual_scale=float("inf")), INVALID),
    (dict(residual_scale=float("nan")), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(kind=2), UNSUPPORTED),
]
BAD_AFFINE = [dict(gamma=(1 << 43) + 4), dict(gate=(1 << 43) + 8), dict(post_gamma=1 << 43), dict(post_beta=1 << 43),
              dict(post=1, post_beta=(1 << 43) + 4)]


def _norm_calls(lib, d, need=BIG):
    return (lib.dpsgd_residual_norm_forward(d, at(1), at(2), at(3), at(4), at(5), None),
            lib.dpsgd_residual_norm_backward(d, at(1), at(2), at(3), at(4), at(5), at(6), at(7), None, None, None,
                                             None, None, at(8), need, None))


@pytest.mark.parametrize("kw,status", BAD_NORM)
def test_residual_norm_refuses_bad_descriptors(lib, kw, status):
    d = ctypes.byref(_norm(**kw))
    assert lib.dpsgd_residual_norm_workspace_bytes(d) == 0
    assert _norm_calls(lib, d) == (status, status)


@pytest.mark.parametrize("kw", BAD_AFFINE)
def test_residual_norm_refuses_bad_parameters(lib, kw):
    assert _norm_calls(lib, ctypes.byref(_norm(**kw))) == (INVALID, INVALID)


def test_residual_norm_refuses_bad_arguments(lib):
    d = ctypes.byref(_norm(post=1))
    good = [d, at(1), at(2), at(3), at(4), at(5), None]

    def forward(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.dpsgd_residual_norm_forward(*a)

    assert forward(_0=None) == INVALID and forward(_1=None) == INVALID and forward(_4=None) == INVALID
    for k in range(1, 6):
        assert forward(**{f"_{k}": P(at(k).value + 8)}) == INVALID
    assert forward(_2=None) == INVALID                                 # a norm of no block
    assert forward(_0=ctypes.byref(_norm(gate=1 << 43)), _2=None) == INVALID
    assert forward(_3=at(2)) == INVALID and forward(_4=at(1)) == INVALID and forward(_4=at(3)) == INVALID
    assert forward(_3=P(at(1).value + 16)) == INVALID
    assert forward(_0=ctypes.byref(_norm(gamma=at(4).value))) == INVALID
    need = lib.dpsgd_residual_norm_workspace_bytes(d)
    assert need > 0
    good2 = [d] + [at(k) for k in range(1, 14)] + [need, None]

    def back(**kw):
        a = list(good2)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.dpsgd_residual_norm_backward(*a)

    for k in (0, 2, 3, 5):
        assert back(**{f"_{k}": None}) == INVALID
    for k in range(1, 13):
        assert back(**{f"_{k}": P(at(k).value + 4)}) == INVALID
    assert back(_1=None) == INVALID and back(_7=None) == INVALID       # block and dblock together
    assert back(_0=ctypes.byref(_norm())) == INVALID                   # gradients of a norm that is not there
    assert back(_13=None) == WORKSPACE and back(_14=need - 1) == WORKSPACE
    assert back(_13=P(at(13).value + 8)) == INVALID
    assert back(_6=at(3)) == INVALID and back(_7=at(4)) == INVALID and back(_7=at(1)) == INVALID
    assert back(_6=at(2)) == INVALID and back(_8=at(9)) == INVALID and back(_10=at(13)) == INVALID
    none = [d, at(1), at(2), at(3), at(4), at(5), None, None] + [None] * 5 + [at(13), need, None]
    none[0] = ctypes.byref(_norm())
    none[1] = None
    assert lib.dpsgd_residual_norm_backward(*none) == INVALID          # nothing asked for


@pytest.mark.parametrize("B,S,C", [((1 << 31) - 1, 1, 8), (1 << 26, 1, 8), (1 << 22, 1, 16384), (1 << 23, 2, 16384)])
def test_residual_norm_backward_refuses_what_no_launch_holds(lib, B, S, C):
    """2^32 threads or more: one workgroup an example at least, of 64 threads for narrow
    rows and 1024 for the widest."""
    assert _norm_calls(lib, ctypes.byref(_norm(B=B, S=S, C=C)))[1] == INVALID


# ------------------------------------------------------------------ 8-bit moments


def _arrays():
    layers = (dpsgd.dpsgd_layer * 2)(dpsgd.shape_layer(1, 1, 3, 5, 0, 1), dpsgd.shape_layer(1, 1, 1, 7, 0, 2))
    return layers, [(P * 2)(at(2 * k), at(2 * k + 1)) for k in range(6)]


def _step(lib, layers, arrays, n=2, sigma=0.5, C=1.0, scale=1.0, opt=None, rounding=0):
    opt = dpsgd.make_adamw(1e-3) if opt is None else opt
    return lib.dpsgd_noise_adamw8_multi(layers, n, *arrays, sigma, C, 1, 2, scale,
                                        ctypes.byref(opt) if opt != 0 else None, rounding, 3, None)


def test_adamw8_refuses_bad_arguments(lib):
    layers, arrays = _arrays()
    assert _step(lib, None, arrays) == INVALID and _step(lib, layers, arrays, n=0) == INVALID
    assert _step(lib, layers, arrays, rounding=2) == UNSUPPORTED
    assert _step(lib, layers, arrays, opt=0) == INVALID
    for k in range(5):
        assert _step(lib, layers, arrays[:k] + [None] + arrays[k + 1:]) == INVALID
        for bad in (None, P(at(2).value + 8)):
            assert _step(lib, layers, arrays[:k] + [(P * 2)(at(1), bad)] + arrays[k + 1:]) == INVALID
    assert _step(lib, layers, arrays[:5] + [(P * 2)(None, P(at(3).value + 4))]) == INVALID
    for sigma in (-1.0, float("nan"), float("inf")):
        assert _step(lib, layers, arrays, sigma=sigma) == INVALID
    for C in (0.0, -1.0, float("nan"), float("inf")):
        assert _step(lib, layers, arrays, C=C) == INVALID
    assert _step(lib, layers, arrays, scale=float("nan")) == INVALID
    for kw in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=1.0, beta1=1.0), dict(lr=1.0, beta2=-0.1),
               dict(lr=1.0, eps=0.0), dict(lr=1.0, weight_decay=-1.0), dict(lr=1.0, t=0)):
        assert _step(lib, layers, arrays, opt=dpsgd.make_adamw(**kw)) == INVALID
    layers[1].tensor_id = 1
    assert _step(lib, layers, arrays) == INVALID
    layers[1].tensor_id = 2
    layers[1].d_in = 0
    assert _step(lib, layers, arrays) == INVALID
    assert lib.dpsgd_adamw8_pack_multi(layers, 2, *arrays[:5], None) == INVALID


def test_adamw8_pack_and_unpack_refuse_bad_arguments(lib):
    layers, arrays = _arrays()
    pack, unpack = lib.dpsgd_adamw8_pack_multi, lib.dpsgd_adamw8_unpack_multi
    assert pack(None, 2, *arrays[:5], None) == INVALID and unpack(layers, 0, *arrays[:5], 0, None) == INVALID
    assert unpack(layers, 2, *arrays[:5], 2, None) == UNSUPPORTED
    for k in range(5):
        for bad in (None, (P * 2)(at(1), None), (P * 2)(P(at(1).value + 4), at(2))):
            a = arrays[:k] + [bad] + arrays[k + 1:5]
            assert pack(layers, 2, *a, None) == INVALID
            assert unpack(layers, 2, *a, 0, None) == INVALID


def test_adamw8_refuses_what_no_launch_holds(lib):
    _, arrays = _arrays()
    layers = (dpsgd.dpsgd_layer * 2)(dpsgd.shape_layer(1, 1, 1 << 19, 1 << 20, 0, 1),
                                     dpsgd.shape_layer(1, 1, 1 << 20, 1 << 20, 0, 2))
    assert _step(lib, layers, arrays) == INVALID


# ------------------------------------------------------------------------- binding


def test_binding_refuses_what_the_library_cannot_see():
    import torch
    x = torch.zeros(2, 3, 5)
    with pytest.raises(ValueError):
        dpsgd.make_logits(x)                                           # not on the device
    with pytest.raises(ValueError):
        dpsgd._logit_rows("logits", torch.zeros(6, 5))
    with pytest.raises(ValueError):
        dpsgd._logit_rows("logits", torch.zeros(2, 0, 5))
    with pytest.raises(ValueError):
        dpsgd._logit_rows("logits", torch.zeros(2, 5, 3).transpose(1, 2))      # entries apart
    with pytest.raises(ValueError):
        dpsgd._logit_rows("logits", torch.zeros(2, 4, 5)[:, :3])               # rows unevenly spaced
    with pytest.raises(ValueError):
        dpsgd._logit_rows("logits", torch.zeros(1, 5).expand(2, 3, 5))         # rows over each other
    assert dpsgd._logit_rows("logits", torch.zeros(2, 3, 8)[..., 1:6]) == (2, 3, 5, 8)
    assert dpsgd._logit_rows("logits", torch.zeros(2, 3, 8)[:, -1:]) == (2, 1, 8, 24)
    assert dpsgd._logit_rows("logits", torch.zeros(1, 3, 8)[:, -1:]) == (1, 1, 8, 8)
    assert dpsgd._logit_rows("logits", torch.zeros(4, 3, 1)) == (4, 3, 1, 1)
    assert dpsgd._logit_rows("logits", torch.zeros(4, 3, 2)[..., :1]) == (4, 3, 1, 2)
    with pytest.raises(ValueError):
        dpsgd.make_residual_norm(x, kind="batch")
    with pytest.raises(ValueError):
        dpsgd.make_residual_norm(x.double())
    with pytest.raises(ValueError):
        dpsgd.make_residual_norm(x, gamma=torch.ones(5))               # not on the device
    with pytest.raises(ValueError):
        dpsgd.make_residual_norm(torch.zeros(2, 0, 5))
    L = [dpsgd.shape_layer(1, 1, 3, 5)]
    m, v, exps = dpsgd.make_states8(L, device="cpu")
    assert m[0].shape == (5, 3) and v[0].dtype == torch.uint8 and exps[0].shape == (1, 2)
    with pytest.raises(ValueError):
        dpsgd.dpsgd_adamw8_pack_multi(L, [x], [x], m, v, exps)


class _Elsewhere:
    """A tensor of another device, as far as the refusal looks."""
    is_cuda = True
    device = "cuda:1"

    def get_device(self):
        return 1


def test_tensors_of_another_device_are_refused():
    import torch
    m = dpsgd._load_marshal()
    with pytest.raises(ValueError, match="not the current device"):
        dpsgd._refuse("x", _Elsewhere(), (2, 3), dpsgd._F32, 0)
    with pytest.raises(ValueError, match="device tensor"):
        dpsgd._take(0, ("y", "x"), None, (2,), dpsgd._F32, torch.zeros(2), (2,), dpsgd._F32)
    with pytest.raises(ValueError, match="device tensor"):
        dpsgd._take(None, ("x",), torch.zeros(2), (2,), dpsgd._F32)
    assert dpsgd._take(0, ("x",), None, (2,), dpsgd._F32) == (None,)
    assert m.take(0) == () and m.take(0, 5, (2,), 6) == 0 and m.take(0, None, 0, 0, torch.zeros(1), (1,), 6) == 1
    for bad in ((), (0, None), ("a",), (0, torch.zeros(1), (1,), "f")):
        with pytest.raises(TypeError):
            m.take(*bad)
    assert m.logits(0, torch.zeros(1, 2, 3)) is None and m.logits(0, 5) is None
    with pytest.raises(TypeError):
        m.logits(0)


def test_lists_of_tensors():
    import torch
    m = dpsgd._load_marshal()
    layers = (dpsgd.dpsgd_layer * 2)(dpsgd.shape_layer(1, 1, 3, 2), dpsgd.shape_layer(1, 1, 1, 2))
    buf = (ctypes.c_void_p * 2)()
    none = (dpsgd.dpsgd_layer * 0)()
    cpu = [torch.zeros(6), torch.zeros(2)]
    assert not m.addresses(cpu, layers, 0, 6, -1, buf)                 # not on a device
    assert not m.addresses(cpu[:1], layers, 0, 6, -1, buf) and not m.addresses([], layers, 0, 6, 0, buf)
    assert not m.addresses([1, 2], layers, 0, 6, 0, buf) and m.addresses([], none, 0, 6, 0, buf)
    assert not m.addresses(cpu, layers, 0, 6, 0, (ctypes.c_void_p * 1)()) and list(buf) == [None, None]
    for bad in ((), (1, layers, 0, 6, 0, buf), ([], 1, 0, 6, 0, buf), ([], none, 0, "f", 0, buf),
                ([], none, 0, 6, 0, b"1"), ([], none, 0, 6, 0)):
        with pytest.raises((TypeError, BufferError)):
            m.addresses(*bad)
    for tensors, here in ((cpu, 0), (cpu[:1], 0), (cpu, None), (cpu, -1)):
        with pytest.raises(ValueError):
            dpsgd._tensors("x", tensors, layers, 2, dpsgd._F32, here)


def test_arrays_of_descriptors():
    Ls = [dpsgd.shape_layer(2, 3, k + 1, 5, dpsgd.DPSGD_F32, k) for k in range(4)]
    for layers in (Ls, tuple(Ls), Ls[1], Ls[:1]):
        (a, n), (b, m) = dpsgd._layer_array(layers), dpsgd._array(layers)
        assert n == m and bytes(a) == bytes(b)
    with pytest.raises(TypeError):
        dpsgd._layer_array([Ls[0], b"x" * 56])


def test_own_capture_refuses_rows_without_a_next_token():
    torch = pytest.importorskip("torch")
    from paper_2609_20532_amd import capture as cap
    cfg = cap.GPT2Config(vocab=11, n_ctx=4, n_embd=8, n_layer=1, n_head=2, r=2)
    model = cap.GPT2LoRA(cfg)
    with pytest.raises(ValueError, match="two tokens"):
        cap.capture(model, torch.zeros(3, 1, dtype=torch.int64), own=True)
    assert model.rec.on is False and not model.rec.items
