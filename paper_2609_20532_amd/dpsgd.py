"""Python binding of the C ABI in ``include/dpsgd.h`` (argument marshalling only).

Every function here has the name of the C entry point it calls and does no
arithmetic of the DP-SGD step: it converts torch tensors to device pointers,
fills ``dpsgd_layer`` descriptors, passes torch's current HIP stream, and
raises :class:`DpsgdError` on a non-zero status. torch supplies device memory
and streams only. The library must be built (``paper_2609_20532_amd.build``);
loading fails loudly when it is missing. The calls between and behind a model's
blocks check their tensors through the built module ``_marshal``.
"""

from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libdpsgd.so")

DPSGD_F32 = 0
DPSGD_BF16 = 1
DPSGD_NORM_AUTO = 0
DPSGD_NORM_GHOST = 1
DPSGD_NORM_MATERIALIZE = 2
DPSGD_NORM_CLOSED_FORM = 3   # reported by dpsgd_select_norm_mode for T = 1 layers

DPSGD_I32 = 0
DPSGD_I64 = 1
DPSGD_ACT_NONE = 0
DPSGD_ACT_RELU = 1
DPSGD_ACT_SILU = 2
DPSGD_ACT_GELU = 3
#: Activations of a group norm by name.
ACTIVATIONS = {"none": DPSGD_ACT_NONE, "relu": DPSGD_ACT_RELU, "silu": DPSGD_ACT_SILU,
               "gelu": DPSGD_ACT_GELU}

DPSGD_MOST_ALTERNATIVES = 64   # of dpsgd_token_logprobs
DPSGD_ROW_NORM_LAYER = 0
DPSGD_ROW_NORM_RMS = 1
#: Norms over rows by name.
ROW_NORMS = {"layer": DPSGD_ROW_NORM_LAYER, "rms": DPSGD_ROW_NORM_RMS}
DPSGD_STATE_BLOCK = 256        # entries that share the exponents of 8-bit moments
DPSGD_ROUND_NEAREST = 0
DPSGD_ROUND_STOCHASTIC = 1

DPSGD_OK = 0
DPSGD_ERR_INVALID_ARG = -1
DPSGD_ERR_UNSUPPORTED = -2
DPSGD_ERR_WORKSPACE = -3
DPSGD_ERR_HIP = -4

#: Every symbol the header declares (checked by the CPU test suite).
EXPORTED = (
    "dpsgd_norms_workspace_bytes", "dpsgd_select_norm_mode", "dpsgd_per_example_norms",
    "dpsgd_per_example_norms_multi", "dpsgd_per_example_norms_multi_noalloc",
    "dpsgd_clip_factors", "dpsgd_clip_workspace_bytes",
    "dpsgd_clip_accumulate", "dpsgd_clip_accumulate_multi", "dpsgd_clipped_sum_workspace_bytes",
    "dpsgd_clipped_sum_multi", "dpsgd_add_noise",
    "dpsgd_add_noise_multi", "dpsgd_noise_adamw", "dpsgd_noise_adamw_multi",
    "dpsgd_philox_u32", "dpsgd_gaussian", "dpsgd_status_string", "dpsgd_version",
    "dpsgd_embedding_lookup", "dpsgd_embedding_workspace_bytes", "dpsgd_embedding_norms",
    "dpsgd_embedding_clip_accumulate", "dpsgd_group_norm_workspace_bytes",
    "dpsgd_group_norm_forward", "dpsgd_group_norm_backward", "dpsgd_global_norm_workspace_bytes",
    "dpsgd_global_norm_multi", "dpsgd_global_clip_multi",
    "dpsgd_token_workspace_bytes", "dpsgd_token_logprobs", "dpsgd_token_logprobs_backward",
    "dpsgd_token_loss", "dpsgd_residual_norm_forward", "dpsgd_residual_norm_workspace_bytes",
    "dpsgd_residual_norm_backward", "dpsgd_noise_adamw8_multi", "dpsgd_adamw8_pack_multi",
    "dpsgd_adamw8_unpack_multi",
)


class DpsgdError(RuntimeError):
    def __init__(self, fn: str, status: int, text: str):
        super().__init__(f"{fn} failed: {text} (status {status})")
        self.status = status


class dpsgd_layer(ctypes.Structure):  # noqa: N801 - mirrors the C struct name
    _fields_ = [
        ("A", ctypes.c_void_p),
        ("G", ctypes.c_void_p),
        ("B", ctypes.c_int64),
        ("T", ctypes.c_int64),
        ("d_in", ctypes.c_int64),
        ("d_out", ctypes.c_int64),
        ("dtype", ctypes.c_int32),
        ("tensor_id", ctypes.c_uint32),
    ]


class dpsgd_adamw(ctypes.Structure):  # noqa: N801 - mirrors the C struct name
    _fields_ = [
        ("lr", ctypes.c_float),
        ("beta1", ctypes.c_float),
        ("beta2", ctypes.c_float),
        ("eps", ctypes.c_float),
        ("weight_decay", ctypes.c_float),
        ("t", ctypes.c_uint32),
    ]


class dpsgd_embedding(ctypes.Structure):  # noqa: N801 - mirrors the C struct name
    _fields_ = [
        ("ids", ctypes.c_void_p),
        ("B", ctypes.c_int64),
        ("T", ctypes.c_int64),
        ("n_rows", ctypes.c_int64),
        ("d", ctypes.c_int64),
        ("index_dtype", ctypes.c_int32),
        ("scale", ctypes.c_float),
    ]


class dpsgd_group_norm(ctypes.Structure):  # noqa: N801 - mirrors the C struct name
    _fields_ = [
        ("B", ctypes.c_int64),
        ("S", ctypes.c_int64),
        ("C", ctypes.c_int64),
        ("groups", ctypes.c_int64),
        ("gamma", ctypes.c_void_p),
        ("beta", ctypes.c_void_p),
        ("dtype", ctypes.c_int32),
        ("act", ctypes.c_int32),
        ("eps", ctypes.c_float),
    ]


class dpsgd_logits(ctypes.Structure):  # noqa: N801 - mirrors the C struct name
    _fields_ = [
        ("targets", ctypes.c_void_p),
        ("B", ctypes.c_int64),
        ("T", ctypes.c_int64),
        ("V", ctypes.c_int64),
        ("stride", ctypes.c_int64),
        ("index_dtype", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("scale", ctypes.c_float),
    ]


class dpsgd_residual_norm(ctypes.Structure):  # noqa: N801 - mirrors the C struct name
    _fields_ = [
        ("B", ctypes.c_int64),
        ("S", ctypes.c_int64),
        ("C", ctypes.c_int64),
        ("gamma", ctypes.c_void_p),
        ("beta", ctypes.c_void_p),
        ("post_gamma", ctypes.c_void_p),
        ("post_beta", ctypes.c_void_p),
        ("gate", ctypes.c_void_p),
        ("gate_per_example", ctypes.c_int32),
        ("post", ctypes.c_int32),
        ("kind", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("residual_scale", ctypes.c_float),
        ("eps", ctypes.c_float),
    ]


_lib = None


def _declare(lib):
    P = ctypes.POINTER
    L = P(dpsgd_layer)
    E, N = P(dpsgd_embedding), P(dpsgd_group_norm)
    K, R = P(dpsgd_logits), P(dpsgd_residual_norm)
    vp, i32, i64, u32, u64, f32, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                       ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float,
                                       ctypes.c_size_t)
    sig = {
        "dpsgd_norms_workspace_bytes": (sz, [L, i32, i32]),
        "dpsgd_select_norm_mode": (i32, [L]),
        "dpsgd_per_example_norms": (ctypes.c_int, [L, i32, vp, i32, vp, sz, vp]),
        "dpsgd_per_example_norms_multi": (ctypes.c_int, [L, i32, i32, vp, i32, vp, sz, vp]),
        "dpsgd_per_example_norms_multi_noalloc": (ctypes.c_int, [L, i32, i32, vp, i32, vp]),
        "dpsgd_clip_factors": (ctypes.c_int, [vp, i64, f32, vp, vp, vp]),
        "dpsgd_clip_workspace_bytes": (sz, [L, i32]),
        "dpsgd_clip_accumulate": (ctypes.c_int, [L, vp, f32, vp, i32, vp, vp, vp, sz, vp]),
        "dpsgd_clip_accumulate_multi": (ctypes.c_int,
                                        [L, i32, vp, f32, P(vp), i32, vp, vp, vp, sz, vp]),
        "dpsgd_clipped_sum_workspace_bytes": (sz, [L, i32, i32]),
        "dpsgd_clipped_sum_multi": (ctypes.c_int, [L, i32, i32, f32, P(vp), i32, vp, vp, vp, vp,
                                                   sz, vp]),
        "dpsgd_add_noise": (ctypes.c_int, [L, vp, f32, f32, u64, u32, f32, vp]),
        "dpsgd_add_noise_multi": (ctypes.c_int, [L, i32, P(vp), f32, f32, u64, u32, f32, vp]),
        "dpsgd_noise_adamw": (ctypes.c_int, [L, vp, vp, vp, vp, vp, f32, f32, u64, u32, f32,
                                             P(dpsgd_adamw), vp]),
        "dpsgd_noise_adamw_multi": (ctypes.c_int, [L, i32, P(vp), P(vp), P(vp), P(vp), P(vp),
                                                   f32, f32, u64, u32, f32, P(dpsgd_adamw), vp]),
        "dpsgd_philox_u32": (ctypes.c_int, [vp, i64, i64, u64, u32, u32, vp]),
        "dpsgd_gaussian": (ctypes.c_int, [vp, i64, u64, u32, u32, vp]),
        "dpsgd_embedding_lookup": (ctypes.c_int, [E, vp, i32, vp, i32, vp]),
        "dpsgd_embedding_workspace_bytes": (sz, [E]),
        "dpsgd_embedding_norms": (ctypes.c_int, [E, vp, i32, vp, i32, vp, sz, vp]),
        "dpsgd_embedding_clip_accumulate": (ctypes.c_int, [E, vp, i32, vp, f32, vp, i32, vp, vp,
                                                           vp, sz, vp]),
        "dpsgd_group_norm_workspace_bytes": (sz, [N]),
        "dpsgd_group_norm_forward": (ctypes.c_int, [N, vp, vp, vp, vp, vp, sz, vp]),
        "dpsgd_group_norm_backward": (ctypes.c_int, [N, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
        "dpsgd_global_norm_workspace_bytes": (sz, [L, i32]),
        "dpsgd_global_norm_multi": (ctypes.c_int, [L, i32, P(vp), vp, vp, sz, vp]),
        "dpsgd_global_clip_multi": (ctypes.c_int, [L, i32, P(vp), P(vp), f32, vp, vp, vp, sz, vp]),
        "dpsgd_token_workspace_bytes": (sz, [K, i32]),
        "dpsgd_token_logprobs": (ctypes.c_int, [K, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]),
        "dpsgd_token_logprobs_backward": (ctypes.c_int, [K, vp, vp, vp, vp, vp, vp, vp, i64, vp]),
        "dpsgd_token_loss": (ctypes.c_int, [K, vp, vp, vp, vp, vp, i64, vp, sz, vp]),
        "dpsgd_residual_norm_forward": (ctypes.c_int, [R, vp, vp, vp, vp, vp, vp]),
        "dpsgd_residual_norm_workspace_bytes": (sz, [R]),
        "dpsgd_residual_norm_backward": (ctypes.c_int, [R] + [vp] * 13 + [sz, vp]),
        "dpsgd_noise_adamw8_multi": (ctypes.c_int, [L, i32, P(vp), P(vp), P(vp), P(vp), P(vp),
                                                    P(vp), f32, f32, u64, u32, f32,
                                                    P(dpsgd_adamw), i32, u64, vp]),
        "dpsgd_adamw8_pack_multi": (ctypes.c_int, [L, i32] + [P(vp)] * 5 + [vp]),
        "dpsgd_adamw8_unpack_multi": (ctypes.c_int, [L, i32] + [P(vp)] * 5 + [i32, vp]),
        "dpsgd_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "dpsgd_version": (ctypes.c_int, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args


def load(path: str | None = None):
    """Load ``libdpsgd.so`` (after torch, so both share one HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    import torch  # noqa: F401  (loads the HIP runtime the library links against)

    path = path or LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2609_20532_amd.build`")
    lib = ctypes.CDLL(path)
    _declare(lib)
    if lib.dpsgd_version() != 1:
        raise RuntimeError("libdpsgd version mismatch")
    _lib = lib
    return lib


def _check(fn: str, status: int):
    if status != DPSGD_OK:
        raise DpsgdError(fn, status, _lib.dpsgd_status_string(status).decode())


_raw_stream = None   # torch's (current device, raw handle of its current stream), once CUDA is initialised


def _stream(stream):
    global _raw_stream
    if stream is None:
        # The handle alone: building a torch.cuda.Stream object takes about 3 us
        # a call, a third of a small call's host time.
        if _raw_stream is not None:
            return _raw_stream[1](_raw_stream[0]())
        import torch
        if torch.cuda.is_initialized():
            _raw_stream = (torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# ----------------------------------------------------------------- descriptors


def make_layer(A, G, tensor_id: int) -> dpsgd_layer:
    """Descriptor of one layer from device tensors A [B,T,d_in] and G [B,T,d_out].

    ``tensor_id`` selects the layer's noise stream: the layers of one step
    need distinct ids (the noise calls reject repeats)."""
    import torch
    if A.dim() != 3 or G.dim() != 3 or A.shape[:2] != G.shape[:2]:
        raise ValueError("A must be [B,T,d_in] and G [B,T,d_out] with the same B, T")
    if A.dtype != G.dtype or A.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("A and G must both be float32 or both bfloat16")
    if not (A.is_contiguous() and G.is_contiguous()):
        raise ValueError("A and G must be contiguous")
    if not (A.is_cuda and G.is_cuda):
        raise ValueError("A and G must be device tensors")
    B, T, d_in = A.shape
    return dpsgd_layer(A.data_ptr(), G.data_ptr(), B, T, d_in, G.shape[2],
                       DPSGD_BF16 if A.dtype == torch.bfloat16 else DPSGD_F32, tensor_id)


def shape_layer(B: int, T: int, d_in: int, d_out: int, dtype: int = DPSGD_BF16,
                tensor_id: int = 0) -> dpsgd_layer:
    """Descriptor with no data, for workspace queries and noise calls."""
    return dpsgd_layer(None, None, B, T, d_in, d_out, dtype, tensor_id)


def _array(layers):
    if isinstance(layers, dpsgd_layer):
        layers = [layers]
    arr = (dpsgd_layer * len(layers))(*layers)
    return arr, len(layers)


def _ptr_array(tensors):
    return (ctypes.c_void_p * len(tensors))(*[None if t is None else t.data_ptr() for t in tensors])


# ------------------------------------------------------------- entry points


def dpsgd_norms_workspace_bytes(layers, mode: int = DPSGD_NORM_AUTO) -> int:
    load()
    arr, n = _array(layers)
    return int(_lib.dpsgd_norms_workspace_bytes(arr, n, mode))


def dpsgd_select_norm_mode(layer: dpsgd_layer) -> int:
    load()
    r = int(_lib.dpsgd_select_norm_mode(ctypes.byref(layer)))
    if r < 0:
        _check("dpsgd_select_norm_mode", r)
    return r


def dpsgd_per_example_norms(layer, mode, norms_sq, accumulate=False, workspace=None,
                            stream=None):
    load()
    st = _lib.dpsgd_per_example_norms(ctypes.byref(layer), mode, _ptr(norms_sq), int(accumulate),
                                      _ptr(workspace),
                                      0 if workspace is None else workspace.numel(),
                                      _stream(stream))
    _check("dpsgd_per_example_norms", st)


def dpsgd_per_example_norms_multi(layers, mode, norms_sq, accumulate=False, workspace=None,
                                  stream=None):
    load()
    arr, n = _array(layers)
    st = _lib.dpsgd_per_example_norms_multi(arr, n, mode, _ptr(norms_sq), int(accumulate),
                                            _ptr(workspace),
                                            0 if workspace is None else workspace.numel(),
                                            _stream(stream))
    _check("dpsgd_per_example_norms_multi", st)


#: Bytes of the scratch array of dpsgd_per_example_norms_multi_noalloc.
DPSGD_NOALLOC_SCRATCH_BYTES = 8 << 20


def dpsgd_per_example_norms_multi_noalloc(layers, mode, norms_sq, accumulate=False, stream=None):
    load()
    arr, n = _array(layers)
    st = _lib.dpsgd_per_example_norms_multi_noalloc(arr, n, mode, _ptr(norms_sq), int(accumulate),
                                                    _stream(stream))
    _check("dpsgd_per_example_norms_multi_noalloc", st)


def dpsgd_clip_factors(norms_sq, C: float, factors=None, mask=None, stream=None):
    load()
    st = _lib.dpsgd_clip_factors(_ptr(norms_sq), norms_sq.numel(), C, _ptr(factors), _ptr(mask),
                                 _stream(stream))
    _check("dpsgd_clip_factors", st)


def dpsgd_clip_workspace_bytes(layers) -> int:
    load()
    arr, n = _array(layers)
    return int(_lib.dpsgd_clip_workspace_bytes(arr, n))


def dpsgd_clip_accumulate(layer, norms_sq, C, grad, accumulate=False, factors_out=None,
                          mask_out=None, workspace=None, stream=None):
    load()
    st = _lib.dpsgd_clip_accumulate(ctypes.byref(layer), _ptr(norms_sq), C, _ptr(grad),
                                    int(accumulate), _ptr(factors_out), _ptr(mask_out),
                                    _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                    _stream(stream))
    _check("dpsgd_clip_accumulate", st)


def dpsgd_clip_accumulate_multi(layers, norms_sq, C, grads, accumulate=False, factors_out=None,
                                mask_out=None, workspace=None, stream=None):
    load()
    arr, n = _array(layers)
    st = _lib.dpsgd_clip_accumulate_multi(arr, n, _ptr(norms_sq), C, _ptr_array(grads),
                                          int(accumulate), _ptr(factors_out), _ptr(mask_out),
                                          _ptr(workspace),
                                          0 if workspace is None else workspace.numel(),
                                          _stream(stream))
    _check("dpsgd_clip_accumulate_multi", st)


def dpsgd_clipped_sum_workspace_bytes(layers, mode: int = DPSGD_NORM_AUTO) -> int:
    load()
    arr, n = _array(layers)
    return int(_lib.dpsgd_clipped_sum_workspace_bytes(arr, n, mode))


def dpsgd_clipped_sum_multi(layers, mode, C, grads, norms_sq, accumulate=False, factors_out=None,
                            mask_out=None, workspace=None, stream=None):
    load()
    arr, n = _array(layers)
    st = _lib.dpsgd_clipped_sum_multi(arr, n, mode, C, _ptr_array(grads), int(accumulate),
                                      _ptr(norms_sq), _ptr(factors_out), _ptr(mask_out),
                                      _ptr(workspace),
                                      0 if workspace is None else workspace.numel(),
                                      _stream(stream))
    _check("dpsgd_clipped_sum_multi", st)


def dpsgd_add_noise(layer, grad, sigma, C, seed, step, scale, stream=None):
    load()
    st = _lib.dpsgd_add_noise(ctypes.byref(layer), _ptr(grad), sigma, C, seed, step, scale,
                              _stream(stream))
    _check("dpsgd_add_noise", st)


def dpsgd_add_noise_multi(layers, grads, sigma, C, seed, step, scale, stream=None):
    load()
    arr, n = _array(layers)
    st = _lib.dpsgd_add_noise_multi(arr, n, _ptr_array(grads), sigma, C, seed, step, scale,
                                    _stream(stream))
    _check("dpsgd_add_noise_multi", st)


def make_adamw(lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, t=1) -> dpsgd_adamw:
    return dpsgd_adamw(lr=lr, beta1=beta1, beta2=beta2, eps=eps, weight_decay=weight_decay, t=t)


def dpsgd_noise_adamw(layer, grad, param, exp_avg, exp_avg_sq, sigma, C, seed, step, scale, opt,
                      noisy_out=None, stream=None):
    load()
    st = _lib.dpsgd_noise_adamw(ctypes.byref(layer), _ptr(grad), _ptr(param), _ptr(exp_avg),
                                _ptr(exp_avg_sq), _ptr(noisy_out), sigma, C, seed, step, scale,
                                ctypes.byref(opt), _stream(stream))
    _check("dpsgd_noise_adamw", st)


def dpsgd_noise_adamw_multi(layers, grads, params, exp_avgs, exp_avg_sqs, sigma, C, seed, step,
                            scale, opt, noisy_outs=None, stream=None):
    load()
    arr, n = _array(layers)
    st = _lib.dpsgd_noise_adamw_multi(arr, n, _ptr_array(grads), _ptr_array(params),
                                      _ptr_array(exp_avgs), _ptr_array(exp_avg_sqs),
                                      None if noisy_outs is None else _ptr_array(noisy_outs),
                                      sigma, C, seed, step, scale, ctypes.byref(opt),
                                      _stream(stream))
    _check("dpsgd_noise_adamw_multi", st)


def dpsgd_philox_u32(out, first_block, n_blocks, seed, tensor_id, step, stream=None):
    load()
    st = _lib.dpsgd_philox_u32(_ptr(out), first_block, n_blocks, seed, tensor_id, step,
                               _stream(stream))
    _check("dpsgd_philox_u32", st)


def dpsgd_gaussian(out, n, seed, tensor_id, step, stream=None):
    load()
    st = _lib.dpsgd_gaussian(_ptr(out), n, seed, tensor_id, step, _stream(stream))
    _check("dpsgd_gaussian", st)


# ----------------------------------------- around the linear layers


_codes = {}   # dpsgd_dtype of a torch dtype, names of the other types that arguments may have


def _types():
    if not _codes:
        import torch
        _codes.update({torch.float32: DPSGD_F32, torch.bfloat16: DPSGD_BF16, torch.int32: "i32",
                       torch.int64: "i64", torch.uint8: "u8", "f32": torch.float32,
                       "bf16": torch.bfloat16, "u8": torch.uint8, "i64": torch.int64})
    return _codes


def _dtype_of(t) -> int:
    code = _types().get(t.dtype)
    if code is DPSGD_F32 or code is DPSGD_BF16:
        return code
    raise ValueError(f"float32 or bfloat16 expected, not {t.dtype}")


def _want(name, t, shape, code=None):
    """The address of t; raises ValueError unless it is a contiguous device tensor of
    this shape (and of the type with this code)."""
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, not {list(t.shape)}")
    if code is not None and _types().get(t.dtype) != code:
        raise ValueError(f"{name} must not be {t.dtype}")
    return t.data_ptr()


def _may_want(name, t, shape, code):
    return None if t is None else _want(name, t, shape, code)


def _workspace(workspace):
    """Address and bytes of a workspace; raises ValueError unless the device holds all of
    its bytes in a row."""
    if workspace is None:
        return None, 0
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def make_embedding(ids, table_shape, scale: float = 1.0) -> dpsgd_embedding:
    """Descriptor of a table [n_rows, d] and the ids [B, T] (int32 or int64, on the
    device) that look into it. An id outside the table is an empty position. The
    descriptor keeps ids alive."""
    code = _types().get(ids.dtype)
    if ids.dim() != 2 or (code != "i32" and code != "i64"):
        raise ValueError("ids must be [B, T], int32 or int64")
    if not ids.is_cuda or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous device tensor")
    B, T = ids.shape
    n_rows, d = table_shape
    emb = dpsgd_embedding(ids.data_ptr(), B, T, n_rows, d,
                          DPSGD_I64 if code == "i64" else DPSGD_I32, scale)
    emb.keep = ids
    return emb


def dpsgd_embedding_lookup(emb: dpsgd_embedding, table, out, stream=None):
    lib = _lib or load()
    st = lib.dpsgd_embedding_lookup(
        emb, _want("table", table, (emb.n_rows, emb.d)), _dtype_of(table),
        _want("out", out, (emb.B, emb.T, emb.d)), _dtype_of(out), _stream(stream))
    _check("dpsgd_embedding_lookup", st)


def dpsgd_embedding_workspace_bytes(emb: dpsgd_embedding) -> int:
    return int((_lib or load()).dpsgd_embedding_workspace_bytes(emb))


def dpsgd_embedding_norms(emb: dpsgd_embedding, G, norms_sq, accumulate=False, workspace=None,
                          stream=None):
    lib = _lib or load()
    B = emb.B
    st = lib.dpsgd_embedding_norms(
        emb, _want("G", G, (B, emb.T, emb.d)), _dtype_of(G),
        _want("norms_sq", norms_sq, (B,), DPSGD_F32), int(accumulate), *_workspace(workspace),
        _stream(stream))
    _check("dpsgd_embedding_norms", st)


def dpsgd_embedding_clip_accumulate(emb: dpsgd_embedding, G, norms_sq, C, grad, accumulate=False,
                                    factors_out=None, mask_out=None, workspace=None, stream=None):
    """norms_sq None: the plain sum over the batch (C is not looked at)."""
    lib = _lib or load()
    B, d = emb.B, emb.d
    st = lib.dpsgd_embedding_clip_accumulate(
        emb, _want("G", G, (B, emb.T, d)), _dtype_of(G),
        _may_want("norms_sq", norms_sq, (B,), DPSGD_F32), C,
        _want("grad", grad, (emb.n_rows, d), DPSGD_F32), int(accumulate),
        _may_want("factors_out", factors_out, (B,), DPSGD_F32),
        _may_want("mask_out", mask_out, (B,), "u8"), *_workspace(workspace), _stream(stream))
    _check("dpsgd_embedding_clip_accumulate", st)


def make_group_norm(x, groups: int, gamma=None, beta=None, eps: float = 1e-5,
                    act: str = "none") -> dpsgd_group_norm:
    """Descriptor of a group norm over channels-last rows x [B, ..., C] (every axis
    between the first and the last is a position: [B, S, C], [B, H, W, C]; a
    channels_last tensor [B, C, H, W] is x.permute(0, 2, 3, 1)). act: a name of
    ACTIVATIONS. The descriptor keeps gamma and beta alive."""
    shape, n = x.shape, x.numel()
    if len(shape) < 2 or n == 0:
        raise ValueError("x must be [B, ..., C] with no empty axis")
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
    B, C = shape[0], shape[-1]
    gn = dpsgd_group_norm(B, n // (B * C), C, groups, _may_want("gamma", gamma, (C,), DPSGD_F32),
                          _may_want("beta", beta, (C,), DPSGD_F32), _dtype_of(x),
                          ACTIVATIONS[act], eps)
    gn.keep = (gamma, beta)
    return gn


def _want_rows(name, t, B, C, n, dtype):
    """The address of t, a contiguous device tensor [B, ..., C] of n entries."""
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor")
    shape = t.shape
    if shape[0] != B or shape[-1] != C or t.numel() != n:
        raise ValueError(f"{name} must be [{B}, ({n // (B * C)} positions), {C}], not {list(shape)}")
    if _codes.get(t.dtype) != dtype:
        raise ValueError(f"{name} has another dtype than the descriptor")
    return t.data_ptr()


def dpsgd_group_norm_workspace_bytes(gn: dpsgd_group_norm) -> int:
    return int((_lib or load()).dpsgd_group_norm_workspace_bytes(gn))


def dpsgd_group_norm_forward(gn: dpsgd_group_norm, x, y, mean=None, rstd=None, workspace=None,
                             stream=None):
    lib = _lib or load()
    B, C, dt = gn.B, gn.C, gn.dtype
    n, stat = B * gn.S * C, (B, gn.groups)
    _types()
    st = lib.dpsgd_group_norm_forward(
        gn, _want_rows("x", x, B, C, n, dt), _want_rows("y", y, B, C, n, dt),
        _may_want("mean", mean, stat, DPSGD_F32), _may_want("rstd", rstd, stat, DPSGD_F32),
        *_workspace(workspace), _stream(stream))
    _check("dpsgd_group_norm_forward", st)


def dpsgd_group_norm_backward(gn: dpsgd_group_norm, x, dy, mean, rstd, dx, dgamma, dbeta,
                              workspace=None, stream=None):
    """dgamma and dbeta are per example ([B, C]); affine_layer makes layers of them."""
    lib = _lib or load()
    B, C, dt = gn.B, gn.C, gn.dtype
    n, stat, affine = B * gn.S * C, (B, gn.groups), (B, C)
    _types()
    st = lib.dpsgd_group_norm_backward(
        gn, _want_rows("x", x, B, C, n, dt), _want_rows("dy", dy, B, C, n, dt),
        _want("mean", mean, stat, DPSGD_F32), _want("rstd", rstd, stat, DPSGD_F32),
        _want_rows("dx", dx, B, C, n, dt), _want("dgamma", dgamma, affine, DPSGD_F32),
        _want("dbeta", dbeta, affine, DPSGD_F32), *_workspace(workspace), _stream(stream))
    _check("dpsgd_group_norm_backward", st)


def affine_layer(ones, grad, tensor_id: int) -> dpsgd_layer:
    """The per-example gradients [B, C] of a vector of parameters as a layer (T = 1,
    d_in = 1, activations ones [B]): the norm, clip, noise and step calls take it like
    any other float32 layer. The parameter's own buffers are [C, 1]."""
    B, C = grad.shape
    return make_layer(ones.view(B, 1, 1), grad.view(B, 1, C), tensor_id)


def dpsgd_global_norm_workspace_bytes(layers) -> int:
    lib = _lib or load()
    arr, n = _array(layers)
    return int(lib.dpsgd_global_norm_workspace_bytes(arr, n))


def _sizes(layers):
    return [L.d_in * L.d_out for L in ([layers] if isinstance(layers, dpsgd_layer) else layers)]


def _gradients(name, tensors, sizes):
    """The addresses of contiguous float32 device tensors with these numbers of entries."""
    if len(tensors) != len(sizes):
        raise ValueError(f"{name}: {len(sizes)} tensors expected, not {len(tensors)}")
    f32 = _types()["f32"]
    arr = (ctypes.c_void_p * len(sizes))()
    for k, (t, n) in enumerate(zip(tensors, sizes)):
        if t.dtype is not f32 or not t.is_cuda or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous float32 device tensors of d_out d_in entries")
        arr[k] = t.data_ptr()
    return arr


def _scalar(name, t):
    if t is None:
        return None
    if _types().get(t.dtype) != DPSGD_F32 or not t.is_cuda or t.numel() != 1:
        raise ValueError(f"{name} must be one float32 value on the device")
    return t.data_ptr()


def dpsgd_global_norm_multi(layers, grads, norm_out, workspace=None, stream=None):
    lib = _lib or load()
    arr, n = _array(layers)
    st = lib.dpsgd_global_norm_multi(arr, n, _gradients("grads", grads, _sizes(layers)),
                                     _scalar("norm_out", norm_out), *_workspace(workspace),
                                     _stream(stream))
    _check("dpsgd_global_norm_multi", st)


def dpsgd_global_clip_multi(layers, grads, outs, max_norm: float, norm_out=None, factor_out=None,
                            workspace=None, stream=None):
    """outs may be grads (in place)."""
    lib = _lib or load()
    arr, n = _array(layers)
    sizes = _sizes(layers)
    g = _gradients("grads", grads, sizes)
    o = g if outs is grads else _gradients("outs", outs, sizes)
    st = lib.dpsgd_global_clip_multi(arr, n, g, o, max_norm, _scalar("norm_out", norm_out),
                                     _scalar("factor_out", factor_out), *_workspace(workspace),
                                     _stream(stream))
    _check("dpsgd_global_clip_multi", st)


# -------------------------------------- between and behind the blocks


_device_of = None   # torch's current device, once CUDA is initialised


def _device():
    """The current device, whose stream the calls use; None where there is none."""
    global _device_of
    if _device_of is not None:
        return _device_of()
    import torch
    if not torch.cuda.is_available():
        return None
    torch.cuda.init()
    _device_of = torch._C._cuda_getDevice
    return _device_of()


_marshal = None   # the module of csrc/marshal.cpp
_F32, _BF16, _U8, _I32, _I64 = 6, 15, 0, 3, 4   # its codes of types
_scalar_codes = {}   # by torch type


def _load_marshal():
    global _marshal
    import torch  # noqa: F401  (whose libraries the module links against)
    try:
        from . import _marshal as module
    except ImportError as e:
        raise RuntimeError("paper_2609_20532_amd/_marshal.so is missing: build it with "
                           "`python -m paper_2609_20532_amd.build`") from e
    _scalar_codes.update({torch.float32: _F32, torch.bfloat16: _BF16, torch.uint8: _U8,
                          torch.int32: _I32, torch.int64: _I64})
    _marshal = module
    return module


def _refuse(name, t, shape, code, here):
    """Raises ValueError with what is wrong about t."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.get_device() != here:
        raise ValueError(f"{name} is on {t.device}, which is not the current device")
    if _scalar_codes.get(t.dtype) != code:
        raise ValueError(f"{name} must not be {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if len(shape) == 4 and shape[0] == -1:
        shape = (shape[1], f"({shape[3] // (shape[1] * shape[2])} positions)", shape[2])
    raise ValueError(f"{name} must be {list(shape)}, not {list(t.shape)}")


def _take(here, names, *spec):
    """The addresses of tensors (None for None); raises ValueError unless they are
    contiguous tensors on the device `here`. spec: tensor, shape, type code, in turn; the
    shape (-1, B, C, n) stands for [B, ..., C] with n entries."""
    m = _marshal or _load_marshal()
    got = m.take(-2 if here is None else here, *spec)
    if type(got) is int:
        _refuse(names[got], *spec[3 * got:3 * got + 3], here)
    return got


def _room(workspace, here):
    """Address and bytes of a workspace on the device `here`."""
    if workspace is not None and workspace.get_device() != here:
        _refuse("workspace", workspace, workspace.shape, None, here)
    return _workspace(workspace)


def _logit_rows(name, t):
    """B, T, V and the entries from a row to the next of logits [B, T, V]."""
    if t.dim() != 3 or t.numel() == 0:
        raise ValueError(f"{name} must be [B, T, V] with no empty axis")
    B, T, V = t.shape
    if t.is_contiguous():
        return B, T, V, V
    sB, sT, sV = t.stride()
    stride = sT if T > 1 else (sB if B > 1 else V)
    if (V > 1 and sV != 1) or stride < V or (B > 1 and T > 1 and sB != T * sT):
        raise ValueError(f"{name}: entries of a row must be neighbours, and rows evenly spaced")
    return B, T, V, stride


def _logits_of(name, t, here):
    """Address, B, T, V, entries from row to row and type code of logits."""
    got = (_marshal or _load_marshal()).logits(-2 if here is None else here, t)
    if got is None:
        _logit_rows(name, t)
        _refuse(name, t, t.shape, _scalar_codes.get(t.dtype), here)
    return got


def make_logits(logits, targets=None, scale: float = 1.0) -> dpsgd_logits:
    """Descriptor of logits [B, T, V] (float32 or bfloat16; a view such as x[..., :V] or
    x[:, -1:] is taken as it lies) and the token of each position, targets [B, T] (int32
    or int64, contiguous; one outside [0, V) is an empty position), or None. scale is 1 /
    temperature. The descriptor keeps targets alive, and is for logits of this layout."""
    here = _device()
    _, B, T, V, stride, code = _logits_of("logits", logits, here)
    if code != _F32 and code != _BF16:
        raise ValueError(f"float32 or bfloat16 expected, not {logits.dtype}")
    at, index = None, _I64
    if targets is not None:
        index = _scalar_codes.get(targets.dtype)
        if index != _I64 and index != _I32:
            raise ValueError("targets must be [B, T], int32 or int64")
        at, = _take(here, ("targets",), targets, (B, T), index)
    desc = dpsgd_logits(at, B, T, V, stride, DPSGD_I64 if index == _I64 else DPSGD_I32,
                        DPSGD_F32 if code == _F32 else DPSGD_BF16, scale)
    desc.keep = targets
    return desc


def _take_logits(name, t, desc, here):
    """The address of t, rows like the descriptor's, and the entries from row to row."""
    p, B, T, V, stride, code = _logits_of(name, t, here)
    if B != desc.B or T != desc.T or V != desc.V:
        raise ValueError(f"{name} must be [{desc.B}, {desc.T}, {desc.V}] as the descriptor has it")
    if code != (_BF16 if desc.dtype == DPSGD_BF16 else _F32):
        raise ValueError(f"{name} has another dtype than the descriptor")
    return p, stride


def _described(logits, desc, here):
    """The address of the descriptor's logits."""
    p, stride = _take_logits("logits", logits, desc, here)
    if stride != desc.stride:
        raise ValueError("logits have their rows elsewhere than the descriptor says")
    return p


def dpsgd_token_workspace_bytes(desc: dpsgd_logits, k: int = 0) -> int:
    return int((_lib or load()).dpsgd_token_workspace_bytes(desc, k))


def dpsgd_token_logprobs(desc: dpsgd_logits, logits, logprobs=None, lse=None, entropy=None,
                         top_ids=None, top_logprobs=None, workspace=None, stream=None):
    """Any of the outputs; top_ids (int64) and top_logprobs are [B, T, k]."""
    lib, here = _lib or load(), _device()
    some = top_ids if top_logprobs is None else top_logprobs
    k = 0 if some is None else some.shape[-1]
    if some is not None and k == 0:
        raise ValueError("no alternatives: leave top_ids and top_logprobs out")
    p, rows = _described(logits, desc, here), (desc.B, desc.T)
    tops = (*rows, k)
    lp, ls, en, ids, lps = _take(
        here, ("logprobs", "lse", "entropy", "top_ids", "top_logprobs"), logprobs, rows, _F32,
        lse, rows, _F32, entropy, rows, _F32, top_ids, tops, _I64, top_logprobs, tops, _F32)
    st = lib.dpsgd_token_logprobs(desc, p, lp, ls, en, k, ids, lps, *_room(workspace, here),
                                  _stream(stream))
    _check("dpsgd_token_logprobs", st)


def dpsgd_token_logprobs_backward(desc: dpsgd_logits, logits, lse, dlogits, entropy=None,
                                  grad_logprobs=None, grad_lse=None, grad_entropy=None,
                                  stream=None):
    """dlogits may be logits."""
    lib, here = _lib or load(), _device()
    p, rows = _described(logits, desc, here), (desc.B, desc.T)
    ls, en, gp, gl, ge = _take(
        here, ("lse", "entropy", "grad_logprobs", "grad_lse", "grad_entropy"), lse, rows, _F32,
        entropy, rows, _F32, grad_logprobs, rows, _F32, grad_lse, rows, _F32, grad_entropy, rows, _F32)
    st = lib.dpsgd_token_logprobs_backward(desc, p, ls, en, gp, gl, ge,
                                           *_take_logits("dlogits", dlogits, desc, here),
                                           _stream(stream))
    _check("dpsgd_token_logprobs_backward", st)


def dpsgd_token_loss(desc: dpsgd_logits, logits, dlogits, losses=None, weights=None, logprobs=None,
                     workspace=None, stream=None):
    """Per-example losses [B] and the gradient of their sum; dlogits may be logits."""
    lib, here = _lib or load(), _device()
    p, B = _described(logits, desc, here), desc.B
    rows = (B, desc.T)
    w, loss, lp = _take(here, ("weights", "losses", "logprobs"), weights, rows, _F32, losses, (B,),
                        _F32, logprobs, rows, _F32)
    st = lib.dpsgd_token_loss(desc, p, w, loss, lp, *_take_logits("dlogits", dlogits, desc, here),
                              *_room(workspace, here), _stream(stream))
    _check("dpsgd_token_loss", st)


def make_residual_norm(x, kind: str = "layer", gamma=None, beta=None, gate=None, post: bool = False,
                       post_gamma=None, post_beta=None, residual_scale: float = 1.0,
                       eps: float = 1e-5) -> dpsgd_residual_norm:
    """Descriptor of the residual sum and norms over rows like x's, [B, ..., C] (every
    axis between the first and the last is a position). kind: a name of ROW_NORMS. gate
    is [C] or, one for each example, [B, C]. The descriptor keeps the parameters alive."""
    shape, n, here = x.shape, x.numel(), _device()
    if len(shape) < 2 or n == 0:
        raise ValueError("x must be [B, ..., C] with no empty axis")
    if kind not in ROW_NORMS:
        raise ValueError(f"kind must be one of {sorted(ROW_NORMS)}")
    B, C, code = shape[0], shape[-1], _dtype_of(x)
    each = gate is not None and gate.dim() == 2
    c = (C,)
    at = _take(here, ("gamma", "beta", "post_gamma", "post_beta", "gate"), gamma, c, _F32, beta, c, _F32,
               post_gamma, c, _F32, post_beta, c, _F32, gate, (B, C) if each else c, _F32)
    desc = dpsgd_residual_norm(B, n // (B * C), C, *at, each, bool(post), ROW_NORMS[kind], code,
                               residual_scale, eps)
    desc.keep = (gamma, beta, post_gamma, post_beta, gate)
    return desc


def _layout_of(desc):
    """Shape (for _take) and type code of rows like the descriptor's, and B, S, C."""
    B, S, C = desc.B, desc.S, desc.C
    return (-1, B, C, B * S * C), _BF16 if desc.dtype == DPSGD_BF16 else _F32, B, S, C


def dpsgd_residual_norm_forward(desc: dpsgd_residual_norm, x, block, r, y, stats=None, stream=None):
    """block None: r = residual_scale x; r None: not written. stats: [B, S, 4]."""
    lib, here = _lib or load(), _device()
    rows, code, B, S, _ = _layout_of(desc)
    at = _take(here, ("x", "block", "r", "y", "stats"), x, rows, code, block, rows, code, r, rows,
               code, y, rows, code, stats, (B, S, 4), _F32)
    _check("dpsgd_residual_norm_forward", lib.dpsgd_residual_norm_forward(desc, *at, _stream(stream)))


def dpsgd_residual_norm_workspace_bytes(desc: dpsgd_residual_norm) -> int:
    return int((_lib or load()).dpsgd_residual_norm_workspace_bytes(desc))


def dpsgd_residual_norm_backward(desc: dpsgd_residual_norm, block, r, dy, dr, stats, dx=None,
                                 dblock=None, dgamma=None, dbeta=None, dgate=None,
                                 dpost_gamma=None, dpost_beta=None, workspace=None, stream=None):
    """The gradients of the affine parameters are per example ([B, C]); affine_layer
    makes layers of them. Any of the results may be left out (dblock with block)."""
    lib, here = _lib or load(), _device()
    rows, code, B, S, C = _layout_of(desc)
    one = (B, C)
    at = _take(here, ("block", "r", "dy", "dr", "stats", "dx", "dblock", "dgamma", "dbeta", "dgate",
                      "dpost_gamma", "dpost_beta"), block, rows, code, r, rows, code, dy, rows, code,
               dr, rows, code, stats, (B, S, 4), _F32, dx, rows, code, dblock, rows, code, dgamma, one,
               _F32, dbeta, one, _F32, dgate, one, _F32, dpost_gamma, one, _F32, dpost_beta, one, _F32)
    st = lib.dpsgd_residual_norm_backward(desc, *at, *_room(workspace, here), _stream(stream))
    _check("dpsgd_residual_norm_backward", st)


def make_states8(layers, device="cuda"):
    """8-bit moments of 0 for the layers' tensors: exp_avgs, exp_avg_sqs (uint8 [d_out,
    d_in]) and exponents (uint8 [ceil(d_out d_in / 256), 2])."""
    import torch
    ms, vs, exps = [], [], []
    for L in [layers] if isinstance(layers, dpsgd_layer) else layers:
        for to in (ms, vs):
            to.append(torch.zeros(L.d_out, L.d_in, dtype=torch.uint8, device=device))
        exps.append(torch.zeros(-(-L.d_out * L.d_in // DPSGD_STATE_BLOCK), 2, dtype=torch.uint8,
                                device=device))
    return ms, vs, exps


def _tensors(name, tensors, layers, n, code, here, per_block=0):
    """The addresses of contiguous tensors on the device `here`, one for each of the n
    descriptors in the ctypes array `layers`, with this type code and d_out d_in entries
    (or a pair for every block of them)."""
    m, arr = _marshal or _load_marshal(), (ctypes.c_void_p * n)()
    if not m.addresses(tensors, layers, per_block, code, -2 if here is None else here, arr):
        if len(tensors) != n:
            raise ValueError(f"{name}: {n} tensors expected, not {len(tensors)}")
        for k, t in enumerate(tensors):
            size = layers[k].d_in * layers[k].d_out
            if per_block:
                size = 2 * -(-size // DPSGD_STATE_BLOCK)
            if t.get_device() != here or not t.is_contiguous() or _scalar_codes.get(t.dtype) != code:
                _refuse(f"{name}[{k}]", t, t.shape, code, here)
            if t.numel() != size:
                raise ValueError(f"{name}[{k}] must have {size} entries, not {t.numel()}")
        raise ValueError(f"{name} must be contiguous device tensors")
    return arr


def _layer_array(layers):
    """_array for lists of descriptors, whose bytes are joined (a seventh of its time)."""
    if type(layers) is list and set(map(type, layers)) == {dpsgd_layer}:
        n = len(layers)
        return (dpsgd_layer * n).from_buffer_copy(b"".join(layers)), n
    return _array(layers)


def _states8(exp_avgs, exp_avg_sqs, exponents, layers, n, here):
    return (_tensors("exp_avgs", exp_avgs, layers, n, _U8, here),
            _tensors("exp_avg_sqs", exp_avg_sqs, layers, n, _U8, here),
            _tensors("exponents", exponents, layers, n, _U8, here, 1))


def dpsgd_noise_adamw8_multi(layers, grads, params, exp_avgs, exp_avg_sqs, exponents, sigma, C,
                             seed, step, scale, opt, round_seed=None, noisy_outs=None,
                             stream=None):
    """round_seed: of stochastic rounding of the moments; None rounds to nearest."""
    lib, here = _lib or load(), _device()
    arr, n = _layer_array(layers)
    noisy = None
    if noisy_outs is not None:
        if len(noisy_outs) != n:
            raise ValueError(f"noisy_outs: {n} entries expected, not {len(noisy_outs)}")
        for k, t in enumerate(noisy_outs):
            if t is not None:
                _tensors("noisy_outs", [t], (dpsgd_layer * 1)(arr[k]), 1, _F32, here)
        noisy = _ptr_array(noisy_outs)
    st = lib.dpsgd_noise_adamw8_multi(
        arr, n, _tensors("grads", grads, arr, n, _F32, here),
        _tensors("params", params, arr, n, _F32, here),
        *_states8(exp_avgs, exp_avg_sqs, exponents, arr, n, here), noisy, sigma, C, seed, step,
        scale, ctypes.byref(opt), DPSGD_ROUND_NEAREST if round_seed is None else DPSGD_ROUND_STOCHASTIC,
        0 if round_seed is None else round_seed, _stream(stream))
    _check("dpsgd_noise_adamw8_multi", st)


def dpsgd_adamw8_pack_multi(layers, exp_avgs_in, exp_avg_sqs_in, exp_avgs, exp_avg_sqs, exponents,
                            stream=None):
    """float32 moments to 8 bits."""
    lib, here = _lib or load(), _device()
    arr, n = _layer_array(layers)
    st = lib.dpsgd_adamw8_pack_multi(
        arr, n, _tensors("exp_avgs_in", exp_avgs_in, arr, n, _F32, here),
        _tensors("exp_avg_sqs_in", exp_avg_sqs_in, arr, n, _F32, here),
        *_states8(exp_avgs, exp_avg_sqs, exponents, arr, n, here), _stream(stream))
    _check("dpsgd_adamw8_pack_multi", st)


def dpsgd_adamw8_unpack_multi(layers, exp_avgs, exp_avg_sqs, exponents, exp_avgs_out,
                              exp_avg_sqs_out, stream=None):
    """The moments that 8-bit states stand for, all float32 or all bfloat16 (both exact)."""
    lib, here = _lib or load(), _device()
    arr, n = _layer_array(layers)
    if len(exp_avgs_out) != n or n == 0:
        raise ValueError(f"exp_avgs_out: {n} tensors expected, not {len(exp_avgs_out)}")
    code = _dtype_of(exp_avgs_out[0])
    element = _BF16 if code == DPSGD_BF16 else _F32
    st = lib.dpsgd_adamw8_unpack_multi(
        arr, n, *_states8(exp_avgs, exp_avg_sqs, exponents, arr, n, here),
        _tensors("exp_avgs_out", exp_avgs_out, arr, n, element, here),
        _tensors("exp_avg_sqs_out", exp_avg_sqs_out, arr, n, element, here), code, _stream(stream))
    _check("dpsgd_adamw8_unpack_multi", st)


# ------------------------------------------------------------ whole step


@dataclass
class StepBuffers:
    """Device buffers of one step: norms, factors, mask, workspaces, grads."""

    norms_sq: object
    factors: object
    mask: object
    norms_ws: object
    clip_ws: object
    grads: list
    fused_ws: object = None   # workspace of dpsgd_clipped_sum_multi (alloc_step(fused=True))


def alloc_step(layers, mode: int = DPSGD_NORM_AUTO, device="cuda", fused: bool = False) -> StepBuffers:
    """Allocate (with torch) every buffer a step over ``layers`` needs; with
    ``fused`` also the workspace of the one-call form (run_step(fused=True))."""
    import torch
    B = layers[0].B
    nb = dpsgd_norms_workspace_bytes(layers, mode)
    cb = dpsgd_clip_workspace_bytes(layers)
    fb = dpsgd_clipped_sum_workspace_bytes(layers, mode) if fused else 0
    return StepBuffers(
        norms_sq=torch.empty(B, dtype=torch.float32, device=device),
        factors=torch.empty(B, dtype=torch.float32, device=device),
        mask=torch.empty(B, dtype=torch.uint8, device=device),
        norms_ws=torch.empty(max(nb, 1), dtype=torch.uint8, device=device),
        clip_ws=torch.empty(max(cb, 1), dtype=torch.uint8, device=device),
        grads=[torch.empty((L.d_out, L.d_in), dtype=torch.float32, device=device)
               for L in layers],
        fused_ws=torch.empty(max(fb, 1), dtype=torch.uint8, device=device) if fused else None,
    )


def run_clipped_sum(layers, buf: StepBuffers, C: float, mode: int = DPSGD_NORM_AUTO, stream=None,
                    fused: bool = False):
    """The step up to its commit point: global norms, clip factors and the
    clipped sums in ``buf.grads`` (two ABI calls, or one with ``fused``)."""
    if fused:
        dpsgd_clipped_sum_multi(layers, mode, C, buf.grads, buf.norms_sq, accumulate=False,
                                factors_out=buf.factors, mask_out=buf.mask,
                                workspace=buf.fused_ws, stream=stream)
    else:
        dpsgd_per_example_norms_multi(layers, mode, buf.norms_sq, accumulate=False,
                                      workspace=buf.norms_ws, stream=stream)
        dpsgd_clip_accumulate_multi(layers, buf.norms_sq, C, buf.grads, accumulate=False,
                                    factors_out=buf.factors, mask_out=buf.mask,
                                    workspace=buf.clip_ws, stream=stream)


def run_step(layers, buf: StepBuffers, C: float, sigma: float, seed: int, step: int = 0,
             scale: float = 1.0, mode: int = DPSGD_NORM_AUTO, stream=None, fused: bool = False):
    """One DP-SGD gradient step: global norms, clip + sum, noise (three ABI
    calls, or two with ``fused``: dpsgd_clipped_sum_multi, then the noise)."""
    run_clipped_sum(layers, buf, C, mode, stream, fused)
    dpsgd_add_noise_multi(layers, buf.grads, sigma, C, seed, step, scale, stream=stream)


class StepGraph:
    """The clipped-sum part of a step captured as a HIP graph (torch.cuda.CUDAGraph),
    replayed once per step, followed by the noise call.

    The library makes no allocation, memset or synchronising call while it
    enqueues, so the norms, factors and clipped sums (two ABI calls, or one
    with ``fused``) can be captured. A replay re-runs them with the arguments
    of the capture: the same input and output buffers (refill the inputs in
    place between replays) and the same C. The noise is not captured: it is
    enqueued after each replay with the seed and step that ``replay`` is
    given, because a captured noise kernel would add the same normals at
    every replay. A (seed, step) pair that this object has already released
    is refused: the noise of every release must be fresh."""

    def __init__(self, layers, buf: StepBuffers, C: float, sigma: float, scale: float = 1.0,
                 mode: int = DPSGD_NORM_AUTO, fused: bool = False):
        import torch
        load()
        self._keep = (layers, buf)
        self._noise = (sigma, C, scale)
        self._used = set()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):   # one eager pass first, outside the capture
            run_clipped_sum(layers, buf, C, mode, fused=fused)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            run_clipped_sum(layers, buf, C, mode, fused=fused)

    def replay(self, seed: int, step: int):
        """One step: the captured clipped sums, then noise keyed by (seed, step)."""
        key = (int(seed), int(step))
        if key in self._used:
            raise ValueError(f"noise (seed, step) = {key} was already released by this graph")
        self._used.add(key)
        layers, buf = self._keep
        sigma, C, scale = self._noise
        self.graph.replay()
        dpsgd_add_noise_multi(layers, buf.grads, sigma, C, seed, step, scale)
