"""Refusals of the 8-bit moments' calls that need several launches (CPU only: every call is
refused before its first launch, of which a machine without a GPU would report an error)."""

import ctypes

import pytest

from paper_2609_20532_amd import dpsgd

INVALID = -1
P = ctypes.c_void_p


def _call(name, layers):
    n = len(layers)
    lib, arr = dpsgd.load(), (dpsgd.dpsgd_layer * n)(*layers)
    at = [(P * n)(*(1 << 44 | k << 40 | l << 20 for l in range(n))) for k in range(6)]
    if name == "step":
        opt = dpsgd.make_adamw(1e-3)
        return lib.dpsgd_noise_adamw8_multi(arr, n, *at, 0.5, 1.0, 1, 2, 1.0, ctypes.byref(opt), 0, 3, None)
    if name == "pack":
        return lib.dpsgd_adamw8_pack_multi(arr, n, *at[:5], None)
    return lib.dpsgd_adamw8_unpack_multi(arr, n, *at[:5], 0, None)


@pytest.mark.parametrize("name", ["step", "pack", "unpack"])
@pytest.mark.parametrize("before", [48, 96])
def test_a_call_is_refused_before_its_first_launch(name, before):
    """48 tensors a launch; the last launch would have 2^32 threads."""
    small = [dpsgd.shape_layer(1, 1, 3, 5, 0, k) for k in range(before)]
    assert _call(name, small + [dpsgd.shape_layer(1, 1, 1 << 18, 1 << 18, 0, before)]) == INVALID
