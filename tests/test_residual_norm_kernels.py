"""The residual norm's kernels that the library holds are the ones that some call reaches:
the plans of every width in both types against the built library's own launch stubs (CPU)."""

import re
import shutil
import subprocess

import pytest

from paper_2609_20532_amd import build
from test_lm_ops_index import plan_rows


def _reached(elements):
    """(type, V, vectors a thread, most threads, whole waves) of all widths."""
    out = set()
    for bf16 in (False, True):
        for C in range(1, 16385):
            V, nv, log, threads, _ = plan_rows(C, bf16, elements)
            most = 1024 if threads > 512 else (512 if threads > 256 else 256)
            out.add(("unsigned short" if bf16 else "float", V, nv, most, log >= 6))
    return out


def _compiled():
    nm = shutil.which("nm") or shutil.which("llvm-nm", path="/opt/rocm/llvm/bin")
    if not nm:
        pytest.skip("no nm")
    text = subprocess.run([nm, "-C", build.LIB], capture_output=True, text=True, check=True).stdout
    forward = re.findall(r"__device_stub__rn_forward_kernel<([\w ]+), (\d+), (\d+), (\d+), (true|false)>", text)
    backward = re.findall(r"__device_stub__rn_backward_kernel<([\w ]+), (\d+), (\d+), (\d+), \D*(\d+)\D*, (true|false)>", text)
    key = lambda t, V, nv, most, wide: (t, int(V), int(nv), int(most), wide == "true")
    return ({key(*m) for m in forward}, [{key(*m[:4], m[5]) for m in backward if m[4] == str(kind)} for kind in range(3)])


def test_every_kernel_is_reached_and_there():
    forward, backward = _compiled()
    assert forward == _reached(16)
    for kind in backward:
        assert kind == _reached(8)
