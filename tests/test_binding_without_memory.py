"""Device tensors that have no memory, which the binding's native module looks at before
any call: inside a function transform a tensor has no address, and asking for it throws.
Runs on the CPU, on tensors that only claim to be on a device; each case in a process of
its own, because an exception that passed through the interpreter would end it."""

import subprocess
import sys

import pytest

PRELUDE = """
import ctypes, sys, warnings
warnings.simplefilter("ignore")
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2609_20532_amd import dpsgd
m = dpsgd._load_marshal()
mode = FakeTensorMode()
with mode:
    x = torch.empty(2, 3, 5, device="cuda:0")
    flat = torch.empty(2, 6, device="cuda:0")
layers = (dpsgd.dpsgd_layer * 1)(dpsgd.shape_layer(1, 1, 3, 2))
buf = (ctypes.c_void_p * 1)()

def raises(f, *args):
    try:
        f(*args)
    except RuntimeError as e:
        print("raised", type(e).__name__)
        return
    sys.exit("no error")

def inside(f, t):
    def body(v):
        f(v)
        return v
    with mode:
        torch.func.vmap(body)(t)
"""

CASES = {
    "take in a transform": "inside(lambda v: raises(m.take, 0, v, (3, 5), 6), x)",
    "take behind another tensor": "inside(lambda v: raises(m.take, 0, None, 0, 0, v, (3, 5), 6), x)",
    "logits in a transform": "inside(lambda v: raises(m.logits, 0, v.unsqueeze(0)), x)",
    "addresses in a transform": "inside(lambda v: raises(m.addresses, [v], layers, 0, 6, 0, buf), flat)",
    "take of no memory": "raises(m.take, 0, x, (2, 3, 5), 6)",
    "logits of no memory": "raises(m.logits, 0, x)",
    "addresses of no memory": "raises(m.addresses, [flat[0]], layers, 0, 6, 0, buf)",
}


@pytest.mark.parametrize("name", list(CASES))
def test_a_tensor_without_memory_raises(name):
    # The same call again: nothing of the first one is left behind.
    code = PRELUDE + CASES[name] + "\n" + CASES[name] + "\nprint('whole')\n"
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout[-500:] + run.stderr[-1500:]
    assert run.stdout.count("raised RuntimeError") == 2 and "whole" in run.stdout


def test_empty_tensors_have_no_address():
    """No entries, no memory: no error of this kind (their shapes are refused, or fit)."""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode

    from paper_2609_20532_amd import dpsgd
    m = dpsgd._load_marshal()
    with FakeTensorMode():
        x = torch.empty(0, 5, device="cuda:0")
    assert m.take(0, x, (0, 5), 6) == (0,) and m.take(0, x, (5,), 6) == 0
