"""The package and torch share one HIP runtime, whichever is imported first."""
import subprocess
import sys

import pytest

LOOK = """
import {0}
import {1}
import torch, paper_2608_23805_amd as msi
msi.linear
print(len({{l.split()[-1] for l in open('/proc/self/maps') if 'libamdhip64' in l}}))
"""


@pytest.mark.parametrize("order", [("torch", "paper_2608_23805_amd"), ("paper_2608_23805_amd", "torch")])
def test_one_hip_runtime(order):
    r = subprocess.run([sys.executable, "-c", LOOK.format(*order)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert r.stdout.split()[-1] == "1"


@pytest.mark.gpu
@pytest.mark.parametrize("first", ["torch", "paper_2608_23805_amd"])
def test_calls_after_either_import(first):
    """A projection and a residual step of a process that imports the package before torch, and after it."""
    code = f"""
import {first}
import paper_2608_23805_amd as msi
import torch
x, w = torch.ones((2, 8), device="cuda").bfloat16(), torch.ones((4, 8), device="cuda").bfloat16()
y = torch.empty((2, 4), device="cuda")
msi.linear(x, w, y)
h, xn = torch.zeros((2, 4), device="cuda"), torch.empty((2, 4), dtype=torch.bfloat16, device="cuda")
msi.residual_add(y, h, xn)
torch.cuda.synchronize()
assert torch.all(y == 8) and torch.all(h == 8) and torch.all(xn == 1)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr
