"""Projection: every tile form that the rule chooses, at its row, feature and K edges, and GELU's tails.

A case asserts the form that its sizes are sent to, so that a change of the rule cannot leave a form untested.
The bound of the products is the one of the projection's other tests."""
import ctypes

import numpy as np
import pytest

from _gpu_helpers import log
from test_gpu_linear import _case

pytestmark = pytest.mark.gpu


def _tile(M, N):
    import paper_2608_23805_amd as msi
    v = [ctypes.c_uint32() for _ in range(3)]
    msi._check(msi.lib.msi_debug_linear_tile(M, N, *map(ctypes.byref, v)))
    return tuple(x.value for x in v)


@pytest.mark.parametrize("M,N,tile", [
    (33, 4095, (32, 32, 2)), (70, 5003, (32, 64, 1)), (300, 3000, (64, 64, 1)), (509, 4050, (64, 128, 1)),
    (449, 4033, (64, 128, 1)), (1000, 3001, (128, 128, 1)), (1030, 4097, (128, 128, 2)), (2500, 2500, (128, 128, 2)),
    (4000, 4050, (256, 256, 1)), (3841, 4033, (256, 256, 1)),
])
@pytest.mark.parametrize("K", [8, 64, 72, 136, 200])
def test_form(M, N, tile, K):
    """One stage, odd and even numbers of stages, tails of K inside every form's stages; rows and features that end
    inside a tile, one of them by one row and one feature."""
    assert _tile(M, N) == tile
    _case(M, K, N, act="gelu", residual="bf16", out="bf16")
    _case(M, K, N, residual="f32", out="f32", inplace=True)


def test_forms_of_long_sums():
    """The two-buffer loops over many stages, with and without a tail."""
    for M, N, K in ((4000, 4050, 1096), (4000, 4050, 1024), (509, 4050, 1096), (1030, 4097, 1032)):
        _case(M, K, N, act="silu", residual="f32", out="f32", pad=8)


def _gelu(z):
    """z Phi(z) in 64 bits without cancellation."""
    from scipy.special import log_ndtr
    return z * np.exp(log_ndtr(z))


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("N", [4099, 4100])
def test_gelu_keeps_its_tail(out, N):
    """z Phi(z) to a bound relative to itself, from z = -12.5 on.  x is zero, so z is the bias, exactly.  The value moves by
    z^2 + 1 times a relative change of z (for large negative z); counted in units of 2^-24, a kernel in fp32 that rounds z^2, its
    product with a constant and the exponential (1 ulp), and evaluates the rest with a reciprocal (1 ulp) whose error counts up to
    2.3 times, is off by at most 1.25 z^2 + 16 of them: less than 4 (z^2 + 4)."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case gelu tail {out} N={N}")
    z = np.linspace(-12.5, 12.5, N).astype(np.float32)
    z[:64] = -np.exp2(np.linspace(-30, 3.6, 64)).astype(np.float32)
    x, w = torch.zeros((3, 8), device="cuda").bfloat16(), torch.ones((N, 8), device="cuda").bfloat16()
    y = torch.empty((3, N), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    msi.linear(x, w, y, bias=torch.from_numpy(z).cuda(), act="gelu")
    torch.cuda.synchronize()
    z = z.astype(np.float64)
    want = _gelu(z)
    tol = np.abs(want) * ((z * z + 4) * 2.0 ** -22 + (2.0 ** -8 if out == "bf16" else 2.0 ** -24))
    got = y.double().cpu().numpy()
    worst = int(np.argmax(np.max(np.abs(got - want), axis=0) / np.where(tol > 0, tol, 1)))
    assert np.all(np.abs(got - want) <= tol), (z[worst], got[0, worst], want[worst])


def test_gelu_of_normal_arguments():
    """Over standard-normal arguments the error (root of the mean square, relative to the values') is no larger than what
    0.5 z (1 + erf(z / sqrt 2)) leaves in fp32: 3.8e-8, computed with each operation rounded once."""
    import torch
    import paper_2608_23805_amd as msi
    log("case gelu, normal arguments")
    z = np.random.default_rng(80).standard_normal(1 << 18).astype(np.float32)
    x, w = torch.zeros((1, 8), device="cuda").bfloat16(), torch.ones((len(z), 8), device="cuda").bfloat16()
    y = torch.empty((1, len(z)), device="cuda")
    msi.linear(x, w, y, bias=torch.from_numpy(z).cuda(), act="gelu")
    torch.cuda.synchronize()
    want = _gelu(z.astype(np.float64))
    err = y[0].double().cpu().numpy() - want
    assert np.sqrt((err ** 2).sum() / (want ** 2).sum()) <= 3.8e-8


def test_gelu_of_infinities_and_nan():
    import torch
    import paper_2608_23805_amd as msi
    log("case gelu, infinities")
    x, w = torch.zeros((1, 8), device="cuda").bfloat16(), torch.ones((4, 8), device="cuda").bfloat16()
    y = torch.empty((1, 4), device="cuda")
    msi.linear(x, w, y, bias=torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0], device="cuda"), act="gelu")
    torch.cuda.synchronize()
    v = y[0].cpu().tolist()
    assert v[0] == float("inf") and v[1] == 0.0 and v[2] != v[2] and v[3] == 0.0
