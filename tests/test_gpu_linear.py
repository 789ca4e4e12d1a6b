"""Projection with its epilogue against 64 bits: every kernel's row and feature edges,
activations, residual and output types, strided rows, an output that is its residual.

Bound per element: the fp32 sum of K exact products, each addition off by at most
2^-24 of the running magnitude (K 2^-24 sum |x w|, of which chance leaves far less:
sqrt(K) 2^-22 is taken), the activation's few roundings (2^-20 of |z|, slope at most
1.13), and half a step of the output's type."""
import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import bf16
from _kv_oracle import linear as oracle

pytestmark = pytest.mark.gpu


def _case(M, K, N, act="none", residual="none", out="f32", bias=True, pad=0, inplace=False, seed=0):
    import torch
    import paper_2608_23805_amd as msi
    log(f"case linear M={M} K={K} N={N} {act} {residual} {out} pad={pad} inplace={inplace}")
    g = np.random.default_rng([78, M, K, N, seed])
    x, xh = bf16(g.standard_normal((M, K + pad)))
    w, wh = bf16(g.standard_normal((N, K)) * K ** -0.5)
    b = g.standard_normal(N).astype(np.float32) if bias else None
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    r = rh = None
    if residual != "none":
        r, rh = bf16(g.standard_normal((M, N + pad)))
        r = r.to(types[residual])[:, :N]
        rh = rh[:, :N]
    buf = torch.full((M + 1, N + pad), 7.0, dtype=types[out], device="cuda")
    y = r if inplace else buf[:M, :N]
    want = oracle(xh[:, :K], wh, b, act, rh)
    msi.linear(x[:, :K], w, y, bias=None if b is None else torch.from_numpy(b).cuda(), act=act, residual=r,
               stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    got = y.double().cpu().numpy()
    size = np.abs(xh[:, :K]) @ np.abs(wh).T + (0 if b is None else np.abs(b))
    tol = 1.13 * (K ** 0.5 * 2.0 ** -22 + 2.0 ** -20) * size + (2.0 ** -8 if out == "bf16" else 2.0 ** -23) * np.abs(want) + 1e-30
    if rh is not None:
        tol = tol + 2.0 ** -23 * np.abs(rh)
    assert np.all(np.abs(got - want) <= tol), float(np.max(np.abs(got - want) / tol))
    if not inplace:
        assert torch.all(buf[M] == 7.0) and (pad == 0 or torch.all(buf[:, N:] == 7.0))     # nothing beside the output


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 32, 33, 63, 65, 130])
@pytest.mark.parametrize("K,N", [(8, 1), (72, 31), (512, 256), (1096, 130)])
def test_rows_and_features(M, K, N):
    _case(M, K, N)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("residual,out", [("none", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("M", [5, 70])
def test_epilogue(act, residual, out, M):
    _case(M, 264, 100, act, residual, out)
    _case(M, 264, 101, act, residual, out, bias=False, pad=8)


@pytest.mark.parametrize("M", [4, 70])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_in_place(M, kind):
    _case(M, 128, 192, residual=kind, out=kind, inplace=True)


@pytest.mark.parametrize("M,K,N", [
    (33, 1000, 4095), (70, 392, 5003),                       # 32 x 32, 32 x 64
    (300, 520, 3000), (511, 136, 2048), (260, 264, 8100),    # 64 x 64, 64 x 128
    (1000, 200, 3001), (1030, 200, 4097), (2050, 72, 2050),  # 128 x 128, one and two to a CU
    (4096, 64, 4100), (2100, 136, 8192), (8200, 8, 2049),    # 256 x 256, odd numbers of stages
])
def test_every_tile(M, K, N):
    _case(M, K, N, act="silu", residual="bf16", out="bf16")
    _case(M, K, N, act="none", residual="none", out="f32", pad=8)
    _case(M, K, N, act="none", residual="f32", out="f32", inplace=True)


def test_infinite_activation_arguments():
    """Large magnitudes: the activations' limits, no NaN."""
    import torch
    import paper_2608_23805_amd as msi
    log("case linear activation limits")
    x = torch.full((3, 8), 1.0, device="cuda").bfloat16()
    w = torch.zeros((6, 8), device="cuda").bfloat16()
    b = torch.tensor([-3e38, -200.0, -30.0, 30.0, 200.0, 3e38], device="cuda")
    for act in ("silu", "gelu", "gelu_tanh"):
        y = torch.empty((3, 6), device="cuda")
        msi.linear(x, w, y, bias=b, act=act)
        torch.cuda.synchronize()
        assert torch.isfinite(y).all() and torch.all(y[:, :2].abs() <= 1e-30) and torch.all(y[:, 3:] == b[3:])
