"""Projection with 4-bit weights against 64 bits: every kernel's row and feature edges, groups, lengths of K that end
inside a chunk or a stage, epilogues, strided rows, an output that is its residual, and x that is not finite.

Bound per element, as the bf16 projection's: the fp32 sum of K exact products (a code times x is exact in fp32; a group's
sum times its scale is one rounding more) sqrt(K) 2^-22 sum |x w|, the activation's few roundings (2^-20 of |z|, slope at
most 1.13), and half a step of the output's type."""
import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import bf16
from _kv_oracle import linear as oracle

pytestmark = pytest.mark.gpu


def q4(g, N, K, group, scale=None):
    """Codes [N, K / 2] and scales [N, K / group] on the device, and the weights in 64 bits."""
    import torch
    q = g.integers(-8, 8, (N, K))
    s = (np.exp(g.standard_normal((N, K // group))) * (K ** -0.5 / 5 if scale is None else scale)).astype(np.float16)
    codes = ((q[:, 0::2] & 15) | (q[:, 1::2] & 15) << 4).astype(np.uint8)
    w = (q.reshape(N, -1, group) * s.astype(np.float64)[..., None]).reshape(N, K)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(s).cuda(), w


def _case(M, K, N, group, act="none", residual="none", out="f32", bias=True, pad=0, inplace=False, seed=0):
    import torch
    import paper_2608_23805_amd as msi
    log(f"case linear_q4 M={M} K={K} N={N} group={group} {act} {residual} {out} pad={pad} inplace={inplace}")
    g = np.random.default_rng([81, M, K, N, group, seed])
    x, xh = bf16(g.standard_normal((M, K + pad)))
    w, s, wh = q4(g, N, K, group)
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
    msi.linear_q4(x[:, :K], w, s, y, bias=None if b is None else torch.from_numpy(b).cuda(), act=act, residual=r,
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


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300])
@pytest.mark.parametrize("K,N,group", [(32, 1, 32), (96, 31, 32), (320, 257, 64), (2176, 130, 128), (2080, 33, 32)])
def test_rows_and_features(M, K, N, group):
    _case(M, K, N, group)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("blocks", [1, 2, 3, 7, 8, 9, 15, 16, 17, 33, 64, 65, 129])
def test_lengths(group, blocks):
    """Groups that end inside a chunk, a stage or a panel of scales, wavefronts without a chunk."""
    for M in (1, 20, 40, 140):
        _case(M, group * blocks, 48, group, bias=False)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("residual,out", [("none", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("M", [1, 5, 30, 50, 170])
def test_epilogue(act, residual, out, M):
    _case(M, 256, 100, 32, act, residual, out)
    _case(M, 256, 101, 64, act, residual, out, bias=False, pad=8)


@pytest.mark.parametrize("M", [4, 40, 170])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_in_place(M, kind):
    _case(M, 128, 192, 128, residual=kind, out=kind, inplace=True)


@pytest.mark.parametrize("M,K,N,group", [(3, 1024, 8200, 32), (16, 4096, 2049, 128), (61, 1536, 4100, 64), (33, 512, 20000, 32),
                                         (513, 288, 2100, 32), (1030, 256, 4097, 64), (2050, 640, 1030, 128)])
def test_many_workgroups(M, K, N, group):
    _case(M, K, N, group, act="silu", residual="bf16", out="bf16")
    _case(M, K, N, group, residual="f32", out="f32", inplace=True)


FORMS = [((5, 4096, 300), (0, 16, 1)), ((12, 256, 4200), (0, 32, 1)), ((17, 4128, 300), (0, 16, 1)), ((25, 288, 4001), (0, 16, 1)),
         ((32, 1056, 8190), (0, 32, 1)), ((21, 2400, 5003), (0, 32, 1)), ((32, 1056, 8200), (32, 64, 1)),
         ((9, 8224, 4200), (0, 32, 1)), ((3, 8224, 4200), (0, 16, 1)), ((33, 544, 500), (16, 32, 1)), ((100, 1056, 2000), (32, 32, 1)),
         ((70, 544, 4099), (32, 64, 1)), ((130, 800, 5001), (64, 64, 1)), ((200, 416, 8190), (64, 128, 1)),
         ((61, 4128, 8190), (64, 32, 1)), ((40, 4608, 5001), (64, 32, 1)), ((65, 4128, 5001), (32, 64, 1)),
         ((600, 352, 5003), (128, 128, 1)), ((1100, 672, 4001), (64, 128, 3)), ((990, 416, 8190), (128, 128, 2))]


@pytest.mark.parametrize("size,form", FORMS)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_form(size, form, group):
    """Every kernel at odd edges of rows, features and K (which ends inside a stage, a chunk, a panel), every group."""
    import ctypes
    import paper_2608_23805_amd as msi
    M, K, N = size
    K = -(-K // group) * group
    v = [ctypes.c_uint32() for _ in range(3)]
    assert msi.lib.msi_debug_linear_q4_tile(M, N, K, *map(ctypes.byref, v)) == 0 and tuple(x.value for x in v) == form
    _case(M, K, N, group, act="gelu", residual="bf16", out="bf16")
    _case(M, K, N, group, residual="f32", out="f32", inplace=True)


@pytest.mark.parametrize("M,N", [(2, 40), (12, 4200), (20, 40), (100, 2000), (70, 4099), (130, 5001), (200, 8190), (600, 5003), (1100, 4001), (990, 8190)])
def test_infinities_stay_in_their_rows(M, N):
    """An infinite element of x gives infinities of the weight's sign (NaN where the weight is zero), as the formula does,
    and only in its row; a NaN likewise.  Rows past the end and the tail of K bring nothing of theirs."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case linear_q4 infinities M={M} N={N}")
    g = np.random.default_rng([81, 5, M])
    K = 288
    x, xh = bf16(g.standard_normal((M, K)))
    w, s, wh = q4(g, N, K, 32)
    x[1, K - 1] = float("inf")
    if M > 3:
        x[M - 1, 0] = float("nan")
    y = torch.empty((M, N), device="cuda")
    msi.linear_q4(x, w, s, y)
    torch.cuda.synchronize()
    got = y.cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = np.inf * wh[:, K - 1]
    assert np.array_equal(got[1], want.astype(np.float32), equal_nan=True)
    rest = np.isfinite(got).all(1)
    assert rest.sum() == M - (2 if M > 3 else 1) and (M <= 3 or np.isnan(got[M - 1]).all())


def test_more_features_than_a_grid_of_small_workgroups_holds():
    import torch
    import paper_2608_23805_amd as msi
    log("case linear_q4 many features")
    N, K = (1 << 22) + 17, 32
    gen = torch.Generator(device="cuda").manual_seed(5)
    w = torch.randint(0, 256, (N, K // 2), device="cuda", dtype=torch.uint8, generator=gen)
    s = (torch.rand((N, 1), device="cuda", generator=gen) + 0.5).half()
    x = torch.randn((3, K), device="cuda", generator=gen).bfloat16()
    y = torch.empty((3, N), device="cuda")
    msi.linear_q4(x, w, s, y)
    b = w.to(torch.int32)
    q = torch.stack([(b & 15 ^ 8) - 8, (b >> 4 ^ 8) - 8], -1).view(N, K).float()
    want, size = (q @ x.float().t()).t() * s.float().t(), (q.abs() @ x.float().abs().t()).t() * s.float().t()
    # both sums in fp32, of K products: K 2^-23 of their magnitude
    assert torch.all((y - want).abs() <= K * 2.0 ** -23 * size)


def test_scales_and_rows_of_the_largest_size():
    """Scales at fp16's ends with x of 2^110.  A group's sum, 224 * 2^110, is a number of fp32; times 65504 it is 2^133.8,
    past fp32's 2^128 (and still past it in the sixteenths that codes are), so the fp32 sum of the first feature is infinite
    after its first group, and no finite product brings it back (fused with the addition, the second group's is finite)."""
    import torch
    import paper_2608_23805_amd as msi
    log("case linear_q4 large values")
    for M in (4, 40, 140):
        x = torch.full((M, 64), 2.0 ** 110, device="cuda").bfloat16()
        w = torch.full((3, 32), 0x77, dtype=torch.uint8, device="cuda")
        s = torch.tensor([[65504.0, -65504.0], [2.0 ** -24, 2.0 ** -24], [0.0, 1.0]], device="cuda").half()
        y = torch.empty((M, 3), device="cuda")
        msi.linear_q4(x, w, s, y)
        torch.cuda.synchronize()
        assert not torch.isfinite(y[:, 0]).any()
        assert torch.equal(y[:, 1:], torch.tensor([[448 * 2.0 ** 86, 224 * 2.0 ** 110]] * M, device="cuda"))


def test_equal_calls_give_equal_bits_and_graphs_replay():
    import torch
    import paper_2608_23805_amd as msi
    log("case linear_q4 graph")
    g = np.random.default_rng([81, 7])
    cases = []
    for M in (1, 40, 200):
        x, _ = bf16(g.standard_normal((M, 512)))
        w, s, _ = q4(g, 300, 512, 64)
        cases.append((x, w, s, torch.empty((M, 300), device="cuda")))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for c in cases:
            msi.linear_q4(*c, stream=stream)
    stream.synchronize()
    first = [c[3].clone() for c in cases]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for c in cases:
            msi.linear_q4(*c, stream=torch.cuda.current_stream())
    for _ in range(3):
        for c in cases:
            c[3].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c[3]) for a, c in zip(first, cases))
