"""The attention block's operators at calls that sizes alone do not reach: arrays past 4 GiB, a first call inside a
capture, negative scales, queries that are not numbers."""
import subprocess
import sys

import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup, bf16
from test_gpu_kv_attention import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,rows", [([70, 5], [1, 2]), ([900], [1]), ([70, 300], [40, 33]), ([900, 3], [40, 1])])
def test_negative_scale(lens, rows):
    log(f"case negative scale {lens} {rows}")
    s = Setup(110 + sum(rows), lens, rows, 2, 128, "int8")
    _check(s, s.seqs, s.table, s.lens, s.cu, 3, scale=-0.125)
    _check(s, s.seqs, s.table, s.lens, s.cu, 3, mass_rows=7, decay=0.5, scale=-0.125)


@pytest.mark.parametrize("rows", [[1, 3], [40, 35]])
def test_queries_that_are_not_numbers(rows):
    """A row with NaN or infinities in its query spoils its own output and no other."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case queries not numbers {rows}")
    s = Setup(111, [600, 90], rows, 2, 64, "e4m3")
    q, _ = s.rows(8, 0.5)
    ws = msi.kv_attention_workspace(s.cache, s.seqs, 8)
    outs = []
    for k in range(2):
        out = torch.empty((s.cu[-1], 8, 64), dtype=torch.bfloat16, device="cuda")
        msi.kv_attention(s.cache, s.seqs, q, out, 0.125, workspace=ws)
        torch.cuda.synchronize()
        outs.append(out)
        q = q.clone()
        q[1, 2], q[1, 5, 3], q[s.cu[-1] - 1, 7, 0] = float("nan"), float("inf"), -float("inf")
    same = (outs[0] == outs[1]).all(-1)
    spoilt = torch.zeros_like(same)
    spoilt[1, 2] = spoilt[1, 5] = spoilt[s.cu[-1] - 1, 7] = True
    assert torch.all(same | spoilt) and not torch.isfinite(outs[1][1, 2].float()).any()


FIRST = """
import torch
import paper_2608_23805_amd as msi
x, w = torch.randn(64, 512, device="cuda").bfloat16(), torch.randn(5003, 512, device="cuda").bfloat16()
y = torch.zeros((64, 5003), device="cuda")
c = msi.KvCache.alloc(8, 2, 256, "e4m3")
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
s = msi.KvSeqs(i32([[3, 5, 0]]), i32([150]), i32([0, 150]), n_rows=150, max_rows=150)
kv, q = torch.randn(150, 2, 256, device="cuda").bfloat16(), torch.randn(150, 4, 256, device="cuda").bfloat16()
out = torch.zeros((150, 4, 256), device="cuda").bfloat16()
ws = msi.kv_attention_workspace(c, s, 4, 3)
def run(st):
    msi.linear(x, w, y, stream=st)
    msi.kv_append(c, s, kv, kv, stream=st)
    msi.kv_attention(c, s, q, out, 0.1, mass_rows=3, mass_decay=0.0, workspace=ws, stream=st)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=torch.cuda.Stream()):
    run(torch.cuda.current_stream())
got = []
for k in range(3):
    y.zero_(); out.zero_(); c.mass.zero_()
    if k < 2:
        g.replay()
    else:
        run(None)
    torch.cuda.synchronize()
    got.append((y.clone(), out.clone(), c.mass.clone()))
for k in range(2):
    assert all(torch.equal(a, b) for a, b in zip(got[k], got[2]))
assert got[2][0].any() and got[2][1].any() and got[2][2].any()
"""


def test_first_call_in_a_capture():
    """Kernels with more than 64 KiB of LDS whose first call in the process is recorded into a graph."""
    log("case first call captured")
    r = subprocess.run([sys.executable, "-c", FIRST], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr


def test_pool_past_four_gib():
    """The last pages of a pool of 4.7 GB against the same pages at the start of a small one, every operator."""
    import torch
    import paper_2608_23805_amd as msi
    log("case large pool")
    H, D, P, n = 8, 256, 18000, 14
    g = np.random.default_rng(112)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    k, _ = bf16(g.standard_normal((400, H, D)))
    v, _ = bf16(g.standard_normal((400, H, D)))
    q, _ = bf16(g.standard_normal((400, H, D)) * 0.5)
    results = []
    for pool, first in ((n, 0), (P, P - n)):
        c = msi.KvCache.alloc(pool, H, D, "e4m3")
        c.data.zero_()                                     # (bytes past the last token stay as they were)
        c.scales.zero_()
        table = i32(first + np.arange(7, dtype=np.int32)[None, ::-1])
        dst = i32(first + 7 + np.arange(7, dtype=np.int32)[None])
        r = []
        whole = msi.KvSeqs(table, i32([400]), i32([0, 400]), n_rows=400, max_rows=400, max_len=400)
        one = msi.KvSeqs(table, i32([400]), i32([0, 1]), n_rows=1, max_rows=1, max_len=400)
        msi.kv_append(c, whole, k, v)
        for seqs, rows in ((whole, 400), (one, 1)):
            out = torch.empty((rows, H, D), dtype=torch.bfloat16, device="cuda")
            msi.kv_attention(c, seqs, q[:rows], out, 0.0625, mass_rows=rows, mass_decay=1.0,
                             workspace=msi.kv_attention_workspace(c, seqs, H, rows))
            r.append(out)
        keep, new = torch.zeros((1, H, 200), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        msi.kv_evict(c, whole, dst, new, keep, budget=200, sinks=2, recent=20)
        left = msi.KvSeqs(dst, new, i32([0, 200]), n_rows=200, max_rows=200, max_len=200)
        ko, vo = (torch.empty((200, H, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
        msi.kv_read(c, left, ko, vo)
        torch.cuda.synchronize()
        r += [keep, new, ko, vo] + [t[first:first + 7].clone() for t in (c.data, c.scales, c.mass)]
        results.append(r)
        del c
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert float(results[0][0].abs().max()) > 0


def test_projection_past_four_gib():
    """Outputs past 2^32 bytes: the last rows, and rows around 2^31 elements, against 64 bits."""
    import torch
    import paper_2608_23805_amd as msi
    log("case large projection")
    M, N, K = 66001, 33001, 8
    g = np.random.default_rng(113)
    x, xh = bf16(g.standard_normal((M, K)))
    w, wh = bf16(g.standard_normal((N, K)))
    y = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    msi.linear(x, w, y)
    torch.cuda.synchronize()
    for r in (0, 2 ** 31 // N, 2 ** 31 // N + 1, 40000, M - 2, M - 1):
        want = xh[r] @ wh.T
        tol = K ** 0.5 * 2.0 ** -22 * (np.abs(xh[r]) @ np.abs(wh).T) + 2.0 ** -8 * np.abs(want) + 1e-30
        assert np.all(np.abs(y[r].double().cpu().numpy() - want) <= tol), r
