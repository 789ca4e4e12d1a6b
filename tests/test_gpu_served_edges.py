"""4-bit projections, append with rotation and attention over shared pages at calls that sizes alone do not reach: arrays
past 4 GiB, a first call inside a capture, two streams at once; lists of pages that are read again by every form of the
kernel of many rows."""
import subprocess
import sys

import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup, bf16
from test_gpu_kv_attention import _check

pytestmark = pytest.mark.gpu

FIRST = """
import sys
import torch
import paper_2608_23805_amd as msi
x = torch.randn(64, 512, device="cuda").bfloat16()
w = torch.randint(0, 256, (5003, 256), device="cuda", dtype=torch.uint8)
sc = torch.rand(5003, 16, device="cuda").half()
y = torch.zeros((64, 5003), device="cuda")
D, fmt = int(sys.argv[1]), sys.argv[2]
c = msi.KvCache.alloc(24, 2, D, fmt)
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
s = msi.KvSeqs(i32([[3, 5, 0], [3, 5, 9]]), i32([150, 170]), i32([0, 22, 64]), n_rows=64, max_rows=42)
g2 = msi.KvGroups(i32([0, 2]), i32([2]), max_rows=64, max_blocks=2)
r = msi.KvRotary([0.1] * (D // 4))
pos = i32(list(range(64)))
kv, q = torch.randn(64, 2, D, device="cuda").bfloat16(), torch.randn(64, 16, D, device="cuda").bfloat16()
c.data.random_(0, 120)
c.scales.fill_(0.25)
out, turned = torch.zeros((64, 16, D), device="cuda").bfloat16(), torch.zeros((64, 16, D), device="cuda").bfloat16()
ws = msi.kv_attention_shared_workspace(c, s, g2, 16)
def run(st):
    msi.linear_q4(x, w, sc, y, stream=st)
    msi.kv_append_rotary(c, s, r, pos, q, turned, kv, kv, stream=st)
    msi.kv_attention_shared(c, s, g2, turned, out, 0.1, workspace=ws, stream=st)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=torch.cuda.Stream()):
    run(torch.cuda.current_stream())
got = []
for k in range(4):
    y.zero_(); out.zero_(); turned.zero_()
    if k % 2 == 0:
        g.replay()
    else:
        run(None)
    torch.cuda.synchronize()
    got.append((y.clone(), out.clone(), turned.clone()))
for k in range(1, 4):
    assert all(torch.equal(a, b) for a, b in zip(got[k], got[0])), k
assert all(t.float().abs().sum(-1).gt(0).all() for t in got[0])
"""


@pytest.mark.parametrize("D,fmt", [(256, "e4m3"), (128, "int8"), (256, "int8")])
def test_first_call_in_a_capture(D, fmt):
    """Kernels with more than 64 KiB of LDS whose first call in the process is recorded into a graph."""
    log(f"case served first call captured {D} {fmt}")
    r = subprocess.run([sys.executable, "-c", FIRST, str(D), fmt], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr


@pytest.mark.parametrize("rows", [1, 9])
def test_pool_past_four_gib(rows):
    """The last pages of a pool of 4.7 GB against the same pages at the start of a small one."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case served large pool {rows}")
    H, D, P, n, S, G = 8, 256, 18000, 14, 3, 4
    g = np.random.default_rng(840 + rows)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    N, lens = S * rows, [290 + rows, 260 + rows, 330 + rows]
    k, v = (bf16(g.standard_normal((N, H, D)))[0] for _ in range(2))
    q, _ = bf16(g.standard_normal((N, G * H, D)))
    pos = i32(np.repeat(lens, rows) - np.tile(np.arange(rows)[::-1], S) - 1)
    rotary = msi.KvRotary([1e4 ** (-i / 64) for i in range(64)])
    codes = torch.randint(0, 120, (n, H, 2, 64, D), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    results = []
    for pool, first in ((n, 0), (P, P - n)):
        cache = msi.KvCache.alloc(pool, H, D, "e4m3")
        cache.data[first:] = codes.view(cache.data[first:].dtype)
        cache.scales.fill_(2.0 ** -6)
        table = i32([[first + b for b in ([13, 2, 7, 0] + [3 + s, 8 + s])] for s in range(S)])
        seqs = msi.KvSeqs(table, i32(lens), i32(np.arange(S + 1) * rows), n_rows=N, max_rows=rows)
        groups = msi.KvGroups(i32([0, S]), i32([4]), max_rows=N, max_blocks=4)
        turned, out = torch.zeros_like(q), torch.zeros_like(q)
        msi.kv_append_rotary(cache, seqs, rotary, pos, q, turned, k, v)
        msi.kv_attention_shared(cache, seqs, groups, turned, out, 0.0625, workspace=msi.kv_attention_shared_workspace(cache, seqs, groups, G * H))
        torch.cuda.synchronize()
        results.append((turned.clone(), out.clone(), cache.data[first:].clone(), cache.scales[first:].clone()))
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert results[0][1].float().abs().sum(-1).gt(0).all()


@pytest.mark.parametrize("M", [3, 17, 40])
def test_weights_past_four_gib(M):
    """The last features of a matrix whose codes take 4.4 GB."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case q4 large matrix {M}")
    N, K = 270011, 32768
    gen = torch.Generator(device="cuda").manual_seed(850)
    w = torch.randint(0, 256, (N, K // 2), device="cuda", dtype=torch.uint8, generator=gen)
    s = (torch.rand((N, K // 128), device="cuda", generator=gen) + 0.5).half()
    x = torch.randn((M, K), device="cuda", generator=gen).bfloat16()
    y = torch.zeros((M, N), device="cuda")
    msi.linear_q4(x, w, s, y)
    for at in (slice(0, 40), slice(N // 2, N // 2 + 40), slice(N - 40, N)):
        b = w[at].to(torch.int32).cpu()
        q = torch.stack([(b & 15 ^ 8) - 8, (b >> 4 ^ 8) - 8], -1).view(-1, K).double()
        W, X = q * s[at].double().cpu().repeat_interleave(128, 1), x.double().cpu()
        want, size = X @ W.t(), X.abs() @ W.abs().t()
        # fp32 sums of K exact products and their groups' scaling: (K + 2) 2^-24 of their magnitude, doubled for orders of adding
        assert torch.all((y[:, at].double().cpu() - want).abs() <= 2 * (K + 2) * 2.0 ** -24 * size)


def test_two_streams_at_once():
    """Calls on two streams with workspaces of their own give what one after the other gives."""
    import torch
    import paper_2608_23805_amd as msi
    log("case served two streams")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(860)
    sides = []
    for D, fmt, rows in ((128, "int8", 1), (64, "e4m3", 33)):
        cache = msi.KvCache.alloc(80, 2, D, fmt)
        cache.data.copy_(torch.randint(0, 120, cache.data.shape, device="cuda", generator=gen).to(cache.data.dtype))
        cache.scales.fill_(2.0 ** -5)
        S, P = 6, 40
        table = i32([list(range(P)) + [P + 5 * s + b for b in range(5)] for s in range(S)])
        seqs = msi.KvSeqs(table, i32([P * 64 + 50 + 40 * s for s in range(S)]), i32([rows * s for s in range(S + 1)]), n_rows=S * rows, max_rows=rows)
        groups = msi.KvGroups(i32([0, S]), i32([P]), max_rows=S * rows, max_blocks=P)
        q = torch.randn((S * rows, 8, D), device="cuda", generator=gen).bfloat16()
        w = torch.randint(0, 256, (8 * D, 4 * D), device="cuda", dtype=torch.uint8, generator=gen)
        sc = torch.rand((8 * D, 8 * D // 32), device="cuda", generator=gen).half()
        ws = msi.kv_attention_shared_workspace(cache, seqs, groups, 8)
        sides.append((cache, seqs, groups, q, ws, w, sc, torch.zeros_like(q), torch.zeros((S * rows, 8 * D), device="cuda")))

    def run(side, stream):
        cache, seqs, groups, q, ws, w, sc, out, y = side
        msi.kv_attention_shared(cache, seqs, groups, q, out, 0.125, workspace=ws, stream=stream)
        msi.linear_q4(out.view(len(out), -1), w, sc, y, stream=stream)

    want = []
    for side in sides:
        run(side, None)
        torch.cuda.synchronize()
        want.append((side[7].clone(), side[8].clone()))
        side[7].zero_(), side[8].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sides]
    for _ in range(8):
        for side, st in zip(sides, streams):
            run(side, st)
    torch.cuda.synchronize()
    for side, (out, y) in zip(sides, want):
        assert torch.equal(side[7], out) and torch.equal(side[8], y) and out.any() and y.any()


@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("D,fmt", [(128, "int8"), (256, "int8"), (128, "e4m3"), (256, "e4m3")])
def test_page_lists_of_many_rows(D, fmt, bad):
    """A sequence of 134 blocks that is not cut: the lists of 64 pages are made three times, a bad page in each."""
    log(f"case page lists, many rows, {D} {fmt} bad={bad}")
    lens, rows = [8530] + [3] * 51, [40] + [1] * 51
    s = Setup(870 + D, lens, rows, 1, D, fmt)
    table = s.table.copy()
    if bad:
        for b in (10, 63, 64, 65, 66, 100, 127, 128, 129, 133):
            table[0, b] = 10 ** 6 + b
    _check(s, s.make_seqs(table, s.lens, s.cu), table, s.lens, s.cu, 16, status=int(bad))
