"""AttentionBlock: rows that no sequence of the call answers for, steps without rows, refusals before anything is
written, and the two halves of a step with the caller's own work between them.  Results are compared bit for bit with
the same operators on the good rows alone (a row's result depends on no other row)."""
import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup, bf16

pytestmark = pytest.mark.gpu

HQ, H, D, WIDTH = 4, 2, 64, 128


def _weights(seed):
    g = np.random.default_rng([90, seed])
    wqkv, _ = bf16(g.standard_normal(((HQ + 2 * H) * D, WIDTH)) * WIDTH ** -0.5)
    wo, _ = bf16(g.standard_normal((WIDTH, HQ * D)) * (HQ * D) ** -0.5)
    return wqkv, wo


def _block(s, max_rows, seed=1):
    import paper_2608_23805_amd as msi
    b = msi.AttentionBlock(*_weights(seed), s.cache, HQ, max_rows)
    b.attn.fill_(float("nan"))                                 # an earlier step's rows, or fresh memory
    return b


def _rows(n, seed):
    import torch
    g = np.random.default_rng([91, seed])
    x, _ = bf16(g.standard_normal((n, WIDTH)))
    return x, torch.from_numpy(g.standard_normal((n, WIDTH)).astype(np.float32)).cuda()


def _seqs(s, table, lens, cu, n_rows, max_rows, max_len=256):
    import paper_2608_23805_amd as msi
    import torch
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    return msi.KvSeqs(i32(table), i32(lens), i32(cu), n_rows=n_rows, max_rows=max_rows, max_len=max_len)


@pytest.mark.parametrize("mass_rows", [0, 3])
@pytest.mark.parametrize("rows,lens", [
    ([1, 2, 20, 3], [100, 70, 10, 200]),                       # 20 rows on 10 tokens; 128-row form
    ([1, 2, 4, 3], [100, 70, 3, 200]),                         # 4 rows on 3 tokens; few-rows form
])
def test_rows_that_are_left_out(rows, lens, mass_rows):
    """A broken length, a sequence with more rows than tokens and rows behind the last sequence: nothing is added to
    their h, their pages stay as they were, and the other rows get what they get alone."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case block, rows left out {rows} {mass_rows}")
    most = max(rows)
    s = Setup(92, lens, rows, H, D, "e4m3")
    alone = Setup(92, lens, rows, H, D, "e4m3")
    n = s.cu[-1] + 4
    device = list(lens)
    device[1] = 257                                            # past max_len
    seqs = _seqs(s, s.table, device, s.cu, n, most)
    b = _block(s, n)
    b.reserve(seqs, mass_rows)
    x, h = _rows(n, 1)
    good = list(range(s.cu[0], s.cu[1])) + list(range(s.cu[3], s.cu[4]))
    rest = [r for r in range(n) if r not in good]
    h0 = h.clone()
    x2, h2 = x[good + rest].contiguous(), h[good + rest].contiguous()
    b.step(x, h, seqs, mass_rows=mass_rows, status=s.status)
    b2 = _block(alone, n)
    seqs2 = _seqs(alone, alone.table[[0, 3]], [lens[0], lens[3]], [0, rows[0], rows[0] + rows[3]], n, most)
    b2.reserve(seqs2, mass_rows)
    b2.step(x2, h2, seqs2, mass_rows=mass_rows)
    got, want = s.device_state(), alone.device_state()
    assert got[3] == msi.KV_BAD_LENGTH
    assert torch.equal(h[rest], h0[rest])
    assert torch.equal(h[good], h2[:len(good)]) and torch.equal(x[good], x2[:len(good)])
    for a, c in zip(got[:3], want[:3]):                        # codes, scales, weights
        assert np.array_equal(a, c)
    assert torch.isfinite(x.float()).all()


def test_captured_step_with_fewer_rows():
    """A step captured for eight rows, replayed with fewer sequences' rows in them, with eager steps in between."""
    import torch
    import paper_2608_23805_amd as msi
    log("case block, captured, fewer rows")
    s = Setup(93, [40, 100, 7, 150], [1, 1, 1, 1], H, D, "int8", extra_blocks=1)
    seqs = _seqs(s, s.table, s.lens, s.cu, 8, 2, max_len=192)
    b = _block(s, 8)
    b.reserve(seqs, 1)
    x, h = _rows(8, 2)
    torch.cuda.synchronize()
    keep = (s.data.clone(), s.scales.clone(), s.mass.clone())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        b.step(x, h, seqs, mass_rows=1, stream=torch.cuda.current_stream())
    for t, v in zip((s.data, s.scales, s.mass), keep):
        t.copy_(v)
    for k, cu in enumerate(([0, 1, 2, 3, 4], [0, 2, 2, 3, 3], [0, 0, 1, 1, 3], [0, 0, 0, 0, 0])):
        seqs.cu_rows.copy_(torch.tensor(cu))
        x0, h0 = _rows(8, 3 + k)
        before = (s.data.clone(), s.scales.clone(), s.mass.clone())
        b.attn.fill_(float("nan"))
        x.copy_(x0), h.copy_(h0)
        g.replay()
        torch.cuda.synchronize()
        got = (x.clone(), h.clone(), s.data.clone(), s.scales.clone(), s.mass.clone())
        for t, v in zip((s.data, s.scales, s.mass), before):
            t.copy_(v)
        xe, he = x0.clone(), h0.clone()
        b.attn.fill_(float("nan"))
        b.step(xe, he, seqs, mass_rows=1)
        torch.cuda.synchronize()
        for a, e in zip(got, (xe, he, s.data, s.scales, s.mass)):
            assert torch.equal(a, e), k
        assert torch.equal(he[cu[-1]:], h0[cu[-1]:]) and not (cu[-1] and torch.equal(he[:cu[-1]], h0[:cu[-1]]))


def test_every_row_of_an_attention_call():
    """kv_attention with all_rows: a row of no sequence, or of one that is left out, becomes zero, also where a whole
    call has no sequence with rows; without it such rows stay as they were."""
    import torch
    import paper_2608_23805_amd as msi
    log("case attention, all rows")
    for rows, n in (([1, 3, 2], 200), ([40, 60, 2], 200)):
        s = Setup(94, [100, 50, 64], rows, H, D, "e4m3")
        q, _ = bf16(s.g.standard_normal((n, HQ, D)))
        i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
        for cu in ([0] + [int(c) for c in np.cumsum(rows)], [5, 5 + rows[0], 150, 152], [0, 0, 0, 0]):
            seqs = msi.KvSeqs(i32(s.table), i32(s.lens), i32(cu), n_rows=n, max_rows=max(rows), max_len=128)
            ws = msi.kv_attention_workspace(s.cache, seqs, HQ)
            outs = [torch.full((n, HQ + 1, D), 5.0, dtype=torch.bfloat16, device="cuda")[:, :HQ] for _ in "ab"]
            msi.kv_attention(s.cache, seqs, q, outs[0], 0.125, workspace=ws, status=s.status, all_rows=True)
            msi.kv_attention(s.cache, seqs, q, outs[1], 0.125, workspace=ws)
            torch.cuda.synchronize()
            covered = torch.zeros(n, dtype=torch.bool)
            for i in range(3):
                if 0 <= cu[i + 1] - cu[i] <= min(s.lens[i], max(rows)):
                    covered[cu[i]:cu[i + 1]] = True
            assert torch.all(outs[0][~covered.cuda()] == 0) and torch.equal(outs[0][covered.cuda()], outs[1][covered.cuda()])
            assert torch.all(outs[1][max(cu):] == 5.0)
    # sequences without rows, and no sequences at all
    for S in (3, 0):
        seqs = msi.KvSeqs(i32(s.table[:S]).contiguous(), i32(s.lens[:S]), i32([0] * (S + 1)), n_rows=n, max_rows=0, max_len=0 if S == 0 else 128)
        out = torch.full((n, HQ, D), 5.0, dtype=torch.bfloat16, device="cuda")
        msi.kv_attention(s.cache, seqs, q, out, 0.125, all_rows=True)
        torch.cuda.synchronize()
        assert not out.any()


def test_many_sequences_answer_for_their_rows():
    """Rows told apart over more sequences than a workgroup looks at in one turn."""
    import torch
    import paper_2608_23805_amd as msi
    log("case attention, all rows of many sequences")
    S = 700
    lens = [(i * 7) % 60 + 1 for i in range(S)]
    s = Setup(95, lens, [1] * S, 1, D, "int8")
    seqs = s.make_seqs(s.table, s.lens, s.cu, max_len=64)
    seqs.lens[::11] = 65
    q, _ = s.rows(2)
    out = torch.full((S, 2, D), 5.0, dtype=torch.bfloat16, device="cuda")
    msi.kv_attention(s.cache, seqs, q, out, 0.125, workspace=msi.kv_attention_workspace(s.cache, seqs, 2), all_rows=True)
    torch.cuda.synchronize()
    zero = (out == 0).all(-1).all(-1).cpu().numpy()
    assert np.array_equal(zero, np.arange(S) % 11 == 0)


@pytest.mark.parametrize("most", [2, 100])
def test_more_rows_than_are_cleared_in_a_turn(most):
    """20001 rows of which three sequences bring a few, in both forms and where the call has nothing else to do."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case attention, all of 20001 rows, most={most}")
    s = Setup(100, [100, 128, 64], [1, 1, 1], 1, D, "e4m3")
    n, cu = 20001, [12000, 12001, 12003, 12004]
    q, _ = bf16(s.g.standard_normal((n, 2, D)))
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    for offsets, rows in ((cu, most), ([0] * 4, most), ([0] * 4, 0)):
        seqs = msi.KvSeqs(i32(s.table), i32(s.lens), i32(offsets), n_rows=n, max_rows=rows, max_len=128)
        out = torch.full((n + 1, 2, D), 5.0, dtype=torch.bfloat16, device="cuda")
        msi.kv_attention(s.cache, seqs, q, out[:n], 0.125, workspace=msi.kv_attention_workspace(s.cache, seqs, 2), all_rows=True)
        torch.cuda.synchronize()
        zero = (out == 0).all(-1).all(-1).cpu().numpy()
        want = np.ones(n + 1, dtype=bool)
        want[offsets[0]:offsets[-1]] = False
        want[n] = False
        assert np.array_equal(zero, want) and torch.all(out[n] == 5.0)


def test_step_without_rows():
    import torch
    import paper_2608_23805_amd as msi
    log("case block, no rows")
    s = Setup(96, [100, 0], [0, 0], H, D, "int8")
    b = _block(s, 4)
    seqs = _seqs(s, s.table, s.lens, s.cu, 0, 0, max_len=128)
    b.reserve(seqs, 1)
    x, h = _rows(0, 4)
    before = s.device_state()
    b.step(x, h, seqs, mass_rows=1, status=s.status)
    after = s.device_state()
    assert all(np.array_equal(a, c) for a, c in zip(before, after))


def test_refusals_come_before_any_effect():
    """What a step refuses, it refuses before the cache, the rows or the weights change."""
    import torch
    import paper_2608_23805_amd as msi
    log("case block, refusals")
    s = Setup(97, [100, 60], [1, 1], H, D, "e4m3")
    bare = Setup(97, [100, 60], [1, 1], H, D, "e4m3", mass=False)
    for t, kw in ((bare, dict(mass_rows=1)), (s, dict(mass_rows=1, mass_decay=-1.0)),
                  (s, dict(mass_rows=1, mass_decay=float("inf"))), (s, dict(mass_rows=-1))):
        b = _block(t, 4)
        b.workspace = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        x, h = _rows(2, 5)
        x0, h0, before = x.clone(), h.clone(), t.device_state()
        with pytest.raises(msi.MsiError):
            b.step(x, h, t.seqs, status=t.status, **kw)
        after = t.device_state()
        assert torch.equal(x, x0) and torch.equal(h, h0)
        assert np.array_equal(before[0], after[0]) and np.array_equal(before[1], after[1]) and after[3] == 0


def test_work_between_the_halves():
    """project, the caller's own change of queries and keys, attend: the same as the operators called one by one."""
    import torch
    import paper_2608_23805_amd as msi
    log("case block, halves")
    s, t, u = (Setup(98, [100, 60], [2, 1], H, D, "e4m3") for _ in "abc")
    x, h = _rows(3, 6)
    x1, h1, x2, h2, x3, h3 = (v.clone() for v in (x, h, x, h, x, h))
    # without a change: a step
    b = _block(s, 4)
    b.reserve(s.seqs, 1)
    b.step(x, h, s.seqs, mass_rows=1)
    c = _block(t, 4)
    c.reserve(t.seqs, 1)
    qkv = c.project(x1, t.seqs)
    assert qkv.shape == (3, HQ + 2 * H, D)
    c.attend(x1, h1, t.seqs, mass_rows=1)
    torch.cuda.synchronize()
    assert torch.equal(x, x1) and torch.equal(h, h1)
    assert all(np.array_equal(a, e) for a, e in zip(s.device_state(), t.device_state()))
    # with one: halves of every head's elements exchanged
    t2 = Setup(98, [100, 60], [2, 1], H, D, "e4m3")
    c = _block(t2, 4)
    c.reserve(t2.seqs, 1)
    qk = c.project(x2, t2.seqs)[:, :HQ + H]
    qk.copy_(torch.cat((-qk[..., D // 2:], qk[..., :D // 2]), -1))
    c.attend(x2, h2, t2.seqs, mass_rows=1)
    wqkv, wo = _weights(1)
    qkv = torch.empty((3, HQ + 2 * H, D), dtype=torch.bfloat16, device="cuda")
    msi.linear(x3, wqkv, qkv.view(3, -1))
    qk = qkv[:, :HQ + H]
    qk.copy_(torch.cat((-qk[..., D // 2:], qk[..., :D // 2]), -1))
    msi.kv_append(u.cache, u.seqs, qkv[:, HQ:HQ + H], qkv[:, HQ + H:])
    a = torch.empty((3, HQ, D), dtype=torch.bfloat16, device="cuda")
    msi.kv_attention(u.cache, u.seqs, qkv[:, :HQ], a, D ** -0.5, mass_rows=1,
                     workspace=msi.kv_attention_workspace(u.cache, u.seqs, HQ, 1))
    o = torch.empty((3, WIDTH), device="cuda")
    msi.linear(a.view(3, -1), wo, o)
    msi.residual_add(o, h3, x3)
    torch.cuda.synchronize()
    assert torch.equal(x2, x3) and torch.equal(h2, h3) and not torch.equal(h2, h)
    assert all(np.array_equal(p, e) for p, e in zip(t2.device_state(), u.device_state()))


def test_blocks_that_share_a_workspace():
    """Blocks of one stream with one workspace handed in, and one that is too small."""
    import torch
    import paper_2608_23805_amd as msi
    log("case block, shared workspace")
    pairs = [(Setup(99, [900, 600], [1, 1], H, D, "int8"), Setup(99, [900, 600], [1, 1], H, D, "int8")) for _ in "ab"]
    ws = None
    for k, (s, t) in enumerate(pairs):
        x, h = _rows(2, 7 + k)
        x2, h2 = x.clone(), h.clone()
        b, c = _block(s, 2, k), _block(t, 2, k)
        if ws is None:
            ws = msi.kv_attention_workspace(s.cache, s.seqs, HQ, 1)
        b.step(x, h, s.seqs, mass_rows=1, workspace=ws)
        c.reserve(t.seqs, 1)
        c.step(x2, h2, t.seqs, mass_rows=1)
        torch.cuda.synchronize()
        assert torch.equal(x, x2) and torch.equal(h, h2) and b.workspace is None
        with pytest.raises(msi.MsiError) as e:
            b.step(x, h, s.seqs, mass_rows=1, workspace=ws[:-256])
        assert e.value.status == msi.MSI_E_NOMEM
        assert torch.equal(x, x2) and torch.equal(h, h2)
