"""Attention over shared pages: how its groups and sequences become units, in both of its planners (up to 64 groups and 64
sequences every wavefront lays the units out, a launch of its own does above).  The oracle and the bound are those of
test_gpu_kv_shared.py."""
import ctypes

import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import bf16
from _kv_oracle import attention
from test_gpu_kv_shared import Shared, _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [3, 90])
@pytest.mark.parametrize("own", [20, 0])
def test_more_blocks_than_any_sequence_has(n, own):
    """A group's blocks lie past every sequence of the call: nobody reads them, whatever its table holds there."""
    log(f"case shared blocks past every sequence n={n} own={own}")
    sh = Shared(900 + n, [(n, 0)], [own] * n, [1] * n, 2, 64, "e4m3")
    s = sh.s
    nb = s.table.shape[1]
    s.table = np.concatenate([s.table, s.table * 0 - 7], axis=1)
    s.seqs = s.make_seqs(s.table, s.lens, s.cu)
    sh.nb.fill_(nb + 1 if own else 1)
    for G in (2, 64):
        _check(sh, 2 * G, groups=sh.bounds(max_rows=n, max_blocks=2 * nb))


@pytest.mark.parametrize("n", [3, 90])
def test_no_tokens_and_no_table(n):
    """Bounds without a token need no table, also where groups claim shared blocks: rows see nothing."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case shared no table n={n}")
    sh = Shared(910 + n, [(n, 0)], [0] * n, [1] * n, 2, 64, "e4m3")
    s = sh.s
    sh.nb.fill_(2)
    for G in (2, 64):
        q = torch.randn((n, 2 * G, 64), device="cuda").bfloat16()
        out = torch.full_like(q, 5.0)
        seqs = msi.msi_kv_seqs(n, 4, n, 1, 0, 0, None, s.seqs.lens.data_ptr(), s.seqs.cu_rows.data_ptr())
        groups = msi.msi_kv_groups(1, n, 4, 0, sh.cu.data_ptr(), sh.nb.data_ptr())
        need = ctypes.c_uint64()
        c, sq, gr = s.cache._ref, ctypes.byref(seqs), ctypes.byref(groups)
        assert msi.lib.msi_kv_attention_shared_workspace(c, sq, gr, 2 * G, ctypes.byref(need)) == 0
        ws = torch.full((need.value,), 0xA5, dtype=torch.uint8, device="cuda")
        s.status.zero_()
        a = msi.msi_kv_attention_args(q=q.data_ptr(), out=out.data_ptr(), q_stride=2 * G * 64, out_stride=2 * G * 64, n_q_heads=2 * G,
                                      scale=0.125, workspace=ws.data_ptr(), workspace_bytes=need.value, status=s.status.data_ptr())
        torch.cuda.synchronize()
        assert msi.lib.msi_kv_attention_shared(c, sq, gr, ctypes.byref(a), None) == 0
        torch.cuda.synchronize()
        assert int(s.status) == 0 and torch.all(out == 0.0)


@pytest.mark.parametrize("n", [5, 90])
@pytest.mark.parametrize("first", ["empty", "without rows", "short", "short, other pages", "left out"])
def test_table_of_a_sequence_that_is_attended_by_itself(n, first):
    """The first sequences of a group do not stand behind its shared pages: their tables are their own affair, and the others
    still share."""
    log(f"case shared table n={n} first={first}")
    rows = [1, 1] + [1] * (n - 2)
    if first in ("empty", "without rows"):
        rows[:2] = [0, 0]
    sh = Shared(920 + n, [(n, 3), (2, 1)], [20 + i % 70 for i in range(n + 2)], rows + [1, 1], 2, 64, "e4m3")
    s = sh.s
    for i in (0, 1):
        s.lens[i] = {"empty": 0, "without rows": s.lens[i], "left out": s.lens[i]}.get(first, 70 + i)
        s.table[i, :3] = s.table[n - 1, 3] if first == "short, other pages" else -1
        if first == "short":
            s.table[i, :2] = s.table[n + i, 0], s.table[n - 1, 3]
    if first == "left out":
        s.lens[0] = s.lens[1] = 1 << 20
    max_len = max(x for x in s.lens if x < 1 << 20)
    s.seqs = s.make_seqs(s.table, s.lens, s.cu, max_len=max_len)
    for G in (2, 64):
        if first == "left out":
            q, out, st = _run(sh, 2 * G)
            want, tol, _ = attention(s.host, s.table[2:], s.lens[2:], [c - 2 for c in s.cu[2:]], q[1][2:], 0.125, G)
            assert st == 4 and np.all(np.abs(out.double().cpu().numpy()[2:] - want) <= tol + 2.0 ** -86 * max_len)
            assert (out[:2] == 5.0).all()
        else:
            _check(sh, 2 * G)


@pytest.mark.parametrize("n", [5, 90])
def test_group_that_no_sequence_stands_behind(n):
    """All of a group's sequences are shorter than its shared pages: nobody reads those, and no status tells of them."""
    log(f"case shared nobody behind n={n}")
    sh = Shared(930 + n, [(n, 3), (2, 1)], [20] * (n + 2), [1] * (n + 2), 2, 64, "int8")
    s = sh.s
    s.lens[:n] = [64 + i % 60 for i in range(n)]
    s.table[:n, 2:] = -1
    s.lens[n] += 200
    s.table[n, 1:5] = s.table[n + 1, 1]
    s.table = np.ascontiguousarray(np.concatenate([s.table, s.table * 0 - 1], axis=1))
    s.table[n, 4:6] = s.table[n + 1, 1]
    s.seqs = s.make_seqs(s.table, s.lens, s.cu)
    for G in (2, 64):
        _check(sh, 2 * G)


def test_sequences_past_the_items_of_overlapping_groups():
    """Offsets of rows that fall, so that groups overlap and take more units than their rows allow: what is left for the
    sequences behind them ends with the launch, and a sequence past that is left out as a whole.  (128 heads: 59 groups and
    sequences of 65 packed rows, three tiles of 32 each, where 10 rows allow 79 for the groups and as many for the sequences.
    The groups take 90, so the last 68 of 158 go to the sequences, 22 of them; rows 5 .. 9 belong to the 24th and later ones.)"""
    import torch
    import paper_2608_23805_amd as msi
    log("case shared items of overlapping groups")
    H, G, D, pairs = 128, 13, 256, (23, 7)
    sh = Shared(940, [(1, 2)], [30], [5], H, D, "e4m3")
    s = sh.s
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    cu = [0, 5] * pairs[0] + [5, 10] * pairs[1]
    S = len(cu) - 1
    table = torch.full((S, 80), -1, dtype=torch.int32, device="cuda")
    table[:, :3] = i32(s.table[0, :3])
    seqs = msi.KvSeqs(table, i32([s.lens[0]] * S), i32(cu), n_rows=10, max_rows=5, max_len=64 * 80)
    groups = msi.KvGroups(i32(list(range(S + 1))), i32([2] * S), max_rows=5, max_blocks=80)
    q = bf16(s.g.standard_normal((10, H * G, D)) * 1.5)
    for all_rows in (False, True):
        _, out, st = _run(sh, H * G, seqs=seqs, groups=groups, q=q, all_rows=all_rows)
        assert st == 4
        got = out.double().cpu().numpy()
        for a, z in ((0, 5), (5, 10)):
            want, tol, _ = attention(s.host, s.table, s.lens, [0, 5], q[1][a:z], 0.125, G)
            right = np.all(np.abs(got[a:z] - want) <= tol + 2.0 ** -86 * s.lens[0])
            assert right or np.all(got[a:z] == (0.0 if all_rows else 5.0))
            assert right == (a == 0)


@pytest.mark.parametrize("fmt,D", [("e4m3", 64), ("int8", 128), ("e4m3", 256), ("int8", 256)])
@pytest.mark.parametrize("groups", [[(100, 20)], [(70, 9), (1, 30), (0, 4), (29, 0)], [(49, 3), (51, 40)]])
def test_answers_past_64_sequences(fmt, D, groups):
    """Single tokens of more sequences than a wavefront has lanes: shared pages by 128 rows, own pages by 16 or 32, in launches
    of their own."""
    log(f"case shared plan answers {fmt} D={D} groups={groups}")
    n = sum(k for k, _ in groups)
    _check(Shared(950 + D, groups, [1 + 37 * i % 400 for i in range(n)], [1] * n, 2, D, fmt), 2 * 7)


@pytest.mark.parametrize("fmt,D", [("e4m3", 128), ("int8", 64), ("int8", 256)])
@pytest.mark.parametrize("groups", [[(3, 12), (67, 2)], [(70, 0)], [(35, 25), (35, 1)]])
def test_prompts_past_64_sequences(fmt, D, groups):
    """Some of the sequences are prompts: shared and own pages both by 128 rows."""
    log(f"case shared plan prompts {fmt} D={D} groups={groups}")
    rows = [(40, 1, 7, 0, 33)[i % 5] for i in range(70)]
    _check(Shared(960 + D, groups, [r + 90 * i % 1000 for i, r in enumerate(rows)], rows, 1, D, fmt), 4)


@pytest.mark.parametrize("rows", [[1], [30, 1, 2]])
def test_more_than_64_groups(rows):
    """Groups whose units are cut by the work alone, by 128 rows; single tokens and prompts behind them."""
    log(f"case shared plan groups rows={rows}")
    g = np.random.default_rng(971)
    sizes = [int(v) for v in g.integers(0, 4, 80)]
    sizes[11] = 30
    groups = [(n, int(b)) for n, b in zip(sizes, g.integers(0, 30, 80))]
    n = sum(sizes)
    r = [rows[i % len(rows)] for i in range(n)]
    _check(Shared(970, groups, [a + int(b) for a, b in zip(r, g.integers(0, 200, n))], r, 1, 64, "e4m3"), 8)


@pytest.mark.parametrize("rows", [1, 30])
@pytest.mark.parametrize("cu,blocks,max_rows", [([0, 3, 2, 90], [3, 3, 3], None), ([0, 50, 91], [3, 3], None), ([0, 50, 90], [3, 99], None),
                                                ([0, 50, 90], [3, -1], None), ([0, 60, 90], [3, 3], 40)])
def test_broken_groups_past_64_sequences(cu, blocks, max_rows, rows):
    """The sequences of a group whose numbers break a bound get their own pages, beside those of one that does not."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case shared plan broken groups {cu} {blocks} {max_rows} rows={rows}")
    sh = Shared(980, [(90, 3)], [rows + 5 * i % 150 for i in range(90)], [rows] * 90, 1, 64, "int8")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    g = msi.KvGroups(i32(cu), i32(blocks), max_rows=max_rows * rows if max_rows else sh.s.cu[-1], max_blocks=3)
    _check(sh, 8, groups=g, status=4)


@pytest.mark.parametrize("n,rows", [(6, 1), (6, 40), (80, 1), (80, 40)])
def test_captured_as_sequences_grow_leave_and_come_back(n, rows):
    """Two captured calls with workspaces of their own, replayed in turn with eager calls between: sequences grow past the end
    of a page, the second half leaves for a group of its own, the first sequence falls back within the shared pages (its table its own), the
    shared pages become fewer, and all of it comes back.  Every replay has the eager call's bits, and those are right."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case shared captured n={n} rows={rows}")
    sh = Shared(990 + n + rows, [(n, 3)], [rows + 61 + i % 5 for i in range(n)], [rows] * n, 2, 64, "e4m3")
    s = sh.s
    dev = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    table, lens, cu_seqs = dev(s.table), dev(s.lens), dev([0, n, n])
    blocks = dev([3, 2])
    seqs = msi.KvSeqs(table, lens, s.seqs.cu_rows, n_rows=s.cu[-1], max_rows=rows, max_len=s.table.shape[1] * 64)
    groups = msi.KvGroups(cu_seqs, blocks, max_rows=s.cu[-1], max_blocks=3)
    q = bf16(s.g.standard_normal((s.cu[-1], 8, 64)))
    ws = [msi.kv_attention_shared_workspace(s.cache, seqs, groups, 8) for _ in range(3)]
    outs = [torch.zeros_like(q[0]) for _ in range(3)]
    stream = torch.cuda.Stream()
    graphs = []
    for w, o in zip(ws[:2], outs):
        g = torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=stream):
            msi.kv_attention_shared(s.cache, seqs, groups, q[0], o, 0.125, workspace=w, stream=torch.cuda.current_stream())
        graphs.append(g)
    start = list(s.lens)
    inside = [rows + 20 if i == 0 else x for i, x in enumerate(start)]
    own = s.table.copy()
    own[0, :3] = -1
    own[0, :2] = s.table[0, 3:5] if s.table.shape[1] > 4 else s.table[0, 3]
    steps = [(start, s.table, [0, n, n], 3), ([x + 2 for x in start], s.table, [0, n, n], 3), ([x + 2 for x in start], s.table, [0, n // 2, n], 3),
             (inside, own, [0, n, n], 3), (start, s.table, [0, n, n], 1), (start, s.table, [0, n, n], 3)]
    first = None
    for now, tab, cu, nb in steps:
        for t, v in ((lens, now), (table, tab), (cu_seqs, cu), (blocks, [nb, 2])):
            t.copy_(dev(v))
        for o in outs:
            o.fill_(5.0)
        msi.kv_attention_shared(s.cache, seqs, groups, q[0], outs[2], 0.125, workspace=ws[2], stream=torch.cuda.current_stream())
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])
        want, tol, _ = attention(s.host, tab, now, s.cu, q[1], 0.125, 4)
        assert np.all(np.abs(outs[2].double().cpu().numpy() - want) <= tol + 2.0 ** -86 * max(now))
        first = outs[2].clone() if first is None else first
    assert torch.equal(first, outs[2])
