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
