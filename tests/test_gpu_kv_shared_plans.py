"""Attention over shared pages: how its groups and sequences become units, in both of its planners (up to 64 groups and 64
sequences every wavefront lays the units out, a launch of its own does above).  The oracle and the bound are those of
test_gpu_kv_shared.py."""
import ctypes

import numpy as np
import pytest

from _gpu_helpers import log
from test_gpu_kv_shared import Shared, _check

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
