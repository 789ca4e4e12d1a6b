"""The attention block on the host: which tiles the projection chooses, refusals of the entry points and of
AttentionBlock before anything runs, and what its workspaces add up to.  Nothing here reaches a device."""
import ctypes

import pytest
from test_kv_common import P, _cache, _refused, _seqs


def _cpu_cache(mass=True):
    import paper_2608_23805_amd as msi
    return msi.KvCache.alloc(40, 2, 64, "e4m3", mass=mass, device="cpu")


def _cpu_seqs(max_len=192, n_rows=4, max_rows=3):
    import paper_2608_23805_amd as msi
    import torch
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    return msi.KvSeqs(i32(2, -(-max_len // 64)), i32(2), i32(3), n_rows=n_rows, max_rows=max_rows, max_len=max_len)


def _w(*shape):
    import torch
    return torch.zeros(shape, dtype=torch.bfloat16)


def _block(mass=True, **over):
    import paper_2608_23805_amd as msi
    kw = dict(wqkv=_w(512, 128), wo=_w(128, 256), cache=_cpu_cache(mass), n_q_heads=4, max_rows=8)
    kw.update(over)
    return msi.AttentionBlock(**kw)


def test_sequence_flags():
    import paper_2608_23805_amd as msi
    n = ctypes.c_uint64()
    for flags in (2, 1 << 31):
        _refused(msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs(flags=flags)), 4, 0, ctypes.byref(n)), "flags")
    assert msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs(flags=1)), 4, 0, ctypes.byref(n)) == 0
