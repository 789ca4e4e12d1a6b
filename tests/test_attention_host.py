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


@pytest.mark.parametrize("M,N,tile", [
    (1, 1, (32, 32, 2)), (16, 5120, (32, 32, 2)), (32, 8192, (32, 32, 2)), (32, 8193, (32, 64, 1)), (64, 8192, (32, 64, 1)),
    (64, 8193, (64, 64, 1)), (512, 2048, (64, 64, 1)), (512, 2049, (64, 128, 1)), (512, 4096, (64, 128, 1)),
    (512, 4097, (128, 128, 1)), (2048, 2048, (128, 128, 1)), (2048, 2049, (128, 128, 2)), (2500, 2500, (128, 128, 2)),
    (4096, 4096, (256, 256, 1)), (4096, 8192, (256, 256, 1)), (1 << 29, 1, (128, 128, 2)), (1 << 29, 128, (128, 128, 2)),
    (1 << 20, 1 << 16, (256, 256, 1)),
])
def test_linear_tile(M, N, tile):
    import paper_2608_23805_amd as msi
    v = [ctypes.c_uint32() for _ in range(3)]
    assert msi.lib.msi_debug_linear_tile(M, N, *map(ctypes.byref, v)) == msi.MSI_OK
    assert tuple(x.value for x in v) == tile


def test_linear_tile_refusals():
    import paper_2608_23805_amd as msi
    v = [ctypes.byref(ctypes.c_uint32()) for _ in range(3)]
    for a in ((0, 1), (1, 0), ((1 << 29) + 1, 1), (1 << 29, 129)):
        _refused(msi.lib.msi_debug_linear_tile(*a, *v), "M and N")
    for k in range(3):
        _refused(msi.lib.msi_debug_linear_tile(1, 1, *[None if i == k else p for i, p in enumerate(v)]), "null")


def test_status_words_are_aligned():
    """A status word between two words would be an atomic at an address that has none."""
    import paper_2608_23805_amd as msi
    c, s = ctypes.byref(_cache()), ctypes.byref(_seqs(max_rows=1, max_len=100))
    for f in (msi.lib.msi_kv_append, msi.lib.msi_kv_read):
        _refused(f(c, s, P, P, 128, 128, P + 2, None), "status")
    a = msi.msi_kv_attention_args(q=P, out=2 * P, q_stride=256, out_stride=256, n_q_heads=4, scale=1.0, status=P + 1)
    _refused(msi.lib.msi_kv_attention(c, s, ctypes.byref(a), None), "status")
    e = msi.msi_kv_evict_args(budget=100, sinks=4, recent=10, dst_blocks=2, dst_table=2 * P, new_lens=3 * P, keep=4 * P, status=P + 3)
    _refused(msi.lib.msi_kv_evict(c, s, ctypes.byref(e), None), "status")


def test_sequence_flags():
    import paper_2608_23805_amd as msi
    n = ctypes.c_uint64()
    for flags in (2, 1 << 31):
        _refused(msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs(flags=flags)), 4, 0, ctypes.byref(n)), "flags")
    assert msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs(flags=1)), 4, 0, ctypes.byref(n)) == 0


def test_workspace_of_weights_needs_them():
    import paper_2608_23805_amd as msi
    n = ctypes.c_uint64()
    _refused(msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache(mass=0)), ctypes.byref(_seqs()), 4, 1, ctypes.byref(n)), "mass")
    assert msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache(mass=0)), ctypes.byref(_seqs()), 4, 0, ctypes.byref(n)) == 0


def test_block_construction_refusals():
    """What a step would trip over after it has written the cache is refused when the block is made."""
    import paper_2608_23805_amd as msi
    import torch
    for over in (dict(wqkv=_w(512, 128).float()), dict(wo=_w(128, 256).float()), dict(wqkv=_w(128, 512).t()),
                 dict(wo=_w(256, 128).t()), dict(wqkv=_w(520, 128)), dict(wo=_w(256, 128)), dict(bias=torch.zeros(511)),
                 dict(bias=_w(512)), dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=3e38), dict(n_q_heads=3),
                 dict(n_q_heads=0), dict(wqkv=_w(512, 100), wo=_w(100, 256)), dict(max_rows=-1), dict(wqkv=_w(512)),
                 dict(wo=_w(128 * 256 + 8)[1:1 + 128 * 256].view(128, 256)), dict(wqkv=_w(512 * 128 + 8)[4:4 + 512 * 128].view(512, 128))):
        with pytest.raises(msi.MsiError) as e:
            _block(**over)
        assert e.value.status == msi.MSI_E_INVALID_ARG, over


def test_block_step_refusals():
    """Refusals that need no device come before the first call that does."""
    import paper_2608_23805_amd as msi
    import torch
    x, h, s = _w(4, 128), torch.zeros((4, 128)), _cpu_seqs()
    for match, b, a, kw in (("mass", _block(mass=False), (x, h, s), dict(mass_rows=1)),
                            ("mass_decay", _block(), (x, h, s), dict(mass_rows=1, mass_decay=-0.5)),
                            ("mass_decay", _block(), (x, h, s), dict(mass_rows=1, mass_decay=float("nan"))),
                            ("mass_decay", _block(), (x, h, s), dict(mass_rows=1, mass_decay=1e39)),
                            ("mass_rows", _block(), (x, h, s), dict(mass_rows=-1)),
                            ("x must", _block(), (x.float(), h, s), {}), ("h must", _block(), (x, h.double(), s), {}),
                            ("h must", _block(), (x, h[:3], s), {}), ("status", _block(), (x, h, s), dict(status=x)),
                            ("rows", _block(max_rows=3), (x, h, s), {})):
        with pytest.raises(msi.MsiError, match=match):
            b.step(*a, **kw)


def test_scales_that_no_float_holds():
    """A scale or decay past fp32's range is refused like one that is infinite."""
    import paper_2608_23805_amd as msi
    s = _cpu_seqs()
    for kw in (dict(scale=1e39), dict(scale=1.0, mass_rows=1, mass_decay=1e39), dict(scale=-1e300)):
        with pytest.raises(msi.MsiError) as e:
            msi.kv_attention(_cpu_cache(), s, _w(4, 4, 64), _w(4, 4, 64), **kw)
        assert e.value.status == msi.MSI_E_INVALID_ARG


def test_growing_bounds_do_not_pile_up_workspaces():
    """Captured steps go on using the workspace they were captured with, so a block keeps each; growing bounds must not
    make that a sum over every size."""
    import paper_2608_23805_amd as msi
    b = _block()
    for blocks in range(9, 200):
        s = _cpu_seqs(max_len=64 * blocks, n_rows=2, max_rows=1)
        b.reserve(s, 1)
        assert b.workspace.numel() >= msi.kv_attention_workspace_size(b.cache, s, 4, 1)
    assert sum(w.numel() for w in b._kept) <= 4 * msi.kv_attention_workspace_size(b.cache, s, 4, 1)


def test_tensors_without_elements():
    """A tensor of no rows may have any strides: only its shape counts."""
    import paper_2608_23805_amd as msi
    import torch
    empty = torch.empty_strided((0, 16), (1, 1), dtype=torch.bfloat16)
    rows = torch.empty_strided((0, 2, 64), (1, 1, 1), dtype=torch.bfloat16)
    s = _cpu_seqs(n_rows=0, max_rows=0)
    for f, a in ((msi.linear, (empty, _w(8, 16), torch.empty_strided((0, 8), (1, 1), dtype=torch.bfloat16))),
                 (msi.kv_append, (_cpu_cache(), s, rows, rows)), (msi.kv_read, (_cpu_cache(), s, rows, rows)),
                 (msi.kv_attention, (_cpu_cache(), s, rows, rows, 1.0))):
        with pytest.raises(msi.MsiError, match="HIP device"):          # (and no complaint about strides)
            f(*a)


def test_streams_of_another_device():
    """A kernel goes to its stream's device, which cannot read the tensors of another: refused."""
    import types
    import paper_2608_23805_amd as msi
    import torch
    s, i32 = _cpu_seqs(), lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    other = types.SimpleNamespace(cuda_stream=0, device_index=1)
    kv, q = _w(4, 2, 64), _w(4, 4, 64)
    for f, a, k in ((msi.linear, (_w(4, 16), _w(8, 16), _w(4, 8)), {}), (msi.kv_append, (_cpu_cache(), s, kv, kv), {}),
                    (msi.kv_read, (_cpu_cache(), s, kv, kv), {}), (msi.kv_attention, (_cpu_cache(), s, q, q, 1.0), {}),
                    (msi.kv_evict, (_cpu_cache(), s, i32(2, 2), i32(2), i32(2, 2, 100)), dict(budget=100))):
        with pytest.raises(msi.MsiError, match="stream"):
            f(*a, stream=other, **k)


def test_launch_bounds_of_all_rows():
    """The workgroups that clear rows come on top of the units': both stay in one grid."""
    import paper_2608_23805_amd as msi
    n = ctypes.c_uint64()

    def size(flags, S, rows):
        s = _seqs(n_seqs=S, n_rows=1 << 29, max_rows=rows, max_blocks=1, max_len=64, flags=flags)
        return msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache(n_heads=1)), ctypes.byref(s), 1, 0, ctypes.byref(n))
    assert size(0, 4095, 128 * 4097) == 0                      # 2^24 - 1 workgroups
    _refused(size(1, 4095, 128 * 4097), "under 2^24")
    assert size(1, 4094, 128 * 4097) == 0
