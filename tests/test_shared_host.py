"""Attention over shared pages on the host: refusals by the C entry, the binding and the block, and workspaces that cover
what the device may make of any lengths within the bounds.  Nothing here reaches a device."""
import ctypes

import pytest
from test_attention_host import _block, _cpu_cache, _cpu_seqs, _w
from test_kv_common import P, _cache, _refused, _seqs


def _groups(**over):
    import paper_2608_23805_amd as msi
    kw = dict(n_groups=1, max_rows=5, max_blocks=3, cu_seqs=P, blocks=P)
    kw.update(over)
    return msi.msi_kv_groups(**kw)


def _args(**over):
    import paper_2608_23805_amd as msi
    kw = dict(q=P, out=2 * P, q_stride=256, out_stride=256, n_q_heads=4, scale=1.0, workspace=4 * P, workspace_bytes=1 << 40)
    kw.update(over)
    return msi.msi_kv_attention_args(**kw)


GROUPS = [(dict(n_groups=65536), "n_groups"), (dict(reserved=1), "reserved"), (dict(cu_seqs=None), "null group"), (dict(blocks=None), "null group"),
          (dict(cu_seqs=P + 2), "aligned"), (dict(blocks=P + 1), "aligned")]


@pytest.mark.parametrize("over,match", GROUPS)
def test_group_refusals(over, match):
    import paper_2608_23805_amd as msi
    c, s, g = (ctypes.byref(x) for x in (_cache(), _seqs(), _groups(**over)))
    _refused(msi.lib.msi_kv_attention_shared(c, s, g, ctypes.byref(_args()), None), match)
    n = ctypes.c_uint64()
    _refused(msi.lib.msi_kv_attention_shared_workspace(c, s, g, 4, ctypes.byref(n)), match)


def test_size_refusals():
    import paper_2608_23805_amd as msi
    n = ctypes.c_uint64()
    f = msi.lib.msi_kv_attention_shared_workspace
    big = _seqs(n_rows=1 << 29, max_rows=1 << 20)
    _refused(f(ctypes.byref(_cache(n_heads=1)), ctypes.byref(big), ctypes.byref(_groups()), 16, ctypes.byref(n)), "n_q_heads must be under")
    rows = _seqs(n_rows=1 << 29, max_rows=1)
    _refused(f(ctypes.byref(_cache(n_heads=1)), ctypes.byref(rows), ctypes.byref(_groups(max_rows=1 << 29)), 2, ctypes.byref(n)), "2^29")
    _refused(f(ctypes.byref(_cache(n_heads=256)), ctypes.byref(_seqs(n_seqs=65535, n_rows=65535, max_rows=1)), ctypes.byref(_groups(n_groups=1)), 256,
               ctypes.byref(n)), "row tiles")


def test_argument_refusals():
    import paper_2608_23805_amd as msi
    c, s, g = (ctypes.byref(x) for x in (_cache(), _seqs(), _groups()))
    f = msi.lib.msi_kv_attention_shared
    for over, match in ((dict(mass_rows=1), "mass_rows"), (dict(q=None), "q and out"), (dict(out=P), "out must not"), (dict(n_q_heads=3), "n_q_heads"),
                        (dict(scale=float("inf")), "scale"), (dict(workspace=4 * P + 8), "aligned"), (dict(status=P + 2), "status"),
                        (dict(out_stride=252), "q and out")):
        _refused(f(c, s, g, ctypes.byref(_args(**over)), None), match)
    for over in (dict(workspace=None), dict(workspace_bytes=100)):
        _refused(f(c, s, g, ctypes.byref(_args(**over)), None), "workspace", want=msi.MSI_E_NOMEM)
    _refused(f(c, s, None, ctypes.byref(_args()), None), "null")
    _refused(f(c, s, g, None, None), "null")
    assert f(c, ctypes.byref(_seqs(n_seqs=0)), g, ctypes.byref(_args(q=None)), None) == 0
    assert f(c, ctypes.byref(_seqs(max_rows=0)), g, ctypes.byref(_args(q=None)), None) == 0


@pytest.mark.parametrize("H,G,D", [(1, 1, 64), (8, 4, 128), (2, 8, 256), (3, 7, 128)])
def test_workspace_covers_what_the_device_may_cut(H, G, D):
    """The rule by which the device cuts units (chunks from the work of all owners), run over batches within the bounds: the
    partial results and items never outgrow what the host reserved.  Bytes of a row of results: 4 (D + 2)."""
    import random
    import paper_2608_23805_amd as msi
    r = random.Random(H * G * D)
    for _ in range(300):
        S = r.choice([1, 2, 7, 64, 200])
        most_rows, most_own, most_shared = r.choice([1, 1, 5, 70]), r.choice([1, 9, 40, 900]), r.choice([0, 1, 30, 2000])
        rows = [r.randint(0, most_rows) for _ in range(S)]
        own = [r.randint(0, most_own) for _ in range(S)]
        cut = sorted(r.sample(range(1, S), min(S - 1, r.choice([0, 1, 3]))))
        groups = [(sum(rows[a:z]), r.randint(0, most_shared)) for a, z in zip([0] + cut, cut + [S])]
        n_rows = sum(rows)
        if not n_rows:
            continue
        seqs = _seqs(n_seqs=S, n_rows=n_rows, max_rows=max(rows), max_blocks=most_own + most_shared, max_len=64 * (most_own + most_shared))
        g = _groups(n_groups=len(groups), max_rows=max(n for n, _ in groups), max_blocks=most_shared)
        need = ctypes.c_uint64()
        assert msi.lib.msi_kv_attention_shared_workspace(ctypes.byref(_cache(n_heads=H, head_dim=D)), ctypes.byref(seqs), ctypes.byref(g), H * G,
                                                         ctypes.byref(need)) == 0
        tile = lambda n, most: 16 if n <= 16 else 32 if n <= most else 128  # noqa: E731
        tp, ts = tile(max(n for n, _ in groups) * G, 96 if D == 256 else 64), tile(max(rows) * G, 96)
        both = tp < 128 and ts < 128
        if both:
            tp = ts = max(tp, ts)

        def chunk(work, rows_of_tile):
            if rows_of_tile == 128:
                most = 4 * (256 if D == 256 else 512)      # (the smallest chunk that the balancing may take)
                return max(8, -(-work // most))
            fill = -(-work // 256)
            return max(fill, 4) if fill <= 16 else max(16, -(-work // 2048))
        wp = sum(b * -(-n * G // tp) * H for n, b in groups)
        ws = sum(b * -(-n * G // ts) * H for n, b in zip(rows, own) if n)
        if both:
            wp = ws = wp + ws
        cp, cs = chunk(wp, tp), chunk(ws, ts)
        parts = sum(-(-b // cp) * n * G * H for n, b in groups if n) + sum(-(-b // cs) * n * G * H for n, b in zip(rows, own) if n)
        assert need.value >= parts * 4 * (D + 2) + 64 * (len(groups) + S)


def test_binding_refusals():
    import paper_2608_23805_amd as msi
    import torch
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for a, kw, match in (((i32(3), i32(3)), dict(max_rows=1, max_blocks=1), "cu_seqs"), ((i32(2).long(), i32(1)), dict(max_rows=1, max_blocks=1), "cu_seqs"),
                         ((i32(2), i32(1, 1)), dict(max_rows=1, max_blocks=1), "blocks"), ((i32(2), i32(1)), dict(max_rows=-1, max_blocks=1), "max_rows"),
                         ((i32(2), i32(1)), dict(max_rows=1, max_blocks=1 << 31), "max_rows")):
        with pytest.raises(msi.MsiError, match=match):
            msi.KvGroups(*a, **kw)
    c, s, q = _cpu_cache(), _cpu_seqs(), _w(4, 4, 64)
    g = msi.KvGroups(i32(2), i32(1), max_rows=4, max_blocks=1)
    for a, match in (((c, s, g, q[0], q, 1.0), "q must"), ((c, s, g, q, q[:3], 1.0), "out must"), ((c, s, g, q, q, float("nan")), "scale"),
                     ((c, s, g, q, q, 1.0), "HIP device")):
        with pytest.raises(msi.MsiError, match=match):
            msi.kv_attention_shared(*a)


def test_block_with_rotation_groups_and_4_bit_weights():
    """What a step would trip over later is refused when the block is made, or before the step changes anything."""
    import paper_2608_23805_amd as msi
    import torch
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q4 = lambda n, k, g=32: (torch.zeros((n, k // 2), dtype=torch.uint8), torch.zeros((n, k // g)).half())  # noqa: E731
    r = msi.KvRotary([0.1] * 32, device="cpu")
    for over in (dict(wqkv=q4(512, 128)[:1]), dict(wqkv=list(q4(512, 128))), dict(wo=()), dict(wo=(q4(128, 256)[0], None)),
                 dict(wqkv=(q4(512, 128)[0], torch.zeros((512, 3)).half())), dict(wqkv=(q4(512, 128)[0].int(), q4(512, 128)[1])),
                 dict(wo=(q4(128, 256)[0], q4(128, 256)[1].float())), dict(wo=q4(128, 128)), dict(wqkv=q4(520, 128)),
                 dict(wqkv=q4(512, 128, 16)), dict(rotary=msi.KvRotary([0.1] * 40, device="cpu"))):
        with pytest.raises(msi.MsiError) as e:
            _block(**over)
        assert e.value.status == msi.MSI_E_INVALID_ARG, over
    x, h, s = _w(4, 128), torch.zeros((4, 128)), _cpu_seqs()
    g = msi.KvGroups(i32(2), i32(1), max_rows=4, max_blocks=1)
    for b, kw, match in ((_block(), dict(positions=i32(4)), "rotary"), (_block(rotary=r), {}, "positions"), (_block(rotary=r), dict(positions=i32(3)), "positions"),
                         (_block(), dict(groups=g, mass_rows=1), "mass_rows"), (_block(), dict(groups=g), "reserve")):
        with pytest.raises(msi.MsiError, match=match):
            b.step(x, h, s, **kw)
    b = _block(wqkv=q4(512, 128), wo=q4(128, 256, 128), rotary=r)
    b.reserve(s, groups=g)
    assert b.workspace.numel() >= msi.kv_attention_shared_workspace_size(b.cache, s, g, 4)
    with pytest.raises(msi.MsiError, match="HIP device"):
        b.step(x, h, s, positions=i32(4), groups=g)
