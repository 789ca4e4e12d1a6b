"""Append with rotation on the host: the frequencies' fixed-point turns, and refusals by the C entry and the binding.
Nothing here reaches a device."""
import ctypes
import math

import pytest
from test_attention_host import _cpu_cache, _cpu_seqs, _w
from test_kv_common import P, _cache, _refused, _seqs


def test_turns():
    """Fractions of a turn to 2^-64, whole turns and negative frequencies wrapped."""
    import paper_2608_23805_amd as msi
    f = [1.0, 0.5, 1e-4, 2 * math.pi, 7.0, -1.0, 0.0, 1e300]
    r = msi.KvRotary(f, device="cpu")
    got = [int(x) % 2 ** 64 for x in r.freq]
    assert got[0] == 0x28BE60DB9391054A                            # 2^64 / (2 pi), from its known hexadecimal digits
    assert got[1] == 0x145F306DC9C882A5 and got[5] == 2 ** 64 - got[0] and got[6] == 0
    assert got[4] == round((7 * (got[0] + 0.5)) / 2 ** 64 % 1 * 2 ** 64) or abs(got[4] - 7 * got[0] % 2 ** 64) <= 7
    assert min(got[3], 2 ** 64 - got[3]) < 2 ** 12                 # (2 pi as a double is off by 2^-52 of it)
    assert r.rot_dim == 16 and r.n_axes == 1 and r.axis is None and 0 <= got[7] < 2 ** 64


def test_rotary_refusals():
    import paper_2608_23805_amd as msi
    ok = [0.1] * 16
    for kw, match in ((dict(inv_freq=[]), "multiple of 8"), (dict(inv_freq=[1.0] * 12), "multiple of 8"),
                      (dict(inv_freq=[1.0] * 136), "multiple of 8"), (dict(inv_freq=[1.0] * 7 + [float("nan")]), "finite"),
                      (dict(inv_freq=ok, axes=[0] * 15), "axes"), (dict(inv_freq=ok, axes=[0] * 15 + [4]), "axes"),
                      (dict(inv_freq=ok, axes=[0] * 15 + [-1]), "axes")):
        with pytest.raises(msi.MsiError, match=match):
            msi.KvRotary(device="cpu", **kw)


def _args(**over):
    import paper_2608_23805_amd as msi
    kw = dict(q=P, q_out=2 * P, k=3 * P, v=4 * P, q_stride=256, q_out_stride=256, k_stride=128, v_stride=128, n_q_heads=4,
              rot_dim=64, n_axes=2, freq=5 * P, axis=6 * P, positions=7 * P, position_stride=5)
    kw.update(over)
    return msi.msi_kv_append_rotary_args(**kw)


@pytest.mark.parametrize("over,match", [
    (dict(rot_dim=0), "rot_dim"), (dict(rot_dim=8), "rot_dim"), (dict(rot_dim=72), "rot_dim"), (dict(rot_dim=128), "rot_dim"),
    (dict(n_axes=0), "n_axes"), (dict(n_axes=5), "n_axes"), (dict(interleaved=2), "interleaved"), (dict(n_q_heads=0), "n_q_heads"),
    (dict(n_q_heads=4097), "n_q_heads"), (dict(freq=None), "freq"), (dict(freq=5 * P + 4), "freq"), (dict(axis=6 * P + 1), "freq"),
    (dict(positions=None), "positions"), (dict(positions=7 * P + 2), "positions"), (dict(position_stride=4), "positions"),
    (dict(position_stride=(1 << 32) + 1), "positions"), (dict(q_stride=248), "q and q_out"), (dict(q_out=None), "q and q_out"),
    (dict(q_out=2 * P + 8), "q and q_out"), (dict(q_out_stride=260), "q and q_out"), (dict(q_out=P, q_out_stride=512), "needs its stride"),
    (dict(q_out=3 * P), "q_out must not"), (dict(q_out=4 * P), "q_out must not"), (dict(k=None), "k and v"), (dict(v_stride=120), "k and v"),
    (dict(status=8 * P + 1), "status"),
])
def test_refusals(over, match):
    import paper_2608_23805_amd as msi
    _refused(msi.lib.msi_kv_append_rotary(ctypes.byref(_cache()), ctypes.byref(_seqs()), ctypes.byref(_args(**over)), None), match)


def test_nothing_to_do_and_nulls():
    import paper_2608_23805_amd as msi
    f, c = msi.lib.msi_kv_append_rotary, ctypes.byref(_cache())
    _refused(f(c, ctypes.byref(_seqs()), None, None), "null")
    _refused(f(None, ctypes.byref(_seqs()), ctypes.byref(_args()), None), "null")
    _refused(f(c, None, ctypes.byref(_args()), None), "null")
    for over in (dict(n_seqs=0), dict(max_rows=0), dict(max_len=0)):
        assert f(c, ctypes.byref(_seqs(**over)), ctypes.byref(_args(q=None, k=None, v=None)), None) == 0


def test_binding_refusals():
    import paper_2608_23805_amd as msi
    import torch
    s, c, q, kv = _cpu_seqs(), _cpu_cache(), _w(4, 4, 64), _w(4, 2, 64)
    r, r3 = msi.KvRotary([0.1] * 32, device="cpu"), msi.KvRotary([0.1] * 32, axes=[0] * 30 + [1, 2], device="cpu")
    p = torch.zeros(4, dtype=torch.int32)
    p3 = torch.zeros((3, 4), dtype=torch.int32)
    for a, match in (((c, s, r, None, q, q, kv, kv), "positions"), ((c, s, r, p[:3], q, q, kv, kv), "positions"),
                     ((c, s, r, p.long(), q, q, kv, kv), "positions"), ((c, s, r3, p, q, q, kv, kv), "positions"),
                     ((c, s, r3, p3[:2], q, q, kv, kv), "positions"), ((c, s, r3, p3.t().contiguous().t(), q, q, kv, kv), "contiguous"),
                     ((c, s, r3, p[None].expand(3, 4), q, q, kv, kv), "overlap"), ((c, s, r, p, q[0], q, kv, kv), "q must"),
                     ((c, s, r, p, q, q[:, :3], kv, kv), "q_out must"), ((c, s, r, p, q, q, q, kv), "k must"),
                     ((c, s, msi.KvRotary([0.1] * 40, device="cpu"), p, q, q, kv, kv), "elements rotate"),
                     ((c, s, r, p, q, None, kv, kv), "together"), ((c, s, r, p, None, q, kv, kv), "together"),
                     ((c, s, r, p, q, q, kv, kv), "HIP device"), ((c, s, r3, p3, None, None, kv, kv), "HIP device")):
        with pytest.raises(msi.MsiError, match=match):
            msi.kv_append_rotary(*a)


def test_streams_of_another_device():
    """A kernel goes to its stream's device, which cannot read the tensors of another: refused."""
    import types
    import paper_2608_23805_amd as msi
    import torch
    s, c, q, kv = _cpu_seqs(), _cpu_cache(), _w(4, 4, 64), _w(4, 2, 64)
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    other = types.SimpleNamespace(cuda_stream=0, device_index=1)
    r, g = msi.KvRotary([0.1] * 32, device="cpu"), msi.KvGroups(i32(2), i32(1), max_rows=4, max_blocks=1)
    w4 = torch.zeros((8, 16), dtype=torch.uint8), torch.zeros((8, 1)).half()
    for f, a in ((msi.kv_append_rotary, (c, s, r, i32(4), q, q, kv, kv)), (msi.kv_attention_shared, (c, s, g, q, q, 1.0)),
                 (msi.linear_q4, (_w(4, 32), *w4, _w(4, 8)))):
        with pytest.raises(msi.MsiError, match="stream"):
            f(*a, stream=other)
