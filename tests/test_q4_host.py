"""Refusals of the projection with 4-bit weights, by the C entry and by the binding.  Nothing here reaches a device."""
import ctypes

import pytest
from test_kv_common import P, _refused


def _args(**over):
    import paper_2608_23805_amd as msi
    lin = dict(x=P, w=2 * P, out=3 * P, M=4, N=8, K=64, x_stride=64, out_stride=8, out_dtype=0)
    rest = dict(scales=4 * P, group=32)
    for k, v in over.items():
        (rest if k in ("scales", "group", "reserved") else lin)[k] = v
    return msi.msi_linear_q4_args(linear=msi.msi_linear_args(**lin), **rest)


@pytest.mark.parametrize("over,match", [
    (dict(group=0), "group"), (dict(group=16), "group"), (dict(group=48), "group"), (dict(group=256), "group"),
    (dict(K=0), "multiple of group"), (dict(K=96, group=64, x_stride=96), "multiple of group"), (dict(reserved=1), "reserved"),
    (dict(scales=None), "scales"), (dict(scales=4 * P + 1), "scales"), (dict(w=None), "16-byte"), (dict(w=2 * P + 8), "16-byte"),
    (dict(x=P + 8), "16-byte"), (dict(x_stride=60), "stride"), (dict(out=None), "out needs"), (dict(out_stride=7), "out needs"),
    (dict(activation=9), "activation"), (dict(out_dtype=2), "dtype"), (dict(out=P), "out must not"), (dict(out=2 * P), "out must not"),
    (dict(out=4 * P), "scales"), (dict(bias=5 * P + 2), "bias"), (dict(residual=3 * P, residual_dtype=1, residual_stride=8), "residual that is out"),
    (dict(M=(1 << 29) + 1), "2^29"), (dict(K=(1 << 21) + 32, x_stride=1 << 21), "2^21"),
])
def test_refusals(over, match):
    import paper_2608_23805_amd as msi
    _refused(msi.lib.msi_linear_q4(ctypes.byref(_args(**over)), None), match)


def test_nothing_to_do():
    import paper_2608_23805_amd as msi
    _refused(msi.lib.msi_linear_q4(None, None), "null")
    for over in (dict(M=0), dict(N=0), dict(M=0, x=None, w=None, out=None, scales=None)):
        assert msi.lib.msi_linear_q4(ctypes.byref(_args(**over)), None) == msi.MSI_OK


def test_binding_refusals():
    import paper_2608_23805_amd as msi
    import torch
    x, w, s = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 2)).half()
    y = torch.zeros((4, 8))
    for a, match in (((x, w, s[:, :0], y), "scales must be"), ((x, w, torch.zeros((8, 3)).half(), y), "scales must be"),
                     ((x, w, torch.zeros((8, 64)).half(), y), "scales must be"), ((x, w.int(), s, y), "w must"),
                     ((x, w[:, :31], s, y), "w must"), ((x, w, s.float(), y), "float16"), ((x, w, s[:7], y), "w must"),
                     ((x, w, s.t().contiguous().t(), y), "scales must"), ((x[0], w, s, y), "matrices"), ((x, w, s[0], y), "matrices"),
                     ((x.float(), w, s, y), "x must"), ((x, w, s, y[:, :7]), "out must"), ((x, w, s, y.double()), "out must"),
                     ((x, w, s, y), "HIP device")):
        with pytest.raises(msi.MsiError, match=match):
            msi.linear_q4(*a)
    with pytest.raises(msi.MsiError, match="activation"):
        msi.linear_q4(x, w, s, y, act="relu")
    with pytest.raises(msi.MsiError, match="bias"):
        msi.linear_q4(x, w, s, y, bias=torch.zeros(7))


def test_tiles_of_many_features():
    """A grid holds under 2^32 threads: past 2^22 features few rows go through tiles as well."""
    import paper_2608_23805_amd as msi
    v = [ctypes.c_uint32() for _ in range(3)]
    for M, N, few in ((1, 1 << 22, True), (1, (1 << 22) + 1, False), (16, 1 << 29, False), (17, 1, True), (32, 8192, True),
                      (32, 8193, False), (33, 1, False)):
        assert msi.lib.msi_debug_linear_q4_tile(M, N, 32, *map(ctypes.byref, v)) == msi.MSI_OK
        rows, features, _ = (x.value for x in v)
        assert (rows == 0) == few
        threads = 512 if rows == 0 else 256
        assert -(-N // features) * -(-M // max(rows, 16)) * threads < 1 << 32


def test_tile_refusals():
    import paper_2608_23805_amd as msi
    v = [ctypes.byref(ctypes.c_uint32()) for _ in range(3)]
    for a in ((0, 1, 32), (1, 0, 32), ((1 << 29) + 1, 1, 32), (1 << 29, 129, 32), (1, 1, 0), (1, 1, 40), (1, 1, (1 << 21) + 32)):
        _refused(msi.lib.msi_debug_linear_q4_tile(*a, *v), "M and N")
    for k in range(3):
        _refused(msi.lib.msi_debug_linear_q4_tile(1, 1, 32, *[None if i == k else p for i, p in enumerate(v)]), "null")
