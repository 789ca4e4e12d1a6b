"""Host-only checks of the paged cache: bounds of lengths and pages, the scale rule (g++ with
AddressSanitizer / UndefinedBehaviorSanitizer), and the refusals of the attention block's entry
points, none of which reaches a device."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_bounds_and_scales(tmp_path):
    exe = str(tmp_path / "kv_common_test")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
                    "-o", exe, os.path.join(ROOT, "tests", "cpp", "kv_common_test.cpp")], check=True, capture_output=True,
                   text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


P = 1 << 20                                 # a pointer that no refused call follows


def _cache(**over):
    import paper_2608_23805_amd as msi
    kw = dict(format=0, n_pages=4, n_heads=2, head_dim=64, data=P, scales=P, mass=P)
    kw.update(over)
    return msi.msi_kv_cache(**kw)


def _seqs(**over):
    import paper_2608_23805_amd as msi
    kw = dict(n_seqs=2, max_blocks=3, n_rows=5, max_rows=4, max_len=192, reserved=0, table=P, lens=P, cu_rows=P)
    kw.update(over)
    return msi.msi_kv_seqs(**kw)


def _refused(status, fragment, want=-1):
    import paper_2608_23805_amd as msi
    assert status == want and fragment in msi.last_error(), (status, msi.last_error())


CACHE = [(dict(format=2), "format"), (dict(n_pages=0), "n_pages"), (dict(n_heads=0), "n_heads"), (dict(n_heads=257), "n_heads"),
         (dict(head_dim=96), "head_dim"), (dict(data=0), "null cache"), (dict(scales=0), "null cache"),
         (dict(data=P + 8), "aligned"), (dict(mass=P + 4), "aligned")]
SEQS = [(dict(n_seqs=65536), "n_seqs"), (dict(max_len=193), "max_len"), (dict(lens=0), "null sequence"),
        (dict(table=0), "null sequence"), (dict(cu_rows=0), "cu_rows"), (dict(max_rows=6), "max_rows"),
        (dict(lens=P + 2), "aligned")]


@pytest.mark.parametrize("which", ["append", "read", "attention", "workspace"])
def test_cache_and_sequence_refusals(which):
    import paper_2608_23805_amd as msi
    a = msi.msi_kv_attention_args(q=P, out=2 * P, q_stride=256, out_stride=256, n_q_heads=4, scale=1.0)
    n = ctypes.c_uint64()

    def call(c, s):
        c, s = ctypes.byref(c), ctypes.byref(s)
        if which == "attention":
            return msi.lib.msi_kv_attention(c, s, ctypes.byref(a), None)
        if which == "workspace":
            return msi.lib.msi_kv_attention_workspace(c, s, 4, 0, ctypes.byref(n))
        return getattr(msi.lib, f"msi_kv_{which}")(c, s, P, P, 128, 128, None, None)
    for over, fragment in CACHE:
        _refused(call(_cache(**over), _seqs()), fragment)
    for over, fragment in SEQS:
        _refused(call(_cache(), _seqs(**over)), fragment)
    f = getattr(msi.lib, "msi_kv_attention_workspace" if which == "workspace" else f"msi_kv_{which}")
    rest = {"attention": (ctypes.byref(a), None), "workspace": (4, 0, ctypes.byref(n))}.get(which, (P, P, 128, 128, None, None))
    _refused(f(None, ctypes.byref(_seqs()), *rest), "null cache")
    _refused(f(ctypes.byref(_cache()), None, *rest), "null sequences")


def test_row_refusals():
    import paper_2608_23805_amd as msi
    for f in (msi.lib.msi_kv_append, msi.lib.msi_kv_read):
        for k, v, ks, vs in ((0, P, 128, 128), (P, 0, 128, 128), (P + 8, P, 128, 128), (P, P, 120, 128), (P, P, 128, 132),
                             (P, P, 128, (1 << 21) + 8)):
            _refused(f(ctypes.byref(_cache()), ctypes.byref(_seqs()), k, v, ks, vs, None, None), "k and v")
        # nothing to do: no rows, no sequences, no tokens
        for s in (_seqs(n_rows=0, max_rows=0), _seqs(n_seqs=0), _seqs(max_len=0)):
            assert f(ctypes.byref(_cache()), ctypes.byref(s), 0, 0, 0, 0, None, None) == 0


def test_attention_refusals():
    import paper_2608_23805_amd as msi

    def call(c=None, s=None, **over):
        kw = dict(q=P, out=2 * P, q_stride=256, out_stride=256, n_q_heads=4, scale=1.0)
        kw.update(over)
        return msi.lib.msi_kv_attention(ctypes.byref(c or _cache()), ctypes.byref(s or _seqs(max_rows=1, max_len=100)),
                                        ctypes.byref(msi.msi_kv_attention_args(**kw)), None)
    for over, fragment in ((dict(n_q_heads=3), "n_q_heads"), (dict(n_q_heads=0), "n_q_heads"), (dict(scale=float("nan")), "scale"),
                           (dict(scale=float("inf")), "scale"), (dict(mass_rows=1, mass_decay=-0.5), "mass_decay"),
                           (dict(mass_rows=1, mass_decay=float("nan")), "mass_decay"), (dict(q=0), "q and out"),
                           (dict(out=0), "q and out"), (dict(q_stride=248), "q and out"), (dict(out_stride=260), "q and out"),
                           (dict(out=P), "out must not be q")):
        _refused(call(**over), fragment)
    _refused(call(c=_cache(mass=0), mass_rows=1, mass_decay=1.0), "mass")
    # workspace: needed for weights and long caches, checked against what the size call says
    n = ctypes.c_uint64()
    long = _seqs(max_rows=1)
    long.max_blocks, long.max_len = 1000, 64000
    msi._check(msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache()), ctypes.byref(long), 4, 0, ctypes.byref(n)))
    assert n.value > 0
    _refused(call(s=long), "workspace", msi.MSI_E_NOMEM)
    _refused(call(s=long, workspace=P, workspace_bytes=n.value - 1), "workspace", msi.MSI_E_NOMEM)
    _refused(call(s=long, workspace=P + 4, workspace_bytes=n.value), "aligned")
    msi._check(msi.lib.msi_kv_attention_workspace(ctypes.byref(_cache()), ctypes.byref(_seqs(max_rows=1, max_len=100)), 4, 0,
                                                  ctypes.byref(n)))
    assert n.value == 0
    assert call(s=_seqs(n_seqs=0)) == 0 and call(s=_seqs(n_rows=0, max_rows=0), q=0, out=0) == 0


def test_launch_bounds():
    """Bounds that would ask for more workgroups than a launch has are refused, the largest ones below are not."""
    import paper_2608_23805_amd as msi
    n = ctypes.c_uint64()

    def size(heads, **over):
        c = _cache(n_heads=heads.pop("n_heads", 2))
        return msi.lib.msi_kv_attention_workspace(ctypes.byref(c), ctypes.byref(_seqs(**over)), heads["q"], 1, ctypes.byref(n))
    most = 1 << 29
    _refused(size(dict(q=4), n_rows=most + 1, max_rows=1), "max_rows")
    _refused(size(dict(q=4), n_rows=most, max_rows=most), "heads of a group")
    _refused(size(dict(q=2), n_rows=most, max_rows=most, n_seqs=2), "under 2^24")
    _refused(size(dict(q=256, n_heads=256), n_rows=1 << 20, max_rows=1 << 20, n_seqs=8), "under 2^24")
    _refused(size(dict(q=4), max_blocks=1 << 23, max_len=most, n_seqs=65), "blocks of max_len")
    assert size(dict(q=2), n_rows=most, max_rows=most, n_seqs=1) == 0
    assert size(dict(q=256, n_heads=256), n_rows=65535, max_rows=1, n_seqs=65535) == 0
    a = msi.msi_kv_attention_args(q=P, out=2 * P, q_stride=256, out_stride=256, n_q_heads=4, scale=3e38)
    _refused(msi.lib.msi_kv_attention(ctypes.byref(_cache()), ctypes.byref(_seqs()), ctypes.byref(a), None), "scale")


def test_evict_refusals():
    import paper_2608_23805_amd as msi

    def call(c=None, s=None, **over):
        kw = dict(budget=100, sinks=4, recent=10, dst_blocks=2, dst_table=2 * P, new_lens=3 * P, keep=4 * P)
        kw.update(over)
        return msi.lib.msi_kv_evict(ctypes.byref(c or _cache()), ctypes.byref(s or _seqs(cu_rows=0)),
                                    ctypes.byref(msi.msi_kv_evict_args(**kw)), None)
    for over, fragment in ((dict(budget=0), "budget"), (dict(sinks=91), "budget"), (dict(sinks=0xFFFFFFFF, recent=2), "budget"),
                           (dict(dst_blocks=1), "dst_table"), (dict(dst_table=0), "null"), (dict(new_lens=0), "null"),
                           (dict(keep=0), "null"), (dict(new_lens=P), "new_lens"), (dict(dst_table=P), "new_lens"),
                           (dict(keep=4 * P + 2), "aligned")):
        _refused(call(**over), fragment)
    _refused(call(c=_cache(mass=0)), "mass")
    assert call(s=_seqs(n_seqs=0, cu_rows=0)) == 0


def test_linear_refusals():
    import paper_2608_23805_amd as msi

    def call(**over):
        kw = dict(x=P, w=P, bias=None, residual=None, out=3 * P, M=4, N=6, K=16, activation=0, residual_dtype=0, out_dtype=1,
                  x_stride=16, residual_stride=6, out_stride=6)
        kw.update(over)
        return msi.lib.msi_linear(ctypes.byref(msi.msi_linear_args(**kw)), None)
    for over, fragment in ((dict(K=0), "K must"), (dict(K=12), "K must"), (dict(K=(1 << 21) + 8), "K must"), (dict(M=(1 << 30) + 1), "M and N"),
                           (dict(M=1 << 30, N=1 << 10), "M and N"), (dict(x=0), "x needs"), (dict(x=P + 2), "x needs"),
                           (dict(x_stride=8), "x needs"), (dict(x_stride=20), "x needs"), (dict(w=0), "w must"), (dict(w=P + 8), "w must"),
                           (dict(out=0), "out needs"), (dict(out=3 * P + 1), "out needs"), (dict(out_stride=5), "out needs"),
                           (dict(residual=P, residual_stride=5), "residual needs"), (dict(residual=P + 2), "residual needs"),
                           (dict(residual=P, residual_dtype=2), "dtype"), (dict(out_dtype=2), "dtype"), (dict(activation=4), "activation"),
                           (dict(bias=P + 2), "bias")):
        _refused(call(**over), fragment)
    # out over another operand, or over a residual of another form
    for over, fragment in ((dict(x=2 * P, out=2 * P), "out must not"), (dict(w=2 * P, out=2 * P), "out must not"),
                           (dict(out=2 * P, residual=2 * P), "residual that is out"),
                           (dict(out=2 * P, residual=2 * P, residual_dtype=1, residual_stride=8), "residual that is out"),
                           (dict(M=(1 << 29) + 1), "M and N"), (dict(M=1 << 29, N=129, out_stride=129), "M and N")):
        _refused(call(**over), fragment)
    assert call(M=0) == 0 and call(N=0, x=0, w=0, out=0) == 0
    _refused(msi.lib.msi_linear(None, None), "null")


def test_binding_refusals():
    """The binding checks what the C call cannot see: types, shapes, strides, devices."""
    import torch
    import paper_2608_23805_amd as msi
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)  # noqa: E731
    x, w, out = z(4, 16), z(6, 16), z(4, 6)

    def refuses(f, *a, **k):
        with pytest.raises(msi.MsiError) as e:
            f(*a, **k)
        assert e.value.status == msi.MSI_E_INVALID_ARG
    for a, k in (((x.float(), w, out), {}), ((x, w.float(), out), {}), ((x, w, z(4, 7)), {}), ((x, z(6, 24), out), {}),
                 ((x, w, out.half()), {}), ((x.t().contiguous().t(), w, out), {}), ((x, w, out), dict(act="relu")),
                 ((x, w, out), dict(bias=z(6))), ((x, w, out), dict(bias=z(5, dtype=torch.float32))),
                 ((x, w, out), dict(residual=z(3, 6))), ((x[0], w, out), {}), ((z(1, 16).expand(4, 16), w, out), {}),
                 ((x, w, z(4, 6, dtype=torch.int32)), {}), ((x, z(6, 32)[:, ::2], out), {})):
        refuses(msi.linear, *a, **k)
    data, scales, mass = z(3, 2, 2, 64, 64, dtype=torch.uint8), z(3, 2, 2, dtype=torch.float32), z(3, 2, 64, dtype=torch.float32)
    refuses(msi.KvCache, data, scales, mass, "fp4")
    refuses(msi.KvCache, data.int(), scales)
    refuses(msi.KvCache, data[:, :, :1], scales)
    refuses(msi.KvCache, data, scales[:2])
    refuses(msi.KvCache, data, scales, mass[..., :32])
    cache = msi.KvCache(data, scales, mass)
    i32 = lambda *s: z(*s, dtype=torch.int32)  # noqa: E731
    refuses(msi.KvSeqs, i32(2), i32(2))
    refuses(msi.KvSeqs, i32(2, 3), i32(3))
    refuses(msi.KvSeqs, i32(2, 3).long(), i32(2))
    refuses(msi.KvSeqs, i32(2, 3), i32(2), i32(2))
    refuses(msi.KvSeqs, i32(2, 3), i32(2), i32(3), n_rows=-1)
    s = msi.KvSeqs(i32(2, 3), i32(2), i32(3), n_rows=4, max_rows=3)
    for f in (msi.kv_append, msi.kv_read):
        refuses(f, cache, s, z(4, 2, 64), z(3, 2, 64))
        refuses(f, cache, s, z(4, 2, 64).float(), z(4, 2, 64))
        refuses(f, cache, s, z(4, 2, 64), z(4, 64, 2).transpose(1, 2))
        refuses(f, cache, s, z(4, 2, 64), z(1, 2, 64).expand(4, 2, 64))
        refuses(f, cache, s, z(4, 2, 64), z(4, 2, 64), status=z(1))
    refuses(msi.kv_attention, cache, s, z(4, 4, 64), z(4, 2, 64), 1.0)
    refuses(msi.kv_attention, cache, s, z(4, 256), z(4, 4, 64), 1.0)
    refuses(msi.kv_attention, cache, s, z(4, 4, 64), z(4, 4, 64), 1.0, mass_rows=-1)
    refuses(msi.kv_attention, cache, s, z(4, 4, 64), z(4, 4, 64), 1.0, workspace=z(100))
    refuses(msi.kv_evict, cache, s, i32(3, 2), i32(2), i32(2, 2, 100), budget=100)
    refuses(msi.kv_evict, cache, s, i32(2, 2), i32(3), i32(2, 2, 100), budget=100)
    refuses(msi.kv_evict, cache, s, i32(2, 2), i32(2), i32(2, 2, 99), budget=100)
    refuses(msi.kv_evict, cache, s, i32(2, 2), i32(2), i32(2, 2, 100), budget=100, sinks=-1)
    # host tensors that are right in everything else
    for f, a, k in ((msi.linear, (x, w, out), {}), (msi.kv_append, (cache, s, z(4, 2, 64), z(4, 2, 64)), {}),
                    (msi.kv_read, (cache, s, z(4, 2, 64), z(4, 2, 64)), {}),
                    (msi.kv_attention, (cache, s, z(4, 4, 64), z(4, 4, 64), 1.0), {}),
                    (msi.kv_evict, (cache, s, i32(2, 2), i32(2), i32(2, 2, 100)), dict(budget=100))):
        with pytest.raises(msi.MsiError, match="HIP device"):
            f(*a, **k)
    with pytest.raises(AttributeError):
        msi.no_such_name
