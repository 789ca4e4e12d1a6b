"""Append with rotation.  The queries against 64 bits; the cache byte for byte against the append's oracle, given the keys
that the operator itself rotates when they come as queries; positions far away, negative and of several axes, both orders
of pairs, partial heads, ragged sequences, refused and left-out rows, in place, strided, captured.

Bound of a rotated element: half a step of bf16 (2^-8 of it), and 2^-21 (|a| + |b|) for the two products' and the sum's
roundings, the sine and cosine (2^-23 each) and the angle (2^-33 turns)."""
import fractions
import math

import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup, bf16
from _kv_oracle import B

pytestmark = pytest.mark.gpu

PI2 = fractions.Fraction(6283185307179586476925286766559005768394338798750, 10 ** 48)


def frequencies(rot, theta=10000.0):
    return [theta ** (-2 * i / rot) for i in range(rot // 2)]


def rotate(x, pos, freq, axis, interleaved):
    """x [n, heads, D], pos [axes, n]: (rotated, |a| + |b| of every element's pair), angles reduced in exact arithmetic."""
    half = len(freq)
    n = x.shape[0]
    turn = np.empty((n, half))
    for i, f in enumerate(freq):
        t = fractions.Fraction(f) / PI2
        a = 0 if axis is None else axis[i]
        turn[:, i] = [float(int(p) * t % 1) for p in pos[a]]
    c, s = np.cos(2 * math.pi * turn)[:, None], np.sin(2 * math.pi * turn)[:, None]
    i = np.arange(half)
    one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    out, size = x.copy(), np.abs(x)
    a, b = x[..., one], x[..., two]
    out[..., one], out[..., two] = a * c - b * s, b * c + a * s
    size[..., one] = size[..., two] = np.abs(a) + np.abs(b)
    return out, size


def close(got, want, size):
    return np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * size + 1e-30)


def _check(s, rot, Hq, axis=None, interleaved=False, far=0, inplace=False, pos=None, stride=0, theta=10000.0, status=0):
    import torch
    import paper_2608_23805_amd as msi
    n, H, D = s.cu[-1], s.H, s.D
    q, qh = s.rows(Hq + 2 * H + stride)
    axes = 1 if axis is None else max(axis) + 1
    if pos is None:
        pos = s.g.integers(0, 1 << 15, (axes, n)) + far
    r = msi.KvRotary(frequencies(rot, theta), axes=axis, interleaved=interleaved)
    p = torch.from_numpy(np.asarray(pos, dtype=np.int32)).cuda()
    k, v = q[:, Hq:Hq + H], q[:, Hq + H:Hq + 2 * H]
    # the keys as queries, into an array of its own
    seqs = s.seqs
    kr = torch.full((n, H, D), 3.0, dtype=torch.bfloat16, device="cuda")
    scratch = msi.KvCache(s.data.clone(), s.scales.clone(), None, s.fmt)
    msi.kv_append_rotary(scratch, seqs, r, p, k, kr, k, v)
    qo = q[:, :Hq] if inplace else torch.full((n, Hq, D), 3.0, dtype=torch.bfloat16, device="cuda")
    msi.kv_append_rotary(s.cache, seqs, r, p if axes > 1 else p[0], q[:, :Hq], qo, k, v, status=s.status,
                         stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for got, x in ((qo, qh[:, :Hq]), (kr, qh[:, Hq:Hq + H])):
        want, size = rotate(x, pos, frequencies(rot, theta), axis, interleaved)
        assert close(got.double().cpu().numpy(), want, size)
        if rot < D:
            assert np.array_equal(got.double().cpu().numpy()[..., rot:], x[..., rot:])
    if inplace:
        assert np.array_equal(q[:, Hq:].double().cpu().numpy(), qh[:, Hq:])
    want_status = s.host.append(s.table, s.lens, s.cu, kr.double().cpu().numpy(), qh[:, Hq + H:Hq + 2 * H])
    data, scales, mass, got_status = s.device_state()
    assert got_status == want_status == status
    assert np.array_equal(scales, s.host.scales.astype(np.float32))
    if mass is not None:
        assert np.array_equal(mass, s.host.mass.astype(np.float32))
    assert np.array_equal(data, s.host.data)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (128, 128), (128, 48), (256, 256), (256, 64), (256, 208)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_shapes(fmt, D, rot, interleaved):
    log(f"case rotary {fmt} D={D} rot={rot} interleaved={interleaved}")
    s = Setup(200 + D + rot, [70, 1, 129, 64, 200], [3, 1, 129, 0, 70], 2, D, fmt)
    _check(s, rot, 6, interleaved=interleaved)


@pytest.mark.parametrize("rows", [[1, 1, 1], [2, 1, 3], [17, 16, 1], [33, 64, 65], [128, 1, 127]])
@pytest.mark.parametrize("Hq,H", [(1, 1), (8, 8), (5, 1), (28, 4), (33, 3)])
def test_rows_and_heads(rows, Hq, H):
    log(f"case rotary rows={rows} heads={Hq}/{H}")
    s = Setup(300 + sum(rows) + Hq, [r + 45 * i for i, r in enumerate(rows)], rows, H, 128, "e4m3")
    _check(s, 128, Hq, inplace=True)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axis", [[0] * 5 + [1] * 3 + [2] * 8, [0, 1, 2, 3] * 4, [2] * 16, [0, 1] * 8])
def test_axes(axis, interleaved):
    log(f"case rotary axes={axis} interleaved={interleaved}")
    s = Setup(400 + sum(axis), [100, 40], [70, 9], 2, 64, "int8")
    _check(s, 32, 4, axis=axis, interleaved=interleaved)


def test_positions_of_any_size():
    """The ends of 32 bits, negative ones, frequencies of one radian and more a position."""
    log("case rotary far positions")
    s = Setup(500, [64], [64], 2, 64, "e4m3")
    pos = np.concatenate([np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 1 << 20, 1 << 24, (1 << 24) + 1]),
                          s.g.integers(-2 ** 31, 2 ** 31, 55)])[None]
    _check(s, 64, 3, pos=pos)
    s = Setup(501, [64], [64], 2, 64, "e4m3")
    _check(s, 64, 3, pos=pos, theta=1e-4)


def test_positions_are_not_the_cache_s():
    """A sequence that was cut back: its tokens' places in the cache are not their positions."""
    log("case rotary after eviction")
    s = Setup(502, [90, 300], [5, 100], 2, 128, "e4m3")
    _check(s, 128, 4, far=1 << 20, stride=3)


def test_without_queries():
    import torch
    import paper_2608_23805_amd as msi
    log("case rotary without queries")
    s, t = Setup(503, [90, 10], [5, 10], 2, 64, "e4m3"), Setup(503, [90, 10], [5, 10], 2, 64, "e4m3")
    k, _ = s.rows(2)
    r = msi.KvRotary(frequencies(64))
    p = torch.arange(15, dtype=torch.int32, device="cuda")
    kr = torch.empty_like(k)
    msi.kv_append_rotary(s.cache, s.seqs, r, p, None, None, k, k)
    msi.kv_append_rotary(t.cache, t.seqs, r, p, k, kr, k, k)
    torch.cuda.synchronize()
    assert torch.equal(s.data, t.data) and torch.equal(s.scales, t.scales)


def test_not_numbers():
    """Infinities and NaN: the pair's own elements at most, coded as the append codes them, with its status bit."""
    import torch
    import paper_2608_23805_amd as msi
    log("case rotary not numbers")
    s = Setup(504, [70], [20], 2, 64, "e4m3")
    x, xh = s.rows(4)
    x[3, 0, 5], x[7, 1, 40], x[9, 2, 0], x[2, 3, 63] = float("inf"), float("nan"), -float("inf"), float("inf")
    r = msi.KvRotary(frequencies(32))
    p = torch.arange(20, dtype=torch.int32, device="cuda") + 11
    out = torch.empty_like(x)
    msi.kv_append_rotary(s.cache, s.seqs, r, p, x, out, x[:, 2:], x[:, :2], status=s.status)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    bad = ~np.isfinite(got)
    allowed = np.zeros_like(bad)
    allowed[3, 0, [5, 21]] = allowed[7, 1, 40] = allowed[9, 2, [0, 16]] = allowed[2, 3, 63] = True
    assert not np.any(bad & ~allowed) and bad[2, 3, 63] and bad[7, 1, 40]
    want, size = rotate(np.where(np.isfinite(xh), xh, 0.0), np.arange(20)[None] + 11, frequencies(32), None, False)
    fine = ~allowed
    assert np.all((np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * size + 1e-30)[fine])
    assert s.host.append(s.table, s.lens, s.cu, got[:, 2:], x[:, :2].double().cpu().numpy()) == 2
    data, scales, _, status = s.device_state()
    assert status == 2 and np.array_equal(data, s.host.data) and np.array_equal(scales, s.host.scales.astype(np.float32))


def test_left_out_sequences_and_rows_behind():
    """A sequence that breaks a bound and rows that no sequence brings stay as they were, in the cache and in q_out."""
    import torch
    import paper_2608_23805_amd as msi
    log("case rotary left out")
    s = Setup(505, [70, 90, 30], [4, 6, 5], 2, 64, "e4m3")
    n = 20
    x, _ = bf16(s.g.standard_normal((n, 4, 64)))
    bad = torch.tensor([70, 1000, 30], dtype=torch.int32, device="cuda")
    seqs = msi.KvSeqs(s.seqs.table, bad, s.seqs.cu_rows, n_rows=n, max_rows=6, max_len=128)
    good = msi.KvSeqs(s.seqs.table, s.seqs.lens, s.seqs.cu_rows, n_rows=n, max_rows=6, max_len=128)
    r = msi.KvRotary(frequencies(64))
    p = torch.arange(n, dtype=torch.int32, device="cuda") + 5
    outs, caches = [], []
    for q in (seqs, good):
        out = torch.full_like(x, 9.0)
        c = msi.KvCache(s.data.clone(), s.scales.clone(), None, "e4m3")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        msi.kv_append_rotary(c, q, r, p, x, out, x[:, :2], x[:, 2:], status=st)
        torch.cuda.synchronize()
        assert int(st) == (4 if q is seqs else 0)
        outs.append(out)
        caches.append(c)
    assert torch.all(outs[1][15:] == 9.0) and torch.all(outs[0][4:10] == 9.0)
    assert torch.equal(outs[0][:4], outs[1][:4]) and torch.equal(outs[0][10:], outs[1][10:])
    pages = [int(v) for v in s.table[1] if v >= 0]
    assert torch.equal(caches[0].data[pages], s.data[pages])
    rest = [int(v) for i in (0, 2) for v in s.table[i] if v >= 0]
    assert torch.equal(caches[0].data[rest], caches[1].data[rest])


def test_bad_pages():
    """Nothing is written for a page outside the pool; the queries of its rows are rotated all the same."""
    import torch
    import paper_2608_23805_amd as msi
    log("case rotary bad pages")
    s = Setup(506, [130], [100], 2, 64, "int8")
    s.table[0, 1] = len(s.host.data)
    s.seqs = s.make_seqs(s.table, s.lens, s.cu)
    x, xh = s.rows(4)
    out = torch.empty_like(x)
    r = msi.KvRotary(frequencies(64))
    pos = np.arange(100)[None]
    msi.kv_append_rotary(s.cache, s.seqs, r, torch.from_numpy(pos.astype(np.int32)).cuda(), x, out, x[:, 2:], x[:, :2], status=s.status)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    want, size = rotate(xh, pos, frequencies(64), None, False)
    assert close(got, want, size)
    assert s.host.append(s.table, s.lens, s.cu, got[:, 2:], xh[:, :2]) == 1
    data, scales, _, status = s.device_state()
    assert status == 1 and np.array_equal(data, s.host.data) and np.array_equal(scales, s.host.scales.astype(np.float32))


def test_many_sequences():
    log("case rotary many sequences")
    g = np.random.default_rng(507)
    lens = [int(v) for v in g.integers(1, 200, 300)]
    rows = [int(min(n, v)) for n, v in zip(lens, g.integers(0, 6, 300))]
    s = Setup(508, lens, rows, 1, 64, "e4m3")
    _check(s, 64, 2, interleaved=True)


def test_captured():
    """A captured append, replayed with other positions and lengths between the replays."""
    import torch
    import paper_2608_23805_amd as msi
    log("case rotary captured")
    s = Setup(509, [80, 20], [1, 1], 2, 128, "e4m3", extra_blocks=1)
    x, _ = s.rows(8)
    out = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device="cuda")
    lens, p = s.seqs.lens, torch.tensor([79, 19], dtype=torch.int32, device="cuda")
    seqs = msi.KvSeqs(s.seqs.table, lens, s.seqs.cu_rows, n_rows=2, max_rows=1, max_len=192)
    r = msi.KvRotary(frequencies(128))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        msi.kv_append_rotary(s.cache, seqs, r, p, x[:, :4], out, x[:, 4:6], x[:, 6:], stream=torch.cuda.current_stream())
    twin = msi.KvCache(s.data.clone(), s.scales.clone(), None, "e4m3")
    for _ in range(4):
        want = torch.zeros_like(out)
        msi.kv_append_rotary(twin, seqs, r, p, x[:, :4], want, x[:, 4:6], x[:, 6:])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(s.data, twin.data) and torch.equal(s.scales, twin.scales)
        lens += 1
        p += 3
        x.mul_(1.25)
