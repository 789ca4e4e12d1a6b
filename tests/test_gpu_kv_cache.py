"""The paged 8-bit cache against 64 bits: what append, read and evict leave is compared
byte for byte (codes, scales, weights), so no tolerance enters."""
import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup, bf16
from _kv_oracle import B, evict

pytestmark = pytest.mark.gpu


def _same(s, status=0):
    data, scales, mass, st = s.device_state()
    assert np.array_equal(scales, s.host.scales.astype(np.float32))
    assert np.array_equal(data, s.host.data)
    assert mass is None or np.array_equal(mass.view(np.uint32), s.host.mass.astype(np.float32).view(np.uint32))
    assert st == status


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("H,D", [(1, 64), (3, 128), (2, 256)])
@pytest.mark.parametrize("lens,rows", [
    ([1], [1]), ([64], [1]), ([65], [1]), ([64], [64]), ([127], [64]), ([129], [66]), ([200], [200]),
    ([5, 0, 130, 64, 77], [1, 0, 130, 3, 20]), ([300, 2], [0, 2]),
])
def test_append(fmt, H, D, lens, rows):
    import torch
    import paper_2608_23805_amd as msi
    log(f"case append {fmt} H={H} D={D} lens={lens} rows={rows}")
    s = Setup(len(lens) * 1000 + sum(lens), lens, rows, H, D, fmt)
    # magnitudes that keep, raise and lower the scale the block had
    size = np.exp2(s.g.integers(-6, 7, (s.cu[-1], H, 1)).astype(np.float64))
    k, kh = bf16(s.g.standard_normal((s.cu[-1], H, D)) * size)
    v, vh = bf16(s.g.standard_normal((s.cu[-1], H, D)) * size[::-1])
    msi.kv_append(s.cache, s.seqs, k, v, status=s.status, stream=torch.cuda.current_stream())
    s.host.append(s.table, s.lens, s.cu, kh, vh)
    _same(s)
    # and again: the scales have grown already, so nothing changes
    msi.kv_append(s.cache, s.seqs, k, v, status=s.status, stream=torch.cuda.current_stream())
    _same(s)
    ko, vo = (torch.zeros((s.cu[-1], H, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    msi.kv_read(s.cache, s.seqs, ko, vo, status=s.status, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for i, (n, a) in enumerate(zip(lens, s.cu)):
        r = s.cu[i + 1] - a
        if r:
            kv = s.host.sequence(s.table[i], n)[:, :, n - r:]
            assert np.array_equal(ko[a:a + r].double().cpu().numpy(), kv[0].transpose(1, 0, 2))
            assert np.array_equal(vo[a:a + r].double().cpu().numpy(), kv[1].transpose(1, 0, 2))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_one_by_one(fmt):
    """A block filled token by token, with growing magnitudes: its codes are rounded again at every growth."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case append one by one {fmt}")
    s = Setup(9, [70], [1], 2, 64, fmt, mass=False)
    for n in range(1, 71):
        seqs = s.make_seqs(s.table, [n], [0, 1])
        k, kh = bf16(s.g.standard_normal((1, 2, 64)) * 1.07 ** n)
        v, vh = bf16(s.g.standard_normal((1, 2, 64)) * 1.3 ** -n)
        msi.kv_append(s.cache, seqs, k, v, status=s.status)
        s.host.append(s.table, [n], [0, 1], kh, vh)
    _same(s)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_rounding_and_special_values(fmt):
    """Every bf16 magnitude between 2^-12 and 2^9 against a block maximum that sets the scale to 1, zeros of both
    signs, subnormals, infinities and NaN."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case rounding {fmt}")
    top = 448.0 if fmt == "e4m3" else 127.0
    bits = np.arange(0x3980, 0x4400, dtype=np.uint16)
    vals = (bits.astype(np.uint32) << 16).view(np.float32)
    vals = vals[vals <= top]
    vals = np.concatenate([vals, -vals, [0.0, -0.0, 1e-40, -1e-40, 3e-39]]).astype(np.float32)
    x = np.zeros((64, 1, 128), dtype=np.float32)
    assert len(vals) <= 63 * 128
    x.reshape(-1)[:len(vals)] = vals
    x[63, 0, 0] = top
    s = Setup(10, [64], [64], 1, 128, fmt)
    k, kh = bf16(x)
    y = x.copy()
    y[5, 0, 3], y[5, 0, 4], y[6, 0, 0] = np.inf, -np.inf, np.nan
    v, vh = bf16(y)
    msi.kv_append(s.cache, s.seqs, k, v, status=s.status)
    assert s.host.append(s.table, s.lens, s.cu, kh, vh) == 2
    _same(s, status=2)
    assert float(s.scales[int(s.table[0, 0]), 0, 0]) == 1.0
    codes = s.data[int(s.table[0, 0]), 0, 1, 6, 0].item()
    assert codes == 0


def test_scale_bounds():
    """All zeros, the smallest and the largest bf16: scales stay finite powers of two, at least 2^-64."""
    import torch
    import paper_2608_23805_amd as msi
    log("case scale bounds")
    for fmt in ("e4m3", "int8"):
        for big in (0.0, 1e-45, 2.0 ** -64, 1e-30, 3.38e38):
            s = Setup(11, [3], [3], 1, 64, fmt)
            k, kh = bf16(np.full((3, 1, 64), big))
            msi.kv_append(s.cache, s.seqs, k, k, status=s.status)
            s.host.append(s.table, s.lens, s.cu, kh, kh)
            _same(s)


def test_strided_rows_and_untouched_neighbours():
    """K and V as views of one projection's rows; pages of other sequences and bytes past the last token stay."""
    import torch
    import paper_2608_23805_amd as msi
    log("case append strided")
    s = Setup(12, [70, 3, 64], [10, 3, 5], 2, 128, "e4m3", spare=5)
    qkv, qh = bf16(s.g.standard_normal((18, 7 * 2 * 128)))
    w = qkv.view(18, 7, 2, 128)
    msi.kv_append(s.cache, s.seqs, w[:, 4], w[:, 6], status=s.status)
    h = qh.reshape(18, 7, 2, 128)
    s.host.append(s.table, s.lens, s.cu, h[:, 4], h[:, 6])
    _same(s)


def test_bad_pages_and_lengths():
    """Bad pages and lengths write nothing, raise their bits and leave the other sequences right."""
    import torch
    import paper_2608_23805_amd as msi
    log("case bad pages")
    s = Setup(13, [70, 130, 20], [70, 130, 20], 2, 64, "int8")
    k, kh = s.rows(2)
    v, vh = s.rows(2)
    table = s.table.copy()
    table[1, 1] = 10 ** 6
    table[2, 0] = -5
    seqs = s.make_seqs(table, s.lens, s.cu)
    msi.kv_append(s.cache, seqs, k, v, status=s.status)
    assert s.host.append(table, s.lens, s.cu, kh, vh) == 1
    _same(s, status=1)
    ko, vo = (torch.full((220, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    msi.kv_read(s.cache, seqs, ko, vo, status=s.status)
    torch.cuda.synchronize()
    assert torch.all(ko[70 + 64:70 + 128] == 0) and torch.all(ko[200:] == 0) and torch.all(ko[70 + 128:200] != 9.0)
    # lengths past the bound, negative, and fewer tokens than rows: those sequences are left out
    s.status.zero_()
    bad = s.make_seqs(s.table, [71, -1, 19], s.cu, max_len=70)
    before = s.device_state()
    msi.kv_append(s.cache, bad, k, v, status=s.status)
    after = s.device_state()
    assert np.array_equal(before[0], after[0]) and after[3] == 4
    s.status.zero_()
    bad = s.make_seqs(s.table, s.lens, [0, 70, 60, 220], max_rows=220)       # offsets that fall
    bad.c.max_rows = 100
    ko.fill_(9.0)
    msi.kv_read(s.cache, bad, ko, vo, status=s.status)
    torch.cuda.synchronize()
    assert int(s.status) == 4 and torch.all(ko[70:] == 9.0) and torch.all(ko[:70] != 9.0)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("H,D", [(2, 64), (3, 128), (1, 256)])
@pytest.mark.parametrize("lens,budget,sinks,recent", [
    ([1], 1, 0, 0), ([1, 0, 5], 4, 1, 1), ([64, 65, 63], 64, 0, 0), ([200, 130, 64], 100, 4, 32), ([300], 65, 0, 65),
    ([300, 7], 1, 0, 0), ([1100, 5000], 777, 4, 100), ([130], 129, 0, 0), ([260], 200, 200, 0),
])
def test_evict(fmt, H, D, lens, budget, sinks, recent):
    import torch
    import paper_2608_23805_amd as msi
    log(f"case evict {fmt} H={H} D={D} lens={lens} {budget}/{sinks}/{recent}")
    s = Setup(sum(lens) + budget, lens, [0] * len(lens), H, D, fmt, dst_lens=[min(n, budget) for n in lens])
    # ties: many weights are equal, some zero of either sign
    m = np.round(s.host.mass * 4) / 4
    m[..., ::7] = 0.0
    m[..., ::14] = -0.0
    s.host.mass[:] = m
    s.mass.copy_(torch.from_numpy(s.host.mass))
    keep = torch.full((len(lens), H, budget), 99, dtype=torch.int32, device="cuda")
    new = torch.full((len(lens),), 99, dtype=torch.int32, device="cuda")
    msi.kv_evict(s.cache, s.seqs, torch.from_numpy(s.dst).cuda(), new, keep, budget=budget, sinks=sinks, recent=recent,
                 status=s.status, stream=torch.cuda.current_stream())
    want = evict(s.host, s.table, s.lens, s.dst, budget, sinks, recent)
    torch.cuda.synchronize()
    assert np.array_equal(keep.cpu().numpy(), want)
    assert new.tolist() == [min(n, budget) for n in lens]
    _same(s)


@pytest.mark.parametrize("length", [4095, 4097, 16383, 16385, 65536, 70000, 140000])
@pytest.mark.parametrize("kind", ["spread", "equal", "special"])
def test_evict_long(length, kind):
    """Lengths at the sides of every selection form, and past the longest one that keeps its keys in registers."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case evict long {length} {kind}")
    budget = length // 3
    s = Setup(length, [length], [0], 1, 64, "int8", dst_lens=[budget])
    if kind == "equal":
        s.mass.fill_(0.25)
    elif kind == "special":
        flat = s.mass.view(-1)
        flat[::3] = float("nan")
        flat[1::5] = float("inf")
        flat[2::11] = -float("inf")
        flat[4::13] = -1.5
    m = s.mass.cpu().numpy()
    keep = torch.full((1, 1, budget), 99, dtype=torch.int32, device="cuda")
    new = torch.zeros(1, dtype=torch.int32, device="cuda")
    msi.kv_evict(s.cache, s.seqs, torch.from_numpy(s.dst).cuda(), new, keep, budget=budget, sinks=4, recent=100,
                 status=s.status)
    torch.cuda.synchronize()
    pos = np.arange(length)
    w = m[s.table[0][pos // B], 0, pos % B].astype(np.float64)
    order = np.lexsort((pos, -np.where(np.isnan(w), -np.inf, w), np.isnan(w)))
    fixed = (pos < 4) | (pos >= length - 100)
    order = order[~fixed[order]][:budget - 104]
    want = np.sort(np.concatenate([pos[fixed], order]))
    assert np.array_equal(keep.cpu().numpy()[0, 0], want) and int(new) == budget and int(s.status) == 0


def test_evict_bad_pages():
    import torch
    import paper_2608_23805_amd as msi
    log("case evict bad pages")
    s = Setup(14, [200, 150], [0, 0], 2, 64, "e4m3", dst_lens=[100, 100])
    table, dst = s.table.copy(), s.dst.copy()
    table[0, 1] = 10 ** 6
    dst[1, 0] = -1
    seqs = s.make_seqs(table, s.lens, s.cu)
    keep = torch.zeros((2, 2, 100), dtype=torch.int32, device="cuda")
    new = torch.zeros(2, dtype=torch.int32, device="cuda")
    before = s.device_state()
    msi.kv_evict(s.cache, seqs, torch.from_numpy(dst).cuda(), new, keep, budget=100, status=s.status)
    data, scales, mass, st = s.device_state()
    assert st == 1 and new.tolist() == [100, 100]
    k = keep[0].cpu().numpy()
    assert not np.any((k >= 64) & (k < 128)) and np.all(np.diff(k) > 0)         # its tokens go first
    written = {int(p) for p in s.dst.reshape(-1) if p >= 0} - {int(s.dst[1, 0])}
    untouched = [p for p in range(data.shape[0]) if p not in written]
    assert np.array_equal(data[untouched], before[0][untouched])


def test_evict_bad_page_of_a_short_sequence():
    """A sequence within its budget is copied whole: a bad page of it is reported and its tokens become zeros."""
    import torch
    import paper_2608_23805_amd as msi
    log("case evict bad page, short sequence")
    s = Setup(15, [100], [0], 2, 64, "int8", dst_lens=[100])
    table = s.table.copy()
    table[0, 1] = s.data.shape[0]
    seqs = s.make_seqs(table, s.lens, s.cu)
    keep = torch.zeros((1, 2, 128), dtype=torch.int32, device="cuda")
    new = torch.zeros(1, dtype=torch.int32, device="cuda")
    msi.kv_evict(s.cache, seqs, torch.from_numpy(s.dst).cuda(), new, keep, budget=128, status=s.status)
    data, _, mass, st = s.device_state()
    want = np.concatenate([np.arange(100), np.full(28, -1)])
    assert st == 1 and new.tolist() == [100] and np.all(keep.cpu().numpy() == want)
    assert not data[s.dst[0, 1], :, :, :36].any() and not mass[s.dst[0, 1], :, :36].any()
    assert np.array_equal(mass[s.dst[0, 0]], s.host.mass[table[0, 0]])


def test_evict_captured():
    """An eviction captured once and replayed on changing weights and lengths, eager work in between."""
    import torch
    import paper_2608_23805_amd as msi
    log("case evict graph")
    s = Setup(16, [500, 90], [0, 0], 2, 128, "e4m3", dst_lens=[100, 100])
    keep = torch.zeros((2, 2, 100), dtype=torch.int32, device="cuda")
    new = torch.zeros(2, dtype=torch.int32, device="cuda")
    dst = torch.from_numpy(s.dst).cuda()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        msi.kv_evict(s.cache, s.seqs, dst, new, keep, budget=100, sinks=2, recent=8, status=s.status,
                     stream=torch.cuda.current_stream())
    for k in range(4):
        s.lens = [500 - 37 * k, 90 - k]
        s.seqs.lens.copy_(torch.tensor(s.lens))
        m = np.roll(s.host.mass, 17, axis=-1)
        s.host.mass[:] = m
        s.mass.copy_(torch.from_numpy(m))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = evict(s.host, s.table, s.lens, s.dst, 100, 2, 8)
        assert np.array_equal(keep.cpu().numpy(), want) and new.tolist() == [min(n, 100) for n in s.lens]
        _same(s)
