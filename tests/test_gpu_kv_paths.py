"""Attention over the paged cache: batches and lengths that reach what the other tests' sizes do not (more than 64
sequences, lists of pages that are read again, weights by four blocks at once), values at the ends of the range, and
what a call leaves alone.  Bounds as in the oracle."""
import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup
from _kv_oracle import Cache
from test_gpu_kv_attention import _check

pytestmark = pytest.mark.gpu


def _lens(g, n, most):
    """Empty, one-token, short and cut sequences in turn."""
    return [int(v) for v in np.where(np.arange(n) % 5 == 0, 0, np.where(np.arange(n) % 7 == 1, 1, g.integers(1, most, n)))]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("S", [64, 65, 130])
@pytest.mark.parametrize("rows", [1, 12])
def test_units_of_many_sequences(fmt, S, rows):
    """Units found past the first 64 and 128 sequences; the last sequence is the longest one."""
    log(f"case many sequences {fmt} S={S} rows={rows}")
    g = np.random.default_rng([81, S])
    lens = _lens(g, S, 600)
    lens[0], lens[-1] = 1100, 1500
    n = [min(rows, max(x, 1)) for x in lens]                   # (a row without tokens comes out zero)
    s = Setup(S + rows, lens, n, 1, 64, fmt)
    _check(s, s.seqs, s.table, s.lens, s.cu, 4)
    _check(s, s.seqs, s.table, s.lens, s.cu, 4, mass_rows=2, decay=0.5)


@pytest.mark.parametrize("bad", [False, True])
def test_page_lists_of_many_rows(bad):
    """A sequence of 134 blocks that is not cut: the lists of 64 pages are made three times, a bad page in each."""
    log(f"case page lists, many rows, bad={bad}")
    lens, rows = [8530] + [3] * 51, [40] + [1] * 51
    s = Setup(82, lens, rows, 1, 64, "int8")
    table = s.table.copy()
    if bad:
        for b in (10, 63, 64, 66, 100, 127, 128, 129, 133):
            table[0, b] = 10 ** 6 + b
    seqs = s.make_seqs(table, s.lens, s.cu)
    _check(s, seqs, table, s.lens, s.cu, 16, status=int(bad))
    _check(s, seqs, table, s.lens, s.cu, 16, mass_rows=17, decay=1.0, status=int(bad))


@pytest.mark.parametrize("bad", [False, True])
def test_page_lists_of_few_rows(bad):
    """A sequence of 258 blocks among so many that none is cut: a wavefront's list of 64 pages is made twice."""
    log(f"case page lists, few rows, bad={bad}")
    lens, rows = [16500] + [1] * 1023, [1] * 1024
    s = Setup(83, lens, rows, 8, 64, "e4m3")
    table = s.table.copy()
    if bad:
        for b in (3, 255, 256, 257):
            table[0, b] = -2
    seqs = s.make_seqs(table, s.lens, s.cu)
    _check(s, seqs, table, s.lens, s.cu, 1, status=int(bad))
    _check(s, seqs, table, s.lens, s.cu, 1, mass_rows=1, decay=0.25, status=int(bad))


@pytest.mark.parametrize("D", [64, 256])
def test_weights_by_four_blocks(D):
    """So many blocks that the four wavefronts of a workgroup take one each; sequences that end inside such a group."""
    log(f"case weights, four blocks D={D}")
    s = Setup(84, [8300, 700, 65, 0, 300], [40, 33, 1, 0, 5], 2, D, "e4m3" if D == 64 else "int8")
    for mass_rows, decay in ((33, 1.0), (1, 0.0), (1000, 0.5)):
        _check(s, s.seqs, s.table, s.lens, s.cu, 2, mass_rows=mass_rows, decay=decay)


@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("lens,rows", [([70, 5, 0], [1, 1, 1]), ([70, 5, 0], [40, 3, 0]), ([900, 130], [1, 1]), ([900, 130], [40, 1])])
def test_weights_of_other_tokens_stay(lens, rows, decay):
    """Weights past a sequence's last token and in pages that no sequence of the call holds keep their bits."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case weights that stay {lens} {rows} {decay}")
    s = Setup(85 + sum(rows), lens, rows, 2, 64, "int8", spare=3)
    live = np.zeros(s.host.mass.shape, dtype=bool)
    for i, n in enumerate(lens):
        for t in range(n):
            live[s.table[i, t // 64], :, t % 64] = True
    s.host.mass[~live & (np.arange(64) % 3 == 0)] = np.nan     # bits that arithmetic would not keep
    s.mass.copy_(torch.from_numpy(s.host.mass))
    q, _ = s.rows(4, 0.5)
    out = torch.empty((s.cu[-1], 4, 64), dtype=torch.bfloat16, device="cuda")
    ws = msi.kv_attention_workspace(s.cache, s.seqs, 4, 2)
    msi.kv_attention(s.cache, s.seqs, q, out, 0.125, mass_rows=2, mass_decay=decay, workspace=ws)
    torch.cuda.synchronize()
    got = s.mass.cpu().numpy()
    assert np.array_equal(got.view(np.uint32)[~live], s.host.mass.view(np.uint32)[~live])
    if decay != 1.0:
        assert np.all(got[live] != s.host.mass[live])          # (the others moved)


@pytest.mark.parametrize("fmt,scale", [("e4m3", 2.0 ** 119), ("int8", 2.0 ** 121)])
@pytest.mark.parametrize("lens,rows", [([70, 200], [1, 3]), ([900], [1]), ([70, 300], [40, 33]), ([900], [40])])
def test_values_at_the_ends_of_the_range(fmt, scale, lens, rows):
    """V up to the largest bf16 (every finite value is accepted by the append) in blocks beside ones whose V is as
    small as scales go: results are finite and right, one unit or several, few rows and many."""
    import torch
    log(f"case V at the range's ends {fmt} {lens} {rows}")
    s = Setup(86 + sum(rows), lens, rows, 1, 64, fmt)
    P = s.host.data.shape[0]
    if fmt == "e4m3":
        s.host.data[:, :, 1] = s.g.integers(0x70, 0x7F, s.host.data[:, :, 1].shape).astype(np.uint8)      # 128 .. 448
    else:
        s.host.data[:, :, 1] = s.g.integers(64, 128, s.host.data[:, :, 1].shape).astype(np.uint8)
    s.host.scales[..., 1] = scale
    small = [int(s.table[i, b]) for i in range(len(lens)) for b in range(1, -(-lens[i] // 64), 3)]
    s.host.scales[small, :, 1] = 2.0 ** -64
    assert P > len(small)
    s.data.copy_(torch.from_numpy(s.host.data))
    s.scales.copy_(torch.from_numpy(s.host.scales))
    out = _check(s, s.seqs, s.table, s.lens, s.cu, 4)
    assert torch.isfinite(out).all()
    _check(s, s.seqs, s.table, s.lens, s.cu, 4, mass_rows=50, decay=0.5)
    # and with the small ones alone
    s.host.scales[..., 1] = 2.0 ** -64
    s.scales.copy_(torch.from_numpy(s.host.scales))
    _check(s, s.seqs, s.table, s.lens, s.cu, 4)


@pytest.mark.parametrize("rows", [1, 40])
def test_large_values_behind_others(rows):
    """Blocks of ordinary and of vanishing V, then, past the first 64 blocks, some whose largest elements are at the
    range's end while most of their elements are zero: the other elements' results are those of the ordinary blocks."""
    import torch
    log(f"case large V behind others rows={rows}")
    s = Setup(89 + rows, [8530] + [3] * 51, [rows] + [1] * 51, 1, 64, "int8")
    at = [int(p) for p in s.table[0, :134]]
    for b in (70, 100, 131):
        s.host.data[at[b], :, 1, :, 8:] = 0
        s.host.scales[at[b], :, 1] = 2.0 ** 121
    for b in (0, 5, 63, 64, 99, 101, 130, 133):
        s.host.data[at[b], :, 1] = 0
        s.host.scales[at[b], :, 1] = 2.0 ** -64
    s.data.copy_(torch.from_numpy(s.host.data))
    s.scales.copy_(torch.from_numpy(s.host.scales))
    _check(s, s.seqs, s.table, s.lens, s.cu, 16)
    _check(s, s.seqs, s.table, s.lens, s.cu, 16, mass_rows=5, decay=0.5)


def test_a_chunk_beside_single_tokens():
    """One prompt chunk and single tokens on long and short caches in one call, every kind of cut."""
    log("case chunk beside single tokens")
    lens = [700] + [int(v) for v in np.random.default_rng(87).integers(1, 900, 20)]
    s = Setup(87, lens, [150] + [1] * 20, 2, 128, "e4m3")
    _check(s, s.seqs, s.table, s.lens, s.cu, 4)
    _check(s, s.seqs, s.table, s.lens, s.cu, 4, mass_rows=1, decay=1.0)


def test_eviction_leaves_a_broken_sequence_out():
    """A sequence whose length breaks its bound keeps its entries of new_lens and keep, and its pages; the others are cut."""
    import torch
    import paper_2608_23805_amd as msi
    from _kv_oracle import evict
    log("case eviction, broken length")
    for wrong in (201, -1, 2 ** 31 - 1):
        s = Setup(88, [200, 150, 90], [0, 0, 0], 2, 64, "e4m3", dst_lens=[100, 100, 90])
        seqs = s.make_seqs(s.table, s.lens, s.cu, max_len=200)
        seqs.lens[1] = wrong
        keep = torch.full((3, 2, 100), 77, dtype=torch.int32, device="cuda")
        new = torch.full((3,), 77, dtype=torch.int32, device="cuda")
        msi.kv_evict(s.cache, seqs, torch.from_numpy(s.dst).cuda(), new, keep, budget=100, sinks=4, recent=10, status=s.status)
        host = Cache(s.host.data, s.host.scales, s.host.mass, "e4m3")
        want = evict(host, [s.table[0], s.table[2]], [200, 90], [s.dst[0], s.dst[2]], 100, 4, 10)
        data, scales, mass, st = s.device_state()
        assert st == 4 and new.tolist() == [100, 77, 90]
        k = keep.cpu().numpy()
        assert np.array_equal(k[0], want[0]) and np.array_equal(k[2], want[1]) and np.all(k[1] == 77)
        assert np.array_equal(data, host.data) and np.array_equal(scales, host.scales) and np.array_equal(mass, host.mass)
