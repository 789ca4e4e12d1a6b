"""Attention over the paged 8-bit cache against 64 bits (bounds derived in the oracle)."""
import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup, bf16
from _kv_oracle import attention

pytestmark = pytest.mark.gpu


def _check(s, seqs, table, lens, cu, G, mass_rows=0, decay=1.0, scale=None, q=None, status=0):
    import torch
    import paper_2608_23805_amd as msi
    q, qh = s.rows(s.H * G, 0.5) if q is None else q
    scale = s.D ** -0.5 if scale is None else scale
    out = torch.full((cu[-1] + 2, s.H * G, s.D), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = msi.kv_attention_workspace(s.cache, seqs, s.H * G, mass_rows)
    ws.fill_(255)                                              # NaN: nothing in it may count
    msi.kv_attention(s.cache, seqs, q, out[:cu[-1]], scale, mass_rows=mass_rows, mass_decay=decay, workspace=ws,
                     status=s.status, stream=torch.cuda.current_stream())
    want, tol, mass = attention(s.host, table, lens, cu, qh, np.float64(np.float32(scale)), G, mass_rows, decay)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got[:cu[-1]] - want) <= tol), float(np.max(np.abs(got[:cu[-1]] - want) / tol))
    assert np.all(got[cu[-1]:] == 5.0)
    m = s.mass.cpu().numpy() if s.mass is not None else None
    if mass_rows:
        # probabilities to 2^-16 (see the bound of the outputs), each sum of up to G * rows of them
        live = np.abs(mass - s.host.mass) > 0
        assert np.all(np.abs(m - mass) <= 2.0 ** -16 * np.abs(mass) + 2.0 ** -22 * np.abs(s.host.mass) + 1e-12)
        assert np.array_equal(m[~live & (mass == s.host.mass)], s.host.mass[~live & (mass == s.host.mass)].astype(np.float32)) or decay
        s.host.mass[:] = m
    elif m is not None:
        assert np.array_equal(m, s.host.mass)
    assert int(s.status) == status
    return out


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("H,G,D", [(2, 1, 64), (1, 8, 128), (2, 5, 64), (1, 16, 256), (3, 7, 128), (2, 2, 256)])
@pytest.mark.parametrize("lens,rows", [
    ([1], [1]), ([64], [1]), ([65], [1]), ([0, 3, 200], [1, 1, 1]), ([700, 64, 1, 333], [1, 1, 1, 1]),
    ([130, 5, 64], [3, 5, 2]), ([2100], [1]),
])
def test_few_rows(fmt, H, G, D, lens, rows):
    log(f"case few rows {fmt} H={H} G={G} D={D} lens={lens} rows={rows}")
    s = Setup(sum(lens), lens, rows, H, D, fmt)
    _check(s, s.seqs, s.table, s.lens, s.cu, G)
    _check(s, s.seqs, s.table, s.lens, s.cu, G, mass_rows=1, decay=0.875)
    _check(s, s.seqs, s.table, s.lens, s.cu, G, mass_rows=9, decay=0.0)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("H,G,D", [(2, 1, 64), (1, 8, 128), (1, 3, 256)])
@pytest.mark.parametrize("lens,rows", [
    ([40], [40]), ([64, 200], [64, 100]), ([129, 1, 0, 70], [129, 1, 0, 33]), ([900], [50]), ([50], [60]),
])
def test_many_rows(fmt, H, G, D, lens, rows):
    log(f"case many rows {fmt} H={H} G={G} D={D} lens={lens} rows={rows}")
    s = Setup(sum(lens) + 1, lens, rows, H, D, fmt)
    _check(s, s.seqs, s.table, s.lens, s.cu, G)
    _check(s, s.seqs, s.table, s.lens, s.cu, G, mass_rows=17, decay=1.0)
    _check(s, s.seqs, s.table, s.lens, s.cu, G, mass_rows=1000, decay=0.0)


@pytest.mark.parametrize("fmt,H,G,D,lens,rows", [
    ("e4m3", 2, 8, 64, [700] * 39 + [0], [1] * 40),            # few rows each, many in all
    ("int8", 2, 8, 128, [1200, 600, 3], [50, 20, 60]),         # some rows see nothing
    ("e4m3", 1, 16, 256, [1500, 64], [40, 2]),
    ("int8", 1, 3, 64, [512, 513, 577], [1, 90, 4]),           # at the side where sequences begin to be cut
    ("e4m3", 1, 2, 128, [512, 500], [1, 1]),
])
def test_cut_sequences_with_many_rows(fmt, H, G, D, lens, rows):
    """Units' results joined with rows side by side and one by one, and sequences at the length where cutting begins."""
    log(f"case cut, many rows {fmt} H={H} G={G} D={D} lens={lens[:3]} rows={rows[:3]}")
    s = Setup(sum(lens) + 2, lens, rows, H, D, fmt)
    _check(s, s.seqs, s.table, s.lens, s.cu, G)
    _check(s, s.seqs, s.table, s.lens, s.cu, G, mass_rows=40, decay=0.5)


@pytest.mark.parametrize("decay", [0.0, 0.5])
@pytest.mark.parametrize("lens,rows", [([200, 100, 0, 64], [1, 0, 0, 2]), ([900, 700], [1, 0]), ([300, 90], [40, 0])])
def test_weights_of_sequences_without_rows(lens, rows, decay):
    """A sequence of the call that brings no rows: its weights decay, nothing else happens to it."""
    log(f"case weights without rows {lens} {rows} {decay}")
    s = Setup(sum(lens) + 3, lens, rows, 2, 64, "int8")
    _check(s, s.seqs, s.table, s.lens, s.cu, 4, mass_rows=2, decay=decay)


def test_rows_without_tokens():
    """More rows than tokens: the first ones see nothing and come out zero; a padded sequence of length 0 too."""
    log("case empty rows")
    s = Setup(21, [2, 0, 65], [5, 4, 70], 2, 64, "int8")
    out = _check(s, s.seqs, s.table, s.lens, s.cu, 3, mass_rows=70, decay=1.0)
    assert not out[:3].any() and not out[5:9].any() and not out[9:14].any()
    s = Setup(22, [2, 0], [5, 4], 2, 64, "e4m3")
    out = _check(s, s.seqs, s.table, s.lens, s.cu, 3, mass_rows=5, decay=1.0)
    assert not out[:3].any() and not out[5:9].any()


def test_bytes_past_the_last_token():
    """NaN codes and wild values past a sequence's last token, and tokens that a row does not see, never count."""
    import torch
    import paper_2608_23805_amd as msi
    log("case wild bytes past the end")
    for rows in ([1, 1], [40, 3]):
        s = Setup(23, [70, 5], rows, 2, 128, "e4m3")
        for i, n in enumerate(s.lens):
            p = int(s.table[i, (n - 1) // 64])
            s.data[p, :, :, (n - 1) % 64 + 1:] = 0x7F
        _check(s, s.seqs, s.table, s.lens, s.cu, 4, mass_rows=2, decay=1.0)


@pytest.mark.parametrize("rows", [[1, 1, 1], [40, 33, 50]])
def test_bad_pages_and_lengths(rows):
    log(f"case attention bad pages rows={rows}")
    import torch
    s = Setup(24, [300, 100, 129], rows, 2, 64, "e4m3")
    table = s.table.copy()
    table[0, 2] = 10 ** 6
    table[2, 0] = table[2, 1] = -3
    seqs = s.make_seqs(table, s.lens, s.cu)
    _check(s, seqs, table, s.lens, s.cu, 2, status=1)
    _check(s, seqs, table, s.lens, s.cu, 2, mass_rows=3, decay=1.0, status=1)
    # a length out of bounds: its rows stay as they were
    import paper_2608_23805_amd as msi
    s.status.zero_()
    seqs = s.make_seqs(s.table, [300, 101, 129], s.cu, max_len=300)
    seqs.lens[0] = 301
    q, _ = s.rows(4)
    out = torch.full((s.cu[-1], 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = msi.kv_attention_workspace(s.cache, seqs, 4)
    msi.kv_attention(s.cache, seqs, q, out, 0.1, workspace=ws, status=s.status)
    torch.cuda.synchronize()
    assert int(s.status) == 4 and torch.all(out[:s.cu[1]] == 5.0) and torch.all((out[s.cu[1]:] != 5.0).any(-1))


def test_extreme_scores():
    """Scores far apart (one token takes everything), equal ones, a zero scale, uneven block scales."""
    import torch
    log("case extreme scores")
    for rows in ([1], [40]):
        s = Setup(25, [200], rows, 1, 64, "int8")
        big = bf16(s.g.standard_normal((s.cu[-1], 4, 64)) * 40)
        # p's error follows the score's: up to 2^-24 of |s| (about 3000) for product and sum; the winner takes all here
        from _kv_oracle import attention as exact
        import paper_2608_23805_amd as msi
        out = torch.empty((s.cu[-1], 4, 64), dtype=torch.bfloat16, device="cuda")
        ws = msi.kv_attention_workspace(s.cache, s.seqs, 4)
        msi.kv_attention(s.cache, s.seqs, big[0], out, 1.0, workspace=ws)
        want, tol, _ = exact(s.host, s.table, s.lens, s.cu, big[1], 1.0, 4)
        torch.cuda.synchronize()
        size = np.abs(s.host.sequence(s.table[0], 200)[1]).max()
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol + 2.0 ** -9 * size)
        _check(s, s.seqs, s.table, s.lens, s.cu, 4, scale=0.0)
        wide = 2.0 ** s.g.integers(-40, 20, (s.host.scales.shape[0], 1)).astype(np.float32)
        s.host.scales[..., 1] = wide
        s.scales.copy_(torch.from_numpy(s.host.scales))
        _check(s, s.seqs, s.table, s.lens, s.cu, 4)


def test_queries_and_outputs_in_one_buffer():
    """q as a view of the projection's rows, out as a strided view."""
    import torch
    import paper_2608_23805_amd as msi
    log("case strided q")
    s = Setup(26, [90, 70], [3, 2], 2, 64, "e4m3")
    buf, bh = bf16(s.g.standard_normal((5, 12, 64)) * 0.5)
    wide = torch.full((5, 10, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = msi.kv_attention_workspace(s.cache, s.seqs, 4)
    msi.kv_attention(s.cache, s.seqs, buf[:, 2:6], wide[:, 4:8], 0.125, workspace=ws)
    want, tol, _ = attention(s.host, s.table, s.lens, s.cu, bh[:, 2:6], 0.125, 2)
    torch.cuda.synchronize()
    got = wide.double().cpu().numpy()
    assert np.all(np.abs(got[:, 4:8] - want) <= tol) and np.all(got[:, :4] == 5) and np.all(got[:, 8:] == 5)


@pytest.mark.parametrize("rows", [1, 5, 30])
def test_loose_bounds_and_equal_bits(rows):
    """A table and bounds far larger than the lengths (a captured server's), and the same call twice."""
    import torch
    log(f"case loose bounds rows={rows}")
    s = Setup(27, [150, 900], [rows, rows], 2, 128, "int8", extra_blocks=200)
    seqs = s.make_seqs(s.table, s.lens, s.cu, max_len=200 * 64, max_rows=rows)
    q = s.rows(8, 0.5)
    a = _check(s, seqs, s.table, s.lens, s.cu, 4, mass_rows=rows, decay=0.0, q=q)
    m = s.mass.clone()
    b = _check(s, seqs, s.table, s.lens, s.cu, 4, mass_rows=rows, decay=0.0, q=q)
    assert torch.equal(a, b) and torch.equal(m, s.mass)


def test_graph_and_streams():
    """append, attend and evict captured once, replayed on changing lengths with eager calls in between, and two
    graphs that share a workspace."""
    import torch
    import paper_2608_23805_amd as msi
    log("case graph")
    s = Setup(28, [120, 300], [1, 1], 2, 64, "e4m3", extra_blocks=4)
    seqs = s.make_seqs(s.table, s.lens, s.cu, max_len=64 * s.table.shape[1])
    spare = [p for p in range(s.data.shape[0]) if p not in set(s.table.reshape(-1).tolist())]
    seqs.table[0, 2], seqs.table[1, 5] = spare[0], spare[1]
    qkv = torch.randn(2, 8, 64, device="cuda").bfloat16()
    out = torch.empty((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    ws = msi.kv_attention_workspace(s.cache, seqs, 4, 1)
    side = torch.cuda.Stream()

    def step(stream, o=out):
        msi.kv_append(s.cache, seqs, qkv[:, 4:6], qkv[:, 6:8], stream=stream)
        msi.kv_attention(s.cache, seqs, qkv[:, :4], o, 0.125, mass_rows=1, mass_decay=1.0, workspace=ws, stream=stream)

    graphs, outs = [], [out, torch.empty_like(out)]
    torch.cuda.synchronize()
    keep = (s.data.clone(), s.scales.clone(), s.mass.clone())
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(torch.cuda.current_stream(), o)
        graphs.append(g)
    for t, x in zip((s.data, s.scales, s.mass), keep):
        t.copy_(x)
    for n in range(6):
        seqs.lens.add_(1)
        qkv.copy_(torch.randn(2, 8, 64, device="cuda"))
        before = (s.data.clone(), s.scales.clone(), s.mass.clone())
        graphs[n % 2].replay()
        torch.cuda.synchronize()
        got = (outs[n % 2].clone(), s.data.clone(), s.scales.clone(), s.mass.clone())
        for t, x in zip((s.data, s.scales, s.mass), before):
            t.copy_(x)
        eager = torch.empty_like(out)
        step(torch.cuda.current_stream(), eager)
        torch.cuda.synchronize()
        for a, b in zip(got, (eager, s.data, s.scales, s.mass)):
            assert torch.equal(a, b), n


def test_calls_at_once_on_two_streams():
    """Few-rows and many-rows calls with workspaces of their own, in flight together on two streams; pages shared
    between two sequences where the tokens' weights are not kept."""
    import torch
    import paper_2608_23805_amd as msi
    log("case two streams at once")
    runs = []
    for seed, rows in ((31, [1, 1]), (32, [64, 40])):
        s = Setup(seed, [700, 300], rows, 2, 128, "e4m3")
        table = s.table.copy()
        table[1, :5] = table[0, :5]                        # a common beginning
        seqs = s.make_seqs(table, s.lens, s.cu)
        q = s.rows(8, 0.5)
        out = torch.empty((s.cu[-1], 8, 128), dtype=torch.bfloat16, device="cuda")
        runs.append((s, table, seqs, q, out, msi.kv_attention_workspace(s.cache, seqs, 8), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, table, seqs, q, out, ws, st in runs:
            msi.kv_attention(s.cache, seqs, q[0], out, 0.1, workspace=ws, stream=st)
    torch.cuda.synchronize()
    for s, table, seqs, q, out, ws, st in runs:
        want, tol, _ = attention(s.host, table, s.lens, s.cu, q[1], np.float64(np.float32(0.1)), 4)
        assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)


def test_block_needs_its_workspace():
    """A block's step before ``reserve`` is refused where the attention needs workspace, and no output is touched."""
    import torch
    import paper_2608_23805_amd as msi
    log("case block without workspace")
    s = Setup(33, [700], [1], 2, 64, "int8")
    w = torch.zeros(((4 + 4) * 64, 64), dtype=torch.bfloat16, device="cuda")
    b = msi.AttentionBlock(w, torch.zeros((64, 256), dtype=torch.bfloat16, device="cuda"), s.cache, 4, 2)
    x, h = torch.ones((1, 64), device="cuda").bfloat16(), torch.ones((1, 64), device="cuda")
    before = s.device_state()
    with pytest.raises(msi.MsiError) as e:
        b.step(x, h, s.seqs, mass_rows=1)
    assert e.value.status == msi.MSI_E_NOMEM
    after = s.device_state()
    assert torch.all(h == 1) and torch.all(x == 1) and np.array_equal(before[2], after[2])
    assert np.array_equal(before[0], after[0])             # (nor was the cache)
    b.reserve(s.seqs, 1)
    b.step(x, h, s.seqs, mass_rows=1)
    torch.cuda.synchronize()
    assert torch.all(h == 1)                               # zero weights add nothing
