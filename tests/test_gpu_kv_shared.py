"""Attention of sequences that share their first pages, against the attention's oracle in 64 bits, which reads every
sequence's own table: single tokens, drafts and prompts in every pairing of kernels, ragged and empty groups, groups that a
sequence or the numbers do not allow, rows that no sequence answers for, captured calls.

The bound is the attention's: half a step of bf16 for the output and for every probability, 2^-16 of the latter's sum for
the fp32 arithmetic, joins of partial results among it (one rounding each of a factor and a sum, 2^-23).  Partial results
are kept in units of 2^40 for the sake of V's largest values, so that a product p v under 2^-126 2^40 = 2^-86, which binary32
holds as a subnormal number at best, may vanish: 2^-86 for each token that carries a row."""
import numpy as np
import pytest

from _gpu_helpers import log
from _kv_helpers import Setup, bf16
from _kv_oracle import B, attention

pytestmark = pytest.mark.gpu


class Shared:
    """Sequences of `own` tokens behind their group's shared blocks; groups: (sequences, blocks)."""

    def __init__(self, seed, groups, own, rows, H, D, fmt):
        import torch
        self.groups = groups
        first = [0] + [int(v) for v in np.cumsum([n for n, _ in groups])]
        lead = [b for n, b in groups for _ in range(n)]
        self.s = Setup(seed, [x + B * b for x, b in zip(own, lead)], rows, H, D, fmt, mass=False)
        for a, z, (_, b) in zip(first, first[1:], groups):
            for i in range(a, z):
                self.s.table[i, :b] = self.s.table[a, :b]
        self.first, self.blocks = first, [b for _, b in groups]
        i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
        self.cu, self.nb = i32(first), i32(self.blocks)
        self.s.seqs = self.s.make_seqs(self.s.table, self.s.lens, self.s.cu)

    def bounds(self, seqs=None, max_rows=None, max_blocks=None):
        import paper_2608_23805_amd as msi
        rows = [self.s.cu[z] - self.s.cu[a] for a, z in zip(self.first, self.first[1:])]
        return msi.KvGroups(self.cu, self.nb, max_rows=max(rows + [0]) if max_rows is None else max_rows,
                            max_blocks=max(self.blocks + [0]) if max_blocks is None else max_blocks)


def _run(sh, Hq, scale=0.125, seqs=None, groups=None, all_rows=False, q=None, extra=0):
    import torch
    import paper_2608_23805_amd as msi
    s = sh.s
    seqs, groups = seqs or s.seqs, groups or sh.bounds()
    if q is None:
        q = bf16(s.g.standard_normal((s.cu[-1] + extra, Hq, s.D)) * 1.5)
    out = torch.full((seqs.n_rows, Hq, s.D), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = msi.kv_attention_shared_workspace(s.cache, seqs, groups, Hq)
    guard = torch.full((ws.numel() + 256,), 0xA5, dtype=torch.uint8, device="cuda")       # (and what the workspace held before)
    s.status.zero_()
    msi.kv_attention_shared(s.cache, seqs, groups, q[0], out, scale, workspace=guard[:ws.numel()], status=s.status,
                            stream=torch.cuda.current_stream(), all_rows=all_rows)
    torch.cuda.synchronize()
    assert torch.all(guard[ws.numel():] == 0xA5)
    return q, out, int(s.status)


def _check(sh, Hq, scale=0.125, status=0, **kw):
    q, out, st = _run(sh, Hq, scale, **kw)
    s = sh.s
    assert st == status
    want, tol, _ = attention(s.host, s.table, s.lens, s.cu, q[1][:s.cu[-1]], np.float64(np.float32(scale)), Hq // s.H)
    got = out.double().cpu().numpy()[:s.cu[-1]]
    tol += 2.0 ** -86 * max(s.lens + [1])
    worst = float(np.max(np.abs(got - want) / tol, initial=0.0))
    assert worst <= 1.0
    return q, out


@pytest.mark.parametrize("fmt,D", [("e4m3", 64), ("int8", 64), ("e4m3", 128), ("int8", 128), ("e4m3", 256), ("int8", 256)])
@pytest.mark.parametrize("H,G", [(1, 1), (2, 4), (1, 7)])
def test_shapes(fmt, D, H, G):
    """Single tokens: shared pages by 16, 32 and 128 rows, own pages by 16."""
    for n in (2, 5, 40):
        log(f"case shared {fmt} D={D} H={H} G={G} sequences={n}")
        own = [1 + 13 * i % 150 for i in range(n)]
        _check(Shared(600 + n + D + G, [(n, 3)], own, [1] * n, H, D, fmt), H * G)


@pytest.mark.parametrize("rows", [[1, 1, 1, 1], [5, 4, 1, 3], [9, 30, 2, 17], [70, 1, 129, 64]])
@pytest.mark.parametrize("groups", [[(4, 2)], [(1, 1), (3, 4)], [(2, 0), (2, 3)], [(2, 5), (0, 9), (1, 2), (1, 0)]])
def test_rows_and_groups(rows, groups):
    log(f"case shared rows={rows} groups={groups}")
    own = [r + 30 * i for i, r in enumerate(rows)]
    _check(Shared(700 + sum(rows), groups, own, rows, 2, 128, "e4m3"), 8)


@pytest.mark.parametrize("blocks,own", [(40, 30), (130, 200), (3, 3000), (300, 1)])
@pytest.mark.parametrize("n", [3, 17])
def test_long(blocks, own, n):
    """Many units of the shared pages, of the sequences' own, or of both."""
    log(f"case shared long {blocks} {own} sequences={n}")
    _check(Shared(800 + blocks, [(n, blocks)], [own + i for i in range(n)], [1] * n, 1, 64, "int8"), 4)


def test_long_prompts():
    log("case shared prompts")
    _check(Shared(810, [(2, 20), (2, 7)], [300, 200, 64, 129], [130, 64, 64, 40], 1, 128, "int8"), 4)


def test_many_sequences_and_groups():
    """More owners than the planning workgroup has threads, and lists that are searched twice."""
    log("case shared many sequences")
    g = np.random.default_rng(811)
    sizes = [int(v) for v in g.integers(0, 6, 450)]
    groups = [(n, int(b)) for n, b in zip(sizes, g.integers(0, 4, 450))]
    n = sum(sizes)
    own = [int(v) for v in g.integers(1, 140, n)]
    rows = [int(min(a, b)) for a, b in zip(own, g.integers(0, 3, n))]
    _check(Shared(812, groups, own, rows, 1, 64, "e4m3"), 2)


def test_sequences_outside_groups_and_loose_bounds():
    import paper_2608_23805_amd as msi
    log("case shared outside groups")
    sh = Shared(813, [(2, 2), (2, 3), (2, 1)], [10, 20, 70, 1, 90, 33], [1, 2, 1, 1, 3, 1], 2, 64, "e4m3")
    part = msi.KvGroups(sh.cu[1:3].contiguous(), sh.nb[1:2].contiguous(), max_rows=8, max_blocks=sh.s.table.shape[1])
    _check(sh, 4, groups=part)
    loose = sh.s.make_seqs(sh.s.table, sh.s.lens, sh.s.cu, max_len=64 * sh.s.table.shape[1], max_rows=9)
    _check(sh, 4, groups=sh.bounds(max_rows=9, max_blocks=sh.s.table.shape[1]), seqs=loose)
    none = msi.KvGroups(sh.cu[:1].contiguous(), sh.nb[:0].contiguous(), max_rows=0, max_blocks=0)
    _check(sh, 4, groups=none)


def test_rows_inside_the_shared_pages():
    """A sequence whose rows stand within the shared pages, and one shorter than its rows, are attended by themselves."""
    log("case shared rows inside")
    sh = Shared(814, [(3, 3)], [5, 40, 2], [5, 41, 2], 2, 64, "int8")
    _check(sh, 4)
    sh = Shared(815, [(2, 2), (1, 0)], [9, 0, 2], [3, 1, 5], 2, 64, "int8")
    _check(sh, 4)


@pytest.mark.parametrize("cu,blocks", [([0, 3, 2, 5], [1, 1, 1]), ([0, 2, 9], [1, 1]), ([0, 2, 5], [1, 77]), ([0, 2, 5], [1, -1]),
                                       ([-1, 2, 5], [1, 1]), ([0, 5], [2]), ([0, 2, 1 << 30], [1, 1])])
def test_groups_that_break_a_bound(cu, blocks):
    """Their sequences get their own pages: every row is right, and the status word says so."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case shared broken groups {cu} {blocks}")
    sh = Shared(816, [(5, 1)], [20, 30, 70, 4, 100], [1, 1, 2, 1, 3], 2, 64, "e4m3")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    g = msi.KvGroups(i32(cu), i32(blocks), max_rows=8, max_blocks=1)
    _check(sh, 4, groups=g, status=4)


def test_group_of_too_many_rows():
    log("case shared too many rows")
    sh = Shared(817, [(3, 1), (2, 2)], [20, 30, 70, 4, 100], [1, 1, 1, 2, 3], 2, 64, "e4m3")
    _check(sh, 4, groups=sh.bounds(max_rows=3), status=4)


def test_overlapping_groups():
    """Offsets that fall: nobody shares anything."""
    import torch
    import paper_2608_23805_amd as msi
    log("case shared overlapping groups")
    sh = Shared(818, [(8, 2)], [5 + i for i in range(8)], [1] * 8, 1, 64, "e4m3")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    cu = [0, 8] * 30
    _check(sh, 16, groups=msi.KvGroups(i32(cu), i32([2] * (len(cu) - 1)), max_rows=8, max_blocks=2), status=4)


def test_overlapping_rows_stay_in_bounds():
    """Offsets of rows that fall: what is written is right, or nothing is and the status word tells."""
    import torch
    import paper_2608_23805_amd as msi
    log("case shared overlapping rows")
    sh = Shared(825, [(30, 2)], [5 + i for i in range(30)], [1] * 30, 1, 64, "e4m3")
    s = sh.s
    cu = torch.tensor([0, 8] * 15 + [0], dtype=torch.int32).cuda()
    seqs = msi.KvSeqs(s.seqs.table, s.seqs.lens, cu, n_rows=8, max_rows=8, max_len=s.seqs.max_len)
    for blocks in (0, 2):
        groups = msi.KvGroups(torch.tensor([0, 29], dtype=torch.int32).cuda(), torch.tensor([blocks], dtype=torch.int32).cuda(), max_rows=8,
                              max_blocks=2)
        q, out, st = _run(sh, 4, seqs=seqs, groups=groups, q=bf16(s.g.standard_normal((8, 4, 64))))
        assert st == 4 and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("rows", [[1, 1, 1, 1], [40, 1, 50, 2]])
def test_rows_that_no_sequence_answers_for(rows):
    """Left as they were; with all_rows zeros.  The second sequence breaks a bound."""
    import torch
    import paper_2608_23805_amd as msi
    log(f"case shared other rows {rows}")
    sh = Shared(819, [(3, 2), (1, 1)], [60, 70, 80, 90], rows, 2, 64, "e4m3")
    s = sh.s
    lens = torch.tensor([s.lens[0], 1 << 20] + s.lens[2:], dtype=torch.int32).cuda()
    seqs = msi.KvSeqs(s.seqs.table, lens, s.seqs.cu_rows, n_rows=s.cu[-1] + 7, max_rows=max(rows), max_len=s.seqs.max_len)
    q, plain, st = _run(sh, 4, seqs=seqs, extra=7)
    assert st == 4
    _, cleared, st = _run(sh, 4, seqs=seqs, q=q, all_rows=True)
    assert st == 4
    want, tol, _ = attention(s.host, s.table, s.lens, s.cu, q[1][:s.cu[-1]], 0.125, 2)
    other = list(range(s.cu[1], s.cu[2])) + list(range(s.cu[-1], s.cu[-1] + 7))
    mine = [r for r in range(s.cu[-1]) if r not in other]
    assert torch.all(plain[other] == 5.0) and torch.all(cleared[other] == 0.0)
    for out in (plain, cleared):
        assert np.all((np.abs(out.double().cpu().numpy()[mine] - want[mine]) <= tol[mine]))
    empty = msi.KvSeqs(s.seqs.table[:0].contiguous(), lens[:0].contiguous(), s.seqs.cu_rows[:1].contiguous(), n_rows=3, max_rows=1,
                       max_len=64)
    none = msi.KvGroups(sh.cu[:1].contiguous(), sh.nb[:0].contiguous(), max_rows=0, max_blocks=0)
    out = torch.full((3, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    msi.kv_attention_shared(s.cache, empty, none, q[0][:3], out, 0.125, all_rows=True)
    torch.cuda.synchronize()
    assert torch.all(out == 0.0)


def test_nothing_cached():
    """Sequences without tokens, and bounds that allow none: rows see nothing."""
    import torch
    import paper_2608_23805_amd as msi
    log("case shared nothing cached")
    sh = Shared(826, [(3, 0)], [0, 0, 0], [2, 1, 0], 2, 64, "e4m3")
    for rows, blocks in ((3, 0), (40, 2)):
        seqs = msi.KvSeqs(sh.s.seqs.table[:, :0].contiguous(), sh.s.seqs.lens, sh.s.seqs.cu_rows, n_rows=3, max_rows=2, max_len=0)
        groups = msi.KvGroups(sh.cu, sh.nb, max_rows=rows, max_blocks=blocks)
        for G in (1, 16, 64):
            _, out, st = _run(sh, 2 * G, seqs=seqs, groups=groups)
            assert st == 0 and torch.all(out == 0.0)
            _, out, st = _run(sh, 2 * G, groups=groups)
            assert st == 0 and torch.all(out == 0.0)


def test_bad_pages():
    """A bad shared page is absent for all of the group, a bad own page for its sequence."""
    log("case shared bad pages")
    sh = Shared(820, [(3, 3)], [70, 80, 5], [1, 2, 1], 2, 64, "e4m3")
    sh.s.table[:, 1] = 1 << 29
    sh.s.table[1, 4] = -5
    sh.s.seqs = sh.s.make_seqs(sh.s.table, sh.s.lens, sh.s.cu)
    _check(sh, 4, status=1)
    sh.s.table[:, :] = -1                                    # no page at all: rows see nothing
    sh.s.seqs = sh.s.make_seqs(sh.s.table, sh.s.lens, sh.s.cu)
    _, out = _check(sh, 4, status=1)
    assert (out == 0).all()


@pytest.mark.parametrize("scale", [-0.125, 4.0, 0.0])
def test_scales(scale):
    log(f"case shared scale {scale}")
    for n in (3, 40):
        _check(Shared(821, [(n, 2)], [30] * n, [1] * n, 2, 64, "int8"), 8, scale=scale)


def test_large_values():
    """V scales at the append's upper end in the shared pages, small ones in the others, and the other way round."""
    log("case shared large values")
    for n in (3, 40):
        sh = Shared(822, [(n, 2)], [70] * n, [1] * n, 2, 64, "e4m3")
        shared = [int(p) for p in sh.s.table[0, :2]]
        for at, rest in ((2.0 ** 116, 2.0 ** -20), (2.0 ** -64, 2.0 ** 116)):
            sc = np.full(sh.s.host.scales.shape[:2], rest, dtype=np.float32)
            sc[shared] = at
            sh.s.host.scales[..., 1] = sc
            sh.s.scales[..., 1] = __import__("torch").from_numpy(sc).cuda()
            _check(sh, 8)


def test_same_as_attention_and_equal_bits():
    """Equal calls give equal bits; a call of kv_attention differs by its sums' order only."""
    import torch
    import paper_2608_23805_amd as msi
    log("case shared equal bits")
    for n, r in ((6, 1), (30, 2)):
        sh = Shared(823 + n, [(n, 30)], [100 + i for i in range(n)], [r] * n, 2, 128, "e4m3")
        s = sh.s
        q, one, _ = _run(sh, 8)
        _, two, _ = _run(sh, 8, q=q)
        assert torch.equal(one, two)
        out = torch.empty_like(one)
        ws = msi.kv_attention_workspace(s.cache, s.seqs, 8)
        msi.kv_attention(s.cache, s.seqs, q[0], out, 0.125, workspace=ws)
        torch.cuda.synchronize()
        assert torch.all((out.float() - one.float()).abs() <= 2.0 ** -6 * out.float().abs().amax())


def test_captured():
    """A captured call, replayed as sequences grow, leave their group and come back; two graphs of their own workspaces."""
    import torch
    import paper_2608_23805_amd as msi
    log("case shared captured")
    sh = Shared(824, [(5, 2)], [40, 3, 64, 80, 1], [1] * 5, 2, 64, "e4m3")
    s = sh.s
    seqs = msi.KvSeqs(s.seqs.table, s.seqs.lens, s.seqs.cu_rows, n_rows=5, max_rows=1, max_len=s.table.shape[1] * 64)
    groups = sh.bounds(max_rows=5, max_blocks=2)
    q, _ = bf16(s.g.standard_normal((5, 8, 64)))
    outs = [torch.zeros_like(q) for _ in range(2)]
    ws = [msi.kv_attention_shared_workspace(s.cache, seqs, groups, 8) for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    for o, w in zip(outs, ws):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            msi.kv_attention_shared(s.cache, seqs, groups, q, o, 0.125, workspace=w, stream=torch.cuda.current_stream())
        graphs.append(g)
    for step in range(4):
        if step == 1:
            sh.nb.fill_(1)
        if step == 2:
            sh.cu.copy_(torch.tensor([1, 4]))
        want = torch.zeros_like(q)
        msi.kv_attention_shared(s.cache, seqs, groups, q, want, 0.125,
                                workspace=msi.kv_attention_shared_workspace(s.cache, seqs, groups, 8))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
        lens = [int(v) for v in s.seqs.lens]
        exact, tol, _ = attention(s.host, s.table, lens, s.cu, q.double().cpu().numpy(), 0.125, 4)
        assert np.all(np.abs(want.double().cpu().numpy() - exact) <= tol)
        for o in outs:
            o.zero_()
        s.seqs.lens.sub_(torch.tensor([1, 0, 1, 1, 0], dtype=torch.int32, device="cuda"))
