"""Answers drawn from one prompt, as a served stack runs them: blocks of 4-bit projections, rotation on the way into the
cache, and attention that reads the prompt's pages once, between the routed-expert layers.  The prompt goes through as one
sequence; its pages then serve every answer's table.  Every operator is checked on its own device input (teacher forcing);
the whole run is compared with one that shares nothing."""
import numpy as np
import pytest

import synth
from _gpu_helpers import log
from _kv_helpers import bf16
from _kv_oracle import B, Cache, attention
from _stack import Stack
from test_gpu_kv_rotary import close, frequencies, rotate
from test_gpu_linear_q4 import q4
from test_gpu_stack_attention import _close

pytestmark = pytest.mark.gpu

WL = synth.Workload("shared_decode_bf16", 18, synth.LayerShape(128, 256, 16, 4, 128, "bf16"), prior="zipf", prior_param=1.1,
                    tau=0.3, n_layers=2)
HQ, H, D, ANSWERS, SHARED, ROT = 8, 2, 64, 5, 2, 32


class Served(Stack):
    """The stack with a block before every layer's experts, whose steps take positions and groups."""

    def __init__(self, blocks, *args, **kw):
        super().__init__(*args, **kw)
        self.blocks = blocks

    def step(self, x0, seqs, positions, groups, before, after):
        import torch
        import paper_2608_23805_amd as msi
        n = x0.shape[0]
        cs, side = torch.cuda.current_stream(), torch.cuda.Stream()
        h, x, out = self.h[:n], self.x[:n], self.out[:n]
        r = msi.Routing.alloc(n, self.s.K, self.s.E)
        msi.residual_init(x0, h, x, cs)
        for l in range(self.L):
            before(l)
            self.blocks[l].reserve(seqs, groups=groups)
            self.blocks[l].step(x, h, seqs, stream=cs, positions=positions, groups=groups)
            after(l)
            self.plan.route(x, self.wr[l], self.bias[l], r, self.ws, cs)
            self.plan.forward(l, x, r, self.shared[l], out, self.ws, cs, side)
            msi.residual_add(out, h, x, cs)
        return h, x


def _serve(share, checked):
    import torch
    import paper_2608_23805_amd as msi
    g = np.random.default_rng([82, 1])
    d = WL.shape.d
    weights, blocks = {}, []
    rotary = msi.KvRotary(frequencies(ROT))
    pages = SHARED + 2 * ANSWERS + 1
    for l in range(WL.n_layers):
        wqkv, s1, wh = q4(g, (HQ + 2 * H) * D, d, 64)
        wo, s2, oh = q4(g, d, HQ * D, 128)
        weights[l] = (wh, oh)
        cache = msi.KvCache.alloc(pages, H, D, "e4m3" if l else "int8", mass=False)
        cache.data.random_(0, 255)                           # a pool that held something else
        cache.scales.fill_(float("nan"))
        blocks.append(msi.AttentionBlock((wqkv, s1), (wo, s2), cache, HQ, SHARED * B, rotary=rotary))
    st = Served(blocks, WL, 16)
    order = g.permutation(pages)
    table = np.concatenate([np.tile(order[:SHARED], (ANSWERS, 1)), order[SHARED:SHARED + 2 * ANSWERS].reshape(ANSWERS, 2)], 1).astype(np.int32)
    mirrors = [Cache(b.cache.data.cpu().numpy(), np.ones(b.cache.scales.shape, np.float32), None, b.cache.fmt) for b in blocks]
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    groups = msi.KvGroups(i32([0, ANSWERS]), i32([SHARED]), max_rows=ANSWERS * 3, max_blocks=SHARED) if share else None
    state, results = {}, []

    def run(lens, rows, tab, grp, far):
        cu = [0] + [int(c) for c in np.cumsum(rows)]
        n = cu[-1]
        seqs = msi.KvSeqs(i32(tab), i32(lens), i32(cu), n_rows=n, max_rows=max(rows), max_len=64 * (SHARED + 2))
        pos = np.concatenate([np.arange(x - r, x) for x, r in zip(lens, rows)])[None] + far
        x0, _ = bf16(g.standard_normal((n, d)))

        def before(l):
            torch.cuda.synchronize()
            state["x"] = st.x[:n].double().cpu().numpy() if st.x.dtype == torch.bfloat16 else \
                synth.bf16_bits_to_f32(st.x[:n].cpu().numpy().view(np.uint16)).astype(np.float64)
            state["cache"] = msi.KvCache(blocks[l].cache.data.clone(), blocks[l].cache.scales.clone(), None, blocks[l].cache.fmt)

        def after(l):
            if not checked:
                return
            torch.cuda.synchronize()
            b, m = blocks[l], mirrors[l]
            wh, oh = weights[l]
            qkv = b.qkv[:n].double().cpu().numpy()
            want = (state["x"] @ wh.T).reshape(n, HQ + 2 * H, D)
            size = (np.abs(state["x"]) @ np.abs(wh).T).reshape(n, HQ + 2 * H, D)
            # keys and values lie in the buffer as projected, queries rotated (which adds their rounding once more)
            assert np.all(_close(qkv[:, HQ:], want[:, HQ:], size[:, HQ:], d))
            turned, pair = rotate(want[:, :HQ], pos, frequencies(ROT), None, False)
            assert np.all(np.abs(qkv[:, :HQ] - turned) <= 2.0 ** -8 * (np.abs(turned) + pair) * (1 + 2.0 ** -8)
                          + 2 * (d ** 0.5 * 2.0 ** -22 + 2.0 ** -20) * rotate(size[:, :HQ], pos * 0, frequencies(ROT), None, False)[1] + 1e-30)
            k = torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda")
            raw = b.qkv[:n]
            msi.kv_append_rotary(state["cache"], seqs, rotary, i32(pos[0]), raw[:, HQ:HQ + H], k, raw[:, HQ:HQ + H], raw[:, HQ + H:])
            torch.cuda.synchronize()
            kr, pair = rotate(qkv[:, HQ:HQ + H], pos, frequencies(ROT), None, False)
            assert close(k.double().cpu().numpy(), kr, pair)
            assert m.append(tab, lens, cu, k.double().cpu().numpy(), qkv[:, HQ + H:]) == 0
            live = sorted({int(tab[i][j]) for i, x in enumerate(lens) for j in range(-(-x // B))})
            assert np.array_equal(b.cache.data.cpu().numpy(), m.data)
            assert np.array_equal(b.cache.scales.cpu().numpy()[live], m.scales[live].astype(np.float32))
            want, tol, _ = attention(m, tab, lens, cu, qkv[:, :HQ], np.float64(np.float32(b.scale)), HQ // H)
            attn = b.attn[:n].double().cpu().numpy()
            assert np.all(np.abs(attn - want) <= tol)
            a = attn.reshape(n, -1)
            assert np.all(_close(b.out[:n].cpu().numpy(), a @ oh.T, np.abs(a) @ np.abs(oh).T, HQ * D))

        h, _ = st.step(x0.view(torch.int16), seqs, i32(pos[0]), grp, before, after)
        torch.cuda.synchronize()
        results.append(h.clone())

    run([SHARED * B], [SHARED * B], table[:1], None, 0)        # the prompt
    lens = [SHARED * B + r for r in (3, 1, 2, 3, 1)]
    run(lens, [3, 1, 2, 3, 1], table, groups, 0)               # the questions
    for k in range(3):
        lens = [x + 1 for x in lens]
        run(lens, [1] * ANSWERS, table, groups, 1 << 20 if k == 2 else 0)
    st.close()
    return results


def test_answers_from_one_prompt():
    """What is shared changes the order of sums only: probabilities and outputs are bf16 (2^-8 each) between two layers of
    experts, whose routing the seeds keep away from ties, so the streams stay within 5 % of their root mean square."""
    import torch
    log("case answers from one prompt")
    shared, alone = _serve(True, True), _serve(False, False)
    for a, b in zip(shared, alone):
        assert torch.isfinite(a).all()
        assert (a - b).pow(2).mean().sqrt() <= 0.05 * b.pow(2).mean().sqrt()


def test_block_in_a_graph():
    """A step of a block with everything on, captured and replayed as lengths and positions move; eager steps between."""
    import torch
    import paper_2608_23805_amd as msi
    log("case served block captured")
    g = np.random.default_rng([82, 3])
    d, n = 256, 4
    wqkv, s1, _ = q4(g, (HQ + 2 * H) * D, d, 32)
    wo, s2, _ = q4(g, d, HQ * D, 32)
    rotary = msi.KvRotary(frequencies(ROT), axes=[0] * 8 + [1] * 8)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    data = torch.from_numpy(g.integers(0, 100, (12, H, 2, B, D)).astype(np.uint8)).cuda()
    scales = torch.full((12, H, 2), 2.0 ** -7, device="cuda")
    table = i32([[1, 3 + i, 8 + i] for i in range(n)])
    lens, pos = i32([65, 70, 127, 100]), i32([[9, 8, 7, 6], [1, 2, 3, 4]])
    seqs = msi.KvSeqs(table, lens, i32(range(n + 1)), n_rows=n, max_rows=1, max_len=192)
    groups = msi.KvGroups(i32([0, n]), i32([1]), max_rows=n, max_blocks=1)
    x0, _ = bf16(g.standard_normal((n, d)))
    runs = []
    for _ in range(2):
        cache = msi.KvCache(data.clone(), scales.clone(), None, "int8")
        b = msi.AttentionBlock((wqkv, s1), (wo, s2), cache, HQ, n, rotary=rotary)
        b.reserve(seqs, groups=groups)
        runs.append((b, torch.zeros((n, d), device="cuda"), x0.clone()))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    b, h, x = runs[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.step(x, h, seqs, stream=torch.cuda.current_stream(), positions=pos, groups=groups)
    for _ in range(4):
        c, h1, x1 = runs[1]
        c.step(x1, h1, seqs, positions=pos, groups=groups)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, h1) and torch.equal(x, x1) and torch.equal(b.cache.data, c.cache.data)
        lens += 1
        pos += 5
