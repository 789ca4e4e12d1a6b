"""The attention block's operators run together, as a stack uses them: ragged prompts, single
tokens, an eviction by the weights that the steps before it left, and single tokens on what is
kept.  Every operator is checked on its own device input (teacher forcing): the projections and the attention within
the bounds of their types, the cache byte for byte, the residual step against the oracle."""
import numpy as np
import pytest

import synth
from _gpu_helpers import log
from _kv_helpers import bf16
from _kv_oracle import B, Cache, attention, evict

pytestmark = pytest.mark.gpu

WL = synth.Workload("stack_attention_bf16", 17, synth.LayerShape(64, 256, 16, 4, 128, "bf16"), prior="zipf",
                    prior_param=1.1, tau=0.3, n_layers=2)
HQ, H, D, SEQS, BLOCKS, BUDGET = 4, 2, 64, 4, 3, 20


def _close(got, want, size, K):
    """fp32 sums of K products (sqrt(K) 2^-22 of their magnitude, see the projection's tests), then bf16 or fp32."""
    return np.abs(got - want) <= (K ** 0.5 * 2.0 ** -22 + 2.0 ** -20) * size + 2.0 ** -8 * np.abs(want) + 1e-30


def test_prompt_decode_evict_decode():
    import oracle
    import torch
    import paper_2608_23805_amd as msi
    from _stack_attention import AttentionStack
    log("case stack with attention: prompts, decode, eviction, decode")
    o = oracle.Oracle()
    g = np.random.default_rng([79, 1])
    d = WL.shape.d
    weights = {}

    def block(l):
        wqkv, wh = bf16(g.standard_normal(((HQ + 2 * H) * D, d)) * d ** -0.5)
        wo, oh = bf16(g.standard_normal((d, HQ * D)) * (HQ * D) ** -0.5)
        bias = g.standard_normal((HQ + 2 * H) * D).astype(np.float32) * 0.1
        weights[l] = (wh, oh, bias)
        cache = msi.KvCache.alloc(SEQS * BLOCKS * 2 + 1, H, D, "e4m3" if l else "int8")
        cache.data.random_(0, 255)                       # a pool that held something else
        cache.scales.fill_(float("nan"))
        return msi.AttentionBlock(wqkv, wo, cache, HQ, 64, bias=torch.from_numpy(bias).cuda())

    st = AttentionStack(WL, 16, block=block)
    order = g.permutation(SEQS * BLOCKS * 2 + 1)
    table = order[:SEQS * BLOCKS].reshape(SEQS, BLOCKS).astype(np.int32)
    spare = order[SEQS * BLOCKS:SEQS * BLOCKS * 2].reshape(SEQS, BLOCKS).astype(np.int32)
    mirrors = [Cache(b.cache.data.cpu().numpy(), np.nan_to_num(b.cache.scales.cpu().numpy(), nan=1.0),
                     b.cache.mass.cpu().numpy(), b.cache.fmt) for b in st.blocks]
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
    state = {}

    def run(lens, rows, tab, seed):
        cu = [0] + [int(c) for c in np.cumsum(rows)]
        seqs = msi.KvSeqs(i32(tab), i32(lens), i32(cu), n_rows=cu[-1], max_rows=max(rows), max_len=64 * BLOCKS)
        x0, _ = bf16(np.random.default_rng([79, 2, seed]).standard_normal((cu[-1], d)))
        n = cu[-1]

        def before(l):
            torch.cuda.synchronize()
            state["x"] = synth.bf16_bits_to_f32(st.x[:n].cpu().numpy().view(np.uint16)).astype(np.float64)
            state["h"] = st.h[:n].cpu().numpy()

        def after(l):
            torch.cuda.synchronize()
            b, m = st.blocks[l], mirrors[l]
            wh, oh, bias = weights[l]
            qkv = b.qkv[:n].double().cpu().numpy().reshape(n, -1)
            want = state["x"] @ wh.T + bias
            assert np.all(_close(qkv, want, np.abs(state["x"]) @ np.abs(wh).T + np.abs(bias), d))
            qkv = qkv.reshape(n, HQ + 2 * H, D)
            assert m.append(tab, lens, cu, qkv[:, HQ:HQ + H], qkv[:, HQ + H:]) == 0
            pages = [int(tab[i][k]) for i, x in enumerate(lens) for k in range(-(-x // B))]
            assert np.array_equal(b.cache.data.cpu().numpy(), m.data)
            assert np.array_equal(b.cache.scales.cpu().numpy()[pages], m.scales[pages].astype(np.float32))
            want, tol, mass = attention(m, tab, lens, cu, qkv[:, :HQ], np.float64(np.float32(b.scale)), HQ // H, 1, 1.0)
            attn = b.attn[:n].double().cpu().numpy()
            assert np.all(np.abs(attn - want) <= tol)
            got = b.cache.mass.cpu().numpy()
            assert np.all(np.abs(got - mass) <= 2.0 ** -16 * np.abs(mass) + 1e-12)
            m.mass[:] = got
            a = attn.reshape(n, -1)
            out = b.out[:n].cpu().numpy()
            assert np.all(_close(out, a @ oh.T, np.abs(a) @ np.abs(oh).T, HQ * D))
            hn, xr = o.residual_step(state["h"].astype(np.float64), out.astype(np.float64))
            assert np.array_equal(st.h[:n].cpu().numpy(), state["h"] + out)
            bits = st.x[:n].cpu().numpy().view(np.uint16)
            diff = np.abs(synth.bf16_bits_to_f32(bits).astype(np.float64) - synth.bf16_bits_to_f32(xr))
            assert np.all(diff <= np.abs(synth.bf16_bits_to_f32(xr)) * 2.0 ** -7 + 1e-30) and (bits == xr).mean() >= 0.999

        h, _ = st.step(x0.view(torch.int16), seqs, mass_rows=1, before=before, after=after)
        torch.cuda.synchronize()
        assert torch.isfinite(h).all()

    lens = [30, 20, 13, 1]
    run(lens, lens, table, 0)
    for k in range(3):
        lens = [x + 1 for x in lens]
        run(lens, [1] * SEQS, table, 1 + k)
    seqs = msi.KvSeqs(i32(table), i32(lens), max_len=64 * BLOCKS)
    for l, b in enumerate(st.blocks):
        new = torch.zeros(SEQS, dtype=torch.int32, device="cuda")
        keep = torch.zeros((SEQS, H, BUDGET), dtype=torch.int32, device="cuda")
        msi.kv_evict(b.cache, seqs, i32(spare), new, keep, budget=BUDGET, sinks=2, recent=4)
        want = evict(mirrors[l], table, lens, spare, BUDGET, 2, 4)
        torch.cuda.synchronize()
        assert np.array_equal(keep.cpu().numpy(), want) and new.tolist() == [min(x, BUDGET) for x in lens]
        assert np.array_equal(b.cache.data.cpu().numpy(), mirrors[l].data)
    lens = [min(x, BUDGET) for x in lens]
    for k in range(2):
        lens = [x + 1 for x in lens]
        run(lens, [1] * SEQS, spare, 9 + k)
    st.close()
