"""Performance cases of the attention block's operators: the projection with its
epilogue (``linear``), the paged cache of keys and values in 8 bits
(``kv_append``, ``kv_read``), the attention that reads it (``kv_attention``)
and the eviction that keeps it bounded (``kv_evict``).

A case is one call (or one append and the read of what it changed).  ``op``
names the operator; the sizes beside it are

* ``linear``: M rows, K inputs, N outputs; ``bias``, ``act``, ``residual``
  ("none", "bf16" or "f32") and ``out`` ("bf16" or "f32") choose the epilogue,
* cache operators: ``S`` sequences of at most ``L`` cached tokens, ``lens``
  "full" (all L) or "ragged" (drawn with ``lseed`` over 1 .. L), ``Hkv`` heads of
  ``D`` elements in ``fmt`` ("e4m3" or "int8"), one scale for each block of 64
  tokens, head and K or V,
* ``append``: ``n`` new tokens a sequence at most (ragged as ``lens``),
* ``attention``: ``Hq`` query heads, ``n`` query rows a sequence at most;
  the last ``mass_rows`` rows add to the tokens' accumulated weights, which are
  first scaled by ``decay``,
* ``evict``: ``budget`` tokens kept, the first ``sinks`` and the last ``recent``
  whatever their weights.

Where ``own`` is false ``run`` computes the operators in elementary torch
operations in 32 bits; where it is true it calls the library.
"""
import math
import random

import torch

own = False

BLOCK = 64                              # tokens of a cache block
QMAX = {"e4m3": 448.0, "int8": 127.0}   # largest code
MIN_SCALE = 2.0 ** -64


def _linear(name, M, K, N, bias=True, act="none", residual="none", out="bf16"):
    return {"name": name, "op": "linear", "M": M, "K": K, "N": N, "bias": bias, "act": act, "residual": residual,
            "out": out}


def _append(name, S, L, n, Hkv, D, fmt, lens="ragged", lseed=1):
    return {"name": name, "op": "append", "S": S, "L": L, "n": n, "Hkv": Hkv, "D": D, "fmt": fmt, "lens": lens,
            "lseed": lseed}


def _attention(name, S, L, n, Hq, Hkv, D, fmt, mass_rows=0, decay=1.0, lens="ragged", lseed=1):
    return {"name": name, "op": "attention", "S": S, "L": L, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "fmt": fmt,
            "mass_rows": mass_rows, "decay": decay, "lens": lens, "lseed": lseed}


def _evict(name, S, L, budget, Hkv, D, fmt, sinks=4, recent=128, lens="ragged", lseed=1):
    return {"name": name, "op": "evict", "S": S, "L": L, "budget": budget, "Hkv": Hkv, "D": D, "fmt": fmt,
            "sinks": sinks, "recent": recent, "lens": lens, "lseed": lseed}


def listed():
    return [
        # the query, key and value projection of a decode step of 16 sequences: 16 heads of 256 and 2 + 2 of the cache
        _linear("linear_decode_t16", 16, 2048, 5120),
        # the output projection of a ragged batch, added to the fp32 residual stream
        _linear("linear_t509_residual", 509, 4096, 2048, residual="f32", out="f32"),
        # a dense layer's first product on a chunk of 4096 tokens, with its activation
        _linear("linear_t4096_gelu", 4096, 2048, 8192, act="gelu"),
        # one new token for each of 64 sequences, and the open block of each read back
        _append("append_decode_s64", 64, 8192, 1, 8, 128, "e4m3"),
        # prompts of up to 4096 tokens of 8 sequences, and the whole cache read back
        _append("append_prompt_s8", 8, 4096, 4096, 8, 128, "int8"),
        # a few short sequences: launches and latency
        _attention("attention_short_s4", 4, 200, 1, 8, 8, 64, "e4m3"),
        # one long sequence, one token at a time: the work has to be split along the cache
        _attention("attention_long_s1", 1, 131072, 1, 16, 2, 256, "e4m3", lens="full"),
        # decode of a ragged batch that keeps the weights its eviction goes by
        _attention("attention_decode_s48", 48, 16384, 1, 32, 8, 128, "int8", mass_rows=1, decay=1.0),
        # five drafted tokens of each sequence checked at once, older weights fading
        _attention("attention_draft_s16", 16, 8192, 5, 32, 8, 128, "e4m3", mass_rows=5, decay=0.875),
        # a chunk of 4096 prompt tokens of two sequences on top of what is cached; the last 64 rows weigh the tokens
        _attention("attention_prompt_s2", 2, 8192, 4096, 16, 2, 256, "e4m3", mass_rows=64, decay=0.0, lseed=5),
        # a batch of sequences cut back to 2048 tokens a head
        _evict("evict_s16", 16, 16384, 2048, 8, 128, "e4m3"),
        # one long sequence cut to a quarter
        _evict("evict_long_s1", 1, 65536, 16384, 2, 256, "int8", recent=1024, lens="full"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "append", "attention", "attention", "attention", "evict"])
    if op == "linear":
        M = _log_int(rng, 1, 4096)
        c = _linear("", M, 8 * _log_int(rng, 32, 512), _log_int(rng, 256, 8192), bias=rng.random() < 0.6,
                    act=rng.choice(["none", "none", "silu", "gelu", "gelu_tanh"]),
                    residual=rng.choice(["none", "bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
        if M * c["K"] * c["N"] > 4096 * 2048 * 8192:
            c["N"] = 4096 * 2048 * 8192 // (M * c["K"])
    else:
        D = rng.choice([64, 128, 128, 256])
        Hkv = rng.choice([1, 2, 4, 8]) if D > 64 else rng.choice([2, 5, 8, 12])
        fmt = rng.choice(["e4m3", "int8"])
        lens, lseed = rng.choice(["ragged", "ragged", "full"]), rng.randrange(1, 1 << 16)
        S = _log_int(rng, 1, 64)
        L = max(1, min(_log_int(rng, 1, 65536), 400_000_000 // (S * Hkv * D)))
        if op == "append":
            n = min(L, _log_int(rng, 1, 4096))
            L = max(1, min(L, 32768 * 8 * 128 // (S * Hkv * D)))
            c = _append("", S, L, min(n, L), Hkv, D, fmt, lens, lseed)
        elif op == "attention":
            G = rng.choice([1, 2, 4, 5, 7, 8, 16])
            n = min(L, rng.choice([1, 1, 1, rng.randint(2, 9), _log_int(rng, 10, 2048)]))
            n = max(1, min(n, 2 * 4096 * 8192 * 16 * 256 // (S * L * Hkv * G * D)))
            mass_rows = rng.choice([0, n, rng.randint(1, n)])
            c = _attention("", S, L, n, Hkv * G, Hkv, D, fmt, mass_rows, rng.choice([0.0, 0.875, 1.0]), lens, lseed)
        else:
            budget = max(1, _log_int(rng, 1, L))
            recent = rng.randint(0, budget)
            c = _evict("", S, L, budget, Hkv, D, fmt, min(rng.choice([0, 4]), budget - recent), recent, lens, lseed)
    del c["name"]
    return c


def _lens(c):
    """Cached tokens and new rows of every sequence: plain integers that follow from the case."""
    r = random.Random(c["lseed"])
    full = c["lens"] == "full"
    lens = [c["L"] if full else r.randint(1, c["L"]) for _ in range(c["S"])]
    lens[r.randrange(c["S"])] = c["L"]
    n = c.get("n", 0)
    rows = [min(x, n if full or n == 1 else r.randint(1, n)) if n else 0 for x in lens]
    return lens, rows


def work(c):
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        size = {"none": 0, "bf16": 2, "f32": 4}
        return {"bytes": 2 * (M * K + N * K) + M * N * (size[c["residual"]] + size[c["out"]]) + 4 * N * bool(c["bias"]),
                "flops": 2 * M * K * N}
    lens, rows = _lens(c)
    head = c["Hkv"] * c["D"]
    if c["op"] == "append":            # new rows in, their codes out; codes in and values out of what is read back
        back = sum(_read_rows(c, lens, rows))
        return {"bytes": sum(rows) * head * (4 + 2) + back * head * (2 + 4), "flops": 0}
    if c["op"] == "attention":
        seen = sum(n * x - n * (n - 1) // 2 for n, x in zip(rows, lens))
        weights = (8 if c["decay"] else 4) * sum(lens) * c["Hkv"] if c["mass_rows"] else 0
        return {"bytes": sum(lens) * (2 * head + c["Hkv"] / 8) + 4 * sum(rows) * c["Hq"] * c["D"] + weights,
                "flops": 4 * seen * c["Hq"] * c["D"]}
    kept = sum(min(x, c["budget"]) for x in lens)
    # the weights that are chosen from, the kept tokens' codes in and out, their weights out, and the read
    return {"bytes": sum(lens) * c["Hkv"] * 4 + kept * (head * 4 + c["Hkv"] * 8) + kept * head * (2 + 4), "flops": 0}


def _read_rows(c, lens, rows):
    """Tokens read back after an append: the last block of each sequence for single tokens, otherwise what was written."""
    return [(x - 1) % BLOCK + 1 if c["n"] == 1 else n for x, n in zip(lens, rows)]


# ---------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------

def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _seqs(table, lens, rows):
    cu = [0]
    for n in rows:
        cu.append(cu[-1] + n)
    s = {"table": table, "lens": _int32(lens), "cu": _int32(cu), "rows": cu[-1], "max_rows": max(rows),
         "max_len": max(lens)}
    if own:
        import paper_2608_23805_amd as msi
        s["seqs"] = msi.KvSeqs(table, s["lens"], s["cu"], n_rows=s["rows"], max_rows=s["max_rows"],
                               max_len=s["max_len"])
    return s


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()

    st = {"case": c}
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        types = {"bf16": torch.bfloat16, "f32": torch.float32}
        st.update(x=normal(M, K), w=normal(N, K, scale=K ** -0.5),
                  bias=torch.randn(N, generator=g, device="cuda") if c["bias"] else None,
                  residual=normal(M, N).to(types[c["residual"]]) if c["residual"] != "none" else None,
                  out=torch.empty((M, N), dtype=types[c["out"]], device="cuda"))
        return st
    lens, rows = _lens(c)
    S, H, D = c["S"], c["Hkv"], c["D"]
    need = [-(-x // BLOCK) for x in lens]
    nb, total = max(need), sum(need)
    evict = c["op"] == "evict"
    keep = [-(-min(x, c["budget"]) // BLOCK) for x in lens] if evict else [0] * S
    n_pages = total + sum(keep) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").int().cpu()   # pages as a running server has them
    table, at = torch.full((S, nb), -1, dtype=torch.int32), 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    scales = torch.full((n_pages, H, 2), 1.0, device="cuda")
    data = torch.zeros((n_pages, H, 2, BLOCK, D), dtype=torch.uint8, device="cuda")
    channel = torch.exp2(torch.randn((H, 1, D), generator=g, device="cuda").mul(0.7).clamp(-2, 2))  # uneven channels
    step = max(1, (1 << 27) // (H * 2 * BLOCK * D))
    for p in range(0, n_pages, step):           # filled as appends would have
        part = data[p:p + step]
        x = torch.randn(part.shape, generator=g, device="cuda")
        x[:, :, 0] *= channel
        x = x.bfloat16().float()
        scales[p:p + step] = _least_scale(x.abs().amax((-1, -2)), c["fmt"])
        part.copy_(_encode(x, scales[p:p + step], c["fmt"]))
    mass = torch.exp(torch.randn((n_pages, H, BLOCK), generator=g, device="cuda") * 2.0)
    mass.mul_(torch.rand(mass.shape, generator=g, device="cuda") < 0.9)     # tokens nobody has looked at yet: ties
    st.update(data=data, scales=scales, mass=mass, s=_seqs(table.cuda(), lens, rows))
    if own:
        import paper_2608_23805_amd as msi
        st["cache"] = msi.KvCache(data, scales, mass, fmt=c["fmt"])
    T = sum(rows)
    if c["op"] == "append":
        st["qkv"] = normal(T, 3 * H * D)        # keys and values are views of one projection's rows
        back = _read_rows(c, lens, rows)
        st["back"] = _seqs(st["s"]["table"], lens, back)
        st["k_out"], st["v_out"] = (torch.empty((sum(back), H, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    elif c["op"] == "attention":
        st["q"] = normal(T, c["Hq"], D, scale=2.0)
        st["out"] = torch.empty_like(st["q"])
        st["scale"] = D ** -0.5
        if own:
            st["workspace"] = msi.kv_attention_workspace(st["cache"], st["s"]["seqs"], c["Hq"], c["mass_rows"])
    else:
        kept = [min(x, c["budget"]) for x in lens]
        dst, at = torch.full((S, max(keep)), -1, dtype=torch.int32), total
        for i, k in enumerate(keep):
            dst[i, :k] = order[at:at + k]
            at += k
        st["keep"] = torch.empty((S, H, c["budget"]), dtype=torch.int32, device="cuda")
        st["new_lens"] = torch.empty(S, dtype=torch.int32, device="cuda")
        st["dst"] = _seqs(dst.cuda(), kept, kept)
        st["k_out"], st["v_out"] = (torch.empty((sum(kept), H, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _least_scale(amax, fmt):
    """Least power of two s with amax <= s * QMAX (QMAX = q 2^e, q the significand: the comparison is exact)."""
    q, e = math.frexp(QMAX[fmt])
    m, x = torch.frexp(amax)
    x = torch.where(amax > 0, x - e + (m > q), -64).clamp_min(-64)         # 2^-64 is MIN_SCALE
    return ((x + 127) << 23).to(torch.int32).view(torch.float32)


def _encode(x, scale, fmt):
    y = (x / scale[..., None, None]).clamp(-QMAX[fmt], QMAX[fmt])
    if fmt == "int8":
        return y.round().to(torch.int8).view(torch.uint8)
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes, scale, fmt):
    y = codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()
    return y * scale[..., None, None]


def _tokens(st, s, blocks):
    """K and V of every sequence, padded: [S, Hkv, 64 * blocks, D] float32."""
    pages = s["table"][:, :blocks].clamp_min(0).long()
    x = _decode(st["data"][pages], st["scales"][pages], st["case"]["fmt"])     # [S, nb, H, 2, 64, D]
    S, nb, H, _, B, D = x.shape
    return [x[:, :, :, i].transpose(1, 2).reshape(S, H, nb * B, D) for i in (0, 1)]


def _row_places(s, width):
    """Padded rows of a ragged batch: (row index, valid) [S, width]."""
    r = torch.arange(width, device="cuda")
    cu = s["cu"].long()
    ok = r[None] < (cu[1:] - cu[:-1])[:, None]
    return torch.where(ok, cu[:-1, None] + r[None], 0), ok


def _read_plain(st, s):
    """Values of the last rows of every sequence, in the order of the rows."""
    n, H, D = s["rows"], st["case"]["Hkv"], st["case"]["D"]
    cu = s["cu"].long()
    row = torch.arange(n, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    pos = s["lens"].long()[seq] - (cu[seq + 1] - row)
    page = s["table"][seq, pos // BLOCK].long()
    out = []
    for i in (0, 1):
        codes = st["data"][page, :, i, pos % BLOCK]                       # [n, H, D]
        out.append(_decode(codes[..., None, :], st["scales"][page, :, i], st["case"]["fmt"]).reshape(n, H, D).bfloat16())
    return out


def _append_plain(st, k, v):
    c, s = st["case"], st["s"]
    lens, cu = s["lens"].long(), s["cu"].long()
    n = cu[1:] - cu[:-1]
    first = (lens - n) // BLOCK                                            # first block with a new row
    width = (s["max_rows"] + 2 * BLOCK - 2) // BLOCK
    blk = first[:, None] + torch.arange(width, device="cuda")[None]         # [S, width]
    pos = blk[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")       # [S, width, 64]
    start = (lens - n)[:, None, None]
    new, old = (pos >= start) & (pos < lens[:, None, None]), pos < start
    seq, b = new.any(-1).nonzero(as_tuple=True)                             # blocks that change
    new, old, pos = new[seq, b], old[seq, b], pos[seq, b]
    page = s["table"][seq, blk[seq, b]].long()
    row = torch.where(new, cu[seq][:, None] + pos - (lens - n)[seq][:, None], 0)
    for i, x in enumerate((k, v)):
        x = x.float()[row].transpose(1, 2) * new[:, None, :, None]          # [blocks, H, 64, D]
        codes, was = st["data"][page][:, :, i], st["scales"][page][:, :, i]
        was = torch.where(old.any(-1)[:, None], was, 0.0)
        scale = torch.maximum(_least_scale(x.abs().amax((-1, -2)), c["fmt"]), was)
        again = _encode(_decode(codes, was, c["fmt"]), scale, c["fmt"])
        again = torch.where((scale == was)[..., None, None], codes, again)
        codes = torch.where(old[:, None, :, None], again, codes)
        codes = torch.where(new[:, None, :, None], _encode(x, scale, c["fmt"]), codes)
        st["data"][page, :, i] = codes
        st["scales"][page, :, i] = scale
    token = new[:, None, :].expand(-1, c["Hkv"], -1)
    st["mass"][page] = torch.where(token, 0.0, st["mass"][page])


def _attention_plain(st):
    c, s = st["case"], st["s"]
    S, H, G, D, R = c["S"], c["Hkv"], c["Hq"] // c["Hkv"], c["D"], s["max_rows"]
    nb = -(-s["max_len"] // BLOCK)
    k, v = _tokens(st, s, nb)
    place, ok = _row_places(s, R)
    q = st["q"].float()[place].reshape(S, R, H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, G * R, D)
    lens = s["lens"].long()
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    pos = torch.arange(nb * BLOCK, device="cuda")
    row = torch.arange(R, device="cuda")
    seen = pos[None, None] <= (lens - n)[:, None, None] + row[None, :, None]      # [S, R, L]
    seen = (seen & (pos < lens[:, None])[:, None] & ok[..., None]).repeat(1, G, 1)[:, None]
    v = v * (pos < lens[:, None])[:, None, :, None]
    x = (q @ k.transpose(-1, -2).contiguous()).mul_(st["scale"]).masked_fill_(~seen, -math.inf)
    x.sub_(x.amax(-1, keepdim=True).clamp_min(-3e38)).exp_()
    x.div_(x.sum(-1, keepdim=True).clamp_min(1e-30))
    out = (x @ v).reshape(S, H, G, R, D).permute(0, 3, 1, 2, 4).reshape(S, R, H * G, D)
    st["out"][place[ok]] = out[ok].bfloat16()
    if c["mass_rows"]:
        last = ok & (row[None] >= n[:, None] - c["mass_rows"])
        w = (x.reshape(S, H, G, R, -1) * last[:, None, None, :, None]).sum((2, 3))    # [S, H, L]
        blk = torch.arange(nb, device="cuda")
        seq, b = (blk[None] * BLOCK < lens[:, None]).nonzero(as_tuple=True)
        page = s["table"][seq, b].long()
        w = w.reshape(S, H, nb, BLOCK)[seq, :, b]
        was = st["mass"][page]
        live = (b[:, None] * BLOCK + torch.arange(BLOCK, device="cuda") < lens[seq][:, None])[:, None]
        st["mass"][page] = torch.where(live, was * c["decay"] + w if c["decay"] else w, was)


def _evict_plain(st):
    c, s, d = st["case"], st["s"], st["dst"]
    S, H, D, budget = c["S"], c["Hkv"], c["D"], c["budget"]
    nb = s["table"].shape[1]
    lens = s["lens"].long()
    kept = lens.clamp_max(budget)
    pages = s["table"].clamp_min(0).long()
    mass = st["mass"][pages].transpose(1, 2).reshape(S, H, nb * BLOCK)
    pos = torch.arange(nb * BLOCK, device="cuda")
    safe = (pos < c["sinks"]) | (pos >= lens[:, None] - c["recent"])
    key = torch.where(safe[:, None], math.inf, mass)
    key = torch.where((pos < lens[:, None])[:, None], key, -math.inf)
    order = key.sort(dim=-1, descending=True, stable=True)[1][..., :budget]
    width = d["table"].shape[1] * BLOCK
    rank = torch.arange(order.shape[-1], device="cuda")
    keep = torch.where((rank < kept[:, None])[:, None], order, nb * BLOCK).sort(-1)[0]
    st["keep"].fill_(-1)
    st["keep"][..., :keep.shape[-1]] = torch.where((rank < kept[:, None])[:, None], keep, -1)
    st["new_lens"].copy_(kept)
    # gather the kept tokens, re-encode every block of 64
    keep = torch.nn.functional.pad(keep[..., :width], (0, max(0, width - keep.shape[-1])))
    slot = torch.arange(width, device="cuda")
    live = (slot < kept[:, None])[:, None].expand(S, H, width)
    keep = torch.where(live, keep, 0)
    page = torch.gather(pages[:, None].expand(S, H, nb), 2, keep // BLOCK)
    head = torch.arange(H, device="cuda")[None, :, None]
    seq, b = (slot[::BLOCK][None] < kept[:, None]).nonzero(as_tuple=True)
    to = d["table"][seq, b].long()
    live = live.reshape(S, H, -1, BLOCK)[seq, :, b]                               # [blocks, H, 64]
    for i in (0, 1):
        codes = st["data"][page, head, i, keep % BLOCK].reshape(S, H, -1, BLOCK, D)[seq, :, b]
        scale = st["scales"][page, head, i].reshape(S, H, -1, BLOCK)[seq, :, b]
        x = _decode(codes[..., None, :], scale, c["fmt"])[..., 0, :] * live[..., None]
        new = _least_scale(x.abs().amax((-1, -2)), c["fmt"])
        st["data"][to, :, i] = torch.where(live[..., None], _encode(x, new, c["fmt"]), st["data"][to][:, :, i])
        st["scales"][to, :, i] = new
    m = st["mass"][page, head, keep % BLOCK].reshape(S, H, -1, BLOCK)[seq, :, b]
    st["mass"][to] = torch.where(live, m, st["mass"][to])


def _activate(y, act):
    if act == "silu":
        return y / (1.0 + torch.exp(-y))
    if act == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
    return y


def run(state):
    st, c = state, state["case"]
    if own:
        import paper_2608_23805_amd as msi
        stream = torch.cuda.current_stream()
    if c["op"] == "linear":
        if own:
            msi.linear(st["x"], st["w"], st["out"], bias=st["bias"], act=c["act"], residual=st["residual"],
                       stream=stream)
        else:
            y = st["x"].float() @ st["w"].float().t()
            y = _activate(y if st["bias"] is None else y + st["bias"], c["act"])
            st["out"].copy_(y if st["residual"] is None else y + st["residual"].float())
        return st["out"]
    if c["op"] == "append":
        T, H, D = st["s"]["rows"], c["Hkv"], c["D"]
        _, k, v = st["qkv"].view(T, 3, H, D).unbind(1)
        if own:
            msi.kv_append(st["cache"], st["s"]["seqs"], k, v, stream=stream)
            msi.kv_read(st["cache"], st["back"]["seqs"], st["k_out"], st["v_out"], stream=stream)
            return st["k_out"], st["v_out"], st["scales"], st["mass"]
        _append_plain(st, k, v)
        return *_read_plain(st, st["back"]), st["scales"], st["mass"]
    if c["op"] == "attention":
        if own:
            msi.kv_attention(st["cache"], st["s"]["seqs"], st["q"], st["out"], st["scale"], mass_rows=c["mass_rows"],
                             mass_decay=c["decay"], workspace=st["workspace"], stream=stream)
        else:
            _attention_plain(st)
        return (st["out"], st["mass"]) if c["mass_rows"] else st["out"]
    if own:
        msi.kv_evict(st["cache"], st["s"]["seqs"], st["dst"]["table"], st["new_lens"], st["keep"], budget=c["budget"],
                     sinks=c["sinks"], recent=c["recent"], stream=stream)
        msi.kv_read(st["cache"], st["dst"]["seqs"], st["k_out"], st["v_out"], stream=stream)
        return st["keep"], st["new_lens"], st["k_out"], st["v_out"], st["scales"], st["mass"]
    _evict_plain(st)
    return st["keep"], st["new_lens"], *_read_plain(st, st["dst"]), st["scales"], st["mass"]


# ---------------------------------------------------------------------------
# the definitions in 64 bits, a sequence at a time
# ---------------------------------------------------------------------------

def _power_of_two(e):
    return torch.tensor([2.0 ** i for i in range(-16, 16)], dtype=torch.float64, device=e.device)[e.long() + 16]


def _round_codes(x, fmt):
    """x rounded to the nearest value of the format, ties to even, in 64 bits."""
    x = x.clamp(-QMAX[fmt], QMAX[fmt])
    if fmt == "int8":
        return torch.round(x)
    e = torch.frexp(x)[1].sub(1).clamp_min(-6)                  # normal numbers from 2^-6 on, three bits after the first
    u = _power_of_two(e - 3)
    return torch.round(x / u) * u


def _values(codes, fmt):
    if fmt == "int8":
        return codes.view(torch.int8).double()
    c = codes.to(torch.int64)
    e, m = (c >> 3) & 15, (c & 7).double()
    x = torch.where(e > 0, (1 + m / 8) * _power_of_two(e - 7), m * 2.0 ** -9)
    return torch.where(c >= 128, -x, x)


def _requantised(x, fmt, least=0.0):
    """Nearest representable values of the rows of one block [n, D], and their scale."""
    top = float(x.abs().max()) if x.numel() else 0.0
    s = max(MIN_SCALE, least)
    if top > 0:
        e = math.ceil(math.log2(top)) - int(math.log2(QMAX[fmt])) - 2
        while 2.0 ** e * QMAX[fmt] < top:
            e += 1
        s = max(s, 2.0 ** e)
    return _round_codes(x / s, fmt) * s, s


def _sequence(st, i, length):
    """K and V of sequence i, [Hkv, length, D] each."""
    c, t = st["case"], st["s"]["table"][i].long()
    p = t[torch.arange(length, device="cuda") // BLOCK]
    o = torch.arange(length, device="cuda") % BLOCK
    return [(_values(st["data"][p, :, j, o], c["fmt"]) * st["scales"][p, :, j].double()[..., None]).transpose(0, 1)
            for j in (0, 1)]


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["op"] == "linear":
        y = torch.empty((c["M"], c["N"]), dtype=torch.float64, device="cuda")
        for lo in range(0, c["M"], 512):
            z = st["x"][lo:lo + 512].double() @ st["w"].double().t().contiguous()
            z = z if st["bias"] is None else z + st["bias"].double()
            y[lo:lo + 512] = {"none": lambda a: a, "silu": lambda a: a * torch.sigmoid(a),
                              "gelu": lambda a: a * torch.special.ndtr(a),
                              "gelu_tanh": lambda a: a * torch.sigmoid(
                                  2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a * a * a))}[c["act"]](z)
        return y if st["residual"] is None else y + st["residual"].double()
    lens, rows = _lens(c)
    H, D = c["Hkv"], c["D"]
    scales, mass = st["scales"].double(), st["mass"].double()
    if c["op"] == "append":
        if sum(rows) * H * D > 1 << 22:
            return None                           # a block at a time: too long for the large ones
        qkv = st["qkv"].double().view(-1, 3, H, D)
        out, row = ([], []), 0
        for i, (x, n, back) in enumerate(zip(lens, rows, _read_rows(c, lens, rows))):
            start, base = x - n, (x - n) // BLOCK * BLOCK
            first = min(base, x - back)
            old = _sequence(st, i, start) if start else [torch.empty((H, 0, D), dtype=torch.float64, device="cuda")] * 2
            for j in (0, 1):
                kept = [old[j][:, first:base].clone()] if first < base else []
                for b in range(base // BLOCK, -(-x // BLOCK)):
                    lo, hi = max(start, b * BLOCK), min(x, (b + 1) * BLOCK)
                    p = int(st["s"]["table"][i, b])
                    fresh = qkv[row + lo - start:row + hi - start, 1 + j].transpose(0, 1)
                    both = []
                    for h in range(H):
                        had = old[j][h, b * BLOCK:start] if lo > b * BLOCK else fresh[h][:0]
                        _, s = _requantised(fresh[h], c["fmt"], float(scales[p, h, j]) if len(had) else 0.0)
                        scales[p, h, j] = s
                        both.append(_round_codes(torch.cat([had, fresh[h]]) / s, c["fmt"]) * s)
                    kept.append(torch.stack(both))
                    if j == 0:
                        mass[p, :, lo - b * BLOCK:hi - b * BLOCK] = 0
                out[j].append(torch.cat(kept, 1)[:, x - back - first:].transpose(0, 1))
            row += n
        return torch.cat(out[0]), torch.cat(out[1]), scales, mass
    if c["op"] == "attention":
        G = c["Hq"] // H
        if sum(n * x for n, x in zip(rows, lens)) * c["Hq"] * D > 1 << 41:
            return None
        q = st["q"].double()
        out, row = torch.empty_like(q), 0
        for i, (x, n) in enumerate(zip(lens, rows)):
            k, v = _sequence(st, i, x)
            w = torch.zeros((H, x), dtype=torch.float64, device="cuda")
            for lo in range(0, n, 256):
                hi = min(n, lo + 256)
                pos = torch.arange(x, device="cuda")[None] <= torch.arange(x - n + lo, x - n + hi, device="cuda")[:, None]
                last = (torch.arange(lo, hi, device="cuda") >= n - c["mass_rows"]).double()
                for h in range(H):
                    for a in range(h * G, (h + 1) * G):
                        z = (q[row + lo:row + hi, a] @ k[h].t().contiguous()) * st["scale"]
                        z = torch.softmax(z.masked_fill(~pos, -math.inf), -1)
                        out[row + lo:row + hi, a] = z @ v[h]
                        w[h] += last @ z
            row += n
            p = st["s"]["table"][i].long()[torch.arange(x, device="cuda") // BLOCK]
            o = torch.arange(x, device="cuda") % BLOCK
            mass[p, :, o] = mass[p, :, o] * c["decay"] + w.t()
        return (out, mass) if c["mass_rows"] else out
    if sum(lens) * H * D > 1 << 28:
        return None
    new_k, new_v = [], []
    keep = torch.full((c["S"], H, c["budget"]), -1, dtype=torch.int64)
    for i, x in enumerate(lens):
        kept = min(x, c["budget"])
        k, v = _sequence(st, i, x)
        p = st["s"]["table"][i].long()[torch.arange(x, device="cuda") // BLOCK]
        m = mass[p, :, torch.arange(x, device="cuda") % BLOCK].t().clone()             # [H, x]
        free = m.cpu().tolist()
        to = st["dst"]["table"][i].tolist()
        rows_k, rows_v = [], []
        for h in range(H):
            fixed = set(range(min(c["sinks"], x))) | set(range(max(0, x - c["recent"]), x))
            rest = sorted((t for t in range(x) if t not in fixed), key=lambda t: (-free[h][t], t))
            chosen = sorted((sorted(fixed) + rest)[:kept]) if x > kept else list(range(x))
            keep[i, h, :kept] = torch.tensor(chosen)
            at = keep[i, h, :kept].cuda()
            for j, (src, dst) in enumerate(((k, rows_k), (v, rows_v))):
                parts = []
                for b in range(0, kept, BLOCK):
                    y, s = _requantised(src[h][at[b:b + BLOCK]], c["fmt"])
                    parts.append(y)
                    scales[to[b // BLOCK], h, j] = s
                dst.append(torch.cat(parts))
            pages = torch.tensor(to, device="cuda")[torch.arange(kept, device="cuda") // BLOCK]
            mass[pages, h, torch.arange(kept, device="cuda") % BLOCK] = m[h][at]
        new_k.append(torch.stack(rows_k, 1))
        new_v.append(torch.stack(rows_v, 1))
    return keep, None, torch.cat(new_k), torch.cat(new_v), scales, mass
