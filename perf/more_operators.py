"""Performance cases of operators that a served step of the stack runs: the
projection with 4-bit weights (``linear_q4``), the append that rotates queries
and keys by their positions on the way (``kv_append_rotary``) and the attention
of batches whose sequences share the first pages of their caches
(``kv_attention_shared``).

A case is one call (of the append: the call and the read of the rows it wrote).
``op`` names the operator; the sizes beside it are

* ``q4``: M rows, K inputs, N outputs, one fp16 scale for each ``group`` of
  weights along K; ``bias``, ``act``, ``residual`` ("none", "bf16" or "f32") and
  ``out`` ("bf16" or "f32") choose the epilogue,
* cache operators: ``S`` sequences of at most ``L`` tokens of their own, ``n`` rows
  of the call each at most, ``lens`` "full" or "ragged" (drawn with ``lseed``),
  ``Hq`` query heads over ``Hkv`` heads of ``D`` elements in ``fmt`` ("e4m3" or "int8"),
* ``rotary``: the first ``rot`` elements of a head rotate, in pairs (i, i + rot / 2)
  or, ``interleaved``, (2 i, 2 i + 1); ``axes`` positions a row, whose frequencies
  are ``sections``; positions are ``far`` beyond the cached tokens,
* ``shared``: the sequences are in ``groups`` groups, each with up to ``P`` blocks of 64
  tokens that its sequences share, before the tokens of their own.

Where ``own`` is false ``run`` computes the operators in elementary torch
operations in 32 bits (the angles in 64); where it is true it calls the library.
"""
import math
import random

import torch

own = False

BLOCK = 64                              # tokens of a cache block
QMAX = {"e4m3": 448.0, "int8": 127.0}   # largest code
THETA = 1e6                             # frequencies are THETA^(-2 i / rot)


def _q4(name, M, K, N, group, bias=False, act="none", residual="none", out="bf16"):
    return {"name": name, "op": "q4", "M": M, "K": K, "N": N, "group": group, "bias": bias, "act": act,
            "residual": residual, "out": out}


def _rotary(name, S, L, n, Hq, Hkv, D, rot, fmt, interleaved=False, sections="", far=0, lens="ragged", lseed=1):
    return {"name": name, "op": "rotary", "S": S, "L": L, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot, "fmt": fmt,
            "interleaved": interleaved, "sections": sections, "far": far, "lens": lens, "lseed": lseed}


def _shared(name, groups, S, P, L, n, Hq, Hkv, D, fmt, lens="ragged", lseed=1):
    return {"name": name, "op": "shared", "groups": groups, "S": S, "P": P, "L": L, "n": n, "Hq": Hq, "Hkv": Hkv, "D": D,
            "fmt": fmt, "lens": lens, "lseed": lseed}


def listed():
    return [
        # the query, key and value projection of one token of one sequence: nothing but the weights' bytes
        _q4("q4_decode_t1", 1, 2048, 5120, 32),
        # the output projection of a decode step of 16 sequences, added to the fp32 residual stream
        _q4("q4_decode_t16_residual", 16, 4096, 2048, 128, residual="f32", out="f32"),
        # drafted tokens of a few sequences through a wide layer with an odd number of features
        _q4("q4_draft_t61_silu", 61, 4096, 8199, 64, bias=True, act="silu"),
        # a prompt chunk through a dense layer's first product
        _q4("q4_prompt_t2000_gelu", 2000, 2048, 8192, 128, act="gelu"),
        # one new token for each of 64 sequences
        _rotary("rotary_decode_s64", 64, 8192, 1, 32, 8, 128, 128, "e4m3"),
        # prompts of up to 4096 tokens of 8 sequences, pairs side by side
        _rotary("rotary_prompt_s8", 8, 4096, 4096, 32, 8, 128, 128, "int8", interleaved=True),
        # frames of a video between text: three positions a token, three sections of frequencies
        _rotary("rotary_axes_s3", 3, 2500, 1500, 12, 2, 128, 128, "e4m3", sections="16,24,24"),
        # a chunk of one sequence far beyond what its cut-back cache holds; a quarter of a head rotates
        _rotary("rotary_far_s1", 1, 16384, 1024, 16, 2, 256, 64, "e4m3", far=1 << 20, lens="full"),
        # a few answers to one short question: launches and latency
        _shared("shared_short_s4", 1, 4, 3, 40, 1, 8, 8, 64, "e4m3"),
        # 64 answers drawn from one long prompt
        _shared("shared_decode_s64", 1, 64, 512, 1024, 1, 32, 8, 128, "int8"),
        # four prompts of a system's users, drafted tokens checked at once
        _shared("shared_draft_g4", 4, 48, 256, 700, 5, 16, 2, 256, "e4m3"),
        # questions of up to 256 tokens about one document
        _shared("shared_prompt_s8", 1, 8, 256, 500, 256, 32, 8, 128, "e4m3", lseed=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["q4", "rotary", "shared"])
    if op == "q4":
        group = rng.choice([32, 64, 128])
        M, K = _log_int(rng, 1, 2000), group * _log_int(rng, 256 // group, 8192 // group)
        N = min(_log_int(rng, 256, 8199), 2000 * 2048 * 8192 // (M * K))
        c = _q4("", M, K, N, group, bias=rng.random() < 0.4, act=rng.choice(["none", "none", "silu", "gelu", "gelu_tanh"]),
                residual=rng.choice(["none", "bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
    else:
        D = rng.choice([64, 128, 128, 256])
        Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
        fmt = rng.choice(["e4m3", "int8"])
        lens, lseed = rng.choice(["ragged", "ragged", "full"]), rng.randrange(1, 1 << 16)
        S = _log_int(rng, 1, 64)
        if op == "rotary":
            n = rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 10, 4096)])
            n = max(1, min(n, 400_000_000 // (S * Hkv * (4 * G + 12) * D)))     # bytes, as the largest listed one's
            L = max(n, min(_log_int(rng, 1, 65536), 200_000_000 // (S * Hkv * D)))
            rot = 16 * rng.randint(1, D // 16)
            axes = rng.choice([1, 1, 2, 3]) if rot >= 32 else 1
            cut = sorted(rng.sample(range(1, rot // 2), axes - 1))
            sections = ",".join(str(b - a) for a, b in zip([0] + cut, cut + [rot // 2])) if axes > 1 else ""
            c = _rotary("", S, L, n, Hkv * G, Hkv, D, rot, fmt, rng.random() < 0.4, sections,
                        rng.choice([0, 0, 1 << 14, 1 << 20]), lens, lseed)
        else:
            groups = min(S, rng.choice([1, 1, 2, 5]))
            L = _log_int(rng, 1, 4096)
            n = min(L, rng.choice([1, 1, 1, rng.randint(2, 9), _log_int(rng, 10, 256)]))
            P = _log_int(rng, 1, 512)
            most = 8 * 256 * 32 * 256 * 128                 # the largest listed one's rows times heads times blocks
            P = max(1, min(P, most // (S * n * Hkv * G * D)))
            L = max(n, min(L, 64 * most // (S * n * Hkv * G * D), 100_000_000 // (S * Hkv * D)))
            c = _shared("", groups, S, P, L, n, Hkv * G, Hkv, D, fmt, lens, lseed)
    del c["name"]
    return c


def _lens(c):
    """Own tokens and rows of every sequence: plain integers that follow from the case."""
    r = random.Random(c["lseed"])
    full = c["lens"] == "full"
    lens = [c["L"] if full else r.randint(1, c["L"]) for _ in range(c["S"])]
    lens[r.randrange(c["S"])] = c["L"]
    n = c["n"]
    return lens, [min(x, n if full or n == 1 else r.randint(1, n)) for x in lens]


def _groups(c):
    """First sequence of every group (and the end), and the groups' shared blocks."""
    r = random.Random(c["lseed"] + 7)
    g, S = c["groups"], c["S"]
    first = [0] + sorted(r.sample(range(1, S), g - 1)) + [S]
    blocks = [c["P"] if c["lens"] == "full" else r.randint((c["P"] + 1) // 2, c["P"]) for _ in range(g)]
    blocks[r.randrange(g)] = c["P"]
    return first, blocks


def work(c):
    if c["op"] == "q4":
        M, K, N = c["M"], c["K"], c["N"]
        size = {"none": 0, "bf16": 2, "f32": 4}
        return {"bytes": 2 * M * K + N * K // 2 + 2 * N * (K // c["group"])
                + M * N * (size[c["residual"]] + size[c["out"]]) + 4 * N * bool(c["bias"]), "flops": 2 * M * K * N}
    lens, rows = _lens(c)
    head = c["Hkv"] * c["D"]
    if c["op"] == "rotary":                # queries in and out, keys and values in, their codes out; those in and out again
        axes = len(c["sections"].split(",")) if c["sections"] else 1
        return {"bytes": sum(rows) * (4 * c["Hq"] * c["D"] + 2 * head * (2 + 1) + 2 * head * (1 + 2) + 4 * axes),
                "flops": sum(rows) * (c["Hq"] + c["Hkv"]) * c["rot"] * 3}
    first, blocks = _groups(c)
    shared = sum(b * BLOCK * sum(rows[a:z]) for b, a, z in zip(blocks, first, first[1:]))
    seen = shared + sum(n * x - n * (n - 1) // 2 for n, x in zip(rows, lens))
    tokens = sum(blocks) * BLOCK + sum(lens)
    return {"bytes": tokens * (2 * head + c["Hkv"] / 8) + 4 * sum(rows) * c["Hq"] * c["D"],
            "flops": 4 * seen * c["Hq"] * c["D"]}


# ---------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------

def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(rows):
    cu = [0]
    for n in rows:
        cu.append(cu[-1] + n)
    return cu


def _frequencies(c):
    return [THETA ** (-2 * i / c["rot"]) for i in range(c["rot"] // 2)]


def _axis_of(c):
    """The axis of every frequency."""
    if not c["sections"]:
        return [0] * (c["rot"] // 2)
    return [a for a, n in enumerate(c["sections"].split(",")) for _ in range(int(n))]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()

    st = {"case": c}
    if c["op"] == "q4":
        M, K, N = c["M"], c["K"], c["N"]
        types = {"bf16": torch.bfloat16, "f32": torch.float32}
        w = torch.randn((N, K // c["group"], c["group"]), generator=g, device="cuda") * K ** -0.5
        scales = (w.abs().amax(-1) / 7).half()
        codes = (w / scales.float()[..., None]).round().clamp(-8, 7).to(torch.int8).view(N, K // 2, 2)
        nibbles = (codes[..., 0] & 15) | (codes[..., 1] << 4)
        st.update(x=normal(M, K), w=nibbles.view(torch.uint8).contiguous(), scales=scales,
                  bias=torch.randn(N, generator=g, device="cuda") if c["bias"] else None,
                  residual=normal(M, N).to(types[c["residual"]]) if c["residual"] != "none" else None,
                  out=torch.empty((M, N), dtype=types[c["out"]], device="cuda"))
        return st
    lens, rows = _lens(c)
    S, Hq, H, D = c["S"], c["Hq"], c["Hkv"], c["D"]
    T = sum(rows)
    if c["op"] == "rotary":
        first, blocks, leads = [], [], [0] * S
    else:
        first, blocks = _groups(c)
        leads = [b for b, a, z in zip(blocks, first, first[1:]) for _ in range(a, z)]
    need = [-(-x // BLOCK) for x in lens]
    n_pages = sum(need) + sum(blocks) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").int().cpu()   # pages as a running server has them
    nb = max(a + b for a, b in zip(leads, need))
    table, at = torch.full((S, nb), -1, dtype=torch.int32), 0
    for b, a, z in zip(blocks, first, first[1:]):
        table[a:z, :b] = order[at:at + b]
        at += b
    for i, (lead, k) in enumerate(zip(leads, need)):
        table[i, lead:lead + k] = order[at:at + k]
        at += k
    lens = [lead * BLOCK + x for lead, x in zip(leads, lens)]
    scales = torch.full((n_pages, H, 2), 1.0, device="cuda")
    data = torch.zeros((n_pages, H, 2, BLOCK, D), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // (H * 2 * BLOCK * D))
    for p in range(0, n_pages, step):           # filled as appends would have
        part = data[p:p + step]
        x = torch.randn(part.shape, generator=g, device="cuda").bfloat16().float()
        scales[p:p + step] = _least_scale(x.abs().amax((-1, -2)), c["fmt"])
        part.copy_(_encode(x, scales[p:p + step], c["fmt"]))
    st.update(data=data, scales=scales, table=table.cuda(), lens=_int32(lens), cu=_int32(_starts(rows)), rows=T,
              max_rows=max(rows), max_len=max(lens))
    if own:
        import paper_2608_23805_amd as msi
        st["cache"] = msi.KvCache(data, scales, None, fmt=c["fmt"])
        st["seqs"] = msi.KvSeqs(st["table"], st["lens"], st["cu"], n_rows=T, max_rows=max(rows), max_len=max(lens))
    if c["op"] == "rotary":
        st["qkv"] = normal(T, Hq + 2 * H, D)        # one projection's rows: queries, keys, values
        at = torch.cat([torch.arange(x - n, x) for x, n in zip(lens, rows)]).int() + c["far"]
        where = [at]
        if c["sections"]:                           # frames of 12 x 16 patches: time, height, width
            axes = len(c["sections"].split(","))
            where = [at // 192, at // 16 % 12, at % 16][:axes]
        st["positions"] = torch.stack(where).int().cuda()
        st["freq"] = torch.tensor(_frequencies(c), dtype=torch.float64, device="cuda")
        st["axis"] = torch.tensor(_axis_of(c), device="cuda")
        st["q_out"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        st["k_out"], st["v_out"] = (torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
        if own:
            st["rotary"] = msi.KvRotary(_frequencies(c), axes=_axis_of(c), interleaved=c["interleaved"])
        return st
    st["q"] = normal(T, Hq, D, scale=2.0)
    st["out"] = torch.empty_like(st["q"])
    st["scale"] = D ** -0.5
    st["first"], st["blocks"] = _int32(first), _int32(blocks)
    st["group_rows"] = max(sum(rows[a:z]) for a, z in zip(first, first[1:]))
    st["own_len"] = max(x - b * BLOCK for x, b in zip(lens, leads))
    if own:
        st["groups"] = msi.KvGroups(st["first"], st["blocks"], max_rows=st["group_rows"], max_blocks=max(blocks))
        st["workspace"] = msi.kv_attention_shared_workspace(st["cache"], st["seqs"], st["groups"], Hq)
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _least_scale(amax, fmt):
    """Least power of two s with amax <= s * QMAX, at least 2^-64 (QMAX = q 2^e: the comparison is exact)."""
    q, e = math.frexp(QMAX[fmt])
    m, x = torch.frexp(amax)
    x = torch.where(amax > 0, x - e + (m > q), -64).clamp_min(-64)
    return ((x + 127) << 23).to(torch.int32).view(torch.float32)


def _encode(x, scale, fmt):
    y = (x / scale[..., None, None]).clamp(-QMAX[fmt], QMAX[fmt])
    if fmt == "int8":
        return y.round().to(torch.int8).view(torch.uint8)
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes, scale, fmt):
    y = codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()
    return y * scale[..., None, None]


def _activate(y, act):
    if act == "silu":
        return y / (1.0 + torch.exp(-y))
    if act == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
    return y


def _q4_plain(st):
    c = st["case"]
    codes = st["w"].view(torch.int8)
    codes = torch.stack([(codes << 4) >> 4, codes >> 4], -1).view(c["N"], -1, c["group"])
    w = (codes.float() * st["scales"].float()[..., None]).view(c["N"], c["K"])
    y = st["x"].float() @ w.t()
    y = _activate(y if st["bias"] is None else y + st["bias"], c["act"])
    st["out"].copy_(y if st["residual"] is None else y + st["residual"].float())


def _rotate(x, cos, sin, rot, interleaved):
    """x [T, heads, D] float32, cos and sin [T, 1, rot / 2]."""
    turn, rest = x[..., :rot], x[..., rot:]
    a, b = (turn[..., 0::2], turn[..., 1::2]) if interleaved else turn.chunk(2, -1)
    u, v = a * cos - b * sin, b * cos + a * sin
    turn = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turn, rest], -1)


def _rotary_plain(st, q, k, v):
    c = st["case"]
    angle = st["positions"].double()[st["axis"]].t() * st["freq"]                   # [T, rot / 2]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    st["q_out"].copy_(_rotate(q.float(), cos, sin, c["rot"], c["interleaved"]))
    k = _rotate(k.float(), cos, sin, c["rot"], c["interleaved"]).bfloat16()          # a key is a bf16 number before it is a code
    lens, cu = st["lens"].long(), st["cu"].long()
    n = cu[1:] - cu[:-1]
    first = (lens - n) // BLOCK                                            # first block with a new row
    width = (st["max_rows"] + 2 * BLOCK - 2) // BLOCK
    blk = first[:, None] + torch.arange(width, device="cuda")[None]         # [S, width]
    pos = blk[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")       # [S, width, 64]
    start = (lens - n)[:, None, None]
    new, old = (pos >= start) & (pos < lens[:, None, None]), pos < start
    seq, b = new.any(-1).nonzero(as_tuple=True)                             # blocks that change
    new, old, pos = new[seq, b], old[seq, b], pos[seq, b]
    page = st["table"][seq, blk[seq, b]].long()
    row = torch.where(new, cu[seq][:, None] + pos - (lens - n)[seq][:, None], 0)
    for i, (x, out) in enumerate(((k, st["k_out"]), (v, st["v_out"]))):
        x = x.float()[row].transpose(1, 2) * new[:, None, :, None]          # [blocks, H, 64, D]
        codes, was = st["data"][page][:, :, i], st["scales"][page][:, :, i]
        was = torch.where(old.any(-1)[:, None], was, 0.0)
        scale = torch.maximum(_least_scale(x.abs().amax((-1, -2)), c["fmt"]), was)
        again = _encode(_decode(codes, was, c["fmt"]), scale, c["fmt"])
        codes = torch.where((old[:, None] & (scale > was)[..., None])[..., None], again, codes)
        codes = torch.where(new[:, None, :, None], _encode(x, scale, c["fmt"]), codes)
        st["data"][page, :, i] = codes
        st["scales"][page, :, i] = scale
        y = _decode(codes, scale, c["fmt"]).bfloat16().transpose(1, 2)      # [blocks, 64, H, D]
        out[row[new]] = y[new]


def _tokens(st, table):
    """K and V of the pages of a table [n, blocks]: [n, Hkv, 64 * blocks, D] float32."""
    pages = table.clamp_min(0).long()
    x = _decode(st["data"][pages], st["scales"][pages], st["case"]["fmt"])     # [n, nb, H, 2, 64, D]
    n, nb, H, _, B, D = x.shape
    return [x[:, :, :, i].transpose(1, 2).reshape(n, H, nb * B, D) for i in (0, 1)]


def _partial(st, q, table, seen):
    """Maximum, sum and outputs of padded rows q [n, R, Hkv, G, D] over a table's tokens; seen [n, R, tokens]."""
    n, R, H, G, D = q.shape
    k, v = _tokens(st, table)
    v = v * seen.any(1)[:, None, :, None]
    x = q.permute(0, 2, 1, 3, 4).reshape(n, H, R * G, D) @ k.transpose(-1, -2).contiguous()
    x.mul_(st["scale"]).masked_fill_(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x.sub_(m).exp_()
    back = [y.reshape(n, H, R, G, -1).permute(0, 2, 1, 3, 4) for y in (m, x.sum(-1, keepdim=True), x @ v)]
    return back                                                             # [n, R, H, G, 1 or D]


def _places(starts, width):
    """Rows of a ragged batch, padded: (row index, valid) [n, width]."""
    r = torch.arange(width, device="cuda")
    ok = r[None] < (starts[1:] - starts[:-1])[:, None]
    return torch.where(ok, starts[:-1, None] + r[None], 0), ok


def _shared_plain(st):
    c = st["case"]
    H, G, D, T = c["Hkv"], c["Hq"] // c["Hkv"], c["D"], st["rows"]
    lens, cu, first, blocks = (st[x].long() for x in ("lens", "cu", "first", "blocks"))
    q = st["q"].float().view(T, H, G, D)
    nb = st["table"].shape[1]
    # every group's rows on its shared pages
    place, ok = _places(cu[first], st["group_rows"])
    pos = torch.arange(c["P"] * BLOCK, device="cuda")
    seen = (pos < blocks[:, None] * BLOCK)[:, None].expand(-1, place.shape[1], -1)
    one = [y[ok] for y in _partial(st, q[place], st["table"][first[:-1], :c["P"]], seen)]
    # every sequence's rows on its own pages
    seq = torch.arange(c["S"], device="cuda")
    lead = blocks[torch.searchsorted(first[1:].contiguous(), seq, right=True)]
    place, ok = _places(cu, st["max_rows"])
    blk = lead[:, None] + torch.arange(-(-st["own_len"] // BLOCK), device="cuda")
    table = torch.gather(st["table"], 1, blk.clamp_max(nb - 1))
    pos = lead[:, None] * BLOCK + torch.arange(blk.shape[1] * BLOCK, device="cuda")
    row = torch.arange(place.shape[1], device="cuda")
    seen = pos[:, None] <= (lens - (cu[1:] - cu[:-1]))[:, None, None] + row[None, :, None]
    two = [y[ok] for y in _partial(st, q[place], table, seen)]
    m = torch.maximum(one[0], two[0])
    a, b = torch.exp(one[0] - m), torch.exp(two[0] - m)
    st["out"].copy_(((a * one[2] + b * two[2]) / (a * one[1] + b * two[1])).view(T, H * G, D))


def run(state):
    st, c = state, state["case"]
    if own:
        import paper_2608_23805_amd as msi
        stream = torch.cuda.current_stream()
    if c["op"] == "q4":
        if own:
            msi.linear_q4(st["x"], st["w"], st["scales"], st["out"], bias=st["bias"], act=c["act"], residual=st["residual"],
                          stream=stream)
        else:
            _q4_plain(st)
        return st["out"]
    if c["op"] == "rotary":
        Hq, H = c["Hq"], c["Hkv"]
        q, k, v = st["qkv"][:, :Hq], st["qkv"][:, Hq:Hq + H], st["qkv"][:, Hq + H:]
        if own:
            msi.kv_append_rotary(st["cache"], st["seqs"], st["rotary"], st["positions"], q, st["q_out"], k, v, stream=stream)
            msi.kv_read(st["cache"], st["seqs"], st["k_out"], st["v_out"], stream=stream)
        else:
            _rotary_plain(st, q, k, v)
        return st["q_out"], st["k_out"], st["v_out"], st["scales"]
    if own:
        msi.kv_attention_shared(st["cache"], st["seqs"], st["groups"], st["q"], st["out"], st["scale"],
                                workspace=st["workspace"], stream=stream)
    else:
        _shared_plain(st)
    return st["out"]


# ---------------------------------------------------------------------------
# the definitions in 64 bits, a sequence at a time
# ---------------------------------------------------------------------------

def _power_of_two(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float64), e)


def _round_codes(x, fmt):
    """x rounded to the nearest value of the format, ties to even, in 64 bits."""
    x = x.clamp(-QMAX[fmt], QMAX[fmt])
    if fmt == "int8":
        return torch.round(x)
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -40)))
    e = torch.where(torch.exp2(e) > x.abs(), e - 1, e)
    e = torch.where(torch.exp2(e + 1) <= x.abs(), e + 1, e).clamp_min(-6)   # normal numbers from 2^-6 on, three bits after the first
    u = torch.exp2(e - 3)
    return torch.round(x / u) * u


def _values(codes, fmt):
    if fmt == "int8":
        return codes.view(torch.int8).double()
    c = codes.to(torch.int64)
    e, m = (c >> 3) & 15, (c & 7).double()
    x = torch.where(e > 0, (1 + m / 8) * _power_of_two(e - 7), m * 2.0 ** -9)
    return torch.where(c >= 128, -x, x)


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["op"] == "q4":
        N, K = c["N"], c["K"]
        byte = st["w"].to(torch.int64)
        q = torch.empty((N, K), dtype=torch.float64, device="cuda")
        for j in (0, 1):
            nib = (byte >> 4 * j) % 16
            q[:, j::2] = torch.where(nib >= 8, nib - 16, nib).double()
        w = (q.view(N, -1, c["group"]) * st["scales"].double().unsqueeze(-1)).view(N, K).t().contiguous()
        act = {"none": lambda a: a, "silu": lambda a: a * torch.sigmoid(a), "gelu": lambda a: a * torch.special.ndtr(a),
               "gelu_tanh": lambda a: a * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a * a * a))}[c["act"]]
        z = st["x"].double() @ w
        y = act(z if st["bias"] is None else z + st["bias"].double())
        return y if st["residual"] is None else y + st["residual"].double()
    own_lens, rows = _lens(c)
    H, D, Hq = c["Hkv"], c["D"], c["Hq"]
    if c["op"] == "rotary":
        half, T = c["rot"] // 2, sum(rows)
        qkv, scales = st["qkv"].double(), st["scales"].double()
        i = torch.arange(half, device="cuda")
        one, two = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
        turn = st["positions"].double()[_axis_of(c), :].t().unsqueeze(1) * torch.tensor(_frequencies(c), dtype=torch.float64,
                                                                                        device="cuda")
        z = torch.polar(torch.ones_like(turn), turn) * torch.complex(qkv[:, :Hq + H, one], qkv[:, :Hq + H, two])
        qkv[:, :Hq + H, one], qkv[:, :Hq + H, two] = z.real, z.imag
        qkv[:, Hq:] = qkv[:, Hq:].bfloat16().double()                # a key is a bf16 number before it is a code
        back, row = ([], []), 0
        for s, (x, n) in enumerate(zip(own_lens, rows)):
            b0 = (x - n) // BLOCK
            blk = torch.arange(x - n, x, device="cuda") // BLOCK - b0
            pages = st["table"][s, b0:(x - 1) // BLOCK + 1].long()
            for j in (0, 1):
                fresh = qkv[row:row + n, Hq + j * H:Hq + (j + 1) * H]           # [n, H, D]
                top = torch.zeros((len(pages), H), dtype=torch.float64, device="cuda")
                top.index_reduce_(0, blk, fresh.abs().amax(-1), "amax")
                e = torch.ceil(torch.log2(top.clamp_min(2.0 ** -60) / QMAX[c["fmt"]]))
                e = torch.where(torch.exp2(e - 1) * QMAX[c["fmt"]] >= top, e - 1, e)
                e = torch.where(torch.exp2(e) * QMAX[c["fmt"]] < top, e + 1, e).clamp_min(-64)
                scale = torch.exp2(e)
                if (x - n) % BLOCK:
                    scale[0] = torch.maximum(scale[0], scales[pages[0], :, j])
                scales[pages, :, j] = scale
                mine = scale[blk][..., None]
                back[j].append(_round_codes(fresh / mine, c["fmt"]) * mine)
            row += n
        return qkv[:, :Hq], torch.cat(back[0]), torch.cat(back[1]), scales
    if work(c)["flops"] > 1 << 41:
        return None
    G, first = Hq // H, _groups(c)[0]
    q, out, row = st["q"].double(), torch.empty((sum(rows), Hq, D), dtype=torch.float64, device="cuda"), 0
    for s, n in enumerate(rows):
        x = int(st["lens"][s])
        lead = first[[a <= s < z for a, z in zip(first, first[1:])].index(True)]
        if lead == s:
            kept = {}                                                # the group's shared tokens, once
        t = torch.arange(x, device="cuda")
        page, at = st["table"][s].long()[t // BLOCK], t % BLOCK
        many = int(st["blocks"][first.index(lead)]) * BLOCK
        pos = t <= x - n + torch.arange(n, device="cuda")[:, None]
        for h in range(H):
            if h not in kept:
                kept[h] = [_values(st["data"][page[:many], h, j, at[:many]], c["fmt"])
                           * st["scales"][page[:many], h, j].double()[:, None] for j in (0, 1)]
            k, v = [torch.cat([kept[h][j], _values(st["data"][page[many:], h, j, at[many:]], c["fmt"])
                               * st["scales"][page[many:], h, j].double()[:, None]]) for j in (0, 1)]
            z = torch.einsum("nad,td->ant", q[row:row + n, h * G:(h + 1) * G], k) * st["scale"]
            p = torch.softmax(z.masked_fill(~pos, -math.inf), -1)
            out[row:row + n, h * G:(h + 1) * G] = (p.reshape(-1, x) @ v).view(G, n, D).transpose(0, 1)
        row += n
    return out
