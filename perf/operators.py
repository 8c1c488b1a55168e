"""The operators of a step of tree speculation, as they are measured: rotary positions, the paged (quantised) key/value cache, attention of
a tree of drafted tokens over it, and the verification of such a tree.

Sequences are ragged: rows [row_start[b], row_start[b + 1]) are sequence b's, and they stand at positions first_pos[b], first_pos[b] + 1, ...
of its cache.  A tree's node 0 is its root (the last final token); every other node names its parent, which has a lower index.  A window
of drafts is a tree without branches.  Shapes come from this repository's configurations (workload/configs.py: 4 heads of 64 in fp32, 20
heads of 64, 32 heads of 128 with 32 or 8 key/value heads, vocabularies of 4 096 to 65 536, windows of 16 and 32, images of 576 to 4 096
tokens) or are generic.
"""
import math

import numpy as np
import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------------------------------ cases
def _rotary(seqs, rows, heads, kv_heads, hd, rotary, interleaved, scaling, dtype, far):
    return dict(op="rotary", seqs=seqs, rows=rows, heads=heads, kv_heads=kv_heads, hd=hd, rotary=rotary, interleaved=interleaved,
                scaling=scaling, dtype=dtype, far=far)


def _cache(seqs, nodes, node_spread, back, ctx, kv_heads, hd, page, dtype, cache, branch):
    """branch 0: no compaction; else the written rows are trees with up to `branch` children a node, and one path of each is kept."""
    return dict(op="cache", seqs=seqs, nodes=nodes, node_spread=node_spread, back=back, ctx=ctx, kv_heads=kv_heads, hd=hd, page=page,
                dtype=dtype, cache=cache, branch=branch)


def _attend(seqs, nodes, node_spread, ctx, ctx_spread, heads, kv_heads, hd, page, cache, branch):
    return dict(op="attend", seqs=seqs, nodes=nodes, node_spread=node_spread, ctx=ctx, ctx_spread=ctx_spread, heads=heads,
                kv_heads=kv_heads, hd=hd, page=page, cache=cache, dtype="f32" if cache == "f32" else "bf16", branch=branch)


def _verify(seqs, nodes, node_spread, vocab, branch, depth, sampled):
    """sampled: the children were drawn from a draft model's distribution (q); else they are its likeliest tokens (no q)."""
    return dict(op="verify", seqs=seqs, nodes=nodes, node_spread=node_spread, vocab=vocab, branch=branch, depth=depth, sampled=sampled)


def listed():
    return [
        # the queries and keys of one token of each of eight sequences: what every layer of a decoding step runs, pure latency
        dict(_rotary(8, 1, 32, 8, 128, 128, False, "none", "bf16", 4096), name="rotary_token"),
        # a prompt of two long documents: half of each head turns, neighbouring pairs, scaled by parts, positions up to 200 000
        dict(_rotary(2, 6001, 32, 8, 128, 64, True, "parts", "bf16", 200000), name="rotary_prompt"),
        # one token of each of eight sequences written into the fp8 cache and read back
        dict(_cache(8, 1, 0, 0, 2352, 8, 128, 64, "bf16", "fp8", 0), name="cache_token"),
        # trees of up to 49 drafts written, the accepted path kept, and the last page's worth of each sequence read back
        dict(_cache(6, 49, 30, 64, 700, 20, 64, 64, "f32", "fp8", 3), name="cache_tree"),
        # prompts of about 4 000 tokens quantised as they are written, and handed to a kernel that wants them plain
        dict(_cache(4, 4099, 500, 0, 0, 8, 128, 64, "bf16", "fp8", 0), name="cache_prompt"),
        # a single token of the narrow model at the end of a 24 x 24 image: the smallest call
        dict(_attend(1, 1, 0, 577, 0, 20, 20, 64, 64, "bf16", 1), name="attend_token"),
        # the tiny fp32 model's window of 16
        dict(_attend(1, 16, 0, 288, 0, 4, 4, 64, 64, "f32", 1), name="attend_window_f32"),
        # four long conversations, one token each, grouped heads, fp8: the cache's bytes and nothing else
        dict(_attend(4, 1, 0, 32801, 9000, 32, 8, 128, 64, "fp8", 1), name="attend_token_long"),
        # eight images of the wide model at different stages, trees of up to 33 drafts, bf16
        dict(_attend(8, 33, 20, 2352, 1500, 32, 32, 128, 64, "bf16", 3), name="attend_tree"),
        # throughput: sixteen sequences, trees of up to 61 drafts, grouped heads, fp8
        dict(_attend(16, 61, 17, 8211, 3000, 32, 8, 128, 64, "fp8", 4), name="attend_tree_batch"),
        # one window of 16 sampled drafts over the narrow vocabulary
        dict(_verify(1, 16, 0, 16384, 1, 15, True), name="verify_window"),
        # sixteen trees of sampled drafts over the wide vocabulary
        dict(_verify(16, 61, 17, 65536, 4, 6, True), name="verify_trees"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(("rotary", "cache", "attend", "attend", "attend", "verify"))
    seqs = _log_int(rng, 1, 24)
    kv_heads = _log_int(rng, 1, 20)
    heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 5, 8))
    hd = rng.choice((32, 64, 64, 96, 128, 128, 192, 256))
    page = rng.choice((32, 64, 64, 96, 128))
    if op == "rotary":
        return _rotary(seqs, _log_int(rng, 1, 4000), heads, kv_heads, hd, 2 * rng.randint(1, hd // 2) if rng.random() < 0.5 else hd,
                       rng.random() < 0.5, rng.choice(("none", "linear", "base", "parts")), rng.choice(("f32", "bf16")),
                       _log_int(rng, 1, 1000000))
    if op == "cache":
        branch = rng.choice((0, 0, 1, 2, 4))
        nodes = _log_int(rng, 1, 4096 if branch == 0 else 250)
        return _cache(seqs, nodes, rng.randint(0, nodes), rng.randint(0, 100), rng.randint(100, 4000), kv_heads, hd, page,
                      rng.choice(("f32", "bf16")), rng.choice(("fp8", "fp8", "bf16", "f32")), branch)
    if op == "attend":
        nodes = 1 if rng.random() < 0.3 else _log_int(rng, 1, 250)
        ctx = _log_int(rng, 1, 40000) - 1
        return _attend(seqs, nodes, rng.randint(0, nodes), ctx, rng.randint(0, ctx), heads, kv_heads, hd, page,
                       rng.choice(("fp8", "fp8", "bf16", "bf16", "f32")), rng.choice((1, 2, 4)))
    nodes = _log_int(rng, 1, 128)
    return _verify(seqs, nodes, rng.randint(0, nodes), _log_int(rng, 500, 70000), rng.choice((1, 2, 3, 5)), rng.randint(1, 8),
                   rng.random() < 0.7)


def draw(rng):
    """One more case over the ranges of the listed ones, none dearer than the dearest of its operator (and fp32 attention, whose products
    run at a sixteenth of the rate, a sixteenth of that)."""
    limit = {}
    for c in listed():
        w = work(c)
        if c["op"] not in limit or w["bytes"] + w["flops"] / 300 > sum(limit[c["op"]]):
            limit[c["op"]] = (w["bytes"], w["flops"] / 300)
    while True:
        c = _draw_once(rng)
        w = work(c)
        share = 1 / 16 if c["op"] == "attend" and c["cache"] == "f32" else 1
        rows = c["seqs"] * c["nodes"] if c["op"] == "verify" else 0
        if w["bytes"] + w["flops"] / 300 <= share * sum(limit[c["op"]]) and rows * c.get("vocab", 0) <= 16 * 61 * 65536:
            return c


# ----------------------------------------------------------------------------------------------------------------------- inputs
def _spread(n, spread, seqs):
    return [n - (spread * s // (seqs - 1) if seqs > 1 else 0) for s in range(seqs)]


def _starts(counts):
    return [0] + np.cumsum(counts).tolist()


def _tree(rng, n, branch, depth=1 << 30):
    """Parents of n nodes (-1: the root), at most `branch` children a node and `depth` levels below the root, while there is room."""
    parents, level, children = [-1], [0], [0]
    while len(parents) < n:
        free = [i for i in range(len(parents)) if children[i] < branch and level[i] < depth] or [0]
        # a tree grows at its likelier nodes: early in a level, and rather deep than wide
        j = free[min(int(rng.exponential(2.0)), len(free) - 1)] if rng.random() < 0.5 else free[-1 - min(int(rng.exponential(2.0)), len(free) - 1)]
        children[j] += 1
        parents.append(j)
        level.append(level[j] + 1)
        children.append(0)
    return parents[:n]


def _path(rng, parents):
    """A path from the root, as a verification would leave it: some children down."""
    path = [0] if parents else []
    while path and rng.random() < 0.8:
        below = [i for i, p in enumerate(parents) if p == path[-1]]
        if not below:
            break
        path.append(below[0] if rng.random() < 0.7 else below[-1])
    return path


def _mask_words(parents, words):
    """Bit j of row i: node j is node i or one of its ancestors."""
    rows = np.zeros((len(parents), words), dtype=np.uint32)
    for i, p in enumerate(parents):
        if p >= 0:
            rows[i] = rows[p]
        rows[i, i // 32] |= np.uint32(1 << (i % 32))
    return rows


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device="cuda")


def _frequencies(c):
    """Radians a position, float64: theta^(-2i/r), stretched for a context `factor` times the one that the model was trained on."""
    r, theta, factor, trained = c["rotary"], 10000.0, 8.0, 8192.0
    i = torch.arange(r // 2, dtype=torch.float64)
    if c["scaling"] == "base":
        theta = theta * factor ** (r / (r - 2)) if r > 2 else theta
    f = theta ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        f = f / factor
    if c["scaling"] == "parts":
        turns = trained * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    return f


def _magnitude(c):
    return 1.0 if c["scaling"] != "parts" else 0.1 * math.log(8.0) + 1.0


def _rows(g, n, heads, hd, dtype, loud=0.0):
    """Rows of projected queries, keys or values; some dimensions of keys are much louder than the others."""
    x = torch.randn((n, heads, hd), generator=g, device="cuda")
    if loud:
        x = x * (1.0 + loud * (torch.rand((heads, hd), generator=g, device="cuda") > 0.95).float())
    return x.to(TORCH[dtype])


def _table(rng, lengths, page):
    """Pages in no order, a few more than needed; a row's unused entries are -1."""
    need = [-(-n // page) for n in lengths]
    total = sum(need) + 3
    perm = rng.permutation(total)
    table = np.full((len(lengths), max(1, max(need))), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, total


def _new_cache(c, table, n_pages):
    """The framework's cache, or pages of plain values (fp8: codes and the exponents of their scales)."""
    shape = (n_pages, c["kv_heads"], c["page"])
    if own:
        import paper_2512_07503_amd as sjd
        return sjd.KvCache(c["cache"], n_pages, c["page"], c["kv_heads"], c["hd"], _ints(table))
    kind = {"fp8": torch.float8_e4m3fn, "bf16": torch.bfloat16, "f32": torch.float32}[c["cache"]]
    pages = [torch.zeros(shape + (c["hd"],), device="cuda").to(kind) for _ in range(2)]
    scales = [torch.zeros(shape, dtype=torch.int32, device="cuda") for _ in range(2)]
    return dict(table=_ints(table).long(), pages=pages, scales=scales, page=c["page"])


def _fill(c, cache, k, v, counts, first):
    starts, first = _ints(_starts(counts)), _ints(first)
    if own:
        import paper_2512_07503_amd as sjd
        sjd.op_cache_write(cache, k, v, starts, first)
    else:
        _plain_write(cache, k, v, *_places(starts, first, int(k.shape[0])))


def _inputs(case, seed):
    """Everything that follows from the seed alone, as plain tensors and lists."""
    c, g, rng = case, _generator(seed), np.random.RandomState(seed % (1 << 31))
    if c["op"] == "rotary":
        n = c["seqs"] * c["rows"]
        first = rng.randint(0, c["far"], size=c["seqs"])
        positions = np.concatenate([np.arange(c["rows"]) + f for f in first])
        qkv = torch.randn((n, (c["heads"] + 2 * c["kv_heads"]) * c["hd"]), generator=g, device="cuda").to(TORCH[c["dtype"]])
        return dict(positions=positions, qkv=qkv)
    counts = _spread(c["nodes"], c["node_spread"], c["seqs"])
    if c["op"] == "verify":
        parents = [_tree(rng, m, c["branch"], c["depth"] if c["branch"] > 1 else m) if m else [] for m in counts]
        starts = _starts(counts)
        n, V = starts[-1], c["vocab"]
        z = torch.randn((n, V), generator=g, device="cuda") * 2.5
        p = torch.softmax(z, dim=1)
        # the draft model sees the same context, less sharply
        q = torch.softmax(0.8 * z + 1.2 * torch.randn((n, V), generator=g, device="cuda"), dim=1)
        del z
        above = [starts[b] + j if j >= 0 else starts[b] for b, t in enumerate(parents) for j in t]
        rank = [t[:i].count(j) for t in parents for i, j in enumerate(t)]
        rows = torch.tensor(above, device="cuda")
        if c["sampled"]:
            # siblings are drawn one by one from their parent's distribution
            order = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
            tokens = torch.zeros(n, dtype=torch.int64, device="cuda")
            for at in range(0, n, 256):
                cdf = torch.cumsum(q[rows[at:at + 256]].double(), dim=1)
                x = (order[at:at + 256] * cdf[:, -1])[:, None]
                tokens[at:at + 256] = torch.searchsorted(cdf, x, right=True)[:, 0].clamp(max=V - 1)
        else:
            best = torch.topk(q, max(rank) + 1, dim=1).indices
            tokens = best[rows, torch.tensor(rank, device="cuda")]
        tokens = tokens.int()
        words = torch.randint(-(1 << 31), 1 << 31, (n,), generator=g, device="cuda", dtype=torch.int64).int()
        draws = torch.randint(-(1 << 62), 1 << 62, (c["seqs"],), generator=g, device="cuda", dtype=torch.int64) * 2
        return dict(counts=counts, parents=parents, tokens=tokens, p=p, q=q if c["sampled"] else None, words=words, draws=draws)
    ctx = _spread(c["ctx"], c["ctx_spread"], c["seqs"]) if c["op"] == "attend" else [c["ctx"]] * c["seqs"]
    back = ctx if c["op"] == "attend" else [min(c["back"], x) for x in ctx]
    if c["op"] == "cache" and c["branch"] == 0 and c["nodes"] > 250:
        ctx, back = [0] * c["seqs"], [0] * c["seqs"]     # a prompt starts its sequence
    parents = [_tree(rng, m, c["branch"]) if m else [] for m in counts] if c["branch"] else [[] for _ in counts]
    table, n_pages = _table(rng, [x + m for x, m in zip(ctx, counts)], c["page"])
    d = dict(counts=counts, ctx=ctx, back=back, parents=parents, table=table, n_pages=n_pages, n=sum(counts))
    for name, m in (("old", sum(back)), ("new", d["n"])):
        d[name] = (_rows(g, m, c["kv_heads"], c["hd"], c["dtype"], 7.0), _rows(g, m, c["kv_heads"], c["hd"], c["dtype"]))
    if c["op"] == "attend":
        d["q"] = _rows(g, d["n"], c["heads"], c["hd"], c["dtype"])
    else:
        d["paths"] = [_path(rng, t) for t in parents]
    return d


def prepare(case, seed):
    c, d = case, _inputs(case, seed)
    if own:
        import paper_2512_07503_amd as sjd
    if c["op"] == "rotary":
        n, hd = d["qkv"].shape[0], c["hd"]
        split = d["qkv"].view(n, -1, hd)        # queries and keys are parts of the fused projection's rows
        state = dict(case=c, q=split[:, :c["heads"]], k=split[:, c["heads"]:c["heads"] + c["kv_heads"]], positions=_ints(d["positions"]))
        if own:
            state["table"] = sjd.rope_table(c["rotary"], theta=10000.0, scaling=c["scaling"], factor=8.0, trained_ctx=8192.0,
                                            low_turns=1.0, high_turns=32.0)
        else:
            state["table"] = _frequencies(c).cuda()
        return state
    if c["op"] == "verify":
        return dict(case=c, starts=_ints(_starts(d["counts"])), parents=_ints([j for t in d["parents"] for j in t]), tokens=d["tokens"],
                    p=d["p"], q=d["q"], words=d["words"], draws=d["draws"], fan=max(t.count(j) for t in d["parents"] for j in [-1] + t))
    cache = _new_cache(c, d["table"], d["n_pages"])
    _fill(c, cache, *d["old"], d["back"], [x - b for x, b in zip(d["ctx"], d["back"])])
    state = dict(case=c, cache=cache, starts=_ints(_starts(d["counts"])), first=_ints(d["ctx"]))
    if c["op"] == "attend":
        _fill(c, cache, *d["new"], d["counts"], d["ctx"])
        words = -(-c["nodes"] // 32)
        mask = np.concatenate([_mask_words(t, words) for t in d["parents"]]) if c["branch"] > 1 else None
        state.update(q=d["q"], mask=None if mask is None else torch.from_numpy(mask.view(np.int32)).cuda(), counts=d["counts"], ctx=d["ctx"])
        return state
    # what is read back: the rows written and up to `back` positions ahead of them
    counts = [b + m for b, m in zip(d["back"], d["counts"])]
    longest = max([len(p) for p in d["paths"]] + [1])
    path = np.full((c["seqs"], longest), -1, dtype=np.int32)
    for b, p in enumerate(d["paths"]):
        path[b, :len(p)] = p
    state.update(k=d["new"][0], v=d["new"][1], read_starts=_ints(_starts(counts)), read_n=sum(counts),
                 read_first=_ints([x - b for x, b in zip(d["ctx"], d["back"])]), path=_ints(path), path_len=_ints([len(p) for p in d["paths"]]))
    kept = np.array([(b, j) for b, p in enumerate(d["paths"]) for j in range(len(p))], dtype=np.int64).reshape(-1, 2)
    state["kept"] = torch.from_numpy(kept[:, 0].copy()).cuda(), torch.from_numpy(kept[:, 1].copy()).cuda()
    return state


# ------------------------------------------------------------------------------------------------------------------ plain forms
def _places(starts, first, n):
    """Sequence and position of every row."""
    rows = torch.arange(n, device="cuda")
    seq = torch.searchsorted(starts[1:].long(), rows, right=True)
    return seq, first.long()[seq] + rows - starts.long()[seq]


def _exponent(x):
    """Smallest e (from -100 to 119) with max |x| <= 448 * 2^e, over the last dimension."""
    mantissa, e = torch.frexp(x.float().abs().amax(dim=-1))
    return torch.where(mantissa <= 0.875, e - 9, e - 8).clamp(-100, 119).int()


def _power(e):
    """2^e in float32, from its bits: a power function may be off in the last one, and a value halfway between two codes then moves."""
    return ((e + 127) << 23).int().view(torch.float32)


def _plain_write(cache, k, v, seq, pos):
    page, slot = cache["table"][seq, pos // cache["page"]], pos % cache["page"]
    for pages, scales, x in zip(cache["pages"], cache["scales"], (k, v)):
        if pages.dtype == torch.float8_e4m3fn:
            e = _exponent(x)
            scales[page, :, slot] = e
            x = (x.float() * _power(-e)[..., None]).clamp(-448.0, 448.0)
        pages.view(torch.uint8 if pages.dtype == torch.float8_e4m3fn else pages.dtype)[page, :, slot] = \
            x.to(pages.dtype).view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else x.to(pages.dtype)


def _plain_read(cache, seq, pos):
    page, slot = cache["table"][seq, pos // cache["page"]], pos % cache["page"]
    out = []
    for pages, scales in zip(cache["pages"], cache["scales"]):
        if pages.dtype == torch.float8_e4m3fn:
            x = pages.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
            out.append(x * _power(scales[page, :, slot])[..., None])
        else:
            out.append(pages[page, :, slot].float())
    return out


def _plain_compact(cache, first, path, kept):
    seq, j = kept
    src, dst = first.long()[seq] + path.long()[seq, j], first.long()[seq] + j
    page = cache["page"]
    for store in cache["pages"] + cache["scales"]:
        store = store.view(torch.uint8) if store.dtype == torch.float8_e4m3fn else store
        store[cache["table"][seq, dst // page], :, dst % page] = store[cache["table"][seq, src // page], :, src % page]


def _plain_rotary(x, positions, frequencies, interleaved, magnitude):
    angle = positions.double()[:, None] * frequencies
    cos, sin = (torch.cos(angle) * magnitude).float()[:, None], (torch.sin(angle) * magnitude).float()[:, None]
    r = 2 * frequencies.shape[0]
    y = x.float().clone()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if interleaved else (y[..., :r // 2], y[..., r // 2:r])
    turned = a * cos - b * sin, b * cos + a * sin
    y[..., :r] = torch.stack(turned, dim=-1).flatten(-2) if interleaved else torch.cat(turned, dim=-1)
    return y.to(x.dtype)


def _plain_attend(s):
    c = s["case"]
    out = torch.empty_like(s["q"])
    at, bits = 0, torch.arange(32, device="cuda")
    for b, (n, ctx) in enumerate(zip(s["counts"], s["ctx"])):
        if n == 0:
            continue
        pos = torch.arange(ctx + n, device="cuda")
        k, v = _plain_read(s["cache"], torch.full_like(pos, b), pos)
        q = s["q"][at:at + n].float().view(n, c["kv_heads"], -1, c["hd"]).permute(1, 0, 2, 3).flatten(1, 2)
        score = torch.matmul(q, k.permute(1, 2, 0).contiguous()) / math.sqrt(c["hd"])
        if s["mask"] is None:
            sees = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        else:
            sees = ((s["mask"][at:at + n, :, None] >> bits) & 1).flatten(1)[:, :n].bool()
        sees = torch.cat([torch.ones((n, ctx), dtype=torch.bool, device="cuda"), sees], dim=1)
        group = c["heads"] // c["kv_heads"]
        score = torch.where(sees.repeat_interleave(group, dim=0)[None], score, torch.full_like(score, -math.inf))
        weight = torch.exp(score - score.amax(dim=-1, keepdim=True))
        o = torch.matmul(weight, v.permute(1, 0, 2).contiguous()) / weight.sum(dim=-1, keepdim=True)
        out[at:at + n] = o.view(c["kv_heads"], n, group, c["hd"]).permute(1, 0, 2, 3).reshape(n, c["heads"], c["hd"]).to(out.dtype)
        at += n
    return out


def _product_high(u, z):
    """floor(u z / 2^64) of an unsigned 64-bit u (in the bits of an int64) and 0 <= z < 2^48, in digits of 16 bits."""
    u = [(u >> (16 * i)) & 0xFFFF for i in range(4)]
    z = [(z >> (16 * i)) & 0xFFFF for i in range(3)]
    carry, out = torch.zeros_like(u[0]), torch.zeros_like(u[0])
    for k in range(7):
        digit = carry + sum(u[i] * z[k - i] for i in range(4) if 0 <= k - i < 3) if k < 6 else carry
        carry = digit >> 16
        if k >= 4:
            out = out + ((digit & 0xFFFF) << (16 * (k - 4)))
    return out


def _weights(rho):
    return (rho.clamp(0.0, 1.0) * 2.0 ** 44).long()


def _plain_verify(s):
    c = s["case"]
    B, N, V = c["seqs"], c["nodes"], c["vocab"]
    starts, p, q = s["starts"].long(), s["p"], s["q"]
    counts = starts[1:] - starts[:-1]
    n = p.shape[0]
    node = torch.arange(N, device="cuda")[None].expand(B, N)
    inside = node < counts[:, None]
    row = (starts[:-1, None] + node).clamp(max=n - 1)
    parents = torch.where(inside, s["parents"].long()[row], torch.full_like(node, -2))
    earlier = (parents[:, :, None] == parents[:, None, :]) & (node[:, None, :] < node[:, :, None])
    rank = earlier.sum(dim=2)
    depth = c["depth"] if c["branch"] > 1 else N
    path = torch.full((B, depth + 1), -1, dtype=torch.int64, device="cuda")
    some = counts > 0
    path[:, 0] = torch.where(some, torch.zeros_like(counts), path[:, 0])
    length = some.long()
    cur = torch.zeros_like(counts)
    moving = some.clone()
    rho = p[row[:, 0]].double()
    for level in range(1, depth + 1):
        total = torch.ones(B, dtype=torch.float64, device="cuda")
        base = p[row.gather(1, cur[:, None])[:, 0]].double()
        rho = torch.where(moving[:, None], base, rho)
        prop = q[row.gather(1, cur[:, None])[:, 0]].double() if q is not None else None
        testing, found, at = moving.clone(), torch.zeros_like(moving), cur.clone()
        for k in range(s["fan"]):
            match = (parents == cur[:, None]) & (rank == k)
            testing = testing & match.any(dim=1)
            child = match.long().argmax(dim=1)
            r = row.gather(1, child[:, None])[:, 0]
            x = s["tokens"].long()[r][:, None]
            chance = ((s["words"].long()[r] & 0xFFFFFFFF).double() + 0.5) * 2.0 ** -32
            rho_x = rho.gather(1, x)[:, 0]
            q_x = prop.gather(1, x)[:, 0] if q is not None else torch.ones_like(rho_x)
            accept = testing & (chance * q_x * total < rho_x)
            found, at = found | accept, torch.where(accept, child, at)
            testing = testing & ~accept
            if q is not None:
                less = (rho - total[:, None] * prop).clamp(min=0.0)
            else:
                less = rho.scatter(1, x, 0.0)
            rho = torch.where(testing[:, None], less, rho)
            total = torch.where(testing, _weights(less).sum(dim=1).double() * 2.0 ** -44, total)
        cur = at
        moving = found
        path[:, level] = torch.where(found, cur, path[:, level])
        length = length + found.long()
    # the deepest level's acceptances draw from their own rows
    rho = torch.where(moving[:, None], p[row.gather(1, cur[:, None])[:, 0]].double(), rho)
    w = _weights(rho)
    w = torch.where(w.sum(dim=1, keepdim=True) > 0, w, _weights(p[row.gather(1, cur[:, None])[:, 0]].double()))
    cdf = torch.cumsum(w, dim=1)
    t = _product_high(s["draws"], cdf[:, -1])
    token = (cdf <= t[:, None]).sum(dim=1)
    token = torch.where(some, token, torch.full_like(token, -1))
    return path.int(), length.int(), token.int()


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2512_07503_amd as sjd
    if c["op"] == "rotary":
        if own:
            return sjd.op_rotary(s["q"], s["k"], s["positions"], s["table"], interleaved=c["interleaved"], magnitude=_magnitude(c))
        return tuple(_plain_rotary(x, s["positions"], s["table"], c["interleaved"], _magnitude(c)) for x in (s["q"], s["k"]))
    if c["op"] == "cache":
        if own:
            sjd.op_cache_write(s["cache"], s["k"], s["v"], s["starts"], s["first"])
            if c["branch"]:
                sjd.op_cache_compact(s["cache"], s["first"], s["path"], s["path_len"])
            return sjd.op_cache_read(s["cache"], s["read_starts"], s["read_first"], s["read_n"], dtype=s["k"].dtype)
        _plain_write(s["cache"], s["k"], s["v"], *_places(s["starts"], s["first"], s["k"].shape[0]))
        if c["branch"]:
            _plain_compact(s["cache"], s["first"], s["path"], s["kept"])
        return tuple(x.to(s["k"].dtype) for x in _plain_read(s["cache"], *_places(s["read_starts"], s["read_first"], s["read_n"])))
    if c["op"] == "attend":
        if own:
            return sjd.op_tree_attention(s["q"], s["cache"], s["starts"], s["first"], mask=s["mask"], max_rows=c["nodes"], max_ctx=c["ctx"])
        return _plain_attend(s)
    if own:
        return sjd.op_tree_verify(s["tokens"], s["parents"], s["starts"], s["p"], s["q"], s["words"], s["draws"], max_rows=c["nodes"],
                                  max_path=(c["depth"] if c["branch"] > 1 else c["nodes"]) + 1)
    return _plain_verify(s)


# ------------------------------------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    size = {"f32": 4, "bf16": 2, "fp8": 1}
    if c["op"] == "rotary":
        n, heads = c["seqs"] * c["rows"], c["heads"] + c["kv_heads"]
        return dict(bytes=2 * n * heads * c["hd"] * size[c["dtype"]] + 4 * n, flops=3 * n * heads * c["rotary"])
    counts = _spread(c["nodes"], c["node_spread"], c["seqs"])
    if c["op"] == "verify":
        # a row of each distribution a sequence; the tests along the path read single values
        live = sum(1 for m in counts if m)
        rows = 2 if c["sampled"] else 1
        return dict(bytes=live * rows * c["vocab"] * 4 + 12 * sum(counts), flops=3.0 * live * c["vocab"])
    entry = 2 * c["kv_heads"] * (c["hd"] * size[c["cache"]] + (1 if c["cache"] == "fp8" else 0))    # a position's keys and values
    if c["op"] == "cache":
        plain = 2 * c["kv_heads"] * c["hd"] * size[c["dtype"]]
        back = c["seqs"] * min(c["back"], c["ctx"]) if not (c["branch"] == 0 and c["nodes"] > 250) else 0
        n = sum(counts)
        return dict(bytes=n * (plain + entry) + (n + back) * (plain + entry), flops=2.0 * n * 2 * c["kv_heads"] * c["hd"])
    ctx = _spread(c["ctx"], c["ctx_spread"], c["seqs"])
    cached = sum(x + m for x, m in zip(ctx, counts) if m)
    seen = sum(m * (x + 1) for x, m in zip(ctx, counts))
    return dict(bytes=cached * entry + 2 * sum(counts) * c["heads"] * c["hd"] * size[c["dtype"]], flops=4.0 * seen * c["heads"] * c["hd"])


# ------------------------------------------------------------------------------------------------------------------------ exact
def _exact_stored(c, x):
    """What the cache holds for x, in float64."""
    x = x.double()
    if c["cache"] == "f32":
        return x
    if c["cache"] == "bf16":
        return x.bfloat16().double()
    def two_to(e):
        return ((e.long() + 1023) << 52).view(torch.float64)

    top = x.abs().amax(dim=-1, keepdim=True)
    e = (torch.frexp(top).exponent - 9).clamp(-100, 119)      # top < 512 * 2^e
    e = torch.where(448.0 * two_to(e) < top, e + 1, e).clamp(-100, 119)
    y = (x / two_to(e)).clamp(-448.0, 448.0)
    step = two_to((torch.frexp(y).exponent - 1).clamp(min=-6) - 3)      # three bits behind the leading one
    return torch.round(y / step) * step * two_to(e)


def _exact_verify(c, d):
    # The distributions stay on the GPU; a sequence's visited rows come to the host one at a time.  The word of a test and the
    # products with the remaining mass are formed in the order of the definition: ((r q) S) against rho.
    depth = c["depth"] if c["branch"] > 1 else c["nodes"]
    starts = _starts(d["counts"])
    tokens, words, draws = (d[k].cpu().numpy() for k in ("tokens", "words", "draws"))
    path, length, token = np.full((c["seqs"], depth + 1), -1, np.int32), np.zeros(c["seqs"], np.int32), np.full(c["seqs"], -1, np.int32)
    for b, parents in enumerate(d["parents"]):
        if not parents:
            continue
        cur, walk = 0, [0]
        while True:
            target = d["p"][starts[b] + cur].cpu().numpy().astype(np.float64)
            draft = d["q"][starts[b] + cur].cpu().numpy().astype(np.float64) if d["q"] is not None else None
            rho, mass, step = target.copy(), 1.0, None
            for i in [i for i, j in enumerate(parents) if j == cur] if len(walk) <= depth else []:
                x = int(tokens[starts[b] + i])
                r = (float(int(words[starts[b] + i]) & 0xFFFFFFFF) + 0.5) / 2.0 ** 32
                if r * (draft[x] if draft is not None else 1.0) * mass < rho[x]:
                    step = i
                    break
                if draft is not None:
                    rho = np.maximum(rho - mass * draft, 0.0)
                else:
                    rho[x] = 0.0
                mass = float(np.floor(np.minimum(rho, 1.0) * 2.0 ** 44).sum()) / 2.0 ** 44
            if step is None:
                break
            cur = step
            walk.append(step)
        w = np.floor(np.minimum(rho, 1.0) * 2.0 ** 44).astype(np.int64)
        if w.sum() == 0:
            w = np.floor(np.minimum(target, 1.0) * 2.0 ** 44).astype(np.int64)
        cdf = np.cumsum(w)
        u = int(draws[b]) & 0xFFFFFFFFFFFFFFFF
        token[b] = np.searchsorted(cdf, (u * int(cdf[-1])) >> 64, side="right")
        path[b, :len(walk)], length[b] = walk, len(walk)
    return path, length, token


def exact(case, seed):
    c, d = case, _inputs(case, seed)
    if c["op"] == "verify":
        return tuple(torch.from_numpy(x).cuda() for x in _exact_verify(c, d))
    if c["op"] == "rotary":
        n, hd, r = d["qkv"].shape[0], c["hd"], c["rotary"]
        x = d["qkv"].view(n, -1, hd)[:, :c["heads"] + c["kv_heads"]].double()
        angle = torch.from_numpy(d["positions"]).cuda().double()[:, None] * _frequencies(c).cuda()
        turn = torch.polar(torch.full_like(angle, _magnitude(c)), angle)[:, None]
        first = torch.arange(0, r, 2, device="cuda") if c["interleaved"] else torch.arange(r // 2, device="cuda")
        second = first + (1 if c["interleaved"] else r // 2)
        y = x.clone()
        for at in range(0, n, 2048):      # complex numbers: a pair is turned by a product
            z = torch.complex(x[at:at + 2048][..., first], x[at:at + 2048][..., second]) * turn[at:at + 2048]
            y[at:at + 2048, :, first], y[at:at + 2048, :, second] = z.real, z.imag
        return y[:, :c["heads"]], y[:, c["heads"]:]
    old, new = ([_exact_stored(c, x) for x in d[name]] for name in ("old", "new"))
    oat, nat = _starts(d["back"]), _starts(d["counts"])
    if c["op"] == "cache":
        out = ([], [])
        for b in range(c["seqs"]):
            for side in (0, 1):
                rows = new[side][nat[b]:nat[b + 1]].clone()
                if c["branch"] and d["paths"][b]:
                    rows[:len(d["paths"][b])] = new[side][nat[b]:nat[b + 1]][d["paths"][b]]
                out[side].append(torch.cat([old[side][oat[b]:oat[b + 1]], rows]))
        return torch.cat(out[0]), torch.cat(out[1])
    out = torch.zeros((d["n"], c["heads"], c["hd"]), dtype=torch.float64, device="cuda")
    for b, parents in enumerate(d["parents"]):
        n, ctx = d["counts"][b], d["ctx"][b]
        if n == 0:
            continue
        k, v = (torch.cat([old[side][oat[b]:oat[b + 1]], new[side][nat[b]:nat[b + 1]]]).permute(1, 0, 2) for side in (0, 1))
        hidden = torch.ones((n, n), dtype=torch.bool)
        for i in range(n):
            j = i
            while j >= 0:
                hidden[i, j] = False
                j = parents[j]
        hidden = torch.cat([torch.zeros((n, ctx), dtype=torch.bool), hidden], dim=1).cuda()
        q = d["q"][nat[b]:nat[b + 1]].double()
        for h in range(c["heads"]):
            of = h // (c["heads"] // c["kv_heads"])
            logits = (q[:, h] @ k[of].T / math.sqrt(c["hd"])).masked_fill(hidden, -math.inf)
            out[nat[b]:nat[b + 1], h] = torch.softmax(logits, dim=-1) @ v[of]
    return out
