"""The operators of scoring and prefilling prompts, as they are measured: norms of queries and keys for each head with the position rotation
in the same pass, causal attention over packed prompts, and log probabilities of given tokens with entropy and top alternatives.

Sequences are ragged: rows [row_start[b], row_start[b + 1]) are sequence b's queries, and where a sequence continues what is cached, its keys and
values are rows [kv_start[b], kv_start[b + 1]), the last of which are its queries' own.  Shapes come from this repository's configurations
(workload/configs.py: 4 heads of 64 in fp32, 20 heads of 64, 32 heads of 128 with 32 or 8 key/value heads, vocabularies of 16 384 to 184 622 with
a sampled range, prompts of 64 and 120 tokens, images of 2 352) or are generic.
"""
import math

import numpy as np
import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ------------------------------------------------------------------------------------------------------------------------ cases
def _norm(seqs, rows, heads, kv_heads, hd, rotary, interleaved, norm, per_head, bias, dtype, far):
    return dict(op="norm", seqs=seqs, rows=rows, heads=heads, kv_heads=kv_heads, hd=hd, rotary=rotary, interleaved=interleaved, norm=norm,
                per_head=per_head, bias=bias, dtype=dtype, far=far)


def _attend(seqs, rows, spread, prefix, prefix_spread, heads, kv_heads, hd, dtype):
    """prefix 0: the keys are the queries' own; else that many cached ones come before them (prefix_spread fewer for the last sequence)."""
    return dict(op="attend", seqs=seqs, rows=rows, spread=spread, prefix=prefix, prefix_spread=prefix_spread, heads=heads, kv_heads=kv_heads,
                hd=hd, dtype=dtype)


def _score(rows, vocab, lo, hi, top, dtype):
    """Ids outside [lo, hi) are masked: their logits are -inf."""
    return dict(op="score", rows=rows, vocab=vocab, lo=lo, hi=hi, top=top, dtype=dtype)


def listed():
    return [
        # one token of each of eight sequences: what every layer of a decoding step runs, pure latency
        dict(_norm(8, 1, 32, 8, 128, 128, False, "rms", False, False, "bf16", 4096), name="norm_token"),
        # two long documents, grouped heads, one gain for all heads
        dict(_norm(2, 6001, 32, 8, 128, 128, False, "rms", False, False, "bf16", 200000), name="norm_prompt"),
        # four images of the wide model, mean and variance, a gain and a bias for each head
        dict(_norm(4, 2352, 32, 32, 128, 128, False, "layer", True, True, "bf16", 100), name="norm_image"),
        # one prompt of the narrow model: the smallest call
        dict(_attend(1, 120, 0, 0, 0, 20, 20, 64, "bf16"), name="attend_prompt"),
        # the tiny fp32 model's prompts and images as one batch
        dict(_attend(8, 288, 256, 0, 0, 4, 4, 64, "f32"), name="attend_f32"),
        # a batch of twelve prompts between a caption and an image, no two alike
        dict(_attend(12, 2352, 2291, 0, 0, 32, 32, 128, "bf16"), name="attend_packed"),
        # one long document, grouped heads
        dict(_attend(1, 16001, 0, 0, 0, 32, 8, 128, "bf16"), name="attend_long"),
        # the next 500 rows of two long documents that are cached already
        dict(_attend(2, 500, 87, 30011, 9000, 32, 8, 128, "bf16"), name="attend_chunk"),
        # a decoding step's rows, with five alternatives: latency
        dict(_score(8, 16384, 0, 16384, 5, "f32"), name="score_token"),
        # windows of 32 of eight sequences, twenty alternatives each
        dict(_score(256, 65536, 0, 65536, 20, "f32"), name="score_window"),
        # only a part of a wide vocabulary may be sampled; odd rows, whose addresses are not aligned
        dict(_score(33, 184621, 151854, 184621, 20, "bf16"), name="score_masked"),
        # a prompt of 4 099 tokens scored
        dict(_score(4099, 65536, 0, 65536, 0, "bf16"), name="score_prompt"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(("norm", "attend", "attend", "score"))
    if op == "score":
        rows, vocab = _log_int(rng, 1, 5000), _log_int(rng, 500, 200000)
        lo = 0 if rng.random() < 0.5 else rng.randint(0, vocab // 2)
        hi = vocab if rng.random() < 0.5 else rng.randint(lo + 1, vocab)
        return _score(rows, vocab, lo, hi, rng.choice((0, 0, 1, 5, 8, 20, 64)), rng.choice(("f32", "bf16")))
    seqs = _log_int(rng, 1, 24)
    kv_heads = _log_int(rng, 1, 20)
    heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 5, 8))
    hd = rng.choice((32, 64, 64, 96, 128, 128, 192, 256))
    if op == "norm":
        return _norm(seqs, _log_int(rng, 1, 6000), heads, kv_heads, hd, 2 * rng.randint(1, hd // 2) if rng.random() < 0.3 else hd,
                     rng.random() < 0.4, rng.choice(("rms", "layer")), rng.random() < 0.4, rng.random() < 0.4, rng.choice(("f32", "bf16")),
                     _log_int(rng, 1, 1000000))
    rows = _log_int(rng, 1, 8000)
    prefix = 0 if rng.random() < 0.6 else _log_int(rng, 1, 40000)
    return _attend(seqs, rows, rng.randint(0, rows), prefix, rng.randint(0, prefix), heads, kv_heads, hd, rng.choice(("bf16", "bf16", "bf16", "f32")))


def draw(rng):
    """One more case over the ranges of the listed ones, none dearer than the dearest of its operator (and fp32 attention, whose products
    run at a sixteenth of the rate, a sixteenth of that)."""
    limit = {}
    for c in listed():
        w = work(c)
        limit[c["op"]] = max(limit.get(c["op"], 0.0), w["bytes"] + w["flops"] / 300)
    while True:
        c = _draw_once(rng)
        w = work(c)
        share = 1 / 16 if c["op"] == "attend" and c["dtype"] == "f32" else 1
        if w["bytes"] + w["flops"] / 300 <= share * limit[c["op"]]:
            return c


# ----------------------------------------------------------------------------------------------------------------------- inputs
def _spread(n, spread, seqs):
    return [n - (spread * s // (seqs - 1) if seqs > 1 else 0) for s in range(seqs)]


def _lengths(c):
    """Queries and keys of every sequence."""
    rows = _spread(c["rows"], c["spread"], c["seqs"])
    return rows, [n + p for n, p in zip(rows, _spread(c["prefix"], c["prefix_spread"], c["seqs"]))]


def _starts(counts):
    return [0] + np.cumsum(counts).tolist()


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device="cuda")


def _frequencies(r):
    return 10000.0 ** (-2.0 * torch.arange(r // 2, dtype=torch.float64, device="cuda") / r)


def _inputs(case, seed):
    """Everything that follows from the seed alone, as plain tensors."""
    c, g, rng = case, _generator(seed), np.random.RandomState(seed % (1 << 31))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if c["op"] == "norm":
        n, kind = c["seqs"] * c["rows"], TORCH[c["dtype"]]
        first = rng.randint(0, c["far"], size=c["seqs"])
        positions = np.concatenate([np.arange(c["rows"]) + f for f in first])
        # queries, keys and values of a fused projection; heads differ in size, and their elements are not centred
        heads = c["heads"] + 2 * c["kv_heads"]
        qkv = ((normal(n, heads, c["hd"]) + 0.3) * torch.exp(normal(heads, 1))).to(kind)
        gains = [(1.0 + 0.3 * normal(*((h, c["hd"]) if c["per_head"] else (c["hd"],)))).to(kind) for h in (c["heads"], c["kv_heads"])]
        biases = [(0.1 * normal(*x.shape)).to(kind) if c["bias"] else None for x in gains]
        return dict(positions=positions, qkv=qkv, gains=gains, biases=biases)
    if c["op"] == "attend":
        rows, keys = _lengths(c)
        kind = TORCH[c["dtype"]]
        if c["prefix"]:
            q = (2.0 * normal(sum(rows), c["heads"], c["hd"])).to(kind)      # scores of a few units, as trained heads have
            k, v = (normal(sum(keys), c["kv_heads"], c["hd"]).to(kind) for _ in range(2))
        else:       # parts of a fused projection's rows
            qkv = normal(sum(rows), c["heads"] + 2 * c["kv_heads"], c["hd"])
            qkv[:, :c["heads"]] *= 2.0
            qkv = qkv.to(kind)
            q, k, v = qkv.split([c["heads"], c["kv_heads"], c["kv_heads"]], dim=1)
        return dict(rows=rows, keys=keys, q=q, k=k, v=v)
    n, V, kind = c["rows"], c["vocab"], TORCH[c["dtype"]]
    z = torch.empty((n, V), dtype=kind, device="cuda")
    for at in range(0, n, 512):
        part = normal(min(512, n - at), V) * 2.5
        part[:, :c["lo"]] = -math.inf
        part[:, c["hi"]:] = -math.inf
        z[at:at + 512] = part.to(kind)
    # half of the tokens are the likeliest ones
    tokens = torch.randint(c["lo"], c["hi"], (n,), generator=g, device="cuda")
    best = torch.cat([z[at:at + 512].argmax(dim=1) for at in range(0, n, 512)])
    tokens = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, best, tokens)
    return dict(z=z, tokens=tokens.int())


def prepare(case, seed):
    c, d = case, _inputs(case, seed)
    if c["op"] == "norm":
        split = d["qkv"]
        state = dict(case=c, q=split[:, :c["heads"]], k=split[:, c["heads"]:c["heads"] + c["kv_heads"]], positions=_ints(d["positions"]),
                     gains=d["gains"], biases=d["biases"])
        if own:
            import paper_2512_07503_amd as sjd
            state["table"] = sjd.rope_table(c["rotary"], theta=10000.0)
        else:
            state["table"] = _frequencies(c["rotary"])
        return state
    if c["op"] == "attend":
        return dict(case=c, q=d["q"], k=d["k"], v=d["v"], starts=_ints(_starts(d["rows"])), kv_starts=_ints(_starts(d["keys"])), rows=d["rows"],
                    keys=d["keys"])
    return dict(case=c, z=d["z"], tokens=d["tokens"])


# ------------------------------------------------------------------------------------------------------------------ plain forms
def _plain_norm_rotary(x, positions, frequencies, interleaved, norm, gain, bias):
    y = x.float()
    if norm == "layer":
        y = y - y.mean(dim=-1, keepdim=True)
    y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + 1e-5) * gain.float()
    if bias is not None:
        y = y + bias.float()
    angle = positions.double()[:, None] * frequencies
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    r = 2 * frequencies.shape[0]
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if interleaved else (y[..., :r // 2], y[..., r // 2:r])
    turned = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack(turned, dim=-1).flatten(-2) if interleaved else torch.cat(turned, dim=-1)
    return torch.cat([turned, y[..., r:]], dim=-1).to(x.dtype)


def _plain_attend(s):
    c = s["case"]
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    group, at, kat = c["heads"] // c["kv_heads"], 0, 0
    for n, total in zip(s["rows"], s["keys"]):
        k = s["k"][kat:kat + total].float().permute(1, 2, 0).contiguous()
        v = s["v"][kat:kat + total].float().permute(1, 0, 2).contiguous()
        step = max(1, (1 << 30) // max(1, c["heads"] * total))
        for i in range(0, n, step):
            m = min(step, n - i)
            q = s["q"][at + i:at + i + m].float().view(m, c["kv_heads"], group, c["hd"]).permute(1, 2, 0, 3).flatten(1, 2)
            score = torch.matmul(q, k).view(c["kv_heads"], group, m, total) / math.sqrt(c["hd"])
            hidden = torch.arange(total, device="cuda")[None] > torch.arange(i, i + m, device="cuda")[:, None] + (total - n)
            score = score.masked_fill(hidden, -math.inf)
            weight = torch.exp(score - score.amax(dim=-1, keepdim=True))
            o = torch.matmul(weight.flatten(1, 2), v).view(c["kv_heads"], group, m, c["hd"]) / weight.sum(dim=-1, keepdim=True)
            out[at + i:at + i + m] = o.permute(2, 0, 1, 3).flatten(1, 2).to(out.dtype)
        at, kat = at + n, kat + total
    return out


def _order(z):
    """Whole numbers in the order of the floats (-0 is 0)."""
    bits = (z + 0.0).view(torch.int32)
    return torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)


def _plain_score(s):
    z, tokens, top = s["z"].float(), s["tokens"].long()[:, None], s["case"]["top"]
    best = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - best)
    total = e.sum(dim=1, keepdim=True)
    rest = torch.log(total)
    of_token = z.gather(1, tokens)
    ids = torch.arange(z.shape[1], device="cuda")
    rank = ((z > of_token) | ((z == of_token) & (ids < tokens))).sum(dim=1)
    entropy = rest - torch.where(e > 0, e * (z - best), torch.zeros_like(e)).sum(dim=1, keepdim=True) / total
    result = (of_token - best - rest)[:, 0], rank.int(), entropy[:, 0]
    if not top:
        return result
    key = (_order(z).long() << 32) + ((1 << 24) - ids)       # equal logits: the lower id first
    at = torch.topk(key, min(top, z.shape[1]), dim=1).indices
    at = torch.cat([at, at.new_zeros((at.shape[0], top - at.shape[1]))], dim=1)
    of_top = z.gather(1, at)
    real = (of_top > -math.inf) & (torch.arange(top, device="cuda") < z.shape[1])
    return result + (torch.where(real, at, torch.full_like(at, -1)).int(), torch.where(real, of_top - best - rest, torch.full_like(of_top, -math.inf)))


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2512_07503_amd as sjd
    if c["op"] == "norm":
        if own:
            return sjd.op_norm_rotary(s["q"], s["k"], s["positions"], s["table"], s["gains"][0], s["gains"][1], q_bias=s["biases"][0],
                                      k_bias=s["biases"][1], norm=c["norm"], eps=1e-5, interleaved=c["interleaved"])
        return tuple(_plain_norm_rotary(x, s["positions"], s["table"], c["interleaved"], c["norm"], s["gains"][i], s["biases"][i])
                     for i, x in enumerate((s["q"], s["k"])))
    if c["op"] == "attend":
        if own:
            return sjd.op_prompt_attention(s["q"], s["k"], s["v"], s["starts"], kv_start=s["kv_starts"] if c["prefix"] else None,
                                           max_rows=c["rows"], max_kv=max(s["keys"]))
        return _plain_attend(s)
    if own:
        logprob, rank, entropy, ids, alternatives = sjd.op_token_logprobs(s["z"], s["tokens"], n_top=c["top"])
        return (logprob, rank, entropy) + ((ids, alternatives) if c["top"] else ())
    return _plain_score(s)


# ------------------------------------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    if c["op"] == "norm":
        elements = c["seqs"] * c["rows"] * (c["heads"] + c["kv_heads"]) * c["hd"]
        return dict(bytes=2 * elements * SIZE[c["dtype"]] + 4 * c["seqs"] * c["rows"], flops=8.0 * elements)
    if c["op"] == "attend":
        rows, keys = _lengths(c)
        seen = sum(n * (t - n) + n * (n + 1) / 2 for n, t in zip(rows, keys))
        size = SIZE[c["dtype"]] * c["hd"]
        live = sum(t for n, t in zip(rows, keys) if n)
        return dict(bytes=2 * size * (sum(rows) * c["heads"] + live * c["kv_heads"]), flops=4.0 * seen * c["heads"] * c["hd"])
    return dict(bytes=c["rows"] * (c["vocab"] * SIZE[c["dtype"]] + 16 + 8 * c["top"]), flops=5.0 * c["rows"] * c["vocab"])


# ------------------------------------------------------------------------------------------------------------------------ exact
def exact(case, seed):
    c, d = case, _inputs(case, seed)
    if c["op"] == "norm":
        out, at, r = [], 0, c["rotary"]
        positions = torch.from_numpy(d["positions"]).cuda().double()
        first = torch.arange(0, r, 2, device="cuda") if c["interleaved"] else torch.arange(r // 2, device="cuda")
        second = first + (1 if c["interleaved"] else r // 2)
        turn = torch.polar(torch.ones((len(d["positions"]), r // 2), dtype=torch.float64, device="cuda"), positions[:, None] * _frequencies(r))
        for heads, gain, bias in zip((c["heads"], c["kv_heads"]), d["gains"], d["biases"]):
            y = torch.empty((len(d["positions"]), heads, c["hd"]), dtype=torch.float64, device="cuda")
            for i in range(0, y.shape[0], 2048):
                x = d["qkv"][i:i + 2048, at:at + heads].double()
                centre = x.mean(dim=-1, keepdim=True) if c["norm"] == "layer" else torch.zeros_like(x[..., :1])
                x = (x - centre) / torch.sqrt(((x - centre) ** 2).sum(dim=-1, keepdim=True) / c["hd"] + 1e-5) * gain.double()
                x = x + bias.double() if bias is not None else x
                z = torch.complex(x[..., first], x[..., second]) * turn[i:i + 2048, None]      # a pair is turned by a product
                x[..., first], x[..., second] = z.real, z.imag
                y[i:i + 2048] = x
            out.append(y)
            at += heads
        return tuple(out)
    if c["op"] == "attend":
        out, at, kat = torch.zeros(d["q"].shape, dtype=torch.float64, device="cuda"), 0, 0
        for n, total in zip(d["rows"], d["keys"]):
            for h in range(c["heads"] if n else 0):
                of = h // (c["heads"] // c["kv_heads"])
                keys, values = d["k"][kat:kat + total, of].double(), d["v"][kat:kat + total, of].double()
                for i in range(0, n, 4096):
                    m = min(4096, n - i)
                    logits = d["q"][at + i:at + i + m, h].double() @ keys.T / math.sqrt(c["hd"])
                    sees = torch.ones((m, total), dtype=torch.bool, device="cuda").tril(i + total - n)
                    out[at + i:at + i + m, h] = torch.softmax(torch.where(sees, logits, -math.inf), dim=-1) @ values
            at, kat = at + n, kat + total
        return out
    n, top, parts = c["rows"], c["top"], []
    for i in range(0, n, 256):
        z = d["z"][i:i + 256].double()
        logp = z - torch.logsumexp(z, dim=1, keepdim=True)
        token = d["tokens"][i:i + 256].long()[:, None]
        mine = logp.gather(1, token)
        entropy = -torch.where(logp > -math.inf, torch.exp(logp) * logp, 0.0).sum(dim=1)
        before = (z > z.gather(1, token)).sum(dim=1) + ((z == z.gather(1, token)).cumsum(dim=1).gather(1, token)[:, 0] - 1)
        part = [mine[:, 0], before.int(), entropy]
        if top:
            order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
            order = torch.nn.functional.pad(order, (0, top - order.shape[1]))
            value = logp.gather(1, order)
            value[:, c["vocab"]:] = -math.inf
            part += [torch.where(value > -math.inf, order, -1).int(), value]
        parts.append(part)
    return tuple(torch.cat(x) for x in zip(*parts))
