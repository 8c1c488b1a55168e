"""The operators of a step of tree speculation together, as a serving loop uses them: rotate, write, attend, verify, keep the accepted path.
Against the same loop in 64 bits over plain arrays; run eagerly, captured and replayed, and on another stream."""
import numpy as np
import pytest

import tree_oracle
from test_gpu_cache import host, i32, make

pytestmark = pytest.mark.gpu
H, HKV, HD, V = 4, 2, 64, 300


class Loop:
    """Trees of the same shape for every sequence; a step's projections are given.  All state lives on the device."""

    def __init__(self, kind, seqs, nodes, seed):
        import paper_2512_07503_amd as sjd
        import torch
        self.rng = np.random.default_rng(seed)
        self.kind, self.seqs, self.nodes = kind, seqs, nodes
        self.td = torch.float32 if kind == "f32" else torch.bfloat16
        self.parents = tree_oracle.random_tree(self.rng, nodes, 3)
        mask, self.depth = sjd.tree_masks(self.parents)
        self.cache, _ = make(kind, 64, HKV, HD, [400] * seqs, seed)
        n = seqs * nodes
        self.mask = torch.from_numpy(np.tile(mask, (seqs, 1)).view(np.int32)).cuda()
        self.depths = i32(np.tile(self.depth, seqs))
        self.parents_dev, self.starts = i32(np.tile(self.parents, seqs)), i32(np.arange(seqs + 1) * nodes)
        self.seq = torch.arange(seqs, device="cuda").repeat_interleave(nodes)
        self.table = sjd.rope_table(HD, theta=500.0)
        self.ctx = i32([0, 31, 60, 7][:seqs])
        # inputs of a step
        self.q, self.k, self.v = (torch.zeros((n, h, HD), dtype=self.td, device="cuda") for h in (H, HKV, HKV))
        self.tokens, self.words = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        self.p, self.qd = torch.zeros((n, V), device="cuda"), torch.zeros((n, V), device="cuda")
        self.draws = torch.zeros(seqs, dtype=torch.int64, device="cuda")

    def feed(self):
        import torch
        n = self.seqs * self.nodes
        for x in (self.q, self.k, self.v):
            x.copy_(torch.from_numpy(self.rng.standard_normal(x.shape).astype(np.float32)))
        z = torch.from_numpy(self.rng.standard_normal((n, V)).astype(np.float32)).cuda() * 2
        self.p.copy_(torch.softmax(z, 1))
        self.qd.copy_(torch.softmax(z + 0.7 * torch.from_numpy(self.rng.standard_normal((n, V)).astype(np.float32)).cuda(), 1))
        q = self.qd.double().cpu().numpy()
        above = [b * self.nodes + max(j, 0) for b in range(self.seqs) for j in self.parents]
        self.tokens.copy_(torch.tensor([min(int(np.searchsorted(np.cumsum(q[r]) / q[r].sum(), self.rng.random(), side="right")), V - 1) for r in above]))
        self.words.copy_(torch.from_numpy(self.rng.integers(0, 1 << 32, n, dtype=np.uint64).astype(np.uint32).view(np.int32)))
        self.draws.copy_(torch.from_numpy(self.rng.integers(0, 1 << 64, self.seqs, dtype=np.uint64).view(np.int64)))

    def step(self):
        import paper_2512_07503_amd as sjd
        positions = self.ctx[self.seq] + self.depths
        q, k = sjd.op_rotary(self.q, self.k, positions, self.table)
        sjd.op_cache_write(self.cache, k, self.v, self.starts, self.ctx)
        out = sjd.op_tree_attention(q, self.cache, self.starts, self.ctx, mask=self.mask, max_rows=self.nodes, max_ctx=400)
        path, length, token = sjd.op_tree_verify(self.tokens, self.parents_dev, self.starts, self.p, self.qd, self.words, self.draws, max_rows=self.nodes, max_path=8)
        sjd.op_cache_compact(self.cache, self.ctx, path, length)
        self.ctx += length
        return q, k, out, path, length, token


class Plain:
    """The same in 64 bits.  It stores the keys that the GPU rotated (they are rounded; their own test holds them to 64 bits)."""

    def __init__(self, loop):
        self.l = loop
        self.store = [[np.zeros((c, HKV, HD)) for c in loop.ctx.cpu().tolist()] for _ in range(2)]

    def step(self, outs):
        l = self.l
        q, k, out, path, length, token = (x.double().cpu().numpy() for x in outs)
        sees = tree_oracle.ancestors(l.parents)
        for b in range(l.seqs):
            r = slice(b * l.nodes, (b + 1) * l.nodes)
            ctx = len(self.store[0][b])
            pos = ctx + l.depth
            for got, x in ((q, l.q), (k, l.k)):
                want, size = tree_oracle.rotary(host(x)[r], pos, tree_oracle.frequencies(HD, 500.0), False)
                assert (np.abs(got[r] - want) <= 2.0 ** -21 * size + (2.0 ** -24 if l.kind == "f32" else 2.0 ** -8) * np.abs(want)).all()
            kk, vv = (np.concatenate([s[b], tree_oracle.store(l.kind, x[r])]) for s, x in zip(self.store, (k, host(l.v))))
            want, size, dot = tree_oracle.attention(q[r], kk, vv, np.concatenate([np.ones((l.nodes, ctx), dtype=bool), sees], axis=1), HD ** -0.5)
            rel = 2 * (HD + 4) * 2.0 ** -24 * dot + 2 * (ctx + l.nodes + 8) * 2.0 ** -24 + 2.0 ** -21
            tol = rel * size if l.kind == "f32" else (rel + 2.0 ** -8) * size + 2.0 ** -8 * np.abs(want)
            assert (np.abs(out[r] - want) <= tol).all(), b
            way, x = tree_oracle.verify(l.tokens.cpu().numpy()[r], l.parents, l.p.cpu().numpy()[r], l.qd.cpu().numpy()[r], l.words.cpu().numpy()[r], int(l.draws[b]), 8)
            assert path[b, :int(length[b])].tolist() == way and (path[b, int(length[b]):] == -1).all() and int(token[b]) == x
            for side, full in enumerate((kk, vv)):
                self.store[side][b] = np.concatenate([full[:ctx], full[ctx:][way]])


def start(kind, seqs=4, nodes=21, seed=0):
    import paper_2512_07503_amd as sjd
    import torch
    l = Loop(kind, seqs, nodes, seed)
    plain = Plain(l)
    # a prompt: ctx tokens of each sequence
    for b, c in enumerate(l.ctx.cpu().tolist()):
        for side in range(2):
            plain.store[side][b] = l.rng.standard_normal((c, HKV, HD)).astype(np.float32)
    k, v = (torch.from_numpy(np.concatenate(plain.store[s]).astype(np.float32)).cuda().to(l.td) for s in range(2))
    counts = l.ctx.cpu().tolist()
    sjd.op_cache_write(l.cache, k, v, i32(np.concatenate([[0], np.cumsum(counts)])), i32([0] * seqs))
    for side, x in enumerate((k, v)):
        x, at = tree_oracle.store(kind, host(x)), np.concatenate([[0], np.cumsum(counts)])
        plain.store[side] = [x[at[b]:at[b + 1]] for b in range(seqs)]
    return l, plain


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
def test_steps(kind):
    l, plain = start(kind)
    total = 0
    for _ in range(6):
        l.feed()
        outs = l.step()
        plain.step(outs)
        total += int(outs[4].sum())
    assert total > 6 * 4                 # some drafts were accepted, so paths were kept
    assert l.ctx.cpu().tolist() == [len(s) for s in plain.store[0]]


@pytest.mark.parametrize("kind", ["fp8", "f32"])
def test_steps_captured_and_replayed(kind):
    """One graph, replayed with eager work and synchronizations in between; lengths grow on the device."""
    import torch
    l, plain = start(kind, seed=1)
    l.feed()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plain.step(l.step())             # warm-up: an eager step on another stream
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = l.step()
    for i in range(5):
        l.feed()
        graph.replay()
        torch.cuda.synchronize()
        plain.step(outs)
        if i == 2:
            l.feed()
            plain.step(l.step())         # an eager step between replays
    assert l.ctx.cpu().tolist() == [len(s) for s in plain.store[0]]


def test_two_graphs():
    """Two loops captured into a graph each and replayed in turn, and on two streams at once: their workspaces are their own."""
    import torch
    loops = [start(kind, seed=s) for s, kind in enumerate(("fp8", "bf16"))]
    graphs, outs = [], []
    for l, plain in loops:
        l.feed()
        plain.step(l.step())
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(l.step())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for i in range(4):
        for l, _ in loops:
            l.feed()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s if i % 2 else torch.cuda.default_stream()):
                g.replay()
        torch.cuda.synchronize()
        for (l, plain), o in zip(loops, outs):
            plain.step(o)
