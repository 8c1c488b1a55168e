"""Attention of trees over the paged cache on the GPU, against 64 bits."""
import numpy as np
import pytest

import tree_oracle
from test_gpu_cache import host, i32, make, rows

pytestmark = pytest.mark.gpu


class Case:
    """Sequences with ctx[b] cached tokens and n[b] tree rows, written to a fresh cache.  sees[b]: bool [n, n], None: a window."""

    def __init__(self, kind, H, Hkv, hd, page, ctx, n, sees=None, seed=0, edit=None, spare=2):
        import paper_2512_07503_amd as sjd
        self.kind, self.ctx, self.n, self.sees = kind, ctx, n, sees
        self.H, self.Hkv, self.hd = H, Hkv, hd
        rng = np.random.default_rng(seed)
        self.dtype = "f32" if kind == "f32" else "bf16"
        total = [c + m for c, m in zip(ctx, n)]
        self.cache, self.table = make(kind, page, Hkv, hd, total, seed, spare)
        k, v = rows(rng, sum(total), Hkv, hd, self.dtype), rows(rng, sum(total), Hkv, hd, self.dtype)
        self.at = np.concatenate([[0], np.cumsum(total)])
        if edit:
            edit(k, v, self.at)
        sjd.op_cache_write(self.cache, k, v, i32(self.at), i32([0] * len(ctx)))
        self.k, self.v = (tree_oracle.store(kind, host(x)) for x in (k, v))
        self.starts = np.concatenate([[0], np.cumsum(n)])
        import torch
        self.q = torch.from_numpy(rng.standard_normal((sum(n), H, hd)).astype(np.float32)).cuda()
        self.q = self.q if self.dtype == "f32" else self.q.bfloat16()
        self.mask = None
        if sees is not None:
            words = max(1, -(-max(n) // 32))
            m = np.concatenate([tree_oracle.pack_mask(s, words) for s in sees])
            self.mask = torch.from_numpy(m.view(np.int32)).cuda()

    def args(self):
        return self.q, self.cache, i32(self.starts), i32(self.ctx)

    def run(self, **kw):
        import paper_2512_07503_amd as sjd
        kw = {**dict(mask=self.mask, max_rows=max(max(self.n), 1), max_ctx=max(self.ctx)), **kw}
        return sjd.op_tree_attention(*self.args(), **kw)

    def check(self, got, scale=None, rows_of=None):
        """fp32: a score is a sum of hd products, (hd + 4) 2^-24 of sum |q k| off, and so, relatively, is each probability, twice for the sum that divides;
        sums of T terms add T 2^-24 each way, the exponential 2^-21.  Otherwise each probability p becomes p (1 + d), |d| <= 2^-8, in bf16, in the
        products and in the sum: off by sum p d (v - out) / (1 + sum p d), at most 2^-8 (sum p |v| + |out|) but for 2^-16 of it, which the next bound's
        slack covers (a result's rounding is 2^-8 / (1 + 2^-8) of it at most); and the result is rounded, 2^-8 of it."""
        got = host(got)
        scale = self.hd ** -0.5 if scale is None else scale
        for b, (c, m) in enumerate(zip(self.ctx, self.n)):
            if m == 0:
                continue
            q = host(self.q[self.starts[b]:self.starts[b + 1]])
            k, v = self.k[self.at[b]:self.at[b + 1]], self.v[self.at[b]:self.at[b + 1]]
            s = np.tril(np.ones((m, m), dtype=bool)) if self.sees is None else self.sees[b][:, :m]
            sees = np.concatenate([np.ones((m, c), dtype=bool), s], axis=1)
            want, size, dot = tree_oracle.attention(q, k, v, sees, scale)
            g = got[self.starts[b]:self.starts[b + 1]]
            same_classes = np.array_equal(np.isnan(g), np.isnan(want)) and np.array_equal(np.isinf(g), np.isinf(want))
            assert same_classes, (b, np.argwhere(np.isnan(g) != np.isnan(want))[:5], np.argwhere(np.isinf(g) != np.isinf(want))[:5])
            ok = np.isfinite(want)
            assert np.array_equal(g[~ok & ~np.isnan(want)], want[~ok & ~np.isnan(want)])
            rel = 2 * (self.hd + 4) * 2.0 ** -24 * dot + 2 * (c + m + 8) * 2.0 ** -24 + 2.0 ** -21
            tol = rel * size if self.kind == "f32" else (rel + 2.0 ** -8) * size + 2.0 ** -7 * np.abs(np.where(ok, want, 0.0))
            off = np.where(ok, np.abs(np.where(ok, g, 0.0) - np.where(ok, want, 0.0)) - tol, -1.0)
            assert off.max() <= 1e-30, (b, off.max(), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("kind", ["fp8", "bf16"])
@pytest.mark.parametrize("hd", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("n", [1, 40, 90])
def test_one_visible_token_gives_its_value(kind, hd, n):
    """The weight is p / p for whatever bf16 p has become: 1 within 2^-22 in fp32, and the value, a bf16 number, is the nearest one to what comes out."""
    c = Case(kind, 2, 1, hd, 32, [0, 0], [n, n], [np.eye(n, dtype=bool)] * 2, seed=n)
    want = np.concatenate([np.repeat(c.v[c.at[b]:c.at[b + 1]], 2, axis=1) for b in range(2)])
    assert np.array_equal(host(c.run()), want)


def trees(ns, seed=0, branch=3):
    rng = np.random.default_rng(seed)
    return [tree_oracle.ancestors(tree_oracle.random_tree(rng, m, branch)) if m else np.zeros((0, 0), dtype=bool) for m in ns]


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,hd", [(4, 2, 32), (2, 2, 64), (3, 1, 96), (8, 2, 128), (5, 1, 192), (2, 1, 256)])
def test_ragged_trees(kind, H, Hkv, hd):
    """Contexts of nothing, within a block, at its end, over pages; trees of none, one, a few and more than a tile of rows."""
    n = [1, 0, 7, 33, 1, 12, 40]
    c = Case(kind, H, Hkv, hd, 64, [0, 9, 31, 32, 95, 130, 0], n, trees(n))
    c.check(c.run())


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
def test_windows(kind):
    """No mask: rows see their predecessors.  One token, the paper's windows, grouped heads by three, pages of 96."""
    for n, ctx, H, Hkv, hd, page in (([1], [0], 4, 4, 64, 32), ([1, 1, 1], [31, 32, 600], 6, 2, 64, 96), ([16], [577], 20, 20, 64, 64), ([96, 3], [70, 700], 2, 1, 128, 64),
                                     ([250], [31], 3, 1, 64, 32), ([32, 31], [0, 1], 8, 1, 128, 128)):
        c = Case(kind, H, Hkv, hd, page, ctx, n, seed=n[0])
        c.check(c.run())


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
def test_long_contexts_are_split(kind):
    """Few rows over long contexts: the work is split over the context and joined.  Whatever max_ctx says, the result is the same to rounding."""
    n = [1, 5]
    c = Case(kind, 8, 2, 64, 64, [5000, 1500], n, trees(n))
    for max_ctx in (0, 100, 5000, 100000):
        c.check(c.run(max_ctx=max_ctx))
    c.check(c.run(max_rows=64))


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
@pytest.mark.parametrize("n", [64, 130])
def test_many_rows(kind, n):
    """Several tiles of rows a key/value head, on contexts that are split and that are not."""
    c = Case(kind, 8, 2, 128, 64, [1700, 333], [n, n - 9], trees([n, n - 9]))
    c.check(c.run())
    c = Case(kind, 4, 4, 64, 32, [70] * 3, [n, 0, 1], trees([n, 0, 1]))
    c.check(c.run())


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
def test_rows_that_see_nothing_and_arbitrary_masks(kind):
    """Masks need not be trees: rows without a bit, with bits of later nodes, with bits behind the last node (which count for nothing)."""
    rng = np.random.default_rng(1)
    n = [20, 6, 40]
    sees = [rng.random((m, 64)) < 0.3 for m in n]
    sees[0][3] = sees[2][0] = sees[2][39] = False
    c = Case(kind, 4, 2, 64, 64, [0, 50, 0], n, sees)
    got = c.run()
    c.check(got)
    assert (got[3] == 0).all() and (got[26] == 0).all()


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
def test_infinities_and_nan_stay_with_the_rows_that_see_them(kind, hd):
    """Values that are NaN or infinite, keys that are NaN: rows that do not see them are as without them, in the same block of tokens and the same tile of rows;
    rows that see them get what the formula gives.  (fp8 stores NaN for either.)"""
    n = [40, 12]

    def edit(k, v, at):
        for node, kv, j, x in ((3, v, 5, np.nan), (7, v, 6, np.inf), (9, v, 6, -np.inf), (11, v, 40, np.inf), (11, k, 0, np.nan), (33, v, hd - 1, -np.inf)):
            kv[at[0] + 70 + node, :, j] = x
        v[at[1] + 4, 0, 3] = np.nan              # a cached token: every row of the second sequence sees it
    c = Case(kind, 4, 2, hd, 64, [70, 61], n, trees(n, 3), edit=edit)
    c.check(c.run())


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
def test_what_lies_behind_a_sequence_does_not_matter(kind):
    """Pages full of NaN behind the last token and in pages that the table does not list."""
    n = [1, 9]
    c = Case(kind, 4, 2, 64, 64, [40, 64], n, trees(n))
    keep = c.run()
    import paper_2512_07503_amd as sjd
    import torch
    total = [x + m for x, m in zip(c.ctx, c.n)]
    room = c.table.shape[1] * 64
    blank = sum(min(room, -(-t // 64) * 64) - t for t in total)
    pad = [min(room, -(-t // 64) * 64) - t for t in total]
    bad = torch.full((blank, 2, 64), float("nan"), device="cuda")
    sjd.op_cache_write(c.cache, bad, bad, i32(np.concatenate([[0], np.cumsum(pad)])), i32(total))
    used = set(c.table[c.table >= 0].tolist())
    per = c.cache.pages.numel() // c.cache.desc.n_pages
    for p in set(range(c.cache.desc.n_pages)) - used:
        c.cache.pages[p * per:(p + 1) * per] = 255
    got = c.run()
    assert torch.equal(got, keep)
    c.check(got)


def test_pages_out_of_range_are_not_seen():
    """A context with entries outside the pool: as if those tokens were not there."""
    import paper_2512_07503_amd as sjd
    import torch
    for kind in ("fp8", "bf16", "f32"):
        c = Case(kind, 4, 2, 64, 32, [200, 40], [5, 1], trees([5, 1]))
        table = c.table.copy()
        table[0, 2], table[0, 4], table[1, 0] = -7, 1 << 30, c.cache.desc.n_pages
        c.cache.page_table.copy_(i32(table))
        got = host(c.run())
        for b, gone in ((0, list(range(64, 96)) + list(range(128, 160))), (1, list(range(32)))):
            m, ctx = c.n[b], c.ctx[b]
            sees = np.concatenate([np.ones((m, ctx), dtype=bool), c.sees[b]], axis=1)
            sees[:, gone] = False
            want, size, _ = tree_oracle.attention(host(c.q[c.starts[b]:c.starts[b + 1]]), c.k[c.at[b]:c.at[b + 1]], c.v[c.at[b]:c.at[b + 1]], sees, 0.125)
            tol = 2.0 ** -14 * size if kind == "f32" else 2.0 ** -8 * (size + np.abs(want)) + 2.0 ** -14 * size
            assert (np.abs(got[c.starts[b]:c.starts[b + 1]] - want) <= tol).all()
        # lengths that leave the table are cut to it, negative ones to nothing
        out = torch.full_like(c.q, 3.0)
        sjd.op_tree_attention(c.q, c.cache, i32(c.starts), i32([2147483647, -5]), mask=c.mask, max_rows=5, max_ctx=100, out=out)
        assert torch.isfinite(out).all()


def test_strides_outputs_and_scale():
    """Queries out of a fused projection, unaligned rows, a given scale, rows of no sequence left alone, rows behind max_rows left alone."""
    import torch
    for kind, pad in (("bf16", 8), ("bf16", 1), ("f32", 4), ("f32", 3), ("fp8", 5)):
        n = [3, 8]
        c = Case(kind, 4, 2, 64, 64, [50, 7], n, trees(n))
        buf = torch.zeros((13, 4 * 64 + pad), dtype=c.q.dtype, device="cuda")
        view = buf[:, pad // 2:pad // 2 + 256].unflatten(1, (4, 64))
        view[1:12] = c.q
        out = torch.full((13, 4 * 64 + pad), 9.0, dtype=c.q.dtype, device="cuda")
        o = out[:, pad - pad // 2:pad - pad // 2 + 256].unflatten(1, (4, 64))
        import paper_2512_07503_amd as sjd
        mask = torch.cat([c.mask[:1], c.mask, c.mask[:1]])
        sjd.op_tree_attention(view, c.cache, i32([1, 4, 12]), i32(c.ctx), mask=mask, max_rows=8, max_ctx=50, scale=0.25, out=o)
        c.check(o[1:12], scale=0.25)
        rest = out.clone()
        rest[1:12, pad - pad // 2:pad - pad // 2 + 256] = 9.0
        assert (rest == 9.0).all()
        o.fill_(9.0)
        sjd.op_tree_attention(view, c.cache, i32([1, 4, 12]), i32(c.ctx), mask=mask, max_rows=5, max_ctx=50, scale=0.25, out=o)
        assert (o[9:12] == 9.0).all() and not (o[4:9] == 9.0).all()


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
def test_in_place_and_beside_the_queries(kind):
    """Results over the queries that they come from, and between them in the rows of one buffer: split and whole, few rows and many."""
    import paper_2512_07503_amd as sjd
    import torch
    for ctx, n in (([5, 90], [3, 8]), ([3000, 40], [2, 5]), ([300, 40], [40, 90])):
        c = Case(kind, 4, 2, 64, 64, ctx, n, trees(n))
        kw = dict(mask=c.mask, max_rows=max(n), max_ctx=max(ctx))
        want, q = c.run(), c.q.clone()
        assert torch.equal(sjd.op_tree_attention(q, c.cache, i32(c.starts), i32(ctx), out=q, **kw), want)
        both = torch.empty((sum(n), 2, 4, 64), dtype=c.q.dtype, device="cuda")
        both[:, 0] = c.q
        sjd.op_tree_attention(both[:, 0], c.cache, i32(c.starts), i32(ctx), out=both[:, 1], **kw)
        assert torch.equal(both[:, 1], want) and torch.equal(both[:, 0], c.q)


def test_large_scores():
    """Scores in the thousands: one token takes all, without overflow."""
    for kind in ("fp8", "bf16", "f32"):
        c = Case(kind, 2, 1, 64, 64, [300], [4], trees([4]))
        c.q *= 64
        got = host(c.run())
        assert np.isfinite(got).all()
        sees = np.concatenate([np.ones((4, 300), dtype=bool), c.sees[0]], axis=1)
        want, size, dot = tree_oracle.attention(host(c.q), c.k, c.v, sees, 0.125)
        rel = 2 * 68 * 2.0 ** -24 * dot + 2.0 ** -12
        assert (np.abs(got - want) <= (rel + 2.0 ** -8) * (size + np.abs(want))).all()


def test_a_long_cache_behind_4_gib():
    import paper_2512_07503_amd as sjd
    c = Case("bf16", 8, 4, 128, 64, [700], [3], trees([3]), spare=40000)
    assert c.cache.pages.numel() > 1 << 32 and int(c.table.max()) > 1 << 14
    c.check(c.run())


def test_two_calls_at_once_with_their_own_workspaces():
    """Two streams, each with its own workspace (what the binding takes by itself); results as one after the other."""
    import torch
    n = [1, 2]
    cases = [Case(kind, 8, 2, 128, 64, [9000, 4000], n, trees(n), seed=s) for s, kind in enumerate(("fp8", "bf16"))]
    alone = [c.run() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    args = [c.args() for c in cases]
    torch.cuda.synchronize()
    outs = []
    import paper_2512_07503_amd as sjd
    for _ in range(5):
        for c, a, s in zip(cases, args, streams):
            with torch.cuda.stream(s):
                outs.append(sjd.op_tree_attention(*a, mask=c.mask, max_rows=2, max_ctx=9000))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert torch.equal(o, alone[i % 2])
        cases[i % 2].check(o)


def test_refusals():
    import paper_2512_07503_amd as sjd
    import torch
    c = Case("fp8", 4, 2, 64, 64, [9000], [2], trees([2]))
    q, cache, starts, ctx = c.args()
    for a in [(q.float(), cache, starts, ctx), (q[:, :3], cache, starts, ctx), (q[..., :32], cache, starts, ctx), (q, cache, starts[:1], ctx), (q, cache, starts.long(), ctx),
              (q, cache, starts, ctx.cpu()), (q[0], cache, starts, ctx)]:
        with pytest.raises(sjd.SjdError):
            sjd.op_tree_attention(*a, max_rows=2, max_ctx=100)
    for kw in (dict(mask=c.mask[:1]), dict(mask=c.mask.long()), dict(out=q.float()), dict(out=q[:1]), dict(max_rows=0), dict(scale=-1.0),
               dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(sjd.SjdError):
            sjd.op_tree_attention(q, cache, starts, ctx, **{**dict(max_rows=2, max_ctx=9000), **kw})
