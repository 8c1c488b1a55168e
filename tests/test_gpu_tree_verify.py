"""Verification of trees of drafts on the GPU: paths, lengths and tokens identical to a plain implementation in doubles and integers."""
import numpy as np
import pytest

import tree_oracle
from test_gpu_cache import i32

pytestmark = pytest.mark.gpu


def problem(rng, V, ns, branch, sampled, sharp=2.0, agree=0.8, pad=0, off=0):
    import torch
    parents = [tree_oracle.random_tree(rng, m, branch) if m else [] for m in ns]
    starts = np.concatenate([[0], np.cumsum(ns)])
    n = int(starts[-1])
    z = rng.standard_normal((n, V)) * sharp
    soft = lambda x: (np.exp(x - x.max(axis=1, keepdims=True)) / np.exp(x - x.max(axis=1, keepdims=True)).sum(axis=1, keepdims=True)).astype(np.float32)
    p, q = soft(z), soft(agree * z + (1 - agree) * 4 * rng.standard_normal((n, V)))
    tokens = np.zeros(n, dtype=np.int32)
    for b, t in enumerate(parents):
        rank = {}
        for i, j in enumerate(t):
            row = q[starts[b] + max(j, 0)].astype(np.float64)
            if sampled:
                tokens[starts[b] + i] = min(int(np.searchsorted(np.cumsum(row) / row.sum(), rng.random(), side="right")), V - 1)
            else:
                rank[j] = rank.get(j, -1) + 1
                tokens[starts[b] + i] = np.argsort(-row)[min(rank[j], V - 1)]
    words = rng.integers(0, 1 << 32, n, dtype=np.uint64).astype(np.uint32)
    draws = rng.integers(0, 1 << 64, len(ns), dtype=np.uint64)

    def dev(x):
        buf = torch.zeros((n, V + pad + off), device="cuda")
        buf[:, off:off + V] = torch.from_numpy(x)
        return buf[:, off:off + V]
    return dict(parents=parents, starts=starts, tokens=tokens, p=p, q=q if sampled else None, words=words, draws=draws, pd=dev(p), qd=dev(q) if sampled else None)


def run(d, max_rows=None, max_path=None, **kw):
    import paper_2512_07503_amd as sjd
    import torch
    return sjd.op_tree_verify(i32(d["tokens"]), i32([j for t in d["parents"] for j in t]), i32(d["starts"]), d["pd"], d["qd"],
                              torch.from_numpy(d["words"].view(np.int32)).cuda(), torch.from_numpy(d["draws"].view(np.int64)).cuda(), max_rows=max_rows,
                              max_path=max_path, **kw)


def check(d, got, max_path=None):
    path, length, token = (x.cpu().numpy() for x in got)
    depth = path.shape[1]
    lengths = []
    for b, t in enumerate(d["parents"]):
        r = slice(d["starts"][b], d["starts"][b + 1])
        want, x = tree_oracle.verify(d["tokens"][r], t, d["p"][r], None if d["q"] is None else d["q"][r], d["words"][r], d["draws"][b], depth)
        assert path[b, :length[b]].tolist() == want and (path[b, length[b]:] == -1).all(), (b, path[b], want)
        assert int(token[b]) == x, (b, token[b], x)
        lengths.append(len(want))
    return lengths


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("V,ns,branch", [(1, [1, 3], 2), (7, [5, 1, 0, 9], 2), (500, [1, 16, 40], 1), (2048, [30, 31], 3), (2049, [33, 2], 5), (5000, [64, 64, 10], 8),
                                         (16384, [16], 1), (70001, [12, 30], 4)])
def test_paths_and_tokens(V, ns, branch, sampled):
    seen = []
    for seed in range(6):
        d = problem(np.random.default_rng(1000 * seed + V), V, ns, branch, sampled, sharp=(0.5, 2.0, 5.0)[seed % 3], agree=(0.2, 0.9)[seed % 2])
        seen += check(d, run(d))
    if V > 100 and sampled:           # (a chosen draft is accepted with its own probability only)
        assert max(seen) > 1


@pytest.mark.parametrize("sampled", [True, False])
def test_wide_nodes(sampled):
    """A root with more children than a wavefront has lanes, duplicates among their tokens."""
    for seed in range(4):
        rng = np.random.default_rng(seed)
        d = problem(rng, 300, [90, 3], 200, sampled, sharp=1.0, agree=0.1)
        d["parents"][0] = [-1] + [0] * 80 + [1, 2, 3, 4, 4, 4, 80, 80, 81]
        d["tokens"][5:40:3] = d["tokens"][4]
        check(d, run(d))


def test_the_largest_tree():
    d = problem(np.random.default_rng(3), 64, [1024, 1000], 2, True, sharp=1.0, agree=1.0)
    check(d, run(d, max_rows=1024))
    d["parents"] = [list(range(-1, 1023)), list(range(-1, 999))]
    d["qd"].copy_(d["pd"])
    d["q"] = d["p"]                    # q = p: a test fails only where r >= 1 in doubles, so a path is as long as the drafts
    assert check(d, run(d, max_rows=1024)) == [1024, 1000]


def test_lengths_are_cut():
    """max_path ends a walk before its drafts do, and the token then comes from the last node's p; rows behind max_rows do not count."""
    rng = np.random.default_rng(4)
    d = problem(rng, 200, [40, 40], 1, True, agree=1.0)
    d["qd"].copy_(d["pd"])
    d["q"] = d["p"]
    assert check(d, run(d, max_path=7)) == [7, 7] and check(d, run(d, max_path=1)) == [1, 1]
    path, length, token = run(d, max_rows=5)
    assert (length.cpu() == 5).all() and (path.cpu()[:, :5] == np.arange(5)).all()


def test_degenerate_distributions():
    """Rows of zeros, q above p everywhere, certainty, NaN and negatives, tokens outside the vocabulary, weights above 1."""
    import torch
    rng = np.random.default_rng(5)
    for sampled in (True, False):
        d = problem(rng, 300, [6] * 8, 3, sampled)
        p = d["p"]
        p[0:6] = 0.0                                       # nothing to draw: token -1
        if sampled:
            d["q"][6:12] = 1.0                             # residual 0: drawn from p
        p[12:18] = 0.0
        p[12:18, 299] = 1.0                                # certain, the last id
        p[18:24, ::3] = np.nan
        p[24:30, ::2] = -1.0
        p[30:36] *= 1000.0
        d["tokens"][36:48:2] = (-1, 300, 2147483647, -2147483648, 299, 0)
        d["draws"][:] = [0, 1 << 63, (1 << 64) - 1, (1 << 64) - 1, 0, 5, 1 << 40, (1 << 64) - 1]
        d["pd"].copy_(torch.from_numpy(p))
        if sampled:
            d["qd"].copy_(torch.from_numpy(d["q"]))
        lengths = check(d, run(d))
        assert len(lengths) == 8


def test_bad_parents_are_nobodys_children():
    d = problem(np.random.default_rng(6), 100, [12], 2, True, agree=1.0)
    d["parents"][0] = [-1, 0, 5, -3, 1, 7, 2147483647, 4, -2147483648, 9, 12, 3]
    check(d, run(d))
    d["parents"][0] = [3, 0, 0, 1, 1, 3, 3, 5, 5, 6, 7, 8]    # the root's parent is not looked at
    check(d, run(d))


def test_strided_and_unaligned_rows():
    for pad, off in ((4, 4), (1, 0), (3, 1), (0, 2)):
        d = problem(np.random.default_rng(pad), 1003, [9, 30], 3, True, pad=pad, off=off)
        check(d, run(d))


def test_distribution_is_the_targets():
    """The first new token (the accepted child's, else the drawn one) is distributed as p of the root, whatever the proposals: chi-square of 65 536 draws
    over 12 ids with 11 degrees of freedom stays below 45 (probability 5e-6 of more)."""
    import torch
    rng = np.random.default_rng(7)
    V, B = 12, 65535
    p = rng.dirichlet(np.ones(V)).astype(np.float32)
    q = rng.dirichlet(np.ones(V)).astype(np.float32)
    for sampled in (True, False):
        if sampled:
            kids = np.searchsorted(np.cumsum(q.astype(np.float64)) / q.sum(dtype=np.float64), rng.random((B, 3)), side="right").clip(0, V - 1)
        else:
            kids = np.tile(np.argsort(-q)[:3], (B, 1))
        tokens = np.concatenate([np.zeros((B, 1), dtype=np.int64), kids], axis=1).astype(np.int32).ravel()
        import paper_2512_07503_amd as sjd
        pd, qd = (torch.from_numpy(x).cuda().expand(4 * B, V).contiguous() for x in (p, q))
        path, length, token = sjd.op_tree_verify(i32(tokens), i32([-1, 0, 0, 0] * B), i32(np.arange(B + 1) * 4), pd, qd if sampled else None,
                                                 torch.from_numpy(rng.integers(0, 1 << 32, 4 * B, dtype=np.uint64).astype(np.uint32).view(np.int32)).cuda(),
                                                 torch.from_numpy(rng.integers(0, 1 << 64, B, dtype=np.uint64).view(np.int64)).cuda(), max_rows=4, max_path=2)
        path, length, token = (x.cpu().numpy() for x in (path, length, token))
        first = np.where(length == 2, tokens.reshape(B, 4)[np.arange(B), path[:, 1].clip(0)], token)
        counts = np.bincount(first, minlength=V)
        expect = p.astype(np.float64) / p.sum(dtype=np.float64) * B
        assert ((counts - expect) ** 2 / expect).sum() < 45.0
        # chosen drafts are accepted with the probability that one of them is the target's token (five standard deviations: 0.01)
        assert (length == 2).mean() > 0.3 if sampled else abs((length == 2).mean() - p[kids[0]].sum()) < 0.01


def test_refusals():
    import paper_2512_07503_amd as sjd
    import torch
    d = problem(np.random.default_rng(8), 50, [5], 2, True)
    good = [i32(d["tokens"]), i32(d["parents"][0]), i32(d["starts"]), d["pd"], d["qd"], torch.zeros(5, dtype=torch.int32, device="cuda"),
            torch.zeros(1, dtype=torch.int64, device="cuda")]
    sjd.op_tree_verify(*good)
    for i, bad in ((0, good[0].long()), (1, good[1][:4]), (2, good[2].cpu()), (3, good[3].double()), (3, good[3].t()), (4, good[4][:, :40]), (5, good[5].long()), (6, good[6].int()),
                   (6, torch.zeros(2, dtype=torch.int64, device="cuda"))):
        a = list(good)
        a[i] = bad
        with pytest.raises(sjd.SjdError):
            sjd.op_tree_verify(*a)
    for kw in (dict(max_rows=0), dict(max_rows=1025), dict(max_path=0), dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(sjd.SjdError):
            sjd.op_tree_verify(*good, **kw)
