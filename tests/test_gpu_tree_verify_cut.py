"""Walks that max_path ends: the children of the last node are not tested, and the next token comes from that node's p, whatever the tests would have said."""
import numpy as np
import pytest

import tree_oracle
from test_gpu_cache import i32
from test_gpu_tree_verify import check, problem, run

pytestmark = pytest.mark.gpu


def test_a_rejected_child_behind_the_cut():
    """p = (1/2, 1/2), q = (1, 0), a child with token 0 whose test fails (7/8 is not below 1/2): with room for the root alone it is not tested, and the draw's
    word 0 gives token 0 of p; with room for it its rejection leaves (0, 1/2)."""
    import paper_2512_07503_amd as sjd
    import torch
    p, q = torch.full((2, 2), 0.5, device="cuda"), torch.tensor([[1.0, 0.0]] * 2, device="cuda")
    words, draw = i32([0, -0x20000000]), torch.zeros(1, dtype=torch.int64, device="cuda")
    for drafts in (q, None):
        for max_path, want in ((1, 0), (2, 1)):
            path, length, token = sjd.op_tree_verify(i32([1, 0]), i32([-1, 0]), i32([0, 2]), p, drafts, words, draw, max_rows=2, max_path=max_path)
            assert path.tolist() == [[0] + [-1] * (max_path - 1)] and length.tolist() == [1] and token.tolist() == [want]


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("max_path", [1, 2, 3])
def test_rejected_children_behind_the_cut(max_path, sampled):
    """Trees whose distributions differ enough that many cut nodes have children that are all rejected."""
    behind = 0
    for seed in range(6):
        d = problem(np.random.default_rng(100 * seed + max_path), 300, [1, 9, 30, 14, 0, 40] * 4, 1 + seed % 4, sampled, sharp=(4.0, 2.0)[seed % 2], agree=(0.5, 0.9)[seed % 2])
        lengths = check(d, run(d, max_path=max_path))
        for b, t in enumerate(d["parents"]):
            r = slice(d["starts"][b], d["starts"][b + 1])
            if lengths[b] == max_path:        # would have ended there with more room, too, and has children
                longer, _ = tree_oracle.verify(d["tokens"][r], t, d["p"][r], None if d["q"] is None else d["q"][r], d["words"][r], d["draws"][b], max_path + 1)
                behind += len(longer) == max_path and longer[-1] in t
    assert behind >= 3, behind


@pytest.mark.parametrize("sampled", [True, False])
def test_distribution_where_the_path_has_room_for_the_root_alone(sampled):
    """The token is then distributed as p of the root: chi-square of 65 535 draws over 12 ids, 11 degrees of freedom, stays below 45 (probability 5e-6
    of more)."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(17)
    V, B = 12, 65535
    p, q = (rng.dirichlet(np.ones(V)).astype(np.float32) for _ in range(2))
    if sampled:
        kids = np.searchsorted(np.cumsum(q.astype(np.float64)) / q.sum(dtype=np.float64), rng.random((B, 2)), side="right").clip(0, V - 1)
    else:
        kids = np.tile(np.argsort(-q)[:2], (B, 1))
    tokens = np.concatenate([np.zeros((B, 1), dtype=np.int64), kids], axis=1).astype(np.int32).ravel()
    pd, qd = (torch.from_numpy(x).cuda().expand(3 * B, V).contiguous() for x in (p, q))
    words = torch.from_numpy(rng.integers(0, 1 << 32, 3 * B, dtype=np.uint64).astype(np.uint32).view(np.int32)).cuda()
    draws = torch.from_numpy(rng.integers(0, 1 << 64, B, dtype=np.uint64).view(np.int64)).cuda()
    path, length, token = sjd.op_tree_verify(i32(tokens), i32([-1, 0, 0] * B), i32(np.arange(B + 1) * 3), pd, qd if sampled else None, words, draws, max_rows=3, max_path=1)
    assert (length == 1).all() and (path == 0).all()
    counts = np.bincount(token.cpu().numpy(), minlength=V)
    expect = p.astype(np.float64) / p.sum(dtype=np.float64) * B
    assert ((counts - expect) ** 2 / expect).sum() < 45.0
