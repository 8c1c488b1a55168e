"""Row ranges that do not ascend, so that sequences share rows: what comes out for those is not specified, but it lies within the trees and the vocabulary, and
the other sequences are as ever."""
import numpy as np
import pytest

import tree_oracle
from test_gpu_cache import i32
from test_gpu_tree_verify import problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sampled", [True, False])
def test_sequences_that_share_rows(sampled):
    import paper_2512_07503_amd as sjd
    import torch
    V, n = 300, 1000
    d = problem(np.random.default_rng(9), V, [n, 40], 2, sampled, agree=1.0)
    d["parents"][0][1:] = [max(i - 50, 0) for i in range(1, n)]       # far steps
    starts = [900, 1000, 0, 1000, 1040]
    draws = torch.from_numpy(np.arange(4, dtype=np.int64) << 60).cuda()
    path, length, token = sjd.op_tree_verify(i32(d["tokens"]), i32(sum(d["parents"], [])), i32(starts), d["pd"], d["qd"], torch.from_numpy(d["words"].view(np.int32)).cuda(),
                                             draws, max_rows=1000)
    path, length, token = (x.cpu().numpy() for x in (path, length, token))
    rows = [100, 0, 1000, 40]
    for b, m in enumerate(rows):
        assert 0 <= length[b] <= m and (path[b, length[b]:] == -1).all() and (path[b, :length[b]] >= 0).all() and (path[b, :length[b]] < max(m, 1)).all()
        assert -1 <= token[b] < V
    r = slice(1000, 1040)
    want, x = tree_oracle.verify(d["tokens"][r], d["parents"][1], d["p"][r], None if d["q"] is None else d["q"][r], d["words"][r], 3 << 60, path.shape[1])
    assert path[3, :length[3]].tolist() == want and token[3] == x and length[1] == 0 and token[1] == -1
