"""Attention of sequences whose context length is negative: like their rows in the cache, they lie outside as a whole and see nothing."""
import pytest

from test_gpu_cache import i32
from test_gpu_tree_attention import Case, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
@pytest.mark.parametrize("n,max_ctx", [([5, 3, 1], 100), ([90, 40, 7], 100), ([2, 5, 1], 9000)])
@pytest.mark.parametrize("window", [True, False])
def test_negative_lengths_see_nothing(kind, n, max_ctx, window):
    import paper_2512_07503_amd as sjd
    import torch
    c = Case(kind, 4, 2, 64, 64, [50, 70, 33], n, None if window else trees(n))
    kw = dict(mask=c.mask, max_rows=max(n), max_ctx=max_ctx)
    want = c.run(**kw)
    c.check(want)
    for bad in (-1, -5, -(1 << 31)):
        got = sjd.op_tree_attention(c.q, c.cache, i32(c.starts), i32([50, bad, bad]), **kw)
        assert torch.equal(got[:n[0]], want[:n[0]]) and (got[n[0]:] == 0).all(), bad
