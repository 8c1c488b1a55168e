"""Arguments of the tree operators' bindings that a call could take for something else than was meant."""
import pytest

from test_gpu_cache import i32
from test_gpu_tree_attention import Case, trees

pytestmark = pytest.mark.gpu


def test_a_mask_without_words_is_refused():
    """Its pointer is null, which in the C ABI stands for a window."""
    import paper_2512_07503_amd as sjd
    import torch
    c = Case("bf16", 4, 2, 64, 64, [40, 3], [5, 1], trees([5, 1]))
    for mask in (torch.empty((6, 0), dtype=torch.int32, device="cuda"), c.mask[:, :0].contiguous()):
        with pytest.raises(sjd.SjdError):
            c.run(mask=mask)
    c.check(c.run())


def test_a_cache_keeps_its_tensors():
    """The library holds their addresses: another tensor in their place would be ignored, and the old one's memory given to somebody else."""
    c = Case("bf16", 4, 2, 64, 64, [40, 3], [5, 1], trees([5, 1]))
    for name in ("page_table", "pages"):
        with pytest.raises(AttributeError):
            setattr(c.cache, name, getattr(c.cache, name).clone())
    want = c.run()
    # the table's contents may change: two pages trade places, and so do their bytes
    per = c.cache.pages.numel() // c.cache.desc.n_pages
    a, b = int(c.table[0, 0]), int(c.table[1, 0])
    pages = c.cache.pages.view(-1, per)
    pages[[a, b]] = pages[[b, a]]
    table = c.table.copy()
    table[0, 0], table[1, 0] = b, a
    c.cache.page_table.copy_(i32(table))
    assert (c.run() == want).all()


def test_lengths_of_a_long_loop_leave_nothing_behind():
    """A loop that says at every step how long its contexts are: what a cache and the binding remember of that has a bound."""
    import paper_2512_07503_amd as sjd
    c = Case("bf16", 4, 2, 64, 64, [40], [1])
    q = c.q[:0]
    for max_ctx in range(2000):
        sjd.op_tree_attention(q, c.cache, i32([0, 0]), i32([40]), max_rows=1, max_ctx=max_ctx)
    assert sum(len(x) for x in vars(c.cache).values() if isinstance(x, dict)) <= 256
    assert sjd.binding._attention_bytes.cache_info().currsize <= 256
