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
