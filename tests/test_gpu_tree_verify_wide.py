"""Nodes with as many chosen children as a tree may have, every one of them rejected."""
import numpy as np
import pytest

from test_gpu_tree_verify import check, problem, run

pytestmark = pytest.mark.gpu


def test_a_thousand_chosen_children():
    """Tokens with repeats and outside the vocabulary among them; the root's children up to one that is accepted, or none.  What is taken off per child is carried from
    one to the next, so a call is far from 100 ms; taken off anew for each it is a sum of sums over the children before, seconds."""
    import torch
    for accepted in (None, 1000):
        rng = np.random.default_rng(5)
        d = problem(rng, 5000, [1024, 3], 2000, False, sharp=0.3)
        d["parents"][0] = [-1] + [0] * 1023
        d["tokens"][1:1024] = rng.permutation(5000)[:1023]
        d["tokens"][20:1000:7] = d["tokens"][19]
        d["tokens"][30:1000:50] = (5000, -1) * 10
        d["words"][1:1024] = 0xFFFFFFFF          # r = 1 - 2^-33: not below rho while it is below all that is left
        if accepted:
            d["words"][accepted] = 0
        assert check(d, run(d, max_rows=1024))[0] == (2 if accepted else 1)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        run(d, max_rows=1024)
        end.record()
        torch.cuda.synchronize()
        assert begin.elapsed_time(end) < 100.0
