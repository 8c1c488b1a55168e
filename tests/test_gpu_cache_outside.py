"""Sequences whose first position lies outside every cache: negative, or beyond 2^30.  They lie outside as a whole: nothing of them is written, and their
rows are read as zeros."""
import numpy as np
import pytest

import tree_oracle
from test_gpu_cache import KINDS, TYPES, host, i32, make, rows, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hkv,hd", [(2, 64), (1, 256), (40, 32)])
def test_rows_outside_are_read_as_zeros(kind, dtype, Hkv, hd):
    """Beside sequences that are there, which stay as they are; rows of no sequence are not written.  The last one starts inside and leaves its table."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(hd)
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    first = [0, -3, 40, -1, -(1 << 31), 1 << 30, 7, (1 << 30) + 1, (1 << 31) - 1, 60]
    n = [10, 10, 33, 1, 100, 70, 0, 5, 64, 50]
    cache, _ = make(kind, 32, Hkv, hd, [96] * len(n))
    starts = np.concatenate([[0], np.cumsum(n)]) + 2
    total = int(starts[-1]) + 3
    k, v = rows(rng, total, Hkv, hd, dtype), rows(rng, total, Hkv, hd, dtype)
    sjd.op_cache_write(cache, k, v, i32(starts), i32(first))
    out = tuple(torch.full((total, Hkv, hd), 5.0, dtype=td, device="cuda") for _ in range(2))
    sjd.op_cache_read(cache, i32(starts), i32(first), total, dtype=td, out=out)
    for g, x in zip(out, (k, v)):
        want = tree_oracle.store(kind, host(x))
        want = tree_oracle.bf16_store(want) if dtype == "bf16" else want
        want[:2] = want[-3:] = 5.0
        for b, f in enumerate(first):
            if f < 0 or f >= 1 << 30:
                want[starts[b]:starts[b + 1]] = 0.0
        want[starts[9] + 36:starts[10]] = 0.0          # positions from 96 on
        assert same(g, want)
