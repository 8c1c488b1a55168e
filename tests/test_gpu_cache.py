"""The paged cache of the tree operators on the GPU: what is written, read back and moved, bit for bit against a plain implementation."""
import numpy as np
import pytest

import tree_oracle

pytestmark = pytest.mark.gpu
KINDS, TYPES = ("fp8", "bf16", "f32"), ("f32", "bf16")


def i32(x):
    import torch
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def make(kind, page, Hkv, hd, lengths, seed=0, spare=2):
    """A cache whose sequences hold up to lengths[b] tokens, pages in no order; -> (cache, host page table)."""
    import paper_2512_07503_amd as sjd
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lengths]
    total = sum(need) + spare
    perm, table, at = rng.permutation(total), np.full((len(lengths), max(1, max(need))), -1, dtype=np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return sjd.KvCache(kind, total, page, Hkv, hd, i32(table)), table


def rows(rng, n, Hkv, hd, dtype):
    import torch
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    x = rng.standard_normal((n, Hkv, hd)) * 2.0 ** rng.integers(-8, 9, (n, Hkv, 1))
    return torch.from_numpy(x.astype(np.float32)).cuda().to(td)


def same(got, want):
    """Equal as numbers, NaN for NaN."""
    got = got.double().cpu().numpy()
    return got.shape == want.shape and np.array_equal(got, want, equal_nan=True)


def host(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hkv,hd,page", [(1, 32, 32), (3, 64, 64), (2, 96, 96), (2, 128, 64), (1, 192, 32), (1, 256, 128)])
def test_write_and_read_ragged_rows(kind, dtype, Hkv, hd, page):
    """Lengths from none to several pages, first positions within, at and across blocks and pages; in two writes, the second behind the first; every
    position is read back, and those that nobody wrote still hold zeros."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(hd + len(kind))
    first, n1, n2 = [0, 5, 31, 32, 33, 60, 0, 90], [1, 0, 2, 70, 33, 9, 200, 1], [40, 1, 1, 3, 0, 130, 7, 64]
    length = [a + b + c + 3 for a, b, c in zip(first, n1, n2)]
    cache, _ = make(kind, page, Hkv, hd, length)
    want = [[np.zeros((m, Hkv, hd)) for m in length] for _ in range(2)]
    at = list(first)
    for counts in (n1, n2):
        k, v = rows(rng, sum(counts), Hkv, hd, dtype), rows(rng, sum(counts), Hkv, hd, dtype)
        starts = np.concatenate([[0], np.cumsum(counts)])
        sjd.op_cache_write(cache, k, v, i32(starts), i32(at))
        for side, x in enumerate((k, v)):
            x = tree_oracle.store(kind, host(x))
            for b in range(len(first)):
                want[side][b][at[b]:at[b] + counts[b]] = x[starts[b]:starts[b + 1]]
        at = [a + c for a, c in zip(at, counts)]
    starts = np.concatenate([[0], np.cumsum(length)])
    for out in (torch.float32, torch.bfloat16):
        got = sjd.op_cache_read(cache, i32(starts), i32([0] * len(first)), sum(length), dtype=out)
        for side in range(2):
            w = np.concatenate(want[side])
            assert same(got[side], tree_oracle.bf16_store(w) if out == torch.bfloat16 else w), (side, out)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hkv,hd", [(9, 32), (5, 64), (3, 96), (5, 128), (2, 192), (2, 256)])
def test_write_and_read_of_many_sequences(kind, dtype, Hkv, hd):
    """Enough tiles that a workgroup takes several heads (and a last one fewer), some of whose elements are no numbers; rows aligned and not."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(hd + len(kind))
    seqs = 2100 // Hkv
    n = rng.integers(0, 5, seqs)
    n[::50] = rng.integers(30, 100, len(n[::50]))
    n[:3] = 64, 32, 33
    first = rng.integers(0, 70, seqs)
    first[:3] = 0, 32, 31
    total = int(n.sum())
    starts = np.concatenate([[0], np.cumsum(n)])
    tiles = np.where(n > 0, (first + n - 1) // 32 - first // 32 + 1, 0).sum()
    bound = min((total + 30 * min(seqs, total)) // 32 + min(seqs, total), total)
    assert tiles <= bound and 2 * bound * Hkv >= 4096
    cache, _ = make(kind, 64, Hkv, hd, first + n)
    k, v = (rows(rng, total, 1, Hkv * hd + 1, dtype)[:, 0] for _ in range(2))
    k, v = k[:, :Hkv * hd].contiguous().unflatten(1, (Hkv, hd)), v[:, 1:].unflatten(1, (Hkv, hd))
    bad = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda").to(k.dtype)
    k[5, Hkv - 1, 3:6] = bad
    v[7, 0, hd - 3:] = bad
    sjd.op_cache_write(cache, k, v, i32(starts), i32(first))
    got = sjd.op_cache_read(cache, i32(starts), i32(first), total, dtype=torch.float32)
    for g, x in zip(got, (k, v)):
        assert same(g, tree_oracle.store(kind, host(x)))


def test_fp8_codes_at_their_edges():
    """Halfway cases, smallest codes, powers of two around the scale's steps, zeros, the largest floats, infinities and NaN."""
    import paper_2512_07503_amd as sjd
    import torch
    hd = 32
    lines = [np.zeros(hd), np.full(hd, -0.0), np.full(hd, 1e-45), np.full(hd, 2.0 ** -100), np.linspace(-448, 448, hd), np.linspace(-447.9, 449, hd),
             np.concatenate([[448.0], 2.0 ** -9 * np.arange(31) * 0.5]), np.concatenate([[256.0], 17 + 0.5 * np.arange(31)]),
             np.concatenate([[3e38], np.linspace(-3.4e38, 3.4e38, 31)]), np.concatenate([[np.inf, -np.inf, np.nan], np.linspace(-1, 1, 29)]),
             np.concatenate([[np.nan] * 32]), np.concatenate([[1.0], np.full(31, 2.0 ** -20)]), np.linspace(-1, 1, hd) * 2.0 ** 119]
    rng = np.random.default_rng(3)
    lines += [np.ldexp(rng.integers(-1024, 1025, hd) / 1024.0, int(e)) for e in rng.integers(-120, 120, 60)]     # many exact ties
    x = np.stack(lines).astype(np.float32)[:, None, :]
    n = len(x)
    cache, _ = make("fp8", 32, 1, hd, [n])
    k = torch.from_numpy(x).cuda()
    sjd.op_cache_write(cache, k, torch.flip(k, (0,)), i32([0, n]), i32([0]))
    gk, gv = sjd.op_cache_read(cache, i32([0, n]), i32([0]), n, dtype=torch.float32)
    want = tree_oracle.fp8_store(x)
    assert same(gk, want) and same(gv, want[::-1])


@pytest.mark.parametrize("kind", KINDS)
def test_strided_and_unaligned_rows(kind):
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(1)
    Hkv, hd, n = 2, 64, 50
    for dtype, pad, off in (("bf16", 8, 8), ("bf16", 3, 1), ("f32", 4, 4), ("f32", 1, 3)):
        buf = rows(rng, n, 1, 2 * Hkv * hd + pad + off, dtype)[:, 0]
        k = buf[:, off:off + Hkv * hd].unflatten(1, (Hkv, hd))
        v = buf[:, off + Hkv * hd:off + 2 * Hkv * hd].unflatten(1, (Hkv, hd))
        cache, _ = make(kind, 64, Hkv, hd, [n + 7])
        sjd.op_cache_write(cache, k, v, i32([0, n]), i32([7]))
        got = sjd.op_cache_read(cache, i32([0, n]), i32([7]), n, dtype=torch.float32)
        for g, x in zip(got, (k, v)):
            assert same(g, tree_oracle.store(kind, host(x))), (dtype, pad)


@pytest.mark.parametrize("kind", KINDS)
def test_pages_out_of_range_and_lengths_out_of_range(kind):
    """Entries outside the pool, positions outside the table, row_start that leaves the rows: writes are dropped, reads give zeros, and rows of no
    sequence are left as they were."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(2)
    Hkv, hd, page, n = 2, 64, 32, 96
    table = np.array([[0, 99, 2], [-1, 3, 1 << 30], [4, 5, 6]], dtype=np.int32)
    cache = sjd.KvCache(kind, 7, page, Hkv, hd, i32(table))
    k, v = rows(rng, 3 * n, Hkv, hd, "f32"), rows(rng, 3 * n, Hkv, hd, "f32")
    sjd.op_cache_write(cache, k, v, i32([0, n, 2 * n, 3 * n]), i32([0, 0, 20]))       # the third runs past its table
    out = tuple(torch.full((3 * n, Hkv, hd), 5.0, device="cuda") for _ in range(2))
    sjd.op_cache_read(cache, i32([0, n, 2 * n, 3 * n]), i32([0, 0, 20]), 3 * n, out=out)
    for g, x in zip(out, (k, v)):
        w = tree_oracle.store(kind, host(x))
        w[32:64] = 0
        w[n:n + 32] = w[n + 64:2 * n] = 0
        w[2 * n + 76:] = 0
        assert same(g, w)
    before = cache.pages.clone()
    for starts, first in (([0, 0, 0, 0], [0, 0, 0]), ([-5, 0, 0, 0], [0, 0, 0]), ([9, 3, 3, 3], [0, 0, 0]), ([0, 3, 3, 3], [-1, 0, 0]), ([0, 3, 3, 3], [1 << 30, 0, 0]),
                          ([0, 3, 3, 3], [2147483647, 0, 0]), ([0, -2147483648, -2147483648, -2147483648], [5, 5, 5]), ([3 * n] * 3 + [2147483647], [0, 0, 0])):
        sjd.op_cache_write(cache, k, v, i32(starts), i32(first))
        assert torch.equal(cache.pages, before), (starts, first)
    out = tuple(torch.full((10, Hkv, hd), 5.0, device="cuda") for _ in range(2))
    sjd.op_cache_read(cache, i32([2, 4, 4, 5]), i32([0, 0, 0]), 10, out=out)          # rows 0, 1 and from 5 on belong to nobody
    for g, x in zip(out, (k, v)):
        assert (g[:2] == 5).all() and (g[5:] == 5).all()
        assert same(g[2:4], tree_oracle.store(kind, host(x))[:2])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hd,page", [(32, 32), (128, 64), (256, 32)])
def test_compact(kind, hd, page):
    """Paths of none, one and many nodes, across pages, longer than what a workgroup holds at a time; entries that do not ascend end a path."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(hd)
    Hkv, n = 2, 300
    first = [0, 31, 7, 64, 1, 2]
    cache, _ = make(kind, page, Hkv, hd, [f + n for f in first])
    k, v = rows(rng, 6 * n, Hkv, hd, "f32"), rows(rng, 6 * n, Hkv, hd, "f32")
    starts = np.arange(7) * n
    sjd.op_cache_write(cache, k, v, i32(starts), i32(first))
    paths = [[], [0], sorted(rng.choice(n, 200, replace=False).tolist()), [0, 3, 40, 41, 299], [0, 2, 9, 9, 12], [1, 5, -1, 20]]
    kept = [[], [0], paths[2], paths[3], [0, 2, 9], [1, 5]]
    path = np.full((6, 210), -1, dtype=np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    sjd.op_cache_compact(cache, i32(first), i32(path), i32([len(p) for p in paths]))
    got = sjd.op_cache_read(cache, i32(starts), i32(first), 6 * n, dtype=torch.float32)
    for g, x in zip(got, (k, v)):
        x = tree_oracle.store(kind, host(x))
        for b, p in enumerate(kept):
            w = x[starts[b]:starts[b + 1]].copy()
            w[:len(p)] = w[p]
            assert same(g[starts[b]:starts[b + 1]], w), b
    # lengths and paths out of range move nothing that they should not
    before = cache.pages.clone()
    sjd.op_cache_compact(cache, i32([-1, 1 << 30, 2147483647, 0, 0, 0]), i32(np.full((6, 4), 2147483647)), i32([4, 4, 4, -3, 0, 4]))
    assert torch.equal(cache.pages, before)


def test_offsets_beyond_32_bits():
    """Pages more than 4 GiB behind the first, in bf16 elements and fp8 bytes."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(5)
    for kind, n_pages in (("fp8", 70000), ("bf16", 70000)):
        cache = sjd.KvCache(kind, n_pages, 64, 4, 128, i32([[n_pages - 1, 5, n_pages - 3]]))
        assert cache.pages.numel() > 1 << 32
        k, v = rows(rng, 150, 4, 128, "bf16"), rows(rng, 150, 4, 128, "bf16")
        sjd.op_cache_write(cache, k, v, i32([0, 150]), i32([0]))
        got = sjd.op_cache_read(cache, i32([0, 150]), i32([0]), 150, dtype=torch.float32)
        for g, x in zip(got, (k, v)):
            assert same(g, tree_oracle.store(kind, host(x))), kind
        del cache


def test_many_sequences():
    """More sequences than the 64 that a wavefront looks at at a time, most of them empty."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(6)
    seqs, Hkv, hd = 300, 1, 64
    counts = [int(x) for x in rng.integers(0, 3, seqs) * rng.integers(0, 30, seqs)]
    first = rng.integers(0, 64, seqs).tolist()
    cache, _ = make("fp8", 64, Hkv, hd, [f + c for f, c in zip(first, counts)])
    n, starts = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    k, v = rows(rng, n, Hkv, hd, "bf16"), rows(rng, n, Hkv, hd, "bf16")
    sjd.op_cache_write(cache, k, v, i32(starts), i32(first))
    got = sjd.op_cache_read(cache, i32(starts), i32(first), n, dtype=torch.float32)
    assert same(got[0], tree_oracle.fp8_store(host(k))) and same(got[1], tree_oracle.fp8_store(host(v)))
