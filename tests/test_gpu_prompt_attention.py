"""Attention of packed prompts on the GPU, against 64 bits."""
import numpy as np
import pytest

import prompt_oracle

pytestmark = pytest.mark.gpu


def i32(x):
    import torch
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def host(t):
    return t.double().cpu().numpy()


def starts(n, first=0):
    return first + np.concatenate([[0], np.cumsum(n)]).astype(np.int64)


class Case:
    """n[b] queries and t[b] keys of every sequence (t None: the same rows), after `lead` rows of nobody and before `trail` more.  Rows are parts of a fused
    projection's with `pad` elements more."""

    def __init__(self, dtype, H, Hkv, hd, n, t=None, seed=0, lead=0, trail=0, pad=0, edit=None, loud=1.5):
        import torch
        rng = np.random.default_rng(seed)
        self.dtype, self.H, self.Hkv, self.hd, self.n, self.t = dtype, H, Hkv, hd, n, n if t is None else t
        self.own = t is None
        td = torch.float32 if dtype == "f32" else torch.bfloat16
        make = lambda rows, width: torch.from_numpy(rng.standard_normal((rows, width)).astype(np.float32)).cuda().to(td)
        part = lambda x, lo, h: x[:, lo * hd:(lo + h) * hd].unflatten(1, (h, hd))
        rows = lead + sum(n) + trail
        if self.own:
            x = make(rows, (H + 2 * Hkv) * hd + pad)
            x[:, :H * hd] *= loud
            self.q, self.k, self.v = part(x, 0, H), part(x, H, Hkv), part(x, H + Hkv, Hkv)
        else:
            kv = lead + sum(self.t) + trail
            self.q = part(make(rows, H * hd + pad) * loud, 0, H)
            self.k, self.v = part(make(kv, Hkv * hd + pad), 0, Hkv), part(make(kv, Hkv * hd + pad), 0, Hkv)
        self.at, self.kat = starts(n, lead), starts(self.t, lead)
        if edit:
            edit(self)

    def run(self, **kw):
        import paper_2512_07503_amd as sjd
        kw = {**dict(max_rows=max(max(self.n), 1), max_kv=max(max(self.t), 1)), **kw}
        return sjd.op_prompt_attention(self.q, self.k, self.v, i32(self.at), None if self.own else i32(self.kat), **kw)

    def check(self, got, scale=None, oracle=prompt_oracle.attention):
        """fp32: a score is a sum of hd products, (hd + 4) 2^-24 of sum |q k| off, and so, relatively, is each probability, twice for the sum that divides;
        sums of T terms add T 2^-24 each way, the exponential 2^-21.  bf16: each probability p becomes p (1 + d), |d| <= 2^-8, in the products and in the sum: off by
        sum p d (v - out) / (1 + sum p d), at most 2^-8 (sum p |v| + |out|) but for 2^-16 of it, which the next bound's slack covers (a result's rounding is
        2^-8 / (1 + 2^-8) of it at most); and the result is rounded, 2^-8 of it."""
        got, scale = host(got), self.hd ** -0.5 if scale is None else scale
        for b in range(len(self.n)):
            if self.n[b] == 0:
                continue
            rows, keys = slice(self.at[b], self.at[b + 1]), slice(self.kat[b], self.kat[b + 1])
            want, size, dot = oracle(host(self.q[rows]), host(self.k[keys]), host(self.v[keys]), scale)
            g = got[rows]
            assert np.array_equal(np.isnan(g), np.isnan(want)) and np.array_equal(np.isinf(g), np.isinf(want)), b
            ok = np.isfinite(want)
            assert np.array_equal(g[~ok & ~np.isnan(want)], want[~ok & ~np.isnan(want)])
            rel = 2 * (self.hd + 4) * 2.0 ** -24 * dot + 2 * (self.t[b] + 8) * 2.0 ** -24 + 2.0 ** -21
            tol = rel * size if self.dtype == "f32" else (rel + 2.0 ** -8) * size + 2.0 ** -7 * np.abs(np.where(ok, want, 0.0))
            off = np.where(ok, np.abs(np.where(ok, g, 0.0) - np.where(ok, want, 0.0)) - tol, -1.0)
            assert off.max() <= 1e-30, (b, off.max(), np.unravel_index(off.argmax(), off.shape))


HEADS = [(4, 2, 32), (2, 2, 64), (3, 1, 96), (8, 2, 128), (5, 1, 192), (2, 1, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,hd", HEADS)
def test_packed(dtype, H, Hkv, hd):
    """Prompts of none, one, a few rows, and more than a tile of them; ends within blocks and at their borders."""
    c = Case(dtype, H, Hkv, hd, [1, 0, 7, 33, 64, 1, 130, 65, 0, 300])
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,hd", HEADS)
def test_behind_what_is_cached(dtype, H, Hkv, hd):
    """Queries that follow keys of their own sequence; sequences with fewer keys than queries, whose first ones see nothing; without keys at all."""
    n = [1, 5, 0, 40, 70, 9, 33, 128]
    c = Case(dtype, H, Hkv, hd, n, [200, 5, 9, 39, 0, 300, 65, 129], seed=1)
    c.check(c.run())
    got = host(c.run())
    assert (got[c.at[3]:c.at[3] + 1] == 0).all() and (got[c.at[4]:c.at[5]] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,hd", [(8, 1, 64), (4, 4, 128), (2, 1, 256), (1, 1, 32)])
@pytest.mark.parametrize("n,t", [([1], [3000]), ([3, 1, 0, 20], [2500, 700, 1000, 20]), ([150], [2200])])
def test_few_rows_behind_many_keys(dtype, H, Hkv, hd, n, t):
    """The keys are split and joined.  Whatever is expected of the sizes, the result is the same to rounding."""
    c = Case(dtype, H, Hkv, hd, n, t, seed=2)
    for max_rows, max_kv in ((max(n), max(t)), (1, 100), (0, 0), (100000, 100000), (1, 1 << 30)):
        if max_kv == 1 << 30 and Hkv > 1:
            continue
        c.check(c.run(max_rows=max_rows, max_kv=max_kv))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_prompts(dtype):
    c = Case(dtype, 2, 1, 64, [1100, 900], seed=3)
    c.check(c.run())
    c = Case(dtype, 1, 1, 128, [2000], seed=4)
    c.check(c.run())
    c = Case(dtype, 12, 1, 64, [700, 3], seed=5)
    c.check(c.run())


def test_a_first_row_gives_its_value():
    """One visible key: the weight is p / p for whatever bf16 p has become."""
    for hd in (32, 64, 96, 128, 192, 256):
        c = Case("bf16", 2, 1, hd, [50, 1, 200], seed=hd)
        got = c.run()
        for b in range(3):
            assert (got[c.at[b]] == c.v[c.at[b]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,pad", [(64, 0), (128, 8), (96, 4), (64, 3), (32, 1), (256, 2)])
def test_strides_and_alignment(dtype, hd, pad):
    for t in (None, [70, 200]):
        c = Case(dtype, 4, 2, hd, [70, 150], t, seed=6, pad=pad)
        c.check(c.run())
        import torch
        out = torch.zeros((220, 4 * hd + 5), dtype=c.q.dtype, device="cuda")
        part = out[:, 1:1 + 4 * hd].unflatten(1, (4, hd))
        assert c.run(out=part).data_ptr() == part.data_ptr()
        c.check(part)
        assert (out[:, :1] == 0).all() and (out[:, 1 + 4 * hd:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dtype):
    """Over the queries, within the fused projection; with splits, too."""
    for n, t in (([300, 20], None), ([2, 30], [1500, 3000])):
        c = Case(dtype, 4, 2, 64, n, t, seed=7)
        want = c.run().clone()
        k, v = c.k.clone(), c.v.clone()
        c.run(out=c.q)
        assert (c.q == want).all() and (c.k == k).all() and (c.v == v).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_nobody(dtype):
    """Rows ahead of the first sequence and behind the last are neither read for others nor written; row_start may reach beyond the rows."""
    import torch

    def edit(c):
        for x in (c.q, c.k, c.v):
            x[:c.at[0]] = float("nan")
            x[c.at[-1]:] = float("nan")
    for t in (None, [80, 70]):
        c = Case(dtype, 4, 2, 64, [70, 65], t, seed=8, lead=5, trail=40)
        if t is None:
            edit(c)
        out = torch.full_like(c.q.contiguous(), 7.0)
        c.run(out=out)
        c.check(out)
        assert (out[:5] == 7).all() and (out[c.at[-1]:] == 7).all()
    # cut off at the last row
    c = Case(dtype, 4, 2, 64, [70, 65], seed=9)
    import paper_2512_07503_amd as sjd
    got = sjd.op_prompt_attention(c.q, c.k, c.v, i32([-3, 70, 1000]), max_rows=70, max_kv=70)
    c.check(got)
    # descending: no rows
    out = torch.full_like(c.q.contiguous(), 7.0)
    sjd.op_prompt_attention(c.q, c.k, c.v, i32([70, 70, 3]), out=out)
    assert (out == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,hd", [(4, 2, 64), (3, 1, 128), (1, 1, 96), (2, 2, 256)])
def test_unseen_infinities_and_nan(dtype, H, Hkv, hd):
    """In keys and values behind a query, also of the block that holds its own: the queries ahead of them are what they are without, those behind have them."""
    rng = np.random.default_rng(10)

    def edit(c):
        for b, bad in enumerate((37, 100, 3)):
            r = c.kat[b] + bad
            c.v[r, 0, 5], c.v[r, 0, hd - 1], c.v[r + 2, 0, 0], c.v[r + 9, 0, 31] = float("inf"), float("-inf"), float("nan"), float("inf")
        c.k[c.kat[1] + 120] = float("nan")
    for n, t in (([60, 140, 20], None), ([60, 140, 20], [60, 150, 100])):
        c = Case(dtype, H, Hkv, hd, n, t, seed=11, edit=edit, loud=0.3)
        c.check(c.run(), oracle=prompt_oracle.attention_wild)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_of_splits_that_are_not_finite(dtype):
    """A visible infinity in one split of several."""
    def edit(c):
        c.v[100, 0, 3], c.v[2900, 0, 4], c.v[1500, 1, 5] = float("inf"), float("-inf"), float("nan")
    c = Case(dtype, 4, 2, 64, [3], [3000], seed=12, edit=edit, loud=0.1)
    c.check(c.run(), oracle=prompt_oracle.attention_wild)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top", [124, -80])
def test_large_and_small_values(dtype, top):
    """Scores (base 2) are 0, but for some of up to 7.5 behind the first blocks: below what the reference may lag behind by.  Weights are at most 1, so sums of products with
    values of up to 2^top stay below 2^top (1 + T 2^-7.5) in magnitude, and far below with their random signs."""
    for steps in ((7.5,), (2.5, 5.0, 7.5)):
        def edit(c):
            c.q.zero_()
            c.q[:, :, 0] = 1.0
            c.k.zero_()
            for i, s in enumerate(steps):
                c.k[150 + 70 * i, :, 0] = s
            c.v.copy_((c.v.float() / c.v.float().abs().amax(dim=-1, keepdim=True) * 2.0 ** top).to(c.v.dtype))
        for n, t in (([400], None), ([5], [400])):
            c = Case(dtype, 2, 1, 64, n, t, seed=13, edit=edit)
            got = c.run(scale=float(np.log(2.0)))
            assert np.isfinite(host(got)).all()
            c.check(got, scale=float(np.log(2.0)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sharp_rows(dtype):
    """Scores of hundreds: one key takes all, the others underflow; maxima that climb from block to block."""
    def edit(c):
        import torch
        c.k *= torch.linspace(1, 40, c.k.shape[0], device="cuda")[:, None, None].to(c.k.dtype)
    c = Case(dtype, 2, 1, 64, [500], seed=14, edit=edit)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    rng = np.random.default_rng(15)
    n = rng.integers(0, 4, 300).tolist()
    n[170] = 90
    c = Case(dtype, 2, 1, 32, n, seed=15)
    c.check(c.run())
    c = Case(dtype, 2, 1, 32, n, [m + int(x) for m, x in zip(n, rng.integers(0, 9, 300))], seed=16)
    c.check(c.run())


def test_same_bits_every_time():
    c = Case("bf16", 8, 2, 64, [9, 200], [3000, 1000], seed=17)
    first = c.run().clone()
    for _ in range(5):
        assert (c.run() == first).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_with_the_card_full(dtype):
    """Every block of keys is in LDS before anybody reads it, however long it took to get there."""
    c = Case(dtype, 32, 8, 128, [2900, 1000], seed=21)
    first = c.run().clone()
    for _ in range(10):
        assert (c.run() == first).all()


def test_workspace():
    import paper_2512_07503_amd as sjd
    import torch
    c = Case("bf16", 8, 1, 64, [4], [4000], seed=18)
    need = sjd.binding._prompt_bytes(sjd.BF16, 4, 1, 8, 1, 64, 4, 4000)
    assert need > 0
    guard = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    c.check(c.run(workspace=guard[256:256 + need]))
    assert (guard[:256] == 0x5A).all() and (guard[256 + need:] == 0x5A).all()
    # what it holds from before does not matter
    guard.fill_(0xFF)
    c.check(c.run(workspace=guard[256:256 + need]))
    with pytest.raises(sjd.SjdError) as e:
        c.run(workspace=guard[:need - 16])
    assert e.value.code == sjd.ECAPACITY
    with pytest.raises(sjd.SjdError):
        c.run(workspace=guard[8:8 + need])


def test_scale():
    c = Case("f32", 2, 2, 64, [90], seed=19)
    c.check(c.run(scale=0.3), scale=0.3)


def test_refusals():
    import paper_2512_07503_amd as sjd
    import torch
    c = Case("bf16", 4, 2, 64, [10, 20], seed=20)
    q, k, v, s = c.q, c.k, c.v, i32(c.at)
    for args in [(q.half(), k, v, s), (q.float(), k, v, s), (q, k.float(), v, s), (q, k, v[:-1], s), (q, k[:-1], v[:-1], s), (q, k, v, s.long()), (q, k, v, s.cpu()),
                 (q[..., :48], k[..., :48], v[..., :48], s), (q[:, :3], k, v, s), (q.transpose(0, 1), k, v, s), (q, k, v, s, s[:-1]), (q, k, v, s[:1])]:
        with pytest.raises(sjd.SjdError):
            sjd.op_prompt_attention(*args)
    for kw in [dict(scale=-1.0), dict(scale=float("nan")), dict(max_rows=-1), dict(max_kv=-1), dict(out=q.float()), dict(out=c.v), dict(out=q[:-1])]:
        with pytest.raises(sjd.SjdError):
            sjd.op_prompt_attention(q, k, v, s, **kw)
    whole = torch.zeros((31, 8, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sjd.SjdError):
        sjd.op_prompt_attention(whole[:30, :4], k, v, s, out=whole[1:, :4])


@pytest.mark.parametrize("dtype,stride", [("bf16", 40_000_000), ("f32", 36_000_000)])
def test_rows_far_apart(dtype, stride):
    """Rows of a block of keys more than 2^32 bytes from its first one."""
    import torch

    def far(c):
        x = torch.empty((len(c.k) * stride,), dtype=c.k.dtype, device="cuda").view(len(c.k), stride)
        x[:, :64], x[:, 64:128] = c.k[:, 0], c.v[:, 0]
        c.k, c.v = x[:, :64].unflatten(1, (1, 64)), x[:, 64:128].unflatten(1, (1, 64))
    c = Case(dtype, 2, 1, 64, [3, 20], [66, 4], seed=21, edit=far)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,most", [(63, 80), (64, 300), (65, 300), (150, 150), (4100, 9)])
def test_many_sequences(dtype, n_seqs, most):
    rng = np.random.default_rng(22 + n_seqs)
    n = (rng.integers(0, most, n_seqs) * (rng.random(n_seqs) < 0.7)).tolist()
    c = Case(dtype, 6, 2, 32, n, seed=22, lead=70, trail=9)
    c.check(c.run())
    t = (np.asarray(n) + rng.integers(-3, 200 if n_seqs < 1000 else 4, n_seqs)).clip(0).tolist()
    c = Case(dtype, 3, 3, 32, n, t, seed=23, lead=3, trail=200)
    c.check(c.run())
    c.check(c.run(max_kv=1000))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("max_kv", [100, 100000])
def test_scores_that_are_minus_infinity(dtype, hd, max_kv):
    """The first 70 of 100 keys have no weight, and the others' scores are far below 0: the result is that of the others alone."""
    def edit(c):
        c.q[..., 0], c.q[..., 1] = 1.0, 1.0
        c.k[:70, :, 0] = float("-inf")
        c.k[70:, :, 1] = -300.0 * hd ** 0.5
    c = Case(dtype, 4, 2, hd, [30], [100], seed=24, edit=edit)
    few = Case(dtype, 4, 2, hd, [30], [30], seed=24)
    few.q, few.k, few.v = c.q, c.k[70:], c.v[70:]
    few.check(c.run(max_kv=max_kv))


@pytest.mark.parametrize("n_seqs", [64, 500])
def test_slots_without_rows_do_not_change_the_division(n_seqs):
    """A batch of slots of which few have a row, behind many keys: the same result, and a workspace as for those alone."""
    import paper_2512_07503_amd as sjd
    n, t = [0] * n_seqs, [0] * n_seqs
    n[1], n[40], n[63] = 1, 3, 1
    t[1], t[40], t[63] = 3000, 2000, 50
    c = Case("bf16", 8, 2, 128, n, t, seed=25)
    c.check(c.run())
    assert sjd.binding._prompt_bytes(sjd.BF16, 5, n_seqs, 8, 2, 128, 3, 3000) > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_scores_that_are_far_from_zero(dtype, hd):
    """Scores q_0 k_0 of up to 2^127 in magnitude, exact in fp32 and at least 2^20 apart where they are not equal: a row is the mean of the values whose keys have its largest one.  Their
    weights are the same number, so a sum of T is (T + 16) 2^-24 of sum p |v| off, the quotient 2^-22, and the result is rounded."""
    import torch
    rng = np.random.default_rng(26)
    for top, scale in ((20, np.log(2.0)), (24, None), (28, 0.7), (33, None), (60, None), (119, np.log(2.0))):
        for sign in (1.0, -1.0):
            def edit(c):
                c.q.zero_()
                c.q[:, :, 0] = sign * 2.0 ** top
                c.k[:, :, 0] = torch.from_numpy(rng.integers(1, 200, (len(c.k), c.Hkv)).astype(np.float32)).cuda().to(c.k.dtype)
            for n, t, max_kv in (([150, 1, 40], None, 150), ([5, 40], [2300, 90], 2300), ([5, 40], [2300, 90], 64)):
                c = Case(dtype, 4, 2, hd, n, t, seed=27, edit=edit)
                got = host(c.run(max_kv=max_kv, scale=float(scale or 0.0)))
                assert np.isfinite(got).all(), (top, sign, n)
                for b in range(len(n)):
                    rows, keys = slice(c.at[b], c.at[b + 1]), slice(c.kat[b], c.kat[b + 1])
                    want, size, _ = prompt_oracle.attention(host(c.q[rows]), host(c.k[keys]), host(c.v[keys]), scale or hd ** -0.5)
                    tol = ((c.t[b] + 16) * 2.0 ** -24 + 2.0 ** -22) * size + (2.0 ** -24 if dtype == "f32" else 2.0 ** -8) * np.abs(want) * (1 + 2.0 ** -7)
                    assert (np.abs(got[rows] - want) <= tol).all(), (top, sign, n, np.abs(got[rows] - want).max())


def test_max_rows_changes_nothing():
    """Neither the bits nor the workspace, whose size is asked for once."""
    import paper_2512_07503_amd as sjd
    c = Case("bf16", 8, 2, 64, [5, 3], [3000, 1000], seed=28)
    first = c.run().clone()
    misses = sjd.binding._prompt_bytes.cache_info().misses
    for max_rows in (0, 1, 7, 100000):
        assert (c.run(max_rows=max_rows) == first).all()
    assert sjd.binding._prompt_bytes.cache_info().misses == misses
    for max_rows in (-1, (1 << 29) + 1):
        with pytest.raises(sjd.SjdError):
            c.run(max_rows=max_rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_short_sequences_and_a_long_one(dtype):
    rng = np.random.default_rng(15)
    n = rng.integers(0, 4, 300).tolist()
    n[170] = 90
    c = Case(dtype, 2, 1, 32, n, seed=15)
    c.check(c.run())
    c = Case(dtype, 2, 1, 32, n, [m + int(x) for m, x in zip(n, rng.integers(0, 9, 300))], seed=16)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs", [65, 1000, 70000])
def test_few_rows_in_many_slots(dtype, n_seqs):
    """A row here and there, ahead of everything, and in the last slot, behind keys that are split."""
    n, t = [0] * n_seqs, [0] * n_seqs
    for b, rows, keys in ((0, 1, 900), (1, 2, 0), (n_seqs // 2, 130, 2500), (n_seqs - 2, 3, 3000), (n_seqs - 1, 1, 1)):
        n[b], t[b] = rows, keys
    t[7] = 50                       # (keys that nobody asks about)
    c = Case(dtype, 8, 2, 64, n, t, seed=29, lead=3, trail=2)
    c.check(c.run())
    c.check(c.run(max_kv=100))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_many_scores_near_the_reference(dtype, hd):
    """Scores (base 2) that rise by up to 8 behind the first block, for all keys from there on, for some rows of a tile more than for others, and fall again: the reference is moved by
    whole numbers, and the weights before and behind it add up."""
    import torch
    rng = np.random.default_rng(30)

    def edit(c):
        c.q[..., 0] = torch.from_numpy(rng.integers(0, 3, c.q.shape[:2]).astype(np.float32)).cuda().to(c.q.dtype)
        c.q[..., 1:] = 0
        c.k[..., 0] = 0
        for at, score in ((64, 2.5), (128, 3.5), (200, 4.0), (300, 1.0), (400, 7.0)):
            c.k[at:, :, 0] = score
    for n, t, max_kv in (([500, 90], None, 500), ([30], [500], 500), ([30], [500], 64)):
        c = Case(dtype, 4, 2, hd, n, t, seed=31, edit=edit)
        c.check(c.run(scale=float(np.log(2.0)), max_kv=max_kv), scale=float(np.log(2.0)))
