"""Log probabilities of tokens, entropy and alternatives on the GPU, against 64 bits."""
import numpy as np
import pytest

import prompt_oracle

pytestmark = pytest.mark.gpu


def check(z, tokens, n_top, **kw):
    """z and tokens on the GPU.  A lane adds up V / 256 terms at most, and 64 and 4 lanes and the parts of a row join; a term's exponent is rounded, 2^-24 of it, and its exponential
    is 2^-22 off: the sum is, relatively, (V / 256 + 64) 2^-24 + 2^-22 + 2^-23 E off, E = sum p |ln p - ln p_max|, its logarithm as much absolutely, and 2^-22 of itself and of 1.  A difference
    of logits is rounded once, and a result.  The mean of the exponents has each term off by what a term of the sum is, times it."""
    import paper_2512_07503_amd as sjd
    got = [t.cpu().numpy() for t in sjd.op_token_logprobs(z, tokens, n_top=n_top, **kw)]
    r = prompt_oracle.logprobs(z.double().cpu().numpy(), tokens.cpu().numpy(), n_top)
    finite = ~np.isnan(r["entropy"])
    assert np.array_equal(got[1][finite], r["rank"][finite]) and np.array_equal(got[3], r["ids"])
    V = z.shape[1]
    term = (V / 256 + 64) * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -23 * r["dist"]
    ln_s = term + 2.0 ** -22 * (1 + r["ln_s"])
    for name, have, tol in (("logprob", got[0], ln_s), ("entropy", got[2], ln_s + 2 * term * (1 + r["dist"])), ("top", got[4], ln_s[:, None])):
        want = r[name]
        assert np.array_equal(np.isnan(have), np.isnan(want)) and np.array_equal(have == -np.inf, want == -np.inf), name
        ok = np.isfinite(want)
        off = np.abs(np.where(ok, have, 0) - np.where(ok, want, 0)) - tol - 2.0 ** -22 * np.abs(np.where(ok, want, 0))
        assert off.size == 0 or off.max() <= 0, (name, off.max(), np.unravel_index(off.argmax(), off.shape))
    return got


def tensors(z, tokens, dtype):
    import torch
    t = torch.from_numpy(np.asarray(z, dtype=np.float32)).cuda()
    return t if dtype == "f32" else t.bfloat16(), torch.tensor(np.asarray(tokens, dtype=np.int32), device="cuda")


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 63), (4, 64), (3, 100), (7, 1000), (2, 1023), (2, 4096), (3, 4099), (1, 16384), (3, 16385), (2, 20001), (40, 5003), (5, 70001), (1100, 300), (2, 200003)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_logprobs(dtype, rows, vocab):
    """From one id to many, rows aligned and not; few rows are split, many are not."""
    rng = np.random.default_rng(rows + vocab)
    z, tokens = tensors(2.5 * rng.standard_normal((rows, vocab)), rng.integers(0, vocab, rows), dtype)
    for n_top in (0, 1, 5, 20, 64):
        check(z, tokens, n_top)
    if rows <= 5:
        tokens = z.float().argmax(dim=1).int()
        check(z, tokens, 3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [50, 3001, 40003])
def test_masked_ids(dtype, vocab):
    """Masks that leave a range, few ids, one or none; tokens that are masked, outside, or the only one."""
    rng = np.random.default_rng(vocab)
    z = 2.5 * rng.standard_normal((12, vocab))
    lo = vocab // 3
    z[0, :lo] = -np.inf
    z[1, lo:] = -np.inf
    z[2] = -np.inf
    z[3] = -np.inf
    z[3, vocab - 1] = 1.5
    z[4] = -np.inf
    z[4, 7] = -1e30
    z[5] = -np.inf
    z[5, [3, 11, vocab - 2]] = [2.0, 2.0, 5.0]
    z[6, ::2] = -np.inf
    z[7, lo:lo + 20] = -np.inf
    z[8] = np.finfo(np.float32).min       # (a mask of the lowest value is a distribution, an even one here)
    z[9, 1:] = np.finfo(np.float32).min
    tokens = [lo - 1, lo, 9, vocab - 1, 7, 12, 1, lo + 3, vocab - 1, 0, -1, vocab]
    z, tokens = tensors(z, tokens, dtype)
    # (bf16 rounds the lowest float to -inf: its own lowest value)
    import torch
    z[8:10] = torch.where(z[8:10] == -np.inf, torch.finfo(z.dtype).min, z[8:10].float()).to(z.dtype)
    for n_top in (0, 4, 64):
        check(z, tokens, n_top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [130, 2050, 30000])
def test_equal_logits(dtype, vocab):
    """Ties go to the lower id: rows of one value, of two, of few; -0 is 0."""
    rng = np.random.default_rng(vocab)
    z = np.zeros((8, vocab))
    z[1] = rng.integers(0, 2, vocab)
    z[2] = rng.integers(0, 9, vocab)
    z[3] = np.where(rng.random(vocab) < 0.5, 0.0, -0.0)
    z[4] = -5.0
    z[4, vocab // 2:] = -4.0
    z[5, -3:] = 1.0
    z[6, ::7] = 0.5
    z[7] = -rng.integers(0, 3, vocab)
    z, tokens = tensors(z, rng.integers(0, vocab, 8), dtype)
    for n_top in (1, 5, 33, 64):
        check(z, tokens, n_top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5000, 66000])
def test_orders(dtype, vocab):
    """Ascending rows, of which every step holds larger ones than all before, descending ones, saw teeth: what is collected fills its buffer and is sifted."""
    x = np.linspace(-30, 20, vocab)
    z = np.stack([x, x[::-1], np.sort(np.abs(np.sin(np.arange(vocab)))) * 9, (np.arange(vocab) % 1024) * 0.01, (np.arange(vocab) // 1024) * 0.5,
                  np.where(np.arange(vocab) % 64 < 5, x, -50.0), np.where(np.arange(vocab) % 4 == 0, x, -50.0)])
    z, tokens = tensors(z, np.arange(7) * 700, dtype)
    for n_top in (1, 20, 64):
        check(z, tokens, n_top)
    many = z.repeat(300, 1)          # (enough rows that none is split)
    import paper_2512_07503_amd as sjd
    for n_top in (20, 64):
        want = check(z, tokens, n_top)
        got = sjd.op_token_logprobs(many, tokens.repeat(300), n_top=n_top)
        for a, b in ((1, 1), (3, 3)):
            assert np.array_equal(got[a].cpu().numpy().reshape(300, *want[b].shape), np.broadcast_to(want[b], (300, *want[b].shape)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nan(dtype):
    """+inf or NaN in a row make its numbers NaN, and no other row's."""
    rng = np.random.default_rng(0)
    for vocab in (40, 9001):
        z = rng.standard_normal((6, vocab))
        z[1, vocab - 1], z[2, 3], z[4, 0] = np.nan, np.inf, np.nan
        z[4, 1:] = -np.inf
        z, tokens = tensors(z, [1, 2, 3, 4, 0, 6], dtype)
        for n_top in (0, 7):
            check(z, tokens, n_top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sharp_and_large(dtype):
    """Logits of hundreds and thousands, one id that takes all, a row of almost equal ones."""
    rng = np.random.default_rng(1)
    z = rng.standard_normal((6, 7001))
    z[0] *= 300.0
    z[1] += 5000.0
    z[2, 17] = 60.0
    z[3] *= 1e-6
    z[4] -= 1e5
    z[5] *= 1e30
    z, tokens = tensors(z, [5, 6, 17, 8, 9, 10], dtype)
    check(z, tokens, 10)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    rng = np.random.default_rng(2)
    for pad, first in ((1, 0), (3, 1), (8, 0), (16, 5)):
        z, tokens = tensors(rng.standard_normal((9, 2000 + pad)), rng.integers(0, 2000 - first, 9), dtype)
        check(z[:, first:2000], tokens, 6)


def test_no_rows_and_refusals():
    import paper_2512_07503_amd as sjd
    import torch
    z, tokens = torch.zeros((0, 9), device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    assert [tuple(t.shape) for t in sjd.op_token_logprobs(z, tokens, n_top=3)] == [(0,), (0,), (0,), (0, 3), (0, 3)]
    z, tokens = torch.zeros((4, 9), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for args, kw in [((z.half(), tokens), {}), ((z, tokens.long()), {}), ((z, tokens[:3]), {}), ((z, tokens.cpu()), {}), ((z[0], tokens), {}), ((z.t(), tokens), {}),
                     ((z, tokens), dict(n_top=65)), ((z, tokens), dict(n_top=-1)), ((z[:, :0], tokens), {})]:
        with pytest.raises(sjd.SjdError):
            sjd.op_token_logprobs(*args, **kw)


def test_workspace():
    import paper_2512_07503_amd as sjd
    import torch
    z, tokens = tensors(np.random.default_rng(3).standard_normal((2, 50000)), [5, 49999], "f32")
    need = sjd.binding._logprob_bytes(2, 50000, 9)
    assert need > 0
    guard = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    check(z, tokens, 9, workspace=guard[256:256 + need])
    assert (guard[:256] == 0x5A).all() and (guard[256 + need:] == 0x5A).all()
    with pytest.raises(sjd.SjdError) as e:
        sjd.op_token_logprobs(z, tokens, n_top=9, workspace=guard[:need - 16])
    assert e.value.code == sjd.ECAPACITY


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 5003, 70001])
def test_nothing_is_above_zero(dtype, vocab):
    """Rows of which one id has all the weight, alone or beside ids that are far below or follow at once: ln p is at most 0, as p is at most 1."""
    rng = np.random.default_rng(vocab)
    z = np.full((120, vocab), -np.inf)
    tokens = rng.integers(0, vocab, 120)
    z[40:80] = 2.5 * rng.standard_normal((40, vocab)) - 60.0
    z[np.arange(120), tokens] = 30.0 * rng.standard_normal(120)
    z[80:, 0] = np.where(tokens[80:] == 0, z[80:, 0], z[np.arange(80, 120), tokens[80:]] - rng.uniform(1.0, 8.0, 40))
    z, tokens = tensors(z, tokens, dtype)
    for n_top in (0, 3):
        got = check(z, tokens, n_top)
        assert got[0].max() <= 0 and (not n_top or got[4].max() <= 0) and got[2].min() >= 0
    # (many rows, of which none is split)
    import paper_2512_07503_amd as sjd
    got = sjd.op_token_logprobs(z.repeat(20, 1), tokens.repeat(20), n_top=2)
    assert got[0].max().item() <= 0 and got[4].max().item() <= 0
