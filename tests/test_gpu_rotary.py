"""Rotary positions on the GPU, against 64 bits."""
import math

import numpy as np
import pytest

import tree_oracle

pytestmark = pytest.mark.gpu


def check(x, y, positions, f, interleaved, magnitude, dtype):
    """An angle is off by at most 2^-32 turns; sine and cosine come from it within 4 * 2^-24 (the rest as a float, two constants and the last steps
    of a polynomial, half a step of 2^-24 each, of numbers up to 1), and the products, their sum and the magnitude round once each: 8 * 2^-24 of
    |a| + |b| in all. Then half a step of the output's type, 2^-24 or 2^-8 of the value."""
    want, size = tree_oracle.rotary(x.double().cpu().numpy(), positions, f, interleaved, magnitude)
    off = np.abs(y.double().cpu().numpy() - want)
    half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    assert (off <= 8 * 2.0 ** -24 * size + half * np.abs(want) + 1e-44).all(), off.max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hd,r,scaling", [(64, 64, "none"), (128, 64, "parts"), (128, 128, "linear"), (256, 256, "base"), (32, 32, "none"), (96, 80, "none"), (80, 30, "parts"),
                                          (64, 2, "linear"), (66, 66, "none"), (512, 512, "none"), (7, 4, "none"), (40, 40, "base")])
def test_rotary(dtype, interleaved, hd, r, scaling):
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(hd + r)
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    kw = dict(theta=10000.0, scaling=scaling, factor=8.0)
    f = tree_oracle.frequencies(r, scaling=scaling, factor=8.0, trained=8192.0, low=1.0, high=32.0)
    table = sjd.rope_table(r, trained_ctx=8192.0, low_turns=1.0, high_turns=32.0, **kw)
    for n, H, Hk in ((1, 1, 0), (5, 4, 2), (37, 6, 3), (1100, 2, 1)):
        positions = rng.integers(-5, 1000000, n)
        positions[0] = 0
        pos = torch.tensor(positions.astype(np.int32), device="cuda")
        q = torch.from_numpy(rng.standard_normal((n, H, hd)).astype(np.float32)).cuda().to(td)
        k = torch.from_numpy(rng.standard_normal((n, Hk, hd)).astype(np.float32)).cuda().to(td) if Hk else None
        q2, k2 = sjd.op_rotary(q, k, pos, table, interleaved=interleaved, magnitude=1.25)
        check(q, q2, positions, f, interleaved, 1.25, dtype)
        if Hk:
            check(k, k2, positions, f, interleaved, 1.25, dtype)
        else:
            assert k2 is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_within_a_fused_projection(dtype):
    """Queries and keys are parts of one buffer's rows, turned in place; what lies beside them stays."""
    import paper_2512_07503_amd as sjd
    import torch
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(1)
    for hd, pad in ((64, 0), (64, 3), (128, 8)):
        buf = torch.randn((9, 8 * hd + pad), generator=g, device="cuda").to(td)
        old = buf.clone()
        part = lambda b, lo, hi: b[:, lo * hd:hi * hd].unflatten(1, (hi - lo, hd))
        q, k = part(buf, 0, 4), part(buf, 4, 6)
        positions = np.arange(9) * 1000
        table = sjd.rope_table(hd)
        sjd.op_rotary(q, k, torch.tensor(positions.astype(np.int32), device="cuda"), table, out=(q, k))
        f = tree_oracle.frequencies(hd)
        check(part(old, 0, 4), q, positions, f, False, 1.0, dtype)
        check(part(old, 4, 6), k, positions, f, False, 1.0, dtype)
        assert torch.equal(buf[:, 6 * hd:], old[:, 6 * hd:])


def test_far_positions_and_the_way_back():
    """At 2^31 - 1 positions a float angle has no fraction left; a turn by -pos undoes one by pos."""
    import paper_2512_07503_amd as sjd
    import torch
    hd = 128
    positions = np.array([2147483647, 2147483646, 2000000000, 16777217, -2147483648], dtype=np.int64)
    pos = torch.tensor(positions.astype(np.int32), device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((5, 2, hd), generator=g, device="cuda")
    table = sjd.rope_table(hd)
    turned, _ = sjd.op_rotary(q, None, pos, table)
    # the reference's angle in exact rationals: the table is what the operator is given, and it is within 2^-53 of theta's powers
    turns = table.cpu().numpy().view(np.uint64)
    frac = np.array([[((int(p) * int(t)) % (1 << 64)) / 2.0 ** 64 for t in turns] for p in positions])
    x = q.double().cpu().numpy()
    c, s = np.cos(2 * math.pi * frac)[:, None], np.sin(2 * math.pi * frac)[:, None]
    a, b = x[..., :hd // 2], x[..., hd // 2:]
    want = np.concatenate([a * c - b * s, b * c + a * s], axis=-1)
    size = np.concatenate([np.abs(a) + np.abs(b)] * 2, axis=-1)
    assert (np.abs(turned.double().cpu().numpy() - want) <= 9 * 2.0 ** -24 * size).all()
    back, _ = sjd.op_rotary(turned[:4].contiguous(), None, -pos[:4], table)
    assert (np.abs(back.double().cpu().numpy() - x[:4]) <= 30 * 2.0 ** -24 * size[:4]).all()


def test_no_rows_and_many_rows():
    import paper_2512_07503_amd as sjd
    import torch
    table = sjd.rope_table(64)
    q = torch.zeros((0, 2, 64), device="cuda")
    assert sjd.op_rotary(q, None, torch.zeros(0, dtype=torch.int32, device="cuda"), table)[0].shape == (0, 2, 64)
    n = 70001
    q = torch.randn((n, 1, 64), device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    got, _ = sjd.op_rotary(q, None, pos, table)
    pick = np.concatenate([np.arange(20), np.arange(n - 20, n), np.random.default_rng(0).integers(0, n, 200)])
    check(q[pick], got[pick], pick, tree_oracle.frequencies(64), False, 1.0, "f32")


def test_refusals():
    import paper_2512_07503_amd as sjd
    import torch
    table, pos = sjd.rope_table(64), torch.zeros(4, dtype=torch.int32, device="cuda")
    q = torch.zeros((4, 2, 64), device="cuda")
    for args in [(q.double(), None, pos, table), (q, None, pos.long(), table), (q, None, pos[:3], table), (q, None, pos.cpu(), table), (q, None, pos, table.int()),
                 (q, q.bfloat16(), pos, table), (q, q[:3], pos, table), (q[..., :32], None, pos, table), (q.transpose(0, 1), None, pos[:2], table)]:
        with pytest.raises(sjd.SjdError):
            sjd.op_rotary(*args)
    buf = torch.zeros((5, 2, 64), device="cuda")
    with pytest.raises(sjd.SjdError):
        sjd.op_rotary(buf[:4], None, pos, table, out=(buf[1:],))
