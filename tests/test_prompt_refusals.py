"""What the operators of scoring and prefilling prompts refuse on the host, through the C ABI with pointers that nothing may follow."""
import ctypes as C

import pytest

import paper_2512_07503_amd as sjd

MiB = 1 << 20
p = C.c_void_p
NULL = None


def refused(rc, code=sjd.EINVAL, text=b""):
    assert rc == code, rc
    message = sjd.lib().sjd_last_error(None)
    assert message and text in message, message


def norm_rotary(**c):
    a = {**dict(dtype=sjd.F32, norm=0, eps=1e-5, per_head=0, table=p(64), r=64, pos=p(64), n=3, hd=64, q=p(MiB), qs=256, qg=p(64), qb=NULL, qo=p(2 * MiB), qos=256, H=4, k=p(3 * MiB), ks=128,
                kg=p(64), kb=NULL, ko=p(4 * MiB), kos=128, Hk=2), **c}
    return sjd.lib().sjd_op_norm_rotary(None, a["dtype"], a["norm"], a["eps"], a["per_head"], 0, a["table"], a["r"], 1.0, a["pos"], a["n"], a["hd"], a["q"], a["qs"], a["qg"], a["qb"], a["qo"],
                                        a["qos"], a["H"], a["k"], a["ks"], a["kg"], a["kb"], a["ko"], a["kos"], a["Hk"])


def test_norm_rotary():
    for bad in [dict(dtype=sjd.FP8), dict(dtype=-1), dict(norm=2), dict(norm=-1), dict(eps=0.0), dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-38),
                dict(table=NULL), dict(r=0), dict(r=63), dict(r=66), dict(r=-2), dict(hd=1), dict(hd=514, r=64), dict(pos=NULL), dict(n=-1), dict(n=(1 << 29) + 1), dict(q=NULL), dict(qg=NULL),
                dict(qo=NULL), dict(k=NULL), dict(kg=NULL), dict(ko=NULL), dict(H=0), dict(Hk=-1), dict(H=(1 << 16) + 1), dict(q=p(MiB + 2)), dict(qo=p(2 * MiB + 1)), dict(kg=p(66)),
                dict(qb=p(65)), dict(kb=p(62)), dict(qs=-256), dict(qos=255), dict(kos=127)]:
        refused(norm_rotary(**bad))
    for bad in [dict(qo=p(3 * MiB)), dict(ko=p(MiB + 100 * 4)), dict(qo=p(MiB + 4)), dict(qo=p(MiB), qos=260), dict(ko=p(2 * MiB)), dict(ko=p(2 * MiB + 255 * 4), kos=256),
                dict(qg=p(2 * MiB)), dict(qg=p(4 * MiB + 63 * 4)), dict(kg=p(2 * MiB - 63 * 4)), dict(kb=p(4 * MiB + 128 * 4)), dict(per_head=1, qg=p(2 * MiB - 255 * 4)),
                dict(qb=p(2 * MiB + 3 * 256 * 4 - 4))]:
        refused(norm_rotary(**bad), text=b"overlap")
    assert norm_rotary(n=0, q=NULL, qo=NULL, k=NULL, ko=NULL, pos=NULL) == sjd.OK
    for n in (1 << 27, 1 << 29):
        refused(norm_rotary(dtype=sjd.BF16, n=n, hd=8, r=8, q=p(1 << 40), qs=8, qo=p(1 << 41), qos=8, H=1, Hk=0), text=b"one launch")
        refused(norm_rotary(dtype=sjd.BF16, n=n, hd=2, r=2, q=p(1 << 40), qs=2, qo=p(1 << 41), qos=2, H=1, Hk=0), text=b"one launch")


def attention(**c):
    a = {**dict(dtype=sjd.BF16, q=p(MiB), qs=256, k=p(2 * MiB), ks=128, v=p(3 * MiB), vs=128, out=p(4 * MiB), os=256, rows=p(64), kv=p(64), n=10, nk=20, seqs=2, H=4, Hk=2, hd=64, scale=0.0,
                max_rows=10, max_kv=20, ws=p(8 * MiB), bytes=1 << 40), **c}
    return sjd.lib().sjd_op_prompt_attention(None, a["dtype"], a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["out"], a["os"], a["rows"], a["kv"], a["n"], a["nk"], a["seqs"], a["H"], a["Hk"],
                                             a["hd"], a["scale"], a["max_rows"], a["max_kv"], a["ws"], a["bytes"])


def need(dtype=sjd.BF16, n=10, seqs=2, H=4, Hk=2, hd=64, max_rows=10, max_kv=20):
    b = C.c_uint64(0)
    rc = sjd.lib().sjd_op_prompt_attention_workspace(dtype, n, seqs, H, Hk, hd, max_rows, max_kv, C.byref(b))
    return rc, b.value


def test_attention():
    sizes = [dict(dtype=sjd.FP8), dict(dtype=7), dict(n=-1), dict(n=(1 << 29) + 1), dict(seqs=0), dict(seqs=-1), dict(H=0), dict(H=3), dict(Hk=0), dict(Hk=1 << 16, H=1 << 16), dict(hd=0),
             dict(hd=80), dict(hd=512), dict(max_rows=-1), dict(max_kv=-1), dict(max_kv=(1 << 30) + 1), dict(max_rows=(1 << 29) + 1)]
    for bad in sizes:
        refused(attention(**bad))
        refused(need(**bad)[0])
    refused(sjd.lib().sjd_op_prompt_attention_workspace(sjd.BF16, 10, 2, 4, 2, 64, 10, 20, None))
    for bad in [dict(q=NULL), dict(k=NULL), dict(v=NULL), dict(out=NULL), dict(rows=NULL), dict(nk=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=p(MiB + 1)),
                dict(k=p(MiB + 1)), dict(v=p(MiB + 1)), dict(out=p(MiB + 1)), dict(qs=-1), dict(ks=-1), dict(vs=-128), dict(os=255), dict(dtype=sjd.F32, q=p(MiB + 2))]:
        refused(attention(**bad))
    for bad in [dict(out=p(MiB + 2)), dict(out=p(MiB), os=512), dict(out=p(2 * MiB)), dict(out=p(3 * MiB - 4)), dict(out=p(2 * MiB + 19 * 256 + 254)), dict(out=p(3 * MiB), os=512),
                dict(kv=NULL, out=p(2 * MiB + 9 * 256)), dict(q=p(4 * MiB), out=p(4 * MiB + 2), n=1)]:
        refused(attention(**bad), text=b"overlap")
    assert attention(n=0, q=NULL, k=NULL, v=NULL, out=NULL) == sjd.OK
    for bad in [dict(n=1 << 29, H=16), dict(n=1 << 29, H=64, Hk=64), dict(n=(1 << 20), seqs=1 << 20, H=64, Hk=64), dict(n=1 << 29, seqs=1 << 30)]:
        refused(attention(**bad), text=b"one launch")
        refused(need(**bad)[0], text=b"one launch")


def test_attention_workspace():
    sizes = dict(n=1, seqs=1, H=8, Hk=1, max_rows=1, max_kv=30000)
    rc, bytes_ = need(**sizes)
    assert rc == sjd.OK and bytes_ > 0 and need()[1] == 0
    refused(attention(**sizes, bytes=bytes_ - 1), code=sjd.ECAPACITY)
    refused(attention(**sizes, bytes=bytes_, ws=NULL))
    refused(attention(**sizes, bytes=bytes_, ws=p(MiB + 8)))
    # many rows need none, however long they are
    assert need(n=1 << 20, seqs=4, H=32, Hk=8, hd=128, max_rows=1 << 18, max_kv=1 << 18) == (sjd.OK, 0)


def logprobs(**c):
    a = {**dict(dtype=sjd.F32, z=p(MiB), stride=5000, tok=p(2 * MiB), lp=p(3 * MiB), rank=p(4 * MiB), ent=p(5 * MiB), ids=p(6 * MiB), top=p(7 * MiB), n=10, V=5000, k=5, ws=p(8 * MiB), bytes=1 << 30), **c}
    return sjd.lib().sjd_op_token_logprobs(None, a["dtype"], a["z"], a["stride"], a["tok"], a["lp"], a["rank"], a["ent"], a["ids"], a["top"], a["n"], a["V"], a["k"], a["ws"], a["bytes"])


def test_logprobs():
    for bad in [dict(dtype=sjd.FP8), dict(dtype=5), dict(n=-1), dict(V=0), dict(V=-4), dict(V=(1 << 24) + 1), dict(k=-1), dict(k=65), dict(z=NULL), dict(tok=NULL), dict(lp=NULL), dict(rank=NULL),
                dict(ent=NULL), dict(ids=NULL), dict(top=NULL), dict(z=p(MiB + 2)), dict(dtype=sjd.BF16, z=p(MiB + 1)), dict(stride=-1), dict(lp=p(3 * MiB + 2)), dict(top=p(7 * MiB + 1))]:
        refused(logprobs(**bad))
    for bad in [dict(lp=p(MiB)), dict(rank=p(2 * MiB + 36)), dict(ent=p(3 * MiB - 36)), dict(ids=p(7 * MiB + 196)), dict(top=p(MiB + 10 * 5000 * 4 - 4)), dict(ids=p(2 * MiB - 196))]:
        refused(logprobs(**bad), text=b"overlap")
    assert logprobs(n=0, z=NULL, tok=NULL, lp=NULL, rank=NULL, ent=NULL, ids=NULL, top=NULL) == sjd.OK
    b = C.c_uint64(0)
    L = sjd.lib()
    assert L.sjd_op_token_logprobs_workspace(2, 50000, 5, C.byref(b)) == sjd.OK and b.value > 0
    refused(logprobs(n=2, V=50000, stride=50000, bytes=b.value - 1), code=sjd.ECAPACITY)
    refused(logprobs(n=2, V=50000, stride=50000, bytes=b.value, ws=NULL))
    refused(logprobs(n=2, V=50000, stride=50000, bytes=b.value, ws=p(8 * MiB + 4)))
    for bad in [(-1, 5, 0), (1, 0, 0), (1, 5, 65), (1 << 24, 5, 0)]:
        refused(L.sjd_op_token_logprobs_workspace(*bad, C.byref(b)))
    refused(L.sjd_op_token_logprobs_workspace(2, 50000, 5, None))
    assert L.sjd_op_token_logprobs_workspace(5000, 65536, 20, C.byref(b)) == sjd.OK and b.value == 0


@pytest.mark.parametrize("n_top", [1, 5, 20, 64])
def test_parts_of_a_row_fit_the_join(n_top):
    """The parts' keys, 8 bytes each behind 16 of sums, are at most what the joining workgroup holds."""
    b = C.c_uint64(0)
    for vocab in (1, 5000, 70000, 1 << 24):
        for rows in (1, 3, 100):
            assert sjd.lib().sjd_op_token_logprobs_workspace(rows, vocab, n_top, C.byref(b)) == sjd.OK
            parts = b.value // rows // (16 + 8 * n_top)
            assert b.value == rows * parts * (16 + 8 * n_top) and parts * n_top <= 1024


@pytest.mark.parametrize("dtype", [sjd.BF16, sjd.F32])
@pytest.mark.parametrize("rows", [1, 8, 40])
@pytest.mark.parametrize("max_kv", [3000, 30000, 100000])
def test_slots_without_rows_need_no_workspace(dtype, rows, max_kv):
    """A batch of any number of slots has at most `rows` sequences with rows: its workspace is what so many sequences need, and the call is not refused for its slots."""
    sizes = dict(dtype=dtype, n=rows, H=32, Hk=8, hd=128, max_rows=rows, max_kv=max_kv)
    rc, alone = need(**sizes, seqs=rows)
    assert rc == sjd.OK and alone > 0
    for seqs in (64, 65, 500, 4096, 1 << 20, 1 << 30):
        assert need(**sizes, seqs=seqs) == (sjd.OK, alone), seqs


def test_expected_keys_refuse_no_call():
    """max_kv only chooses how the work is divided: a call that is accepted without splits is accepted whatever it says, with a workspace of at most 32 times the places' partial
    results (1 280 workgroups of 128 rows), and of a few rows with more keys than are split one by one."""
    for dtype, n, H, Hk, hd in [(sjd.F32, 1 << 20, 16, 4, 128), (sjd.F32, 1 << 22, 16, 4, 128), (sjd.F32, 1 << 22, 16, 16, 64), (sjd.F32, 1 << 20, 64, 1, 256), (sjd.F32, 100000, 8, 8, 32),
                                (sjd.BF16, 1 << 22, 16, 4, 128), (sjd.F32, 1, 8, 1, 128)]:
        for seqs in (1, 300):
            assert need(dtype=dtype, n=n, seqs=seqs, H=H, Hk=Hk, hd=hd, max_rows=0, max_kv=0) == (sjd.OK, 0)
            for max_kv in (1 << 16, 1 << 20, 1 << 30):
                rc, bytes_ = need(dtype=dtype, n=n, seqs=seqs, H=H, Hk=Hk, hd=hd, max_rows=n, max_kv=max_kv)
                assert rc == sjd.OK and bytes_ <= 32 * 1280 * 128 * (hd + 2) * 4, (n, max_kv)


def test_max_rows_needs_no_workspace():
    for max_kv in (20, 3000, 1 << 20):
        assert len({need(H=32, Hk=8, hd=128, max_rows=m, max_kv=max_kv) for m in (0, 1, 10, 1 << 29)}) == 1
