"""What the tree operators refuse on the host, through the C ABI with pointers that nothing may follow, and their host-side helpers."""
import ctypes as C
import math

import numpy as np
import pytest

import tree_oracle
import paper_2512_07503_amd as sjd
from paper_2512_07503_amd.binding import KvCacheDesc

ONE, ODD, NULL = C.c_void_p(64), C.c_void_p(65), None      # (aligned, unaligned and no pointer)


def desc(**change):
    d = dict(pages=64, page_table=64, n_pages=4, page_tokens=64, n_kv_heads=2, head_dim=64, dtype=sjd.BF16, n_seqs=2, pages_per_seq=3)
    d.update(change)
    return C.byref(KvCacheDesc(*[d[n] for n, _ in KvCacheDesc._fields_]))


BAD_SHAPES = [dict(dtype=3), dict(dtype=-1), dict(page_tokens=0), dict(page_tokens=48), dict(page_tokens=-32), dict(n_kv_heads=0), dict(head_dim=0),
              dict(head_dim=80), dict(head_dim=512), dict(head_dim=-64)]
BAD_CACHES = BAD_SHAPES + [dict(pages=0), dict(pages=72), dict(page_table=0), dict(n_pages=0), dict(n_seqs=0), dict(pages_per_seq=0),
                           dict(pages_per_seq=1 << 26)]


def refused(rc, code=sjd.EINVAL):
    assert rc == code, rc
    assert sjd.lib().sjd_last_error(None)


def test_page_bytes():
    L, n = sjd.lib(), C.c_uint64(0)
    assert L.sjd_cache_page_bytes(desc(dtype=sjd.FP8), C.byref(n)) == 0 and n.value == 2 * 2 * 64 * (64 + 1)
    assert L.sjd_cache_page_bytes(desc(pages=0, page_table=0, n_pages=0, n_seqs=0), C.byref(n)) == 0 and n.value == 2 * 2 * 64 * 64 * 2
    refused(L.sjd_cache_page_bytes(None, C.byref(n)))
    refused(L.sjd_cache_page_bytes(desc(), None))
    for bad in BAD_SHAPES:
        refused(L.sjd_cache_page_bytes(desc(**bad), C.byref(n)))


def test_cache_rows():
    L = sjd.lib()
    good = dict(cache=desc(), dtype=sjd.F32, k=ONE, ks=128, v=ONE, vs=128, rows=ONE, first=ONE, n=5)

    def write(**c):
        a = {**good, **c}
        return L.sjd_op_cache_write(None, a["cache"], a["dtype"], a["k"], a["ks"], a["v"], a["vs"], a["rows"], a["first"], a["n"])

    def read(**c):
        a = {**good, **c}
        return L.sjd_op_cache_read(None, a["cache"], a["dtype"], a["k"], a["v"], a["rows"], a["first"], a["n"])

    for call in (write, read):
        for bad in [dict(cache=None), dict(dtype=sjd.FP8), dict(dtype=7), dict(k=NULL), dict(v=NULL), dict(rows=NULL), dict(first=NULL), dict(n=-1),
                    dict(n=(1 << 29) + 1), dict(k=ODD), dict(v=ODD)] + [dict(cache=desc(**b)) for b in BAD_CACHES]:
            refused(call(**bad))
        assert call(n=0, k=NULL, v=NULL) == sjd.OK             # nothing to do
    for v in (64, 64 + 4, 64 + 5 * 2 * 64 * 4 - 4):            # keys and values on each other
        refused(read(v=C.c_void_p(v)))


def test_cache_compact():
    L = sjd.lib()
    for a in [(None, ONE, ONE, ONE, 4), (desc(), NULL, ONE, ONE, 4), (desc(), ONE, NULL, ONE, 4), (desc(), ONE, ONE, NULL, 4), (desc(), ONE, ONE, ONE, 0)]:
        refused(L.sjd_op_cache_compact(None, *a))
    for b in BAD_CACHES:
        refused(L.sjd_op_cache_compact(None, desc(**b), ONE, ONE, ONE, 4))


def test_rotary():
    L = sjd.lib()
    Q, QO, K, KO = (C.c_void_p(x << 20) for x in (1, 2, 3, 4))
    good = dict(dtype=sjd.F32, table=ONE, r=64, pos=ONE, n=3, hd=64, q=Q, qs=256, qo=QO, qos=256, H=4, k=K, ks=128, ko=KO, kos=128, Hk=2)

    def call(**c):
        a = {**good, **c}
        return L.sjd_op_rotary(None, a["dtype"], 0, a["table"], a["r"], 1.0, a["pos"], a["n"], a["hd"], a["q"], a["qs"], a["qo"], a["qos"], a["H"], a["k"],
                               a["ks"], a["ko"], a["kos"], a["Hk"])

    for bad in [dict(dtype=sjd.FP8), dict(table=NULL), dict(r=0), dict(r=63), dict(r=66), dict(hd=1, r=2), dict(hd=514, r=2), dict(pos=NULL), dict(n=-1), dict(q=NULL),
                dict(qo=NULL), dict(k=NULL), dict(ko=NULL), dict(H=0), dict(Hk=-1), dict(q=C.c_void_p((1 << 20) + 2)), dict(qos=255), dict(kos=127), dict(qs=-256),
                dict(qo=C.c_void_p((1 << 20) + 64)), dict(qo=Q, qos=300), dict(ko=Q), dict(qo=K, qos=128)]:
        refused(call(**bad))
    assert call(n=0, q=NULL, qo=NULL, k=NULL, ko=NULL, pos=NULL) == sjd.OK


def test_rope_table():
    L = sjd.lib()
    t = np.zeros(64, dtype=np.uint64)
    p = t.ctypes.data
    for a in [(0, 1e4, 0, 1, 0, 0, 1), (63, 1e4, 0, 1, 0, 0, 1), (514, 1e4, 0, 1, 0, 0, 1), (64, 1.0, 0, 1, 0, 0, 1), (64, math.nan, 0, 1, 0, 0, 1), (64, math.inf, 0, 1, 0, 0, 1),
              (64, 1e4, 4, 1, 0, 0, 1), (64, 1e4, -1, 1, 0, 0, 1), (64, 1e4, 1, 0.5, 0, 0, 1), (64, 1e4, 1, math.nan, 0, 0, 1), (2, 1e4, 2, 4, 0, 0, 1),
              (64, 1e4, 3, 4, 0, 1, 32), (64, 1e4, 3, 4, 8192, -1, 32), (64, 1e4, 3, 4, 8192, 32, 32), (64, 1e4, 3, 4, 8192, 1, math.nan)]:
        refused(L.sjd_rope_table(*a, p))
    refused(L.sjd_rope_table(64, 1e4, 0, 1, 0, 0, 1, None))
    for r in (2, 30, 128):
        for name, code in (("none", 0), ("linear", 1), ("base", 2), ("parts", 3)):
            if r == 2 and name == "base":
                continue
            assert L.sjd_rope_table(r, 5e5, code, 8.0, 8192.0, 1.0, 4.0, p) == sjd.OK
            f = tree_oracle.frequencies(r, 5e5, name, 8.0, 8192.0, 1.0, 4.0)
            # (the oracle's powers are doubles; position 10^6 then is 10^6 * 2^-52 radians off at most)
            assert np.allclose(t[:r // 2].astype(np.float64) * 2.0 ** -64 * 2 * math.pi, f, rtol=1e-13, atol=2.0 ** -63)


def test_tree_masks():
    rng = np.random.default_rng(0)
    for n in (0, 1, 5, 32, 33, 100):
        parents = tree_oracle.random_tree(rng, n) if n else []
        mask, depth = sjd.tree_masks(parents, mask_words=4)
        want = tree_oracle.ancestors(parents)
        assert np.array_equal(mask, tree_oracle.pack_mask(want, 4)) and np.array_equal(depth, want.sum(axis=1) - 1 if n else depth)
    L = sjd.lib()
    par = np.array([-1, 0, 2], dtype=np.int32)
    out = np.zeros((3, 1), dtype=np.uint32)
    refused(L.sjd_tree_masks(par.ctypes.data, 3, 1, out.ctypes.data, None))      # node 2 is its own parent
    par[2] = 1
    assert L.sjd_tree_masks(par.ctypes.data, 3, 1, out.ctypes.data, None) == sjd.OK and out[2, 0] == 7
    refused(L.sjd_tree_masks(par.ctypes.data, 3, 0, out.ctypes.data, None))
    refused(L.sjd_tree_masks(None, 3, 1, out.ctypes.data, None))
    refused(L.sjd_tree_masks(par.ctypes.data, 3, 1, None, None))


def test_tree_attention():
    L, need = sjd.lib(), C.c_uint64(0)
    good = dict(cache=desc(), dtype=sjd.BF16, q=ONE, qs=512, out=ONE, os=512, rows=ONE, ctx=ONE, mask=ONE, words=1, n=6, H=8, scale=0.0, max_rows=4, max_ctx=100, ws=ONE,
                wsb=1 << 40)

    def call(**c):
        a = {**good, **c}
        return L.sjd_op_tree_attention(None, a["cache"], a["dtype"], a["q"], a["qs"], a["out"], a["os"], a["rows"], a["ctx"], a["mask"], a["words"], a["n"], a["H"], a["scale"],
                                       a["max_rows"], a["max_ctx"], a["ws"], a["wsb"])

    for bad in [dict(cache=None), dict(dtype=sjd.F32), dict(dtype=sjd.FP8), dict(cache=desc(dtype=sjd.F32)), dict(q=NULL), dict(out=NULL), dict(q=ODD), dict(out=ODD), dict(os=511),
                dict(rows=NULL), dict(ctx=NULL), dict(words=0), dict(mask=C.c_void_p(66)), dict(n=-1), dict(H=0), dict(H=7), dict(scale=-1.0), dict(scale=math.nan),
                dict(scale=math.inf), dict(max_rows=0), dict(max_rows=65537), dict(max_ctx=-1)] + [dict(cache=desc(**b)) for b in BAD_CACHES]:
        refused(call(**bad))
    assert call(n=0, q=NULL, out=NULL) == sjd.OK
    # an output that overlaps the queries, but for the same rows; a stride that goes back
    for bad in [dict(out=C.c_void_p(64 + 2)), dict(os=1024), dict(out=C.c_void_p(64 + 5 * 1024 + 2)), dict(qs=1024, os=1024, out=C.c_void_p(64 + 1022)),
                dict(n=1, out=C.c_void_p(64 + 1022)), dict(qs=-512)]:
        refused(call(**bad))
    long = dict(cache=desc(pages_per_seq=2000), max_ctx=100000)      # split: needs a workspace
    assert L.sjd_op_tree_attention_workspace(long["cache"], 8, 4, 100000, C.byref(need)) == 0 and need.value > 0
    refused(call(**long, wsb=need.value - 1), sjd.ECAPACITY)
    refused(call(**long, ws=NULL))
    refused(call(**long, ws=C.c_void_p(72)))
    refused(L.sjd_op_tree_attention_workspace(long["cache"], 8, 4, 100000, None))
    refused(L.sjd_op_tree_attention_workspace(desc(n_seqs=0), 8, 4, 100, C.byref(need)))
    refused(L.sjd_op_tree_attention_workspace(desc(), 7, 4, 100, C.byref(need)))


def test_tree_verify():
    L, need = sjd.lib(), C.c_uint64(0)
    names = ("tokens", "parents", "rows", "p", "ps", "q", "qs", "aw", "dw", "path", "len", "next", "n", "seqs", "V", "max_rows", "max_path", "ws", "wsb")
    good = dict(tokens=ONE, parents=ONE, rows=ONE, p=ONE, ps=100, q=ONE, qs=100, aw=ONE, dw=ONE, path=ONE, len=ONE, next=ONE, n=6, seqs=2, V=100, max_rows=4, max_path=3, ws=ONE,
                wsb=1 << 40)

    def call(**c):
        a = {**good, **c}
        return L.sjd_op_tree_verify(None, *[a[x] for x in names])

    for bad in [{x: NULL} for x in ("tokens", "parents", "rows", "p", "aw", "dw", "path", "len", "next", "ws")] + [
            {x: C.c_void_p(66)} for x in ("tokens", "parents", "rows", "p", "q", "aw", "dw", "path", "len", "next", "ws")] + [
            dict(dw=C.c_void_p(68)), dict(n=-1), dict(seqs=0), dict(seqs=65536), dict(V=0), dict(V=(1 << 19) + 1), dict(max_rows=0), dict(max_rows=1025), dict(max_path=0)]:
        refused(call(**bad))
    assert L.sjd_op_tree_verify_workspace(6, 2, 100, C.byref(need)) == 0 and need.value > 0
    refused(call(wsb=need.value - 1), sjd.ECAPACITY)
    refused(L.sjd_op_tree_verify_workspace(6, 2, 100, None))
    refused(L.sjd_op_tree_verify_workspace(6, 0, 100, C.byref(need)))


def test_bindings_refuse_host_tensors():
    import torch
    t = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(sjd.SjdError):
        sjd.KvCache("fp8", 4, 64, 2, 64, torch.zeros((2, 3), dtype=torch.int32))
    with pytest.raises(sjd.SjdError):
        sjd.op_rotary(torch.zeros(3, 2, 64), None, t, torch.zeros(32, dtype=torch.int64))
    with pytest.raises(sjd.SjdError):
        sjd.op_tree_verify(t, t, torch.zeros(2, dtype=torch.int32), torch.zeros(3, 9), None, t, torch.zeros(1, dtype=torch.int64))
