"""Sizes whose launch would have more work-items than a launch can have, 2^32 - 1 a dimension, are refused as such, through the C ABI with pointers that nothing
may follow."""
import ctypes as C

import paper_2512_07503_amd as sjd
from test_tree_refusals import ONE, desc

p = C.c_void_p


def refused(rc):
    assert rc == sjd.EINVAL and b"one launch" in sjd.lib().sjd_last_error(None), (rc, sjd.lib().sjd_last_error(None))


def test_rotary():
    for n in (1 << 27, 1 << 29):         # 8 rows a workgroup of 256
        refused(sjd.lib().sjd_op_rotary(None, sjd.BF16, 0, p(64), 2, 1.0, p(64), n, 2, p(1 << 40), 2, p(1 << 41), 2, 1, None, 0, None, 0, 0))


def test_cache():
    L = sjd.lib()
    for n, seqs in ((1 << 29, 1), (1 << 24, 1 << 24), (1 << 29, 1 << 23)):
        c = desc(n_seqs=seqs)
        refused(L.sjd_op_cache_write(None, c, sjd.F32, p(1 << 40), 128, p(1 << 41), 128, ONE, ONE, n))
        refused(L.sjd_op_cache_read(None, c, sjd.F32, p(1 << 42), p(1 << 44), ONE, ONE, n))
    refused(L.sjd_op_cache_compact(None, desc(n_seqs=1 << 24), ONE, ONE, ONE, 4))


def test_attention():
    L, need = sjd.lib(), C.c_uint64(0)
    for seqs, kv, max_rows in ((1 << 24, 1, 1), (1 << 20, 16, 1), (1 << 14, 1, 1 << 16), ((1 << 31) - 1, 65535, 1 << 16)):
        c = desc(n_seqs=seqs, n_kv_heads=kv)
        refused(L.sjd_op_tree_attention_workspace(c, kv, max_rows, 100, C.byref(need)))
        refused(L.sjd_op_tree_attention(None, c, sjd.BF16, p(1 << 40), 64 * kv, p(1 << 41), 64 * kv, ONE, ONE, None, 0, 5, kv, 0.0, max_rows, 100, None, 0))
    refused(L.sjd_op_tree_attention_workspace(desc(n_kv_heads=1), 1 << 20, 1 << 16, 100, C.byref(need)))     # 2^31 tiles of rows
    assert L.sjd_op_tree_attention_workspace(desc(n_seqs=(1 << 24) - 8, n_kv_heads=1), 1, 1, 100, C.byref(need)) == sjd.OK and need.value == 0
