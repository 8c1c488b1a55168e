"""Outputs of one call that lie on each other are refused, through the C ABI with pointers that nothing may follow."""
import ctypes as C

import paper_2512_07503_amd as sjd

MiB = 1 << 20


def rotary(q_out, q_stride, k_out, k_stride, n=3, dtype=sjd.F32):
    """4 query heads and 2 key heads of 64; inputs at 64 and 65 MiB."""
    p = C.c_void_p
    return sjd.lib().sjd_op_rotary(None, dtype, 0, p(64), 64, 1.0, p(64), n, 64, p(64 * MiB), 256, p(q_out), q_stride, 4, p(65 * MiB), 128, p(k_out), k_stride, 2)


def test_rotary():
    for size, dtype in ((4, sjd.F32), (2, sjd.BF16)):
        for q_out, qs, k_out, ks, n in [(MiB, 256, MiB, 256, 3), (MiB, 256, MiB, 128, 3), (MiB, 256, MiB + 255 * size, 128, 1), (MiB + 127 * size, 256, MiB, 128, 1),
                                        (MiB, 256, MiB + 2 * 256 * size + 255 * size, 128, 3),
                                        (MiB, 384, MiB + 255 * size, 384, 3),              # rows of one buffer, an element on each other
                                        (MiB, 383, MiB + 256 * size, 383, 3),              # rows of one buffer too short for both
                                        (MiB, 384, MiB + 256 * size, 400, 3)]:             # between each other's rows, at different strides
            assert rotary(q_out, qs, k_out, ks, n, dtype) == sjd.EINVAL, (q_out, qs, k_out, ks, n)
            assert b"q_out and k_out" in sjd.lib().sjd_last_error(None)
