// What the entry points that turn queries and keys (with a norm or without) check on the host, and how they divide the rows.
#pragma once
#include "kernels_rotary.hip.h"
#include "tree_ops.h"

// wide: rows are 16-byte aligned and come in pieces of 8 elements
inline int rotary_check(const RotaryArgs &a, int32_t dtype, int32_t rotary_dim, bool &w) {
    if (dtype != SJD_F32 && dtype != SJD_BF16) TREE_FAIL(SJD_EINVAL, "rows are SJD_F32 or SJD_BF16");
    if (a.hd < 2 || a.hd > 2 * kRotaryMaxHalf || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > a.hd)
        TREE_FAIL(SJD_EINVAL, "rotary_dim must be even and 2 .. head_dim, head_dim at most 512");
    const int n_rows = a.n_rows;
    if (a.heads[0] < 1 || a.heads[1] < 0 || a.heads[0] > 1 << 16 || a.heads[1] > 1 << 16 || n_rows < 0 || n_rows > 1 << 29)
        TREE_FAIL(SJD_EINVAL, "n_heads must be 1 .. 65536, n_kv_heads 0 .. 65536, n_rows 0 .. 2^29");
    if (!a.table || (n_rows && (!a.positions || !a.x[0] || !a.y[0] || (a.heads[1] && (!a.x[1] || !a.y[1]))))) TREE_FAIL(SJD_EINVAL, "null argument");
    const int size = dtype == SJD_F32 ? 4 : 2;
    w = a.interleaved ? a.hd % 8 == 0 : a.half % 8 == 0 && (a.hd - rotary_dim) % 8 == 0;
    for (int s = 0; s < 2; ++s) {
        const long row = (long)a.heads[s] * a.hd;
        if (!row || !n_rows) continue;
        if ((uintptr_t)a.x[s] % size || (uintptr_t)a.y[s] % size) TREE_FAIL(SJD_EINVAL, "rows are not aligned to their elements");
        if (n_rows > 1 && a.y_stride[s] < row) TREE_FAIL(SJD_EINVAL, "output rows overlap");
        if (n_rows > 1 && a.x_stride[s] < 0) TREE_FAIL(SJD_EINVAL, "negative stride");
        w = w && wide(a.x[s], a.x_stride[s], size, 16) && wide(a.y[s], a.y_stride[s], size, 16);
        for (int o = 0; o < 2; ++o) {
            const long out_row = (long)a.heads[o] * a.hd;
            const bool same = o == s && a.x[s] == a.y[s] && (a.x_stride[s] == a.y_stride[s] || n_rows == 1);
            if (out_row && !same && !rows_apart(a.x[s], a.x_stride[s], row, n_rows, a.y[o], a.y_stride[o], out_row, n_rows, size))
                TREE_FAIL(SJD_EINVAL, "an output overlaps an input");
        }
    }
    if (n_rows && a.heads[1] && !rows_apart(a.y[0], a.y_stride[0], (long)a.heads[0] * a.hd, n_rows, a.y[1], a.y_stride[1], (long)a.heads[1] * a.hd, n_rows, size))
        TREE_FAIL(SJD_EINVAL, "q_out and k_out overlap");
    return SJD_OK;
}

// Rows a workgroup: their sines and cosines are shared by the heads of a row only, so more rows mean nothing but fewer workgroups;
// two for each of the 256 CUs, and few rows are split over their heads' units (of which a row has `units`) instead.  most_rows <= 8.
inline bool rotary_grid(RotaryArgs &a, int most_rows, long units, dim3 &grid) {
    while (a.rows_per_wg < most_rows && a.rows_per_wg * a.half * 2 <= 8 * kRotaryMaxHalf && a.n_rows / (2 * a.rows_per_wg) >= 512) a.rows_per_wg *= 2;
    const unsigned gx = (unsigned)ceil_div(a.n_rows, a.rows_per_wg);
    if (gx > kMaxWorkgroups) return false;
    long gy = gx >= 512 ? 1 : 512 / gx;
    if (gy > (a.rows_per_wg * units + 255) / 256) gy = (a.rows_per_wg * units + 255) / 256;
    grid = dim3(gx, (unsigned)gy);
    return true;
}
