// What the translation units of the operators on the caller's tensors share with each other and with the rest of the library.
#pragma once
#include "common.hip.h"

// where calls without a context leave their error text (sjd_last_error(NULL))
char *sjd_call_error();

#define TREE_FAIL(code, ...)                            \
    do {                                                \
        sjd_set_error(sjd_call_error(), __VA_ARGS__);   \
        return code;                                    \
    } while (0)
#define TREE_TRY(expr) SJD_HIP_TRY(sjd_call_error(), expr)

// A launch has at most 2^32 - 1 work-items a dimension: so many workgroups of 256
constexpr size_t kMaxWorkgroups = (1u << 24) - 1;

inline bool wide(const void *p, int64_t stride, int size, int bytes) { return (uintptr_t)p % bytes == 0 && stride * size % bytes == 0; }

// Do x_rows rows of x and y_rows of y (one at least of either), x_row and y_row elements long, have no element in common?  (Rows with the same stride may
// interleave: parts of a fused projection.)
inline bool rows_apart(const void *x, long x_stride, long x_row, int x_rows, const void *y, long y_stride, long y_row, int y_rows, int size) {
    const uintptr_t x0 = (uintptr_t)x, x1 = x0 + ((uintptr_t)(x_rows - 1) * x_stride + x_row) * size;
    const uintptr_t y0 = (uintptr_t)y, y1 = y0 + ((uintptr_t)(y_rows - 1) * y_stride + y_row) * size;
    if (x1 <= y0 || y1 <= x0) return true;
    if ((x_rows == 1 && y_rows == 1) || x_stride != y_stride || x_stride <= 0) return false;
    const long d = ((long)(y0 - x0) / size % x_stride + x_stride) % x_stride;   // where y's row starts within x's
    return d >= x_row && d + y_row <= x_stride;
}
