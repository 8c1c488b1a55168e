// Rotary positions: pairs of dimensions turned by position * frequency.
//
// The angle is a fixed-point fraction of a turn: position (32 bits) * frequency (2^-64 turns) modulo 2^64, an integer product that is
// exact at any position, where a float angle of a far position has no fraction left.  It is rounded to 32 bits (2^-33 turns; the frequency's
// rounding is another 2^-34 at most), which are split into the nearest quarter
// turn and a rest of at most an eighth, whose sine and cosine are the Taylor polynomials to x^9 and x^10 (|x| <= pi / 4: the next terms
// are below 2^-29 and 2^-33).  Bound by memory: a row's sines and cosines are computed once, in LDS, for all its heads.
// 12 000 rows of 32 + 8 heads of 128 bf16, 246 MB: 51.5 us, 4.8 TB/s, where a copy of the size reaches 5.5; 8 rows: 3.4 us, latency.
#pragma once
#include "common.hip.h"
#include "kernels_cache.hip.h"

struct RotaryArgs {
    const uint64_t *table;
    const int32_t *positions;
    const void *x[2];          // queries, keys
    void *y[2];
    long x_stride[2], y_stride[2];
    int heads[2];
    int n_rows, hd, half;      // half = rotary_dim / 2
    int interleaved, rows_per_wg;
    float magnitude;
};

SJD_D void sincos_turns(uint64_t turns, float &sn, float &cs) {
    const uint32_t t = (uint32_t)((turns + 0x80000000ull) >> 32);
    const uint32_t quarter = (t + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(t - (quarter << 30)) * 0x1.921fb6p-30f;    // 2 pi / 2^32
    const float x2 = x * x;
    float s = fmaf(x2, 1.0f / 362880.0f, -1.0f / 5040.0f);
    s = fmaf(x2, s, 1.0f / 120.0f);
    s = fmaf(x2, s, -1.0f / 6.0f);
    s = fmaf(x * x2, s, x);
    float c = fmaf(x2, -1.0f / 3628800.0f, 1.0f / 40320.0f);
    c = fmaf(x2, c, -1.0f / 720.0f);
    c = fmaf(x2, c, 1.0f / 24.0f);
    c = fmaf(x2, c, -0.5f);
    c = fmaf(x2, c, 1.0f);
    const bool swap = quarter & 1u;
    sn = swap ? c : s;
    cs = swap ? s : c;
    if (quarter & 2u) sn = -sn;                 // quarters 2 and 3
    if ((quarter + 1u) & 2u) cs = -cs;          // quarters 1 and 2
}

constexpr int kRotaryMaxHalf = 256;   // head_dim <= 512

// Workgroup = rows_per_wg rows.  WIDE: 8 dimensions at a time, 16-byte aligned; half (or, interleaved, nothing) a multiple of 8.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
    __shared__ float2 cs[8 * kRotaryMaxHalf];   // (cos, sin) * magnitude of [row][pair]; rows_per_wg * half <= 8 * 256
    const int row0 = blockIdx.x * a.rows_per_wg, rows = min(a.rows_per_wg, a.n_rows - row0), tid = threadIdx.x;
    for (int u = tid; u < rows * a.half; u += 256) {
        const int r = u / a.half, i = u - r * a.half;
        float s, c;
        sincos_turns((uint64_t)(int64_t)a.positions[row0 + r] * a.table[i], s, c);
        cs[u] = float2{c * a.magnitude, s * a.magnitude};
    }
    __syncthreads();
    const int heads = a.heads[0] + a.heads[1], half = a.half;
    // units of a head: WIDE 8 dimensions (of a half layout's turned part 8 + 8), else a pair (or a copied dimension)
    const int turned = WIDE ? (a.interleaved ? a.hd >> 3 : half >> 3) : half;
    const int copied = WIDE ? (a.interleaved ? 0 : (a.hd - 2 * half) >> 3) : a.hd - 2 * half;
    const int per_head = turned + copied, total = rows * heads * per_head;
    for (int u = blockIdx.y * 256 + tid; u < total; u += gridDim.y * 256) {
        const int unit = u % per_head, rh = u / per_head, hh = rh % heads, r = rh / heads;
        const int side = hh >= a.heads[0], h = side ? hh - a.heads[0] : hh;
        const T *x = (const T *)a.x[side] + (size_t)(row0 + r) * a.x_stride[side] + (size_t)h * a.hd;
        T *y = (T *)a.y[side] + (size_t)(row0 + r) * a.y_stride[side] + (size_t)h * a.hd;
        const float2 *w = cs + r * half;
        if constexpr (WIDE) {
            if (unit >= turned) {
                const int j = 2 * half + 8 * (unit - turned);
                float v[8];
                load8(x + j, true, v);
                store8(y + j, true, v);
            } else if (a.interleaved) {
                const int j = 8 * unit;
                float v[8];
                load8(x + j, true, v);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if ((j >> 1) + e < half) {
                        const float2 t = w[(j >> 1) + e];
                        const float v0 = v[2 * e], v1 = v[2 * e + 1];
                        v[2 * e] = fmaf(v0, t.x, -(v1 * t.y));
                        v[2 * e + 1] = fmaf(v1, t.x, v0 * t.y);
                    }
                store8(y + j, true, v);
            } else {
                const int j = 8 * unit;
                float v0[8], v1[8];
                load8(x + j, true, v0);
                load8(x + half + j, true, v1);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 t = w[j + e];
                    const float b0 = v0[e], b1 = v1[e];
                    v0[e] = fmaf(b0, t.x, -(b1 * t.y));
                    v1[e] = fmaf(b1, t.x, b0 * t.y);
                }
                store8(y + j, true, v0);
                store8(y + half + j, true, v1);
            }
        } else {
            if (unit >= turned) y[2 * half + unit - turned] = x[2 * half + unit - turned];
            else {
                const int j0 = a.interleaved ? 2 * unit : unit, j1 = a.interleaved ? 2 * unit + 1 : unit + half;
                const float2 t = w[unit];
                const float b0 = to_float<T>(x[j0]), b1 = to_float<T>(x[j1]);
                const float r0 = fmaf(b0, t.x, -(b1 * t.y)), r1 = fmaf(b1, t.x, b0 * t.y);
                const uint32_t both = pack_bf16(r0, r1);
                if constexpr (sizeof(T) == 4) { y[j0] = r0; y[j1] = r1; }
                else { y[j0] = (T)both; y[j1] = (T)(both >> 16); }
            }
        }
    }
}
