// Norms of queries and keys for each head, and the rotary positions (kernels_rotary.hip.h) in the same pass:
//   y = (x - c) / sqrt(mean((x - c)^2) + eps) * gain + bias,   c = 0 or the mean,   then pairs of y turned.
// A head is held in the registers of a team of lanes, 16 elements each, from the load to the store: read once, written once, rounded once.
//
// What bounds it: memory, and as soon as that is near, the vector units (bf16, 12 000 rows of 40 heads of 128, root mean squares: 40 us, 6.1 TB/s where a copy does 5.0 - 5.5, as half of it
// stays in the card's cache; vector units busy for 75 % of the cycles; 9 408 rows of 64 heads with means, gains and biases 62 us, 5.0 TB/s, 73 %).  A team is as small as a head allows, so that a sum over it is a few
// moves within a wavefront; a team's next head is loaded while this one is worked on (89 -> 49 us); and a row's sines are computed once, by the workgroup, for all of its heads.  Few rows are one head a
// team, and latency (8 rows of 40 heads: 3.6 us).
#pragma once
#include "kernels_rotary.hip.h"
#include "lanes.hip.h"

struct NormRotaryArgs {
    RotaryArgs r;
    const void *gain[2], *bias[2];   // of queries, keys; a bias may be NULL
    int per_head;                    // gains and biases are [heads][hd], else [hd]
    float eps;
};

// The normalised x in its place: z = (x - c) / sqrt(mean((x - c)^2) + eps), of a lane's elements (0 where it has none: bit e of `has`; FULL: it has all).
// With means: c rounded is 2^-24 of it off, which may be many times the deviation, so what it leaves, the mean of the differences from it, is taken off as well: in the same multiplication as the
// scale, unless that mean is most of the differences (heads of nearly one value), of which their spread would be what roundings leave.  Then it is taken off them first, divided without an
// error where it can be: a head of one value is 0 about its mean.
// Squares of elements beyond 2^60 do not fit: then they are taken 2^-72 times as large (the norm does not change, but for eps, which is far below).
template <int N, int TEAM, bool LAYER, bool FULL> SJD_D float norm_moments(float (&x)[N], uint32_t has, float n, float inv, float &off) {
    off = 0.0f;
    float first[2] = {0.0f, 0.0f}, second[2] = {0.0f, 0.0f};      // (two chains of additions each)
    if constexpr (LAYER) {
        float t[2] = {0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < N; ++e) t[e & 1] += x[e];
        float c = lanes_sum<TEAM>(t[0] + t[1]) * inv;
        asm volatile("" : "+v"(c));      // (the rounded one in all differences: fused with one of them the product would not be)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            x[e] = FULL || (has >> e & 1u) ? x[e] - c : 0.0f;
            first[e & 1] += x[e];
        }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) second[e & 1] = fmaf(x[e], x[e], second[e & 1]);
    const float var = lanes_sum<TEAM>(second[0] + second[1]) * inv;
    if constexpr (!LAYER) return var;
    const float sum = lanes_sum<TEAM>(first[0] + first[1]);
    off = sum * inv;
    float less = var - off * off;
    if (less < 0.25f * var) {            // (the same in all of the team)
        off = fmaf(fmaf(-off, n, sum), inv, off);
        first[0] = first[1] = second[0] = second[1] = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            x[e] = FULL || (has >> e & 1u) ? x[e] - off : 0.0f;
            first[e & 1] += x[e];
            second[e & 1] = fmaf(x[e], x[e], second[e & 1]);
        }
        off = lanes_sum<TEAM>(first[0] + first[1]) * inv;
        less = lanes_sum<TEAM>(second[0] + second[1]) * inv - off * off;
    }
    return less < 0.0f ? 0.0f : less;
}
template <int N, int TEAM, bool LAYER, bool FULL> SJD_D void normalise(float (&x)[N], uint32_t has, int hd, float eps) {
    const float n = (float)hd, inv = 1.0f / n;
    float y[N], off;
    if constexpr (LAYER)
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = x[e];
    float var = norm_moments<N, TEAM, LAYER, FULL>(x, has, n, inv, off);
    if (!(var < INFINITY)) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = (LAYER ? y[e] : x[e]) * 0x1p-72f;
        var = norm_moments<N, TEAM, LAYER, FULL>(x, has, n, inv, off);
        eps = 0x1p-126f;
    }
    const float scale = __builtin_amdgcn_rsqf(var + eps), less = -off * scale;     // (within 2^-23; the argument is at least 1e-30)
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = LAYER ? fmaf(x[e], scale, less) : x[e] * scale;
}

// WIDE rows (16-byte aligned, in pieces of 8 elements).  A lane of the team has two pieces: the two halves of 8 turned pairs, or what lies behind the turned part;
// interleaved: 16 elements in a row.
template <typename T, int TEAM, bool LAYER, bool FULL>
__global__ __launch_bounds__(256) void norm_rotary_kernel(NormRotaryArgs p) {
    const RotaryArgs &a = p.r;
    __shared__ float2 cs[8 * kRotaryMaxHalf];   // (cos, sin) * magnitude of [row][pair]; rows_per_wg * half <= 8 * 256
    const int row0 = blockIdx.x * a.rows_per_wg, rows = min(a.rows_per_wg, a.n_rows - row0), tid = threadIdx.x;
    const int half = a.half, heads = a.heads[0] + a.heads[1], hd = a.hd;
    const int unit = tid & (TEAM - 1), turned = a.interleaved ? (hd + 15) >> 4 : half >> 3;
    const bool turn = unit < turned;
    const int j0 = a.interleaved ? 16 * unit : turn ? 8 * unit : 2 * half + 16 * (unit - turned);
    const int j1 = !a.interleaved && turn ? j0 + half : j0 + 8;
    const bool has0 = FULL || j0 < hd, has1 = FULL || j1 < hd;
    // heads of the workgroup's rows, a team's one behind the other: head hh of row r
    const int step = gridDim.y * (256 / TEAM), dr = step / heads, dh = step - dr * heads;
    int r = (blockIdx.y * (256 / TEAM) + tid / TEAM) / heads, hh = blockIdx.y * (256 / TEAM) + tid / TEAM - r * heads;
    Raw8<T> x[2], g[2], b[2];
    auto load = [&]() {
        const int side = hh >= a.heads[0], h = side ? hh - a.heads[0] : hh;
        const T *px = (const T *)a.x[side] + (size_t)(row0 + r) * a.x_stride[side] + (size_t)h * hd;
        const size_t g0 = p.per_head ? (size_t)h * hd : 0;
        const T *pg = (const T *)p.gain[side] + g0, *pb = (const T *)p.bias[side] + g0;
        if (has0) { x[0] = load_raw8(px + j0); g[0] = load_raw8(pg + j0); }
        if (has1) { x[1] = load_raw8(px + j1); g[1] = load_raw8(pg + j1); }
        if (p.bias[side]) {
            if (has0) b[0] = load_raw8(pb + j0);
            if (has1) b[1] = load_raw8(pb + j1);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) b[i] = Raw8<T>{};
        }
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = g[i] = b[i] = Raw8<T>{};
    if (r < rows) load();
    for (int u = tid; u < rows * half; u += 256) {
        const int rr = u / half, i = u - rr * half;
        float s, c;
        sincos_turns((uint64_t)(int64_t)a.positions[row0 + rr] * a.table[i], s, c);
        cs[u] = float2{c * a.magnitude, s * a.magnitude};
    }
    __syncthreads();
    while (r < rows) {
        float v0[8], v1[8], g0[8], g1[8], b0[8], b1[8], v[16];
        unpack8(x[0], v0); unpack8(x[1], v1); unpack8(g[0], g0); unpack8(g[1], g1); unpack8(b[0], b0); unpack8(b[1], b1);
        const float2 *w = cs + r * half;
        const int side = hh >= a.heads[0];
        T *y = (T *)a.y[side] + (size_t)(row0 + r) * a.y_stride[side] + (size_t)(side ? hh - a.heads[0] : hh) * hd;
        r += dr;
        hh += dh;
        if (hh >= heads) { hh -= heads; ++r; }
        if (r < rows) load();          // the next head, while this one is worked on
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = e < 8 ? v0[e & 7] : v1[e & 7];
        normalise<16, TEAM, LAYER, FULL>(v, (has0 ? 0xFFu : 0u) | (has1 ? 0xFF00u : 0u), hd, p.eps);
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = fmaf(v[e], e < 8 ? g0[e & 7] : g1[e & 7], e < 8 ? b0[e & 7] : b1[e & 7]);
        if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((j0 >> 1) + e < half) {
                    const float2 t = w[(j0 >> 1) + e];
                    const float a0 = v[2 * e], a1 = v[2 * e + 1];
                    v[2 * e] = fmaf(a0, t.x, -(a1 * t.y));
                    v[2 * e + 1] = fmaf(a1, t.x, a0 * t.y);
                }
        } else if (turn) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 t = w[j0 + e];
                const float a0 = v[e], a1 = v[8 + e];
                v[e] = fmaf(a0, t.x, -(a1 * t.y));
                v[8 + e] = fmaf(a1, t.x, a0 * t.y);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) { v0[e] = v[e]; v1[e] = v[8 + e]; }
        if (has0) store8(y + j0, true, v0);
        if (has1) store8(y + j1, true, v1);
    }
}

// Any alignment and sizes: a wavefront a head, a lane has pairs lane + 64 n and elements behind the turned part 2 half + lane + 64 n, each loaded by itself.  (bf16, rows of one element more than above: 12 002 of
// 40 heads of 128 39 -> 133 us, 9 408 of 64 with means, gains and biases 56 -> 348; 12 002 of 40 heads of 80 with 32 dimensions turned 32 us, with 30 154.  fp32: 93 -> 164 and 115 -> 305.)
template <typename T, bool LAYER>
__global__ __launch_bounds__(256) void norm_rotary_any_kernel(NormRotaryArgs p) {
    const RotaryArgs &a = p.r;
    const int row = blockIdx.x, lane = threadIdx.x & 63, half = a.half, hd = a.hd, rest = hd - 2 * half, heads = a.heads[0] + a.heads[1];
    float2 w[kRotaryMaxHalf / 64];
#pragma unroll
    for (int n = 0; n < kRotaryMaxHalf / 64; ++n) {
        const int i = lane + 64 * n;
        float s = 0.0f, c = 0.0f;
        if (i < half) sincos_turns((uint64_t)(int64_t)a.positions[row] * a.table[i], s, c);
        w[n] = float2{c * a.magnitude, s * a.magnitude};
    }
    for (int hh = blockIdx.y * 4 + (threadIdx.x >> 6); hh < heads; hh += gridDim.y * 4) {
        const int side = hh >= a.heads[0], h = side ? hh - a.heads[0] : hh;
        const T *x = (const T *)a.x[side] + (size_t)row * a.x_stride[side] + (size_t)h * hd;
        T *y = (T *)a.y[side] + (size_t)row * a.y_stride[side] + (size_t)h * hd;
        const size_t g0 = p.per_head ? (size_t)h * hd : 0;
        const T *gain = (const T *)p.gain[side] + g0, *bias = p.bias[side] ? (const T *)p.bias[side] + g0 : nullptr;
        // elements 0 .. 7: pairs; 8 .. 15: what is not turned
        auto at = [&](int e) { return e < 8 ? (a.interleaved ? 2 * (lane + 64 * (e >> 1)) + (e & 1) : lane + 64 * (e >> 1) + (e & 1) * half) : 2 * half + lane + 64 * (e - 8); };
        auto has = [&](int e) { return e < 8 ? lane + 64 * (e >> 1) < half : lane + 64 * (e - 8) < rest; };
        float v[16];
        uint32_t there = 0u;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            v[e] = has(e) ? to_float<T>(x[at(e)]) : 0.0f;
            there |= has(e) ? 1u << e : 0u;
        }
        normalise<16, 64, LAYER, false>(v, there, hd, p.eps);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (has(e)) v[e] = fmaf(v[e], to_float<T>(gain[at(e)]), bias ? to_float<T>(bias[at(e)]) : 0.0f);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const float a0 = v[2 * n], a1 = v[2 * n + 1];
            v[2 * n] = fmaf(a0, w[n].x, -(a1 * w[n].y));
            v[2 * n + 1] = fmaf(a1, w[n].x, a0 * w[n].y);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (has(e)) {
                if constexpr (sizeof(T) == 4) y[at(e)] = v[e];
                else y[at(e)] = (T)pack_bf16(v[e], v[e]);
            }
    }
}
