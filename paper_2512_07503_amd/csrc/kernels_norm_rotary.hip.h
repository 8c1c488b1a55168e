// Norms of queries and keys for each head, and the rotary positions (kernels_rotary.hip.h) in the same pass:
//   y = (x - c) / sqrt(mean((x - c)^2) + eps) * gain + bias,   c = 0 or the mean,   then pairs of y turned.
// A head is held in the registers of a team of lanes, 16 elements each, from the load to the store: read once, written once, rounded once.
#pragma once
#include "kernels_rotary.hip.h"

struct NormRotaryArgs {
    RotaryArgs r;
    const void *gain[2], *bias[2];   // of queries, keys; a bias may be NULL
    int per_head;                    // gains and biases are [heads][hd], else [hd]
    int layer;                       // subtract the mean
    float eps;
};

// y = ((x * pre - shift) - off) * scale
struct NormStats { float pre, shift, off, scale; };
// From a lane's elements (0 where it has none, has[e] false) and a sum over the lanes of the head.  Squares of elements beyond 2^60 do not fit: then the
// elements are taken 2^-72 times as large (the norm does not change, but for eps, which is far below).  What the mean's rounding leaves, the mean of the
// differences from it, is taken off as well: it would be 2^-24 of the mean, which may be many times the deviation.
template <int N, typename Sum, typename Has> SJD_D NormStats norm_stats(const float (&x)[N], Has has, int hd, bool layer, float eps, Sum sum) {
    NormStats s;
    const float inv = 1.0f / (float)hd;
    auto moments = [&](float pre, float &shift, float &off, float &var) {
        shift = off = 0.0f;
        if (layer) {
            float t = 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) t += x[e] * pre;
            shift = sum(t) * inv;
        }
        float first = 0.0f, second = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float d = has(e) ? x[e] * pre - shift : 0.0f;
            first += d;
            second = fmaf(d, d, second);
        }
        var = sum(second) * inv;
        if (layer) {
            off = sum(first) * inv;
            const float less = var - off * off;
            var = less < 0.0f ? 0.0f : less;
        }
    };
    float var;
    s.pre = 1.0f;
    moments(1.0f, s.shift, s.off, var);
    if (!(var < INFINITY)) {
        s.pre = 0x1p-72f;
        eps = 0x1p-126f;
        moments(s.pre, s.shift, s.off, var);
    }
    s.scale = 1.0f / sqrtf(var + eps);
    return s;
}

// WIDE rows (16-byte aligned, in pieces of 8 elements).  A lane of the team has two pieces: the two halves of 8 turned pairs, or what lies behind the turned part;
// interleaved: 16 elements in a row.
template <typename T, int TEAM>
__global__ __launch_bounds__(256) void norm_rotary_kernel(NormRotaryArgs p) {
    const RotaryArgs &a = p.r;
    __shared__ float2 cs[8 * kRotaryMaxHalf];   // (cos, sin) * magnitude of [row][pair]; rows_per_wg * half <= 8 * 256
    const int row0 = blockIdx.x * a.rows_per_wg, rows = min(a.rows_per_wg, a.n_rows - row0), tid = threadIdx.x;
    const int half = a.half, heads = a.heads[0] + a.heads[1], hd = a.hd;
    for (int u = tid; u < rows * half; u += 256) {
        const int r = u / half, i = u - r * half;
        float s, c;
        sincos_turns((uint64_t)(int64_t)a.positions[row0 + r] * a.table[i], s, c);
        cs[u] = float2{c * a.magnitude, s * a.magnitude};
    }
    __syncthreads();
    const int unit = tid & (TEAM - 1), turned = a.interleaved ? (hd + 15) >> 4 : half >> 3;
    const bool turn = unit < turned;
    const int j0 = a.interleaved ? 16 * unit : turn ? 8 * unit : 2 * half + 16 * (unit - turned);
    const int j1 = !a.interleaved && turn ? j0 + half : j0 + 8;
    const bool has0 = j0 < hd, has1 = j1 < hd;
    const int total = rows * heads, step = gridDim.y * (256 / TEAM);
    for (int u = blockIdx.y * (256 / TEAM) + tid / TEAM; u < total; u += step) {
        const int r = u / heads, hh = u - r * heads, side = hh >= a.heads[0], h = side ? hh - a.heads[0] : hh;
        const T *x = (const T *)a.x[side] + (size_t)(row0 + r) * a.x_stride[side] + (size_t)h * hd;
        T *y = (T *)a.y[side] + (size_t)(row0 + r) * a.y_stride[side] + (size_t)h * hd;
        const size_t g0 = p.per_head ? (size_t)h * hd : 0;
        const T *gain = (const T *)p.gain[side] + g0, *bias = p.bias[side] ? (const T *)p.bias[side] + g0 : nullptr;
        float v[16] = {}, g[16] = {}, b[16] = {};
        float (&v0)[8] = reinterpret_cast<float (&)[8]>(v[0]), (&v1)[8] = reinterpret_cast<float (&)[8]>(v[8]);
        if (has0) load8(x + j0, true, v0);
        if (has1) load8(x + j1, true, v1);
        if (has0) load8(gain + j0, true, reinterpret_cast<float (&)[8]>(g[0]));
        if (has1) load8(gain + j1, true, reinterpret_cast<float (&)[8]>(g[8]));
        if (bias && has0) load8(bias + j0, true, reinterpret_cast<float (&)[8]>(b[0]));
        if (bias && has1) load8(bias + j1, true, reinterpret_cast<float (&)[8]>(b[8]));
        const NormStats s = norm_stats<16>(v, [&](int e) { return e < 8 ? has0 : has1; }, hd, p.layer, p.eps, [](float t) {
#pragma unroll
            for (int d = 1; d < TEAM; d <<= 1) t += __shfl_xor(t, d, 64);
            return t;
        });
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = fmaf((v[e] * s.pre - s.shift - s.off) * s.scale, g[e], b[e]);
        const float2 *w = cs + r * half;
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
                const float a0 = v0[e], a1 = v1[e];
                v0[e] = fmaf(a0, t.x, -(a1 * t.y));
                v1[e] = fmaf(a1, t.x, a0 * t.y);
            }
        }
        if (has0) store8(y + j0, true, v0);
        if (has1) store8(y + j1, true, v1);
    }
}

// Any alignment and sizes: a wavefront a head, a lane has pairs lane + 64 n and elements behind the turned part 2 half + lane + 64 n.
template <typename T>
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
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = has(e) ? to_float<T>(x[at(e)]) : 0.0f;
        const NormStats s = norm_stats<16>(v, has, hd, p.layer, p.eps, [](float t) {
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) t += __shfl_xor(t, d, 64);
            return t;
        });
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (has(e)) v[e] = fmaf((v[e] * s.pre - s.shift - s.off) * s.scale, to_float<T>(gain[at(e)]), bias ? to_float<T>(bias[at(e)]) : 0.0f);
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
