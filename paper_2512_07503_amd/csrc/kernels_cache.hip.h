// Kernels that write, read and compact the paged key/value cache of the tree operators (layout: cache_layout.h).
#pragma once
#include "cache_layout.h"
#include "common.hip.h"

template <int KIND> struct CacheElem;
template <> struct CacheElem<SJD_F32> { typedef float type; };
template <> struct CacheElem<SJD_BF16> { typedef uint16_t type; };
template <> struct CacheElem<SJD_FP8> { typedef uint8_t type; };

// A cache as the kernels see it
struct CacheView {
    unsigned char *pages;
    const int32_t *page_table;
    int n_pages, page_tokens, n_kv, hd, n_seqs, pages_per_seq;
    size_t block_bytes;   // of one (page, kv head)
};

SJD_D int cache_page(const CacheView &c, int b, int pos) {
    return cache_page(c.page_table + (size_t)b * c.pages_per_seq, c.pages_per_seq, c.page_tokens, c.n_pages, pos);
}
SJD_D unsigned char *cache_block(const CacheView &c, int page, int kvh) {
    return c.pages + ((size_t)page * c.n_kv + kvh) * c.block_bytes;
}

// The work of a write or a read is a tile of 32 positions that a block of the layout holds, of one sequence.  Workgroup `tile`
// of the launch finds its own: the wavefront's lanes look at 64 sequences at a time, and a prefix sum over their tiles tells whose
// it is.  -> sequence (-1: there are fewer tiles), its first row, its first position, number of rows, the tile's first position.
struct CacheTile { int b, r0, n, first, t0; };
SJD_D CacheTile cache_find_tile(const int32_t *row_start, const int32_t *first_pos, int n_seqs, int n_rows, long tile) {
    const int lane = threadIdx.x & 63;
    long before = 0;
    for (int s0 = 0; s0 < n_seqs; s0 += 64) {
        const int b = s0 + lane;
        int r0 = 0, n = 0, first = 0;
        if (b < n_seqs) {
            r0 = rows_first(row_start, b, n_rows);
            n = rows_count(row_start, b, n_rows);
            first = first_pos[b];
        }
        const int tiles = cache_tiles(first, n);
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
        const unsigned long long mine = __ballot(before + upto > tile);
        if (mine) {
            const int l = __ffsll((long long)mine) - 1;
            CacheTile f;
            f.b = s0 + l;
            f.r0 = __shfl(r0, l, 64);
            f.n = __shfl(n, l, 64);
            f.first = __shfl(first, l, 64);
            f.t0 = ((f.first >> 5) + (int)(tile - before - (__shfl(upto, l, 64) - __shfl(tiles, l, 64)))) << 5;
            return f;
        }
        before += __shfl(upto, 63, 64);
    }
    return CacheTile{-1, 0, 0, 0, 0};
}

// ----------------------------------------------------------------------------------------------------------------- elements
// 8 consecutive elements of a row; `wide`: rows are 16-byte aligned
SJD_D void load8(const float *p, bool wide, float (&x)[8]) {
    if (wide) {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p[e];
    }
}
SJD_D void load8(const bf16_t *p, bool wide, float (&x)[8]) {
    if (wide) {
        const u32x4 a = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __builtin_bit_cast(float, a[e] << 16);
            x[2 * e + 1] = __builtin_bit_cast(float, a[e] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = bf16_to_float(p[e]);
    }
}
// two floats to bf16, round to nearest even; NaN stays NaN
typedef float cache_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 cache_bf16x2 __attribute__((ext_vector_type(2)));
SJD_D uint32_t pack_bf16(float a, float b) {
    const cache_f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, cache_bf16x2));
}
SJD_D void store8(float *p, bool wide, const float (&x)[8]) {
    if (wide) {
        reinterpret_cast<float4 *>(p)[0] = float4{x[0], x[1], x[2], x[3]};
        reinterpret_cast<float4 *>(p)[1] = float4{x[4], x[5], x[6], x[7]};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = x[e];
    }
}
SJD_D void store8(bf16_t *p, bool wide, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
    if (wide) *reinterpret_cast<u32x4 *>(p) = u32x4{w[0], w[1], w[2], w[3]};
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (bf16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}

SJD_D bool finite_f(float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7F800000u) != 0x7F800000u; }
// The scale's exponent for a largest finite magnitude of amax = mantissa * 2^x, 1/2 <= mantissa < 1 (448 = 0.875 * 2^9)
SJD_D int fp8_exponent(float amax) {
    int x;
    const float mantissa = frexpf(amax, &x);
    return amax > 0.0f ? min(max(mantissa <= 0.875f ? x - 9 : x - 8, kCacheMinExp), kCacheMaxExp) : kCacheMinExp;
}
SJD_D float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
// x / 2^e as an e4m3 operand: what overflows saturates, what is not a number (or infinite) is NaN
SJD_D float fp8_operand(float x, float inv_scale) {
    return finite_f(x) ? fminf(fmaxf(x * inv_scale, -448.0f), 448.0f) : __builtin_nanf("");
}
SJD_D uint32_t pack_fp8(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// Eight elements as the cache holds them, in the order of their dimensions: 32, 16 or 8 bytes
template <int KIND> struct Packed8 { uint32_t w[KIND == SJD_F32 ? 8 : KIND == SJD_BF16 ? 4 : 2]; };
template <int KIND> SJD_D Packed8<KIND> encode8(const float (&x)[8], float inv_scale) {
    Packed8<KIND> p;
    if constexpr (KIND == SJD_F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p.w[e] = __builtin_bit_cast(uint32_t, x[e]);
    } else if constexpr (KIND == SJD_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) p.w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
    } else {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fp8_operand(x[e], inv_scale);
        p.w[0] = pack_fp8(y[0], y[1], y[2], y[3]);
        p.w[1] = pack_fp8(y[4], y[5], y[6], y[7]);
    }
    return p;
}
template <int KIND> SJD_D void decode8(const Packed8<KIND> &p, float scale, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (KIND == SJD_F32) x[e] = __builtin_bit_cast(float, p.w[e]);
        else if constexpr (KIND == SJD_BF16) x[e] = __builtin_bit_cast(float, e & 1 ? p.w[e >> 1] & 0xFFFF0000u : p.w[e >> 1] << 16);
    }
    if constexpr (KIND == SJD_FP8) {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const cache_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)p.w[d], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)p.w[d], true);
            x[4 * d] = lo[0] * scale; x[4 * d + 1] = lo[1] * scale; x[4 * d + 2] = hi[0] * scale; x[4 * d + 3] = hi[1] * scale;
        }
    }
}

struct CacheRowsArgs {
    CacheView c;
    const int32_t *row_start, *first_pos;
    void *k, *v;          // rows: source of a write, destination of a read
    long k_stride, v_stride;
    int n_rows;
    bool k_wide, v_wide;  // rows start 16-byte aligned
};

// ------------------------------------------------------------------------------------------------------------------- write
// Workgroup = (tile of 32 positions, kv head, keys or values).  Eight threads share a token: they load its elements 16 bytes of
// bf16 at a time, agree on its largest magnitude and encode.  Keys go straight to their place, 8 codes (or 8 elements) at a time.  Values turn
// around through LDS: a thread then owns four tokens of one dimension, which are neighbours in the layout.
template <int KIND, typename T>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheRowsArgs a) {
    typedef typename CacheElem<KIND>::type E;
    constexpr int kMaxChunks = 4;                  // of 8 dimensions, per thread: head_dim <= 256
    __shared__ __align__(16) E turn[32 * (256 + 16 / (int)sizeof(E))];   // [token][dimension], rows shifted against each other by 16 bytes
    const CacheTile f = cache_find_tile(a.row_start, a.first_pos, a.c.n_seqs, a.n_rows, blockIdx.x);
    if (f.b < 0) return;
    const int page = cache_page(a.c, f.b, f.t0);
    if (page < 0) return;
    const int kvh = blockIdx.y, hd = a.c.hd, tid = threadIdx.x;
    const bool v = blockIdx.z;
    const int tok = tid >> 3, part = tid & 7;
    const int i = f.t0 + tok - f.first;            // row within the sequence
    const bool live = i >= 0 && i < f.n;
    const bool wide = v ? a.v_wide : a.k_wide;
    const T *src = (const T *)(v ? a.v : a.k) + (size_t)(f.r0 + (live ? i : 0)) * (v ? a.v_stride : a.k_stride) + (size_t)kvh * hd;
    const int chunks = hd >> 3;
    float x[kMaxChunks][8];
#pragma unroll
    for (int c = 0; c < kMaxChunks; ++c)
        if (live && c * 8 + part < chunks) load8(src + (c * 8 + part) * 8, wide, x[c]);
    const int slot = f.t0 % a.c.page_tokens;       // of the tile within its page
    unsigned char *block = cache_block(a.c, page, kvh);
    E *dst = (E *)block + (v ? (size_t)a.c.page_tokens * hd : 0);
    float inv = 1.0f;
    if constexpr (KIND == SJD_FP8) {
        float amax = 0.0f;
#pragma unroll
        for (int c = 0; c < kMaxChunks; ++c)
            if (live && c * 8 + part < chunks)
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, finite_f(x[c][e]) ? fabsf(x[c][e]) : 0.0f);
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) amax = fmaxf(amax, __shfl_xor(amax, d, 64));
        const int e = fp8_exponent(amax);
        inv = power_of_two(-e);
        if (live && part == 0) block[2 * (size_t)a.c.page_tokens * hd + (v ? a.c.page_tokens : 0) + slot + tok] = (unsigned char)(e + 127);
    }
    const int pitch = hd + 16 / (int)sizeof(E);
#pragma unroll
    for (int c = 0; c < kMaxChunks; ++c) {
        if (!live || c * 8 + part >= chunks) continue;
        const int j = (c * 8 + part) * 8;
        const Packed8<KIND> p = encode8<KIND>(x[c], inv);
        E *to = v ? turn + tok * pitch + j : dst + cache_k_index<KIND>(slot + tok, j, hd);
        if constexpr (KIND == SJD_F32) {   // the layout of keys parts the 8 into two pieces of 4
            E *to2 = v ? to + 4 : dst + cache_k_index<KIND>(slot + tok, j + 4, hd);
            *reinterpret_cast<u32x4 *>(to) = u32x4{p.w[0], p.w[1], p.w[2], p.w[3]};
            *reinterpret_cast<u32x4 *>(to2) = u32x4{p.w[4], p.w[5], p.w[6], p.w[7]};
        } else if constexpr (KIND == SJD_BF16) {
            *reinterpret_cast<u32x4 *>(to) = u32x4{p.w[0], p.w[1], p.w[2], p.w[3]};
        } else {
            *reinterpret_cast<uint2 *>(to) = uint2{p.w[0], p.w[1]};
        }
    }
    if (!v) return;
    __syncthreads();
    // four tokens t .. t + 3 of dimension j; the tile's rows are those from `lo` up to `hi`
    const int lo = max(f.first - f.t0, 0), hi = min(f.first + f.n - f.t0, 32);
    for (int u = tid; u < 8 * hd; u += 256) {
        // neighbouring threads: the two g of a lane's half wavefront apart, so that a wavefront's stores fill whole lines
        const int j = u % hd, quad = u / hd, t = 4 * quad;
        if (t + 4 <= lo || t >= hi) continue;
        E q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = t + e >= lo && t + e < hi ? turn[(t + e) * pitch + j] : E(0);
        E *to = dst + cache_v_index<KIND>(slot + t, j, hd);
        if (t >= lo && t + 4 <= hi) {
            if constexpr (KIND == SJD_F32) *reinterpret_cast<float4 *>(to) = float4{q[0], q[1], q[2], q[3]};
            else if constexpr (KIND == SJD_BF16) *reinterpret_cast<uint2 *>(to) = uint2{q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16};
            else *reinterpret_cast<uint32_t *>(to) = q[0] | (uint32_t)q[1] << 8 | (uint32_t)q[2] << 16 | (uint32_t)q[3] << 24;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (t + e >= lo && t + e < hi) to[e] = q[e];
        }
    }
}

// -------------------------------------------------------------------------------------------------------------------- read
// The same tiles the other way round.
template <int KIND, typename T>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheRowsArgs a) {
    typedef typename CacheElem<KIND>::type E;
    __shared__ __align__(16) E turn[32 * (256 + 16 / (int)sizeof(E))];
    const CacheTile f = cache_find_tile(a.row_start, a.first_pos, a.c.n_seqs, a.n_rows, blockIdx.x);
    if (f.b < 0) return;
    const int page = cache_page(a.c, f.b, f.t0);
    const int kvh = blockIdx.y, hd = a.c.hd, tid = threadIdx.x;
    const bool v = blockIdx.z;
    const int slot = f.t0 % a.c.page_tokens, pitch = hd + 16 / (int)sizeof(E);
    const int lo = max(f.first - f.t0, 0), hi = min(f.first + f.n - f.t0, 32);
    const unsigned char *block = page >= 0 ? cache_block(a.c, page, kvh) : nullptr;
    const E *src = (const E *)block + (v ? (size_t)a.c.page_tokens * hd : 0);
    if (v && block) {
        for (int u = tid; u < 8 * hd; u += 256) {
            const int j = u % hd, t = 4 * (u / hd);
            if (t + 4 <= lo || t >= hi) continue;
            const E *from = src + cache_v_index<KIND>(slot + t, j, hd);
            E q[4];
            if constexpr (KIND == SJD_F32) {
                const float4 x = *reinterpret_cast<const float4 *>(from);
                q[0] = x.x; q[1] = x.y; q[2] = x.z; q[3] = x.w;
            } else if constexpr (KIND == SJD_BF16) {
                const uint2 x = *reinterpret_cast<const uint2 *>(from);
                q[0] = (E)x.x; q[1] = (E)(x.x >> 16); q[2] = (E)x.y; q[3] = (E)(x.y >> 16);
            } else {
                const uint32_t x = *reinterpret_cast<const uint32_t *>(from);
                q[0] = (E)x; q[1] = (E)(x >> 8); q[2] = (E)(x >> 16); q[3] = (E)(x >> 24);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) turn[(t + e) * pitch + j] = q[e];
        }
    }
    __syncthreads();
    const int tok = tid >> 3, part = tid & 7, i = f.t0 + tok - f.first;
    if (tok < lo || tok >= hi) return;
    T *dst = (T *)(v ? a.v : a.k) + (size_t)(f.r0 + i) * (v ? a.v_stride : a.k_stride) + (size_t)kvh * hd;
    const bool wide = v ? a.v_wide : a.k_wide;
    float scale = 1.0f;
    if constexpr (KIND == SJD_FP8)
        if (block) scale = power_of_two((int)min((int)block[2 * (size_t)a.c.page_tokens * hd + (v ? a.c.page_tokens : 0) + slot + tok], 254) - 127);
    for (int c = part; c < hd >> 3; c += 8) {
        float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (block) {
            const E *from = v ? turn + tok * pitch + c * 8 : src + cache_k_index<KIND>(slot + tok, c * 8, hd);
            Packed8<KIND> p;
            if constexpr (KIND == SJD_F32) {
                const u32x4 lo4 = *reinterpret_cast<const u32x4 *>(from);
                const u32x4 hi4 = *reinterpret_cast<const u32x4 *>(v ? from + 4 : src + cache_k_index<KIND>(slot + tok, c * 8 + 4, hd));
#pragma unroll
                for (int e = 0; e < 4; ++e) { p.w[e] = lo4[e]; p.w[4 + e] = hi4[e]; }
            } else if constexpr (KIND == SJD_BF16) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(from);
#pragma unroll
                for (int e = 0; e < 4; ++e) p.w[e] = w[e];
            } else {
                const uint2 w = *reinterpret_cast<const uint2 *>(from);
                p.w[0] = w.x; p.w[1] = w.y;
            }
            decode8<KIND>(p, scale, x);
        }
        store8(dst + c * 8, wide, x);
    }
}

// ----------------------------------------------------------------------------------------------------------------- compact
// Workgroup = (sequence, kv head, keys or values), which moves the entries of the path in order, `group` of them at a time: all of a
// group are read before any is written.  The path ascends, so its node j is at least j, and what a later group reads lies
// behind everything that an earlier one wrote.
template <int KIND>
__global__ __launch_bounds__(256) void cache_compact_kernel(CacheView c, const int32_t *first_pos, const int32_t *path, const int32_t *path_len,
                                                            int max_path) {
    typedef typename CacheElem<KIND>::type E;
    constexpr int kPer = 16;                      // elements of a group per thread
    __shared__ int good;
    const int b = blockIdx.x, kvh = blockIdx.y, tid = threadIdx.x, hd = c.hd;
    const bool v = blockIdx.z;
    const int32_t *p = path + (size_t)b * max_path;
    const int first = first_pos[b];
    if (first < 0 || first > (1 << 30)) return;
    if (tid == 0) good = min(max(path_len[b], 0), max_path);
    __syncthreads();
    const int len = good;
    __syncthreads();
    for (int j = tid; j < len; j += 256)
        if (p[j] <= (j ? p[j - 1] : -1) || p[j] > (1 << 30) - 1) atomicMin(&good, j);
    __syncthreads();
    const int n = good, group = 256 * kPer / hd;   // >= 16
    const size_t side = v ? (size_t)c.page_tokens * hd : 0, scales = 2 * (size_t)c.page_tokens * hd + (v ? c.page_tokens : 0);
    for (int j0 = 0; j0 < n; j0 += group) {
        const int m = min(group, n - j0);
        E x[kPer];
        unsigned char s = 0;
#pragma unroll
        for (int r = 0; r < kPer; ++r) {
            const int u = tid + 256 * r, j = j0 + u / hd;
            if (u >= m * hd || p[j] == j) continue;
            const int pos = first + p[j], page = cache_page(c, b, pos);
            if (page >= 0) x[r] = ((const E *)cache_block(c, page, kvh) + side)[cache_index<KIND>(v, pos % c.page_tokens, u % hd, hd)];
        }
        if (KIND == SJD_FP8 && tid < m) {
            const int pos = first + p[j0 + tid], page = cache_page(c, b, pos);
            if (page >= 0) s = cache_block(c, page, kvh)[scales + pos % c.page_tokens];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kPer; ++r) {
            const int u = tid + 256 * r, j = j0 + u / hd;
            if (u >= m * hd || p[j] == j || cache_page(c, b, first + p[j]) < 0) continue;
            const int pos = first + j, page = cache_page(c, b, pos);
            if (page >= 0) ((E *)cache_block(c, page, kvh) + side)[cache_index<KIND>(v, pos % c.page_tokens, u % hd, hd)] = x[r];
        }
        if (KIND == SJD_FP8 && tid < m && cache_page(c, b, first + p[j0 + tid]) >= 0) {
            const int pos = first + j0 + tid, page = cache_page(c, b, pos);
            if (page >= 0) cache_block(c, page, kvh)[scales + pos % c.page_tokens] = s;
        }
        __syncthreads();
    }
}
