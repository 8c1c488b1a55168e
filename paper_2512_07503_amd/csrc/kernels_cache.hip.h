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
            first = cache_first(first_pos[b]);
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
// 8 consecutive elements of a row: from 16-byte aligned rows
template <typename T> struct Raw8 { u32x4 w[sizeof(T) / 2]; };
template <typename T> SJD_D Raw8<T> load_raw8(const T *p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = reinterpret_cast<const u32x4 *>(p)[i];
    return r;
}
SJD_D void unpack8(const Raw8<float> &r, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) { const uint32_t b = r.w[e >> 2][e & 3]; x[e] = __builtin_bit_cast(float, b); }
}
SJD_D void unpack8(const Raw8<bf16_t> &r, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __builtin_bit_cast(float, r.w[0][e] << 16);
        x[2 * e + 1] = __builtin_bit_cast(float, r.w[0][e] & 0xFFFF0000u);
    }
}
// and from any
template <typename T> SJD_D void load8(const T *p, bool wide, float (&x)[8]) {
    if (wide) unpack8(load_raw8(p), x);
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_float<T>(p[e]);
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

// the low bits of a word as an element
template <typename E> SJD_D E as_elem(uint32_t w) {
    if constexpr (sizeof(E) == 4) return __builtin_bit_cast(E, w);
    else return (E)w;
}
SJD_D bool finite_f(float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7F800000u) != 0x7F800000u; }
// The scale's exponent for a largest finite magnitude of amax = mantissa * 2^x, 1/2 <= mantissa < 1: x - 9 for a mantissa of up to 7/8 (448 is
// 7/8 * 2^9), x - 8 above. From amax's bits: x is the exponent field - 126, and 0x1FFFFF carries into the field from a fraction above 0x600000, 7/8.
SJD_D int fp8_exponent(uint32_t amax) { return min(max((int)((amax + 0x1FFFFFu) >> 23) - 135, kCacheMinExp), kCacheMaxExp); }
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
// (`plain`: every x / scale is a number of at most 448 in magnitude)
template <int KIND> SJD_D Packed8<KIND> encode8(const float (&x)[8], float inv_scale, bool plain) {
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
        for (int e = 0; e < 8; ++e) y[e] = x[e] * inv_scale;
        if (!plain)
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
    int group;            // kv heads of a workgroup, <= cache_heads
    bool k_wide, v_wide;  // rows start 16-byte aligned
};

// A workgroup of a write or a read takes a tile of 32 positions, of one kv head or as many as 256 elements of a row hold. Eight threads share a token;
// each has up to kCacheChunks pieces of 8 dimensions, `rounds` of them a head.
constexpr int kCacheChunks = 4;
constexpr int cache_rounds(int hd) { return (hd + 63) >> 6; }
constexpr int cache_heads(int hd) { return kCacheChunks / cache_rounds(hd); }

// Sixteen bytes of the values of a tile, a lane's share: kRuns runs of four tokens, 8 apart, of one dimension. Share `s` of a dimension starts with
// token cache_v_token(s); there are kCacheShares of a tile.
template <int KIND> constexpr int kCacheRuns = KIND == SJD_F32 ? 1 : KIND == SJD_BF16 ? 2 : 4;
template <int KIND> constexpr int kCacheShares = 8 / kCacheRuns<KIND>;
template <int KIND> constexpr int cache_v_token(int s) { return (s >> 1) * 8 * kCacheRuns<KIND> + (s & 1) * 4; }

// ------------------------------------------------------------------------------------------------------------------- write
// Workgroup = (tile of 32 positions, group of kv heads, keys or values). The eight threads of a token load its elements, agree on each head's
// largest magnitude and encode. Keys go straight to their place, 8 codes (or 8 elements) at a time; values go there by way of
// LDS, which holds the tile in the layout's own order, 16-byte shares shuffled so that a wavefront's elements lie in different banks.
// Bound by memory: 15 600 rows of 8 kv heads of 128, bf16 to fp8, 96 MB in all: 28.4 us, 3.4 TB/s, where a copy of the size reaches 5.5. A head a workgroup,
// whose threads have only 32 bytes on their way: 33.1; the loads one behind the other in branches of their own and a largest magnitude that asks of
// every element whether it is finite: 34.0.
template <int KIND> constexpr int cache_turn_share(int s) { return s ^ ((s >> 4 & 3) | (s >> (KIND == SJD_F32 ? 8 : 6) & 1) << 2); }
template <int KIND> constexpr int cache_turn(int e) {   // place of element e of a tile's values
    constexpr int n = 16 / (int)sizeof(typename CacheElem<KIND>::type);
    return cache_turn_share<KIND>(e / n) * n + e % n;
}
template <int KIND, typename T>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheRowsArgs a) {
    typedef typename CacheElem<KIND>::type E;
    __shared__ __align__(16) E turn[32 * 256];
    const CacheTile f = cache_find_tile(a.row_start, a.first_pos, a.c.n_seqs, a.n_rows, blockIdx.x);
    if (f.b < 0) return;
    const int hd = a.c.hd, tid = threadIdx.x, rounds = cache_rounds(hd);
    const int kvh0 = blockIdx.y * a.group, heads = min(a.group, a.c.n_kv - kvh0);
    const bool v = blockIdx.z;
    const int tok = tid >> 3, part = tid & 7;
    const int i = f.t0 + tok - f.first;            // row within the sequence
    const bool live = i >= 0 && i < f.n, wide = v ? a.v_wide : a.k_wide;
    const T *src = (const T *)(v ? a.v : a.k) + (size_t)(f.r0 + (live ? i : 0)) * (v ? a.v_stride : a.k_stride) + (size_t)kvh0 * hd;
    float x[kCacheChunks][8];
    bool mine[kCacheChunks];                       // is there such a piece
    int head[kCacheChunks], round[kCacheChunks];   // its head within the group; its first dimension is 64 round + 8 part
#pragma unroll
    for (int c = 0; c < kCacheChunks; ++c) {
        head[c] = c / rounds;
        round[c] = c - head[c] * rounds;
        mine[c] = live && head[c] < heads && round[c] * 64 + part * 8 < hd;
    }
    if (wide) {                                    // (what is not there loads something that is: no branch parts the loads)
        Raw8<T> raw[kCacheChunks];
#pragma unroll
        for (int c = 0; c < kCacheChunks; ++c) raw[c] = load_raw8(src + (mine[c] ? head[c] * hd + round[c] * 64 + part * 8 : 0));
#pragma unroll
        for (int c = 0; c < kCacheChunks; ++c) unpack8(raw[c], x[c]);
    } else {
#pragma unroll
        for (int c = 0; c < kCacheChunks; ++c)
            if (mine[c]) load8(src + head[c] * hd + round[c] * 64 + part * 8, false, x[c]);
    }
    const int page = cache_page(a.c, f.b, f.t0);
    if (page < 0) return;
    const int slot = f.t0 % a.c.page_tokens;       // of the tile within its page
    const size_t side = v ? (size_t)a.c.page_tokens * hd : 0;
    unsigned char *block = cache_block(a.c, page, kvh0);
    float inv[kCacheChunks] = {1.0f, 1.0f, 1.0f, 1.0f};
    bool plain = true;                             // every element is finite and within the codes' range
    if constexpr (KIND == SJD_FP8) {
        uint32_t amax[kCacheChunks];               // bits of a magnitude
#pragma unroll
        for (int c = 0; c < kCacheChunks; ++c) {
            amax[c] = 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) amax[c] = max(amax[c], __builtin_bit_cast(uint32_t, x[c][e]) & 0x7FFFFFFFu);
            amax[c] = mine[c] ? amax[c] : 0u;
            if (__any(amax[c] >= 0x7F000000u)) {   // something is not finite, or beyond the largest scale: look at the finite ones alone
                plain = false;
                amax[c] = 0u;
                if (mine[c])
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        amax[c] = max(amax[c], finite_f(x[c][e]) ? __builtin_bit_cast(uint32_t, x[c][e]) & 0x7FFFFFFFu : 0u);
            }
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) amax[c] = max(amax[c], (uint32_t)__shfl_xor((int)amax[c], d, 64));
        }
        if (rounds > 1) {                          // over the rounds of a head
            uint32_t own[kCacheChunks];
#pragma unroll
            for (int c = 0; c < kCacheChunks; ++c) own[c] = amax[c];
#pragma unroll
            for (int c = 0; c < kCacheChunks; ++c)
#pragma unroll
                for (int o = 0; o < kCacheChunks; ++o) amax[c] = max(amax[c], head[o] == head[c] ? own[o] : 0u);
        }
        unsigned char *scales = block + 2 * (size_t)a.c.page_tokens * hd + (v ? a.c.page_tokens : 0) + slot + tok;
#pragma unroll
        for (int c = 0; c < kCacheChunks; ++c) {
            const int e = fp8_exponent(amax[c]);
            inv[c] = power_of_two(-e);
            if (mine[c] && part == 0 && round[c] == 0) scales[head[c] * a.c.block_bytes] = (unsigned char)(e + 127);
        }
    }
    if (!v) {
        // 64 dimensions on is 64 * 32 elements on, in any kind's layout
        E *dst = (E *)block + cache_k_index<KIND>(slot + tok, part * 8, hd);
#pragma unroll
        for (int c = 0; c < kCacheChunks; ++c) {
            const Packed8<KIND> p = encode8<KIND>(x[c], inv[c], plain);
            if (!mine[c]) continue;
            E *to = (E *)((unsigned char *)dst + head[c] * a.c.block_bytes) + round[c] * 64 * 32;
            if constexpr (KIND == SJD_F32) {       // the layout parts the 8 into two pieces of 4
                *reinterpret_cast<u32x4 *>(to) = u32x4{p.w[0], p.w[1], p.w[2], p.w[3]};
                *reinterpret_cast<u32x4 *>(to + 32 * 4) = u32x4{p.w[4], p.w[5], p.w[6], p.w[7]};
            } else if constexpr (KIND == SJD_BF16) {
                *reinterpret_cast<u32x4 *>(to) = u32x4{p.w[0], p.w[1], p.w[2], p.w[3]};
            } else {
                *reinterpret_cast<uint2 *>(to) = uint2{p.w[0], p.w[1]};
            }
        }
        return;
    }
#pragma unroll
    for (int c = 0; c < kCacheChunks; ++c) {
        const Packed8<KIND> p = encode8<KIND>(x[c], inv[c], plain);
        if (!mine[c]) continue;
        const int at = (int)cache_v_index<KIND>(tok, round[c] * 64 + part * 8, hd);     // (the 8 are in the same 32: their shares follow each other)
        constexpr int kShare = 16 / (int)sizeof(E);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            turn[head[c] * 32 * hd + cache_turn<KIND>(at + e * kShare)] =
                KIND == SJD_F32 ? as_elem<E>(p.w[e % 8]) : KIND == SJD_BF16 ? as_elem<E>(p.w[e / 2 % 4] >> 16 * (e & 1)) : as_elem<E>(p.w[e / 4 % 2] >> 8 * (e & 3));
    }
    __syncthreads();
    // the tile's rows are those from `lo` up to `hi`
    const int lo = max(f.first - f.t0, 0), hi = min(f.first + f.n - f.t0, 32);
    E *dst = (E *)block + side + (size_t)slot * hd;
    if (lo == 0 && hi == 32) {
        const int n = 32 * hd * (int)sizeof(E) / 16;
        for (int h = 0; h < heads; ++h)
            for (int u = tid; u < n; u += 256)
                reinterpret_cast<u32x4 *>((unsigned char *)dst + h * a.c.block_bytes)[u] = reinterpret_cast<const u32x4 *>(turn + h * 32 * hd)[cache_turn_share<KIND>(u)];
        return;
    }
    for (int u = tid; u < 8 * heads * hd; u += 256) {    // four tokens t .. t + 3 of a dimension, which are neighbours
        const int col = u % (heads * hd), t = u / (heads * hd) * 4, h = col / hd;
        if (t + 4 <= lo || t >= hi) continue;
        const int at = (int)cache_v_index<KIND>(t, col - h * hd, hd);
        const E *q = turn + h * 32 * hd + cache_turn<KIND>(at);
        E *to = (E *)((unsigned char *)dst + h * a.c.block_bytes) + at;
        if (t >= lo && t + 4 <= hi) {
            if constexpr (KIND == SJD_F32) *reinterpret_cast<u32x4 *>(to) = *reinterpret_cast<const u32x4 *>(q);
            else if constexpr (KIND == SJD_BF16) *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(q);
            else *reinterpret_cast<uint32_t *>(to) = *reinterpret_cast<const uint32_t *>(q);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (t + e >= lo && t + e < hi) to[e] = q[e];
        }
    }
}

// -------------------------------------------------------------------------------------------------------------------- read
// The same tiles the other way round; values turn around in LDS rows, shifted against each other by 16 bytes. The sizes above: 18.6 us, 5.2 TB/s
// (a head a workgroup: 22.5).
template <int KIND, typename T>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheRowsArgs a) {
    typedef typename CacheElem<KIND>::type E;
    __shared__ __align__(16) E turn[32 * (256 + 16 / (int)sizeof(E))];
    const CacheTile f = cache_find_tile(a.row_start, a.first_pos, a.c.n_seqs, a.n_rows, blockIdx.x);
    if (f.b < 0) return;
    const int page = cache_page(a.c, f.b, f.t0);
    const int hd = a.c.hd, tid = threadIdx.x, rounds = cache_rounds(hd);
    const int kvh0 = blockIdx.y * a.group, heads = min(a.group, a.c.n_kv - kvh0);
    const bool v = blockIdx.z;
    const int width = heads * hd, slot = f.t0 % a.c.page_tokens, pitch = width + 16 / (int)sizeof(E);
    const int lo = max(f.first - f.t0, 0), hi = min(f.first + f.n - f.t0, 32);
    const size_t side = v ? (size_t)a.c.page_tokens * hd : 0;
    const int tok = tid >> 3, part = tid & 7, i = f.t0 + tok - f.first;
    const bool live = tok >= lo && tok < hi;
    // keys and scales of the thread's pieces: on their way before the values turn around
    Packed8<KIND> p[kCacheChunks];
    unsigned char code[kCacheChunks] = {};
    bool mine[kCacheChunks];
    int head[kCacheChunks], at[kCacheChunks];
#pragma unroll
    for (int c = 0; c < kCacheChunks; ++c) {
        head[c] = c / rounds;
        at[c] = ((c - head[c] * rounds) * 8 + part) * 8;
        mine[c] = live && head[c] < heads && at[c] < hd;
        if (!mine[c] || page < 0) continue;
        const unsigned char *block = cache_block(a.c, page, kvh0 + head[c]);
        if constexpr (KIND == SJD_FP8) code[c] = block[2 * (size_t)a.c.page_tokens * hd + (v ? a.c.page_tokens : 0) + slot + tok];
        if (v) continue;
        const E *from = (const E *)block + cache_k_index<KIND>(slot + tok, at[c], hd);
        if constexpr (KIND == SJD_F32) {
            const u32x4 lo4 = *reinterpret_cast<const u32x4 *>(from);
            const u32x4 hi4 = *reinterpret_cast<const u32x4 *>((const E *)block + cache_k_index<KIND>(slot + tok, at[c] + 4, hd));
#pragma unroll
            for (int e = 0; e < 4; ++e) { p[c].w[e] = lo4[e]; p[c].w[4 + e] = hi4[e]; }
        } else if constexpr (KIND == SJD_BF16) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(from);
#pragma unroll
            for (int e = 0; e < 4; ++e) p[c].w[e] = w[e];
        } else {
            const uint2 w = *reinterpret_cast<const uint2 *>(from);
            p[c].w[0] = w.x; p[c].w[1] = w.y;
        }
    }
    if (v && page >= 0) {
        constexpr int kRuns = kCacheRuns<KIND>, kBatch = kCacheShares<KIND> < 4 ? kCacheShares<KIND> : 4;     // 16 bytes a thread on their way
        const int n = kCacheShares<KIND> * width;
#pragma unroll 1
        for (int u0 = tid; u0 < n; u0 += 256 * kBatch) {
            u32x4 w[kBatch];
            int to[kBatch];                        // its first place in `turn`, -1: not there
#pragma unroll
            for (int r = 0; r < kBatch; ++r) {
                const int u = u0 + 256 * r, col = u % width, t = cache_v_token<KIND>(u / width), h = col / hd;
                to[r] = u < n && t + 8 * (kRuns - 1) + 4 > lo && t < hi ? t * pitch + col : -1;
                if (to[r] < 0) continue;
                w[r] = *reinterpret_cast<const u32x4 *>((const E *)cache_block(a.c, page, kvh0 + h) + side + cache_v_index<KIND>(slot + t, col - h * hd, hd));
            }
#pragma unroll
            for (int r = 0; r < kBatch; ++r) {
                if (to[r] < 0) continue;
#pragma unroll
                for (int e = 0; e < 4 * kRuns; ++e) {
                    E &x = turn[to[r] + ((e >> 2) * 8 + (e & 3)) * pitch];
                    if constexpr (KIND == SJD_F32) { const uint32_t b = w[r][e]; x = __builtin_bit_cast(float, b); }
                    else if constexpr (KIND == SJD_BF16) x = (E)(w[r][e >> 1] >> (16 * (e & 1)));
                    else x = (E)(w[r][e >> 2] >> (8 * (e & 3)));
                }
            }
        }
    }
    __syncthreads();
    T *dst = (T *)(v ? a.v : a.k) + (size_t)(f.r0 + i) * (v ? a.v_stride : a.k_stride) + (size_t)kvh0 * hd;
    const bool wide = v ? a.v_wide : a.k_wide;
#pragma unroll
    for (int c = 0; c < kCacheChunks; ++c) {
        if (!mine[c]) continue;
        float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (page >= 0) {
            if (v) {
                const E *from = turn + tok * pitch + head[c] * hd + at[c];
#pragma unroll
                for (int e = 0; e < (int)(sizeof(Packed8<KIND>) / 8); ++e) {
                    const uint2 w = reinterpret_cast<const uint2 *>(from)[e];
                    p[c].w[2 * e] = w.x; p[c].w[2 * e + 1] = w.y;
                }
            }
            decode8<KIND>(p[c], KIND == SJD_FP8 ? power_of_two(min((int)code[c], 254) - 127) : 1.0f, x);
        }
        store8(dst + head[c] * hd + at[c], wide, x);
    }
}

// ----------------------------------------------------------------------------------------------------------------- compact
// Workgroup = (sequence, kv head, keys or values), which moves the entries of the path in order, `group` of them at a time: all of a
// group are read before any is written. Bound by latency: 6 paths of a few nodes, 20 heads of 64, 5.0 us.  The path ascends, so its node j is at least j, and what a later group reads lies
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
