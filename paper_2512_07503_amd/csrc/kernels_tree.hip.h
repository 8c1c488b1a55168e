// Attention of the rows of trees over a paged cache (layout: cache_layout.h).
//
// Row r of the launch is (node i, query head h) of a sequence; the rows of one kv head, ordered (i, h), are cut into tiles of 32, so
// that the query heads of a group share every key and value that is fetched.  Per block of 32 tokens a wavefront computes
//   S^T (tokens x rows) = K Q^T,   online softmax per row = per accumulator column,   O^T (dimensions x rows) += V^T P^T,
// and P^T needs no data movement: the accumulator registers of S^T are the B operand of the second product.
#pragma once
#include "common.hip.h"
#include "kernels_cache.hip.h"

struct TreeArgs {
    CacheView c;
    const void *q;             // [n_rows][H][hd], rows q_stride apart
    void *out;                 // [n_rows][H][hd], rows out_stride apart
    long q_stride, out_stride;
    const int32_t *row_start, *ctx_len;
    const uint32_t *mask;      // [n_rows][mask_words], NULL: a window
    int mask_words, n_rows, max_rows, H, G;
    int tiles, groups;         // of rows: tiles of 32, and of as many tiles as a workgroup takes
    int n_splits;              // of every sequence's context
    float scale_log2e;
    float *part_o;             // [sequence][kv head][split][tiles][32 * hd]  unnormalised, order of tree_part_index
    float *part_ml;            // [sequence][kv head][split][tiles][2][32]    running maximum (base 2), running sum
    bool q_wide, out_wide;     // rows 16-byte (out: 4 elements) aligned
};

// Rows and length of sequence b.  One whose length is negative is outside as a whole, like its rows in the cache, and sees nothing.
struct TreeSeq { int r0, n, ctx, n_tot; };
SJD_D TreeSeq tree_seq(const TreeArgs &a, int b) {
    TreeSeq s;
    s.r0 = rows_first(a.row_start, b, a.n_rows);
    s.n = min(rows_count(a.row_start, b, a.n_rows), a.max_rows);
    const int cap = a.c.pages_per_seq * a.c.page_tokens;
    const int ctx = a.ctx_len[b];
    s.ctx = min(max(ctx, 0), cap);
    s.n_tot = ctx < 0 ? 0 : min(s.ctx + s.n, cap);
    return s;
}

// What a workgroup of the launch works on: a group of row tiles, of a split of a (sequence, kv head).  The groups of a split read the same keys and
// values: they run on one XCD (workgroups go round the 8 XCDs), near each other in time.
struct TreeWork { int b, kvh, split, group; };
SJD_D TreeWork tree_work(const TreeArgs &a, unsigned id) {
    const unsigned xcd = id & 7, rest = id >> 3, share = rest / a.groups * 8 + xcd;
    TreeWork w;
    w.group = rest % a.groups;
    w.split = share % a.n_splits;
    w.kvh = share / a.n_splits % a.c.n_kv;
    w.b = share / a.n_splits / a.c.n_kv;
    return w;
}
inline unsigned tree_grid(const TreeArgs &a) { return (unsigned)(ceil_div_sz((size_t)a.c.n_seqs * a.c.n_kv * a.n_splits, 8) * 8 * a.groups); }
SJD_D size_t tree_slot(const TreeArgs &a, int b, int kvh, int split, int tile) { return ((((size_t)b * a.c.n_kv + kvh) * a.n_splits + split) * a.tiles + tile); }

// The pages of a sequence, block by block: the lanes hold 64 entries of its table at a time, so that a block's address does not wait for one
struct TreePages {
    const int32_t *table;
    int per_seq, page_tokens, n_pages, idx, slot, base, held;
    SJD_D TreePages(const TreeArgs &a, int b, int blk)
        : table(a.c.page_table + (size_t)b * a.c.pages_per_seq), per_seq(a.c.pages_per_seq), page_tokens(a.c.page_tokens), n_pages(a.c.n_pages) {
        idx = 32 * blk / page_tokens;
        slot = 32 * blk - idx * page_tokens;
        hold();
    }
    SJD_D void hold() {
        base = idx;
        const int i = idx + (int)(threadIdx.x & 63);
        held = i < per_seq ? table[i] : -1;
    }
    // page of the block (its first token: slot), -1 where there is none
    SJD_D int page() {
        if (idx - base >= 64) hold();
        const int p = __builtin_amdgcn_readlane(held, idx - base);
        return (unsigned)p < (unsigned)n_pages ? p : -1;
    }
    SJD_D void advance(int blocks) {
        slot += 32 * blocks;
        while (slot >= page_tokens) { slot -= page_tokens; ++idx; }
    }
};
// Registers that are loaded ahead of a loop: waits for them there.  (Where the first use is in the loop the compiler's wait is, too, and is one
// for everything that the loop has asked for since.)
template <int N> SJD_D void arrived(u32x4 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// ------------------------------------------------------------------------------------------------ one block of 32 tokens
// by value: __builtin_bit_cast of an element of a vector that is named in place takes the vector's first element, whichever is meant
SJD_D float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }

// Keys and values of a block as they come from memory; q operand; by kind
template <int KIND, int HD> struct TreeFrag {
    static constexpr int NK = HD * (KIND == SJD_F32 ? 4 : KIND == SJD_BF16 ? 2 : 1) / 32;   // 16-byte pieces of a lane: keys, and values
    static constexpr int NQ = HD * (KIND == SJD_F32 ? 4 : 2) / 32;
    u32x4 k[NK], v[NK];
    uint32_t k_scale;          // FP8: byte of token lane % 32
    uint32_t v_scale[4];       // FP8: bytes of tokens 8 m + 4 g + (0 .. 3)

    SJD_D void load_k(const TreeArgs &a, const unsigned char *block, int slot, int lane) {
        const u32x4 *p = reinterpret_cast<const u32x4 *>(block + (size_t)slot * HD * (KIND == SJD_F32 ? 4 : KIND == SJD_BF16 ? 2 : 1)) + lane;
#pragma unroll
        for (int i = 0; i < NK; ++i) k[i] = p[i * 64];
        if (KIND == SJD_FP8) k_scale = block[2 * (size_t)a.c.page_tokens * HD + slot + (lane & 31)];
    }
    SJD_D void load_v(const TreeArgs &a, const unsigned char *block, int slot, int lane) {
        const size_t size = KIND == SJD_F32 ? 4 : KIND == SJD_BF16 ? 2 : 1;
        const u32x4 *p = reinterpret_cast<const u32x4 *>(block + ((size_t)a.c.page_tokens + slot) * HD * size) + lane;
#pragma unroll
        for (int i = 0; i < NK; ++i) v[i] = p[i * 64];
        if (KIND == SJD_FP8) {
            const uint32_t *s = reinterpret_cast<const uint32_t *>(block + 2 * (size_t)a.c.page_tokens * HD + a.c.page_tokens + slot + 4 * (lane >> 5));
#pragma unroll
            for (int m = 0; m < 4; ++m) v_scale[m] = s[2 * m];
        }
    }
};

// two dwords of fp8 codes -> 8 bf16, times a power of two
SJD_D bf16x8 fp8_to_bf16(uint32_t lo, uint32_t hi, float scale) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, scale, true);
    const b2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
SJD_D float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }    // 2^(byte - 127)
template <int I> SJD_D float scale_of_byte(uint32_t w) {                                 // of byte I, in one instruction
    float r;
    if constexpr (I == 0) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(23), "v"(w));
    if constexpr (I == 1) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(23), "v"(w));
    if constexpr (I == 2) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(23), "v"(w));
    if constexpr (I == 3) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(r) : "v"(23), "v"(w));
    return r;
}

// q(n): piece n of the query operand
template <int KIND, int HD, typename Q>
SJD_D f32x16 tree_scores(const TreeFrag<KIND, HD> &f, Q q) {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.0f;
    if constexpr (KIND == SJD_F32) {
#pragma unroll
        for (int i = 0; i < HD / 8; ++i) {
            const u32x4 qi = q(i);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(as_float(f.k[i][e]), as_float(qi[e]), s, 0, 0, 0);
        }
    } else if constexpr (KIND == SJD_BF16) {
#pragma unroll
        for (int i = 0; i < HD / 16; ++i)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f.k[i]), __builtin_bit_cast(bf16x8, q(i)), s, 0, 0, 0);
    } else {
        const float ks = scale_of(f.k_scale);
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8_to_bf16(f.k[i][0], f.k[i][1], ks), __builtin_bit_cast(bf16x8, q(2 * i)), s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8_to_bf16(f.k[i][2], f.k[i][3], ks), __builtin_bit_cast(bf16x8, q(2 * i + 1)), s, 0, 0, 0);
        }
    }
    return s;
}

// A operand of the second product for dimension block db, half i of the tokens (not F32)
template <int KIND, int HD> SJD_D bf16x8 tree_values(const TreeFrag<KIND, HD> &f, int db, int i) {
    if constexpr (KIND == SJD_BF16) return __builtin_bit_cast(bf16x8, f.v[i * (HD / 32) + db]);
    else return fp8_to_bf16(f.v[db][2 * i], f.v[db][2 * i + 1], 1.0f);
}

enum { VALUE_FINITE = 0, VALUE_POS_INF = 1, VALUE_NEG_INF = 2, VALUE_NAN = 3 };
SJD_D int value_class(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    if ((u & 0x7F800000u) != 0x7F800000u) return VALUE_FINITE;
    return u & 0x007FFFFFu ? VALUE_NAN : u >> 31 ? VALUE_NEG_INF : VALUE_POS_INF;
}
// is any of a lane's values infinite or NaN
template <int KIND, int HD> SJD_D bool tree_values_wild(const TreeFrag<KIND, HD> &f) {
    bool wild = false;
#pragma unroll
    for (int i = 0; i < TreeFrag<KIND, HD>::NK; ++i)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const uint32_t u = f.v[i][d];
            if constexpr (KIND == SJD_F32) wild |= (u & 0x7F800000u) == 0x7F800000u;
            else if constexpr (KIND == SJD_BF16) wild |= (u & 0x7F80u) == 0x7F80u || (u & 0x7F800000u) == 0x7F800000u;
            else {   // a byte is 0x7F after its sign is cleared: adding 1 carries into its sign
                wild |= (((u & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0u;
            }
        }
    return wild;
}

// infinite and NaN values become 0
template <int KIND, int HD> SJD_D void tree_values_tame(TreeFrag<KIND, HD> &f) {
#pragma unroll
    for (int i = 0; i < TreeFrag<KIND, HD>::NK; ++i)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            uint32_t u = f.v[i][d];
            if constexpr (KIND == SJD_F32) u = (u & 0x7F800000u) == 0x7F800000u ? 0u : u;
            else if constexpr (KIND == SJD_BF16) u &= ((u & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((u & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
            else u &= ~(((((u & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xFFu);
            f.v[i][d] = u;
        }
}

// o + V P for dimension block db
template <int KIND, int HD>
SJD_D f32x16 tree_product(const TreeFrag<KIND, HD> &f, int db, const float (&p32)[16], const u32x4 (&pb)[2], f32x16 o) {
    if constexpr (KIND == SJD_F32) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
            o = __builtin_amdgcn_mfma_f32_32x32x2f32(as_float(f.v[db * 4 + (v >> 2)][v & 3]), p32[v], o, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tree_values<KIND, HD>(f, db, i), __builtin_bit_cast(bf16x8, pb[i]), o, 0, 0, 0);
    }
    return o;
}

// The running state of a wavefront's 32 rows: O^T, maxima (base 2), this lane's half of the sums
template <int HD> struct TreeState {
    f32x16 o[HD / 32];
    float m, l;
    SJD_D void clear() {
#pragma unroll
        for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[db][v] = 0.0f;
        m = -INFINITY;
        l = 0.0f;
    }
};

// Probabilities are 2^(score - m).  A rescaling puts m 8 above the row's maximum, a whole number, so that it is exact, and the next one comes when the
// maximum has grown beyond m: until then probabilities are between 2^-9 and 1 at the maximum, never above 1, and so no sum of products with values overflows that would not
// with the formula's own.  (With m at the maximum and up to 2^8 above it, finite values from 2^120 on became infinite.)  The factor costs neither fp32 sums nor bf16 operands
// a bit but at the lower end of the exponents: values below 2^-117 make subnormal products, which the matrix cores keep (of values of 2^-124 an fp32 row is
// 2^-18 off).
// `pending`: probabilities whose product with values is still to come.
constexpr float kTreeAhead = 8.0f;
template <int HD, typename F> SJD_D void tree_rescale(TreeState<HD> &st, float mx, F pending) {
    if (!__ballot(mx > st.m)) return;
    const float m = fmaxf(st.m, __builtin_ceilf(mx) + kTreeAhead);
    const float alpha = __builtin_amdgcn_exp2f(st.m - (m == -INFINITY ? 0.0f : m));     // (not (-inf) - (-inf))
    st.m = m;
    st.l *= alpha;
    pending(alpha);
#pragma unroll
    for (int db = 0; db < HD / 32; ++db) {
#pragma unroll
        for (int v = 0; v < 16; ++v) st.o[db][v] *= alpha;
        __builtin_amdgcn_sched_barrier(0);
    }
}

// sum + the two bf16 numbers of a pair, in fp32: what the products take is what the sums add, so that the weights of a row add up to 1 whatever their
// rounding (a row that sees one token gives its value, exactly), and one instruction where two additions of unrounded numbers were.
SJD_D float tree_add_pair(float sum, uint32_t pair) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(cache_bf16x2, pair), __builtin_bit_cast(cache_bf16x2, 0x3F803F80u), sum, false);
}

// Softmax of a block's scores into p (and, but for F32, its bf16 operand pb), and the rescaling of the state.  `vis`: bit k = this lane's
// row sees token k of the block.
template <int KIND, int HD>
SJD_D void tree_softmax(TreeFrag<KIND, HD> &f, f32x16 s, bool masked, uint32_t vis, float scale_log2e, TreeState<HD> &st, int lane,
                        float (&p)[16], u32x4 (&pb)[2]) {
    if (masked) {
        const uint32_t mine = vis >> (4 * (lane >> 5));     // bit 8 (v / 4) + v % 4 belongs to register v
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = mine >> (8 * (v >> 2) + (v & 3)) & 1u ? s[v] : -INFINITY;
        if constexpr (KIND == SJD_FP8) {
            // A token that nobody wrote may have a scale of 255, which is no number (and 0 times it none either): 254 in its place
#pragma unroll
            for (int m = 0; m < 4; ++m) f.v_scale[m] ^= (((f.v_scale[m] & 0x7F7F7F7Fu) + 0x01010101u) & f.v_scale[m] & 0x80808080u) >> 7;
        }
    }
    float mx = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * scale_log2e;
    tree_rescale<HD>(st, mx, [](float) {});
    const float m_use = st.m == -INFINITY ? 0.0f : st.m;    // a row that has seen nothing so far: not (-inf) - (-inf)
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        p[v] = __builtin_amdgcn_exp2f(fmaf(s[v], scale_log2e, -m_use));
        if (KIND == SJD_F32) sum += p[v];
    }
    if constexpr (KIND != SJD_F32) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const int v = 8 * i + 2 * d;
                float a = p[v], b = p[v + 1];
                sum = tree_add_pair(sum, pack_bf16(a, b));
                if constexpr (KIND == SJD_FP8) {           // the values' scales, exact: the product takes plain codes
                    a *= d & 1 ? scale_of_byte<2>(f.v_scale[v >> 2]) : scale_of_byte<0>(f.v_scale[v >> 2]);
                    b *= d & 1 ? scale_of_byte<3>(f.v_scale[v >> 2]) : scale_of_byte<1>(f.v_scale[v >> 2]);
                }
                pb[i][d] = pack_bf16(a, b);
            }
    }
    st.l += sum;
}

// Values some of which are infinite or NaN, of tokens that not every row sees: in O += V P their 0 * inf would reach the rows that do
// not.  Which rows see an element of which class is noted in LDS, bit r of wild[class - 1][dimension] for row r, and added at the end; the
// values become 0.  (Rare, so it is kept off the registers of the loop: with a product of ones per class in its place bf16 heads of
// 128 took all 256 and 43 in scratch memory, where they take 216.)
template <int KIND, int HD> SJD_D float tree_value(const TreeFrag<KIND, HD> &f, int db, int m, int e) {   // token 8 m + 4 g + e, dimension 32 db + lane % 32
    if constexpr (KIND == SJD_F32) return as_float(f.v[db * 4 + m][e]);
    else if constexpr (KIND == SJD_BF16) return bf16_to_float((bf16_t)(f.v[(m >> 1) * (HD / 32) + db][(m & 1) * 2 + (e >> 1)] >> (16 * (e & 1))));
    else return (f.v[db][m] >> (8 * e) & 0x7Fu) == 0x7Fu ? __builtin_nanf("") : 0.0f;
}
template <int KIND, int HD>
SJD_D void tree_note_wild(const TreeFrag<KIND, HD> &f, uint32_t vis, uint32_t (&wild)[3][HD], int lane) {
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = (uint32_t)__ballot(vis >> (8 * m + e) & 1u), hi = (uint32_t)__ballot(vis >> (8 * m + 4 + e) & 1u);
            const uint32_t rows = lane < 32 ? lo : hi;
#pragma unroll
            for (int db = 0; db < HD / 32; ++db) {
                const int cls = value_class(tree_value<KIND, HD>(f, db, m, e));
                if (cls != VALUE_FINITE && rows) atomicOr(&wild[cls - 1][db * 32 + (lane & 31)], rows);
            }
        }
}
// what the noted elements make of dimension j of a row
template <int HD> SJD_D float tree_add_wild(float x, const uint32_t (&wild)[3][HD], int row, int j) {
    if (wild[VALUE_POS_INF - 1][j] >> row & 1u) x += INFINITY;
    if (wild[VALUE_NEG_INF - 1][j] >> row & 1u) x -= INFINITY;
    if (wild[VALUE_NAN - 1][j] >> row & 1u) x += __builtin_nanf("");
    return x;
}

// The query operand of tile `tile`: lane's row = 32 tile + lane % 32.  Rows behind the last are zeros.
template <int KIND, int HD>
SJD_D void tree_load_q(const TreeArgs &a, const TreeSeq &s, int kvh, int tile, int lane, u32x4 (&q)[TreeFrag<KIND, HD>::NQ]) {
    const int rho = 32 * tile + (lane & 31), i = rho / a.G, g = rho - i * a.G;
    const bool live = i < s.n;
    constexpr int PIECE = KIND == SJD_F32 ? 4 : 8, SIZE = KIND == SJD_F32 ? 4 : 2;   // elements of 16 bytes
    const char *src = (const char *)a.q + ((size_t)(s.r0 + (live ? i : 0)) * a.q_stride + (size_t)(kvh * a.G + (live ? g : 0)) * HD) * SIZE;
#pragma unroll
    for (int n = 0; n < TreeFrag<KIND, HD>::NQ; ++n) {
        const char *p = src + (size_t)(n * 2 + (lane >> 5)) * PIECE * SIZE;
        u32x4 x = {0u, 0u, 0u, 0u};
        if (live) {
            if (a.q_wide) x = *reinterpret_cast<const u32x4 *>(p);
            else if (KIND == SJD_F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = reinterpret_cast<const uint32_t *>(p)[e];
            } else {
                const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = h[2 * e] | (uint32_t)h[2 * e + 1] << 16;
            }
        }
        q[n] = x;
    }
}

// four dimensions of one output row
template <int KIND> SJD_D void tree_store(const TreeArgs &a, size_t row, int h, int hd, int j, f32x4 t) {
    if constexpr (KIND == SJD_F32) {
        float *p = (float *)a.out + row * a.out_stride + (size_t)h * hd + j;
        if (a.out_wide) *reinterpret_cast<f32x4 *>(p) = t;
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = t[e];
        }
    } else {
        bf16_t *p = (bf16_t *)a.out + row * a.out_stride + (size_t)h * hd + j;
        const uint2 w = {pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3])};
        if (a.out_wide) *reinterpret_cast<uint2 *>(p) = w;
        else {
            p[0] = (bf16_t)w.x; p[1] = (bf16_t)(w.x >> 16); p[2] = (bf16_t)w.y; p[3] = (bf16_t)(w.y >> 16);
        }
    }
}

// Partial results lie in the order in which the lanes hold them: a wavefront's store is 1 KiB
SJD_D int tree_part_index(int row, int j) { return ((j >> 3) * 64 + ((j >> 2) & 1) * 32 + row) * 4; }

// what the noted wild elements and the norm make of the quad of dimensions j of a row, and where it goes: to the output, or to a partial result
template <int KIND, int HD>
SJD_D void tree_finish(const TreeArgs &a, const TreeSeq &s, int kvh, size_t slot, int tile, int row, int j, float norm, bool any_wild, const uint32_t (&wild)[3][HD], f32x4 t) {
    const int rho = 32 * tile + row, node = rho / a.G;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        t[e] = norm == 0.0f ? 0.0f : t[e] * norm;
        if (any_wild) t[e] = tree_add_wild<HD>(t[e], wild, row, j + e);
    }
    if (node >= s.n) return;
    if (a.n_splits > 1) *reinterpret_cast<f32x4 *>(a.part_o + slot * 32 * HD + tree_part_index(row, j)) = t;
    else tree_store<KIND>(a, (size_t)s.r0 + node, kvh * a.G + rho - node * a.G, HD, j, t);
}

// --------------------------------------------------------------------------------------------------- wavefronts over tokens
// Workgroup = tile of 32 rows, of a split; its wavefronts take the blocks in turn and merge through LDS.  For few rows: what bounds it is
// the stream of keys and values.  Four fp8 sequences of 24 000 - 42 000 tokens, 8 kv heads of 128, a token each: 234 MB in 46.2 us, 5.1 TB/s, where a
// copy reaches 5.5.  Eight bf16 trees of 13 - 53 nodes over 850 - 3 850 tokens, 32 heads of 128: 216 MB in 49.5 us, 4.4 TB/s.  With many rows it is
// the order of a block's steps: sixteen fp8 trees of 44 - 78 nodes, 4 query heads a kv head, over 5 200 - 11 200 tokens, 94 GFLOP in 187 us, 0.5 PFLOP/s (a
// large product reaches 1.41).  Scores, softmax and output follow each other, with two wavefronts a SIMD to fill the gaps: of the cycles in which a CU has work
// its matrix cores are busy for 31 %, its vector units for 55 %.  Tried: one line of all sequences' blocks cut into equal shares, 53.7 us for the first, 67.7 for the second,
// as a share then joins several sequences; two tiles of rows a wavefront, 427 us for the third, one wavefront a SIMD and copies between register files.
constexpr int kTreeWaves = 4;

// A lane's registers hold its queries, keys, values and output: from 40 (fp8 heads of 32) to 512 of 512 (fp32 heads of 256).  Wide heads
// leave the queries in LDS, and fp32 heads of 256 ask for keys and values only when the other ones are done with.
template <int KIND, int HD> constexpr bool kTreeQueriesInLds = KIND == SJD_F32 ? HD >= 192 : HD == 256;
template <int KIND, int HD> constexpr bool kTreeLateLoads = KIND == SJD_F32 && HD == 256;
constexpr int tree_waves_per_simd(int kind, int hd) {
    return hd * (kind == SJD_F32 ? 4 : kind == SJD_BF16 ? 2 : 1) / 4 + hd * (kind == SJD_F32 ? 2 : 1) / 4 + hd / 2 <= 191 ? 2 : 1;
}

template <int KIND, int HD>
__global__ __launch_bounds__(kTreeWaves * 64, tree_waves_per_simd(KIND, HD)) void tree_attention_kernel(TreeArgs a) {
    constexpr int DB = HD / 32, NW = kTreeWaves;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 31;
    __shared__ uint32_t wild[3][HD], any_wild;
    __shared__ float ml[NW][2][32];
    __shared__ f32x4 red[NW][4][64];
    constexpr int NL = kTreeQueriesInLds<KIND, HD> ? TreeFrag<KIND, HD>::NQ : 1;
    __shared__ u32x4 q_lds[NL][64];
    const TreeWork w = tree_work(a, blockIdx.x);
    if (w.b >= a.c.n_seqs) return;
    const int tile = w.group, kvh = w.kvh;
    const TreeSeq s = tree_seq(a, w.b);
    if (32 * tile >= s.n * a.G) return;
    const TreeBlocks range = tree_blocks(a.mask, s.ctx, s.n_tot, min((32 * tile + 31) / a.G, s.n - 1), w.split, a.n_splits);
    const int first = range.first, last = range.last;
    const int rho = 32 * tile + row, node = rho / a.G;
    const bool live = node < s.n;
    const uint32_t *mask = a.mask && live ? a.mask + (size_t)(s.r0 + node) * a.mask_words : nullptr;
    TreeState<HD> st;
    st.clear();
    TreeFrag<KIND, HD> f;
    u32x4 q[TreeFrag<KIND, HD>::NQ];
    TreePages pages(a, w.b, min(first + wave, last));
    int blk = first + wave, page = blk < last ? pages.page() : -1;
    tree_load_q<KIND, HD>(a, s, kvh, tile, lane, q);
    if (page >= 0) {
        f.load_k(a, cache_block(a.c, page, kvh), pages.slot, lane);
        if (!kTreeLateLoads<KIND, HD>) f.load_v(a, cache_block(a.c, page, kvh), pages.slot, lane);
    }
    arrived(q);
    for (int i = threadIdx.x; i < 3 * HD; i += NW * 64) (&wild[0][0])[i] = 0u;
    if (threadIdx.x == 0) any_wild = 0u;
    if constexpr (kTreeQueriesInLds<KIND, HD>) {
        if (wave == 0)
#pragma unroll
            for (int n = 0; n < NL; ++n) q_lds[n][lane] = q[n];
    }
    __syncthreads();
    auto query = [&](int n) {
        if constexpr (kTreeQueriesInLds<KIND, HD>) return q_lds[n][lane];
        else return q[n];
    };
    while (blk < last) {
        const int next = blk + NW, t0 = 32 * blk;
        pages.advance(NW);
        const int next_page = next < last ? pages.page() : -1, next_slot = pages.slot;
        const unsigned char *next_block = next_page >= 0 ? cache_block(a.c, next_page, kvh) : nullptr;
        if (page >= 0) {
            const bool masked = t0 + 32 > s.ctx;
            uint32_t vis = 0xFFFFFFFFu;
            if (masked) vis = live ? tree_visible(mask, a.mask_words, s.ctx, s.n_tot, node, t0) : 0u;
            const f32x16 sc = tree_scores<KIND, HD>(f, query);
            if (kTreeLateLoads<KIND, HD>) {
                __builtin_amdgcn_sched_barrier(0);
                f.load_v(a, cache_block(a.c, page, kvh), t0 % a.c.page_tokens, lane);
            } else if (next_page >= 0) f.load_k(a, next_block, next_slot, lane);
            float p[16];
            u32x4 pb[2];
            tree_softmax<KIND, HD>(f, sc, masked, vis, a.scale_log2e, st, lane, p, pb);
            if (masked && __ballot(tree_values_wild<KIND, HD>(f))) {
                if (lane == 0) any_wild = 1;
                tree_note_wild<KIND, HD>(f, vis, wild, lane);
                tree_values_tame<KIND, HD>(f);
            }
#pragma unroll
            for (int db = 0; db < DB; ++db) st.o[db] = tree_product<KIND, HD>(f, db, p, pb, st.o[db]);
            if (kTreeLateLoads<KIND, HD>) {
                __builtin_amdgcn_sched_barrier(0);
                if (next_page >= 0) f.load_k(a, next_block, next_slot, lane);
            } else if (next_page >= 0) f.load_v(a, next_block, next_slot, lane);
        } else if (next_page >= 0) {
            f.load_k(a, next_block, next_slot, lane);
            if (!kTreeLateLoads<KIND, HD>) f.load_v(a, next_block, next_slot, lane);
        }
        blk = next;
        page = next_page;
    }
    st.l += __shfl_xor(st.l, 32, 64);

    // merge: out = sum_w 2^(m_w - m) O_w / sum_w 2^(m_w - m) l_w, 32 dimensions at a time
    if (lane < 32) {
        ml[wave][0][row] = st.m;
        ml[wave][1][row] = st.l;
    }
    __syncthreads();
    float m_all = -INFINITY;
#pragma unroll
    for (int i = 0; i < NW; ++i) m_all = fmaxf(m_all, ml[i][0][row]);
    const float m_use = m_all == -INFINITY ? 0.0f : m_all;
    float denom = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i) denom += __builtin_amdgcn_exp2f(ml[i][0][row] - m_use) * ml[i][1][row];
    const float mine = __builtin_amdgcn_exp2f(st.m - m_use);
    // (denom is NaN, and so is the row, where a score is; it is 0 where the row saw nothing)
    const size_t slot = tree_slot(a, w.b, kvh, w.split, tile);
    const bool split = a.n_splits > 1;
    const float norm = split ? 1.0f : denom == 0.0f ? 0.0f : 1.0f / denom;
    if (split && wave == 0 && lane < 32) {
        float *part = a.part_ml + slot * 64 + row;
        part[0] = m_all;
        part[32] = denom;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        if (db > 0) __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u)
            red[wave][u][lane] = f32x4{st.o[db][4 * u] * mine, st.o[db][4 * u + 1] * mine, st.o[db][4 * u + 2] * mine, st.o[db][4 * u + 3] * mine};
        __syncthreads();
        f32x4 t = red[0][wave][lane];      // NW == 4 quads: wavefront u adds quad u
#pragma unroll
        for (int i = 1; i < NW; ++i) t += red[i][wave][lane];
        tree_finish<KIND, HD>(a, s, kvh, slot, tile, row, db * 32 + 8 * wave + 4 * (lane >> 5), norm, any_wild, wild, t);
    }
}
static_assert(kTreeWaves == 4, "a wavefront adds one quad of a lane's 16 accumulators");

// ------------------------------------------------------------------------------------------------------ wavefronts over rows
// bf16 caches.  Workgroup = a tile of 32 rows for each of its four wavefronts, of a split: every block is fetched once for all of them and read
// from LDS, in the layout of its page, by every wavefront.  While a wavefront turns block j's scores into probabilities, the matrix cores work on
// the scores of block j + 1 and the output of block j - 1, one product between every few instructions.  Sixteen bf16 trees of 44 - 78 nodes, 4 query heads a kv head
// of 128, over 5 200 - 11 200 tokens, 94 GFLOP: 179 us, 0.53 PFLOP/s (by tokens: 207).  Bound by what comes ahead of that in every round, the barrier and the reads of the
// operands from LDS: of the cycles in which a CU has work its LDS is busy for 43 %, its vector units for 35 %, its matrix cores for 33 %.
constexpr int kTreeRowWaves = 4, kTreeRowThreads = 64 * kTreeRowWaves;
constexpr int kTreeRing = 4;     // blocks in LDS: the last one's values, this one, the next one's keys, and the one that is being written

template <int HD> struct TreeLds {
    u32x4 k[kTreeRing][HD * 4], v[kTreeRing][HD * 4];
    // infinities and NaN among the values: bit t of map[class - 1][dimension] for token t of a block
    uint32_t map[kTreeRing][3][HD], mapped[kTreeRing];
    uint32_t wild[kTreeRowWaves][3][HD], any_wild[kTreeRowWaves];
};

// 8 values of dimension 32 db + lane % 32, tokens 8 (2 i + e / 4) + 4 (lane / 32) + e % 4: infinities and NaN become 0 and are noted
template <int HD> SJD_D void tree_tame(u32x4 &x, int i, int db, int lane, uint32_t (&map)[3][HD], uint32_t &mapped) {
    bool wild = false;
#pragma unroll
    for (int d = 0; d < 4; ++d) wild |= (x[d] & 0x7F80u) == 0x7F80u || (x[d] & 0x7F800000u) == 0x7F800000u;
    if (!wild) return;
    mapped = 1u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int cls = value_class(bf16_to_float((bf16_t)(x[e >> 1] >> (16 * (e & 1)))));
        if (cls == VALUE_FINITE) continue;
        atomicOr(&map[cls - 1][db * 32 + (lane & 31)], 1u << (8 * (2 * i + (e >> 2)) + 4 * (lane >> 5) + (e & 3)));
        x[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
    }
}

// A thread's 16-byte pieces of a block on their way to LDS.  A block that is not there becomes zeros.
template <int HD> struct TreeStage {
    static constexpr int PIECES = HD * 4, PER = (PIECES + kTreeRowThreads - 1) / kTreeRowThreads;
    u32x4 k[PER], v[PER];
    SJD_D static bool has(int n) { return PIECES % kTreeRowThreads == 0 || n < PIECES; }
    SJD_D void load(const TreeArgs &a, const unsigned char *block, int slot, int tid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int n = tid + kTreeRowThreads * i;
            k[i] = v[i] = u32x4{0u, 0u, 0u, 0u};
            if (!has(n) || !block) continue;
            k[i] = reinterpret_cast<const u32x4 *>(block + (size_t)slot * HD * 2)[n];
            v[i] = reinterpret_cast<const u32x4 *>(block + ((size_t)a.c.page_tokens + slot) * HD * 2)[n];
        }
    }
    SJD_D void store(TreeLds<HD> &l, int buf, bool tame, int tid) const {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int n = tid + kTreeRowThreads * i, frag = n >> 6;
            if (!has(n)) continue;
            u32x4 x = v[i];
            if (tame) tree_tame<HD>(x, frag / (HD / 32), frag % (HD / 32), n & 63, l.map[buf], l.mapped[buf]);
            l.k[buf][n] = k[i];
            l.v[buf][n] = x;
        }
    }
};

template <int HD>
__global__ __launch_bounds__(kTreeRowThreads, HD <= 128 ? 2 : 1) void tree_attention_rows_kernel(TreeArgs a) {
    constexpr int DB = HD / 32, NQ = HD / 16, NW = kTreeRowWaves, THREADS = kTreeRowThreads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 31, tid = threadIdx.x;
    __shared__ TreeLds<HD> l;
    const TreeWork w = tree_work(a, blockIdx.x);
    if (w.b >= a.c.n_seqs) return;
    const TreeSeq s = tree_seq(a, w.b);
    if (32 * NW * w.group >= s.n * a.G) return;
    const int tile = w.group * NW + wave, node = (32 * tile + row) / a.G;
    const bool live = node < s.n, busy = 32 * tile < s.n * a.G;     // (a wavefront without rows helps to fetch)
    const uint32_t *mask = a.mask && live ? a.mask + (size_t)(s.r0 + node) * a.mask_words : nullptr;
    const TreeBlocks range = tree_blocks(a.mask, s.ctx, s.n_tot, min((32 * NW * (w.group + 1) - 1) / a.G, s.n - 1), w.split, a.n_splits);
    TreePages pages(a, w.b, range.first);
    TreeState<HD> st;
    st.clear();
    u32x4 q[NQ];
    tree_load_q<SJD_BF16, HD>(a, s, w.kvh, tile, lane, q);
    TreeStage<HD> stage;
    for (int i = tid; i < kTreeRing * 3 * HD; i += THREADS) (&l.map[0][0][0])[i] = 0u;
    for (int i = tid; i < NW * 3 * HD; i += THREADS) (&l.wild[0][0][0])[i] = 0u;
    // "the last block's values" of the first one: probabilities of 0 meet them
    for (int i = tid; i < HD * 4; i += THREADS) l.v[kTreeRing - 1][i] = u32x4{0u, 0u, 0u, 0u};
    if (tid < kTreeRing) l.mapped[tid] = 0u;
    if (tid < NW) l.any_wild[tid] = 0u;
    __syncthreads();
    // of this block, the next one, and the one in registers: whether it is there, and whether some row may not see all of it
    bool there[3] = {false, false, false}, part[3] = {false, false, false};
    auto fetch = [&](int blk, int i) {
        if (blk >= range.last) return;
        const int page = pages.page();
        there[i] = page >= 0;
        part[i] = page < 0 || 32 * (blk + 1) > s.ctx;
        stage.load(a, page >= 0 ? cache_block(a.c, page, w.kvh) : nullptr, pages.slot, tid);
        pages.advance(1);
    };
    fetch(range.first, 0);
    if (range.first < range.last) stage.store(l, 0, part[0], tid);
    fetch(range.first + 1, 1);
    if (range.first + 1 < range.last) stage.store(l, 1, part[1], tid);
    fetch(range.first + 2, 2);
    arrived(q);
    __syncthreads();
    f32x16 sc;
    u32x4 p[2] = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};     // probabilities of the last block, still to meet its values
#pragma unroll
    for (int v = 0; v < 16; ++v) sc[v] = 0.0f;
    if (busy && range.first < range.last)
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, l.k[0][n * 64 + lane]), __builtin_bit_cast(bf16x8, q[n]), sc, 0, 0, 0);
    int cur = 0;
    for (int blk = range.first; blk < range.last; ++blk, cur = (cur + 1) & (kTreeRing - 1)) {
        const int before = (cur + kTreeRing - 1) & (kTreeRing - 1), after = (cur + 1) & (kTreeRing - 1), far = (cur + 2) & (kTreeRing - 1);
        __syncthreads();
        if (l.mapped[before]) {          // (rare; the same for all threads: nobody writes it between two barriers)
            __syncthreads();
            for (int i = tid; i < 3 * HD; i += THREADS) (&l.map[before][0][0])[i] = 0u;
            if (tid == 0) l.mapped[before] = 0u;
            __syncthreads();
        }
        // the block after the next, asked for a round ago, goes to LDS, and the one behind it is asked for
        const bool far_there = there[2], far_part = part[2];
        if (blk + 2 < range.last) {
            stage.store(l, far, far_part, tid);
            fetch(blk + 3, 2);
        }
        if (busy) {
            // operands of the products to come: asked for ahead of everything else, they are there when it is done
            u32x4 kf[NQ], vf[NQ];
#pragma unroll
            for (int n = 0; n < NQ; ++n) kf[n] = l.k[after][n * 64 + lane];
#pragma unroll
            for (int n = 0; n < NQ; ++n) vf[n] = l.v[before][n * 64 + lane];
            __builtin_amdgcn_sched_barrier(0);
            if (part[0]) {
                const uint32_t vis = live && there[0] ? tree_visible(mask, a.mask_words, s.ctx, s.n_tot, node, 32 * blk) : 0u;
                const uint32_t mine = vis >> (4 * (lane >> 5));
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[v] = mine >> (8 * (v >> 2) + (v & 3)) & 1u ? sc[v] : -INFINITY;
                if (l.mapped[cur]) {
                    if (lane == 0) l.any_wild[wave] = 1u;
#pragma unroll 1
                    for (int i = 0; i < 3 * HD; ++i) {
                        const uint32_t rows = (uint32_t)__ballot(vis & (&l.map[cur][0][0])[i]);
                        if (lane == 0) (&l.wild[wave][0][0])[i] |= rows;
                    }
                }
            }
            float mx = sc[0];
#pragma unroll
            for (int v = 1; v < 16; ++v) mx = fmaxf(mx, sc[v]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * a.scale_log2e;
            tree_rescale<HD>(st, mx, [&](float alpha) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int d = 0; d < 4; ++d) p[i][d] = pack_bf16(as_float(p[i][d] << 16) * alpha, as_float(p[i][d] & 0xFFFF0000u) * alpha);
            });
            const float m_use = st.m == -INFINITY ? 0.0f : st.m;
            __builtin_amdgcn_sched_barrier(0);
            f32x16 sn;
            float sum = 0.0f;
            u32x4 pn[2];
#pragma unroll
            for (int v = 0; v < 16; ++v) sn[v] = 0.0f;
#pragma unroll
            for (int n = 0; n < NQ; ++n)
                sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[n]), __builtin_bit_cast(bf16x8, q[n]), sn, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    st.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[i * DB + db]), __builtin_bit_cast(bf16x8, p[i]), st.o[db], 0, 0, 0);
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[v] = __builtin_amdgcn_exp2f(fmaf(sc[v], a.scale_log2e, -m_use));
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    pn[i][d] = pack_bf16(sc[8 * i + 2 * d], sc[8 * i + 2 * d + 1]);
                    sum = tree_add_pair(sum, pn[i][d]);
                }
#pragma unroll
            for (int n = 0; n < 2 * NQ; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);      // a matrix product,
                __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);      // a few instructions
                __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);      // and an exponential
            }
            // (without this they are put off to where they are needed, behind the products)
            asm volatile("" : "+v"(pn[0]), "+v"(pn[1]), "+v"(sum));
            __builtin_amdgcn_sched_barrier(0);
            st.l += sum;
            sc = sn;
            p[0] = pn[0];
            p[1] = pn[1];
        }
        there[0] = there[1]; there[1] = far_there;
        part[0] = part[1]; part[1] = far_part;
    }
    if (!busy) return;
    // the last block's values: behind the loop, not as its last round's branch, whose join would copy the output registers every round
    if (range.first < range.last) {
        const u32x4 *vp = &l.v[(cur + kTreeRing - 1) & (kTreeRing - 1)][lane];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int db = 0; db < DB; ++db)
                st.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vp[(i * DB + db) * 64]), __builtin_bit_cast(bf16x8, p[i]), st.o[db], 0, 0, 0);
    }
    const bool split = a.n_splits > 1;
    const float sum = st.l + __shfl_xor(st.l, 32, 64);
    const float norm = split ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum;
    const size_t slot = tree_slot(a, w.b, w.kvh, w.split, tile);
    if (split && lane < 32) {
        float *part_ml = a.part_ml + slot * 64 + row;
        part_ml[0] = st.m;
        part_ml[32] = sum;
    }
    const bool any = l.any_wild[wave];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            tree_finish<SJD_BF16, HD>(a, s, w.kvh, slot, tile, row, db * 32 + 8 * u + 4 * (lane >> 5), norm, any, l.wild[wave],
                                      f32x4{st.o[db][4 * u], st.o[db][4 * u + 1], st.o[db][4 * u + 2], st.o[db][4 * u + 3]});
}

// ------------------------------------------------------------------------------------------------------------------ joining
// Joins the splits of every row: out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  A thread owns four dimensions of a row.  Where a split
// saw nothing of a row l = 0.  Bound by latency: N splits, for most calls all of them, are on their way together with the row's lengths (rows
// that turn out not to be there read what their place in the workspace holds, and drop it): 5.4 us for 16 splits of 128 rows, 8.0 with one after the other.
template <int KIND, int N>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeArgs a) {
    const int quads = a.c.hd >> 2, per = 32 * quads;
    const unsigned wgs = (per + 255) / 256;
    const unsigned pair = blockIdx.x / wgs;
    const int u = (blockIdx.x % wgs) * 256 + threadIdx.x;
    const int tile = pair % a.tiles, kvh = (pair / a.tiles) % a.c.n_kv, b = pair / a.tiles / a.c.n_kv;
    if (u >= per) return;
    const int row = u & 31, j = (u >> 5) * 4;
    const size_t slot0 = tree_slot(a, b, kvh, 0, tile), step = a.tiles;
    float m = -INFINITY, denom = 0.0f;
    f32x4 t = {0.0f, 0.0f, 0.0f, 0.0f};
    int r0 = 0, n = 0;
    for (int i0 = 0; i0 < a.n_splits; i0 += N) {
        float pm[N], pl[N];
        f32x4 po[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const size_t slot = slot0 + min(i0 + i, a.n_splits - 1) * step;
            pm[i] = a.part_ml[slot * 64 + row];
            pl[i] = a.part_ml[slot * 64 + 32 + row];
            po[i] = *reinterpret_cast<const f32x4 *>(a.part_o + slot * per * 4 + tree_part_index(row, j));
        }
        if (i0 == 0) {
            const TreeSeq s = tree_seq(a, b);
            r0 = s.r0;
            n = s.n;
        }
        float m_new = m;
#pragma unroll
        for (int i = 0; i < N; ++i) m_new = fmaxf(m_new, pm[i]);
        const float m_use = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        m = m_new;
        denom *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = finite_f(t[e]) ? t[e] * alpha : t[e];      // (alpha may be 0: not 0 * inf)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i0 + i >= a.n_splits || pl[i] == 0.0f) continue;
            const float w = __builtin_amdgcn_exp2f(pm[i] - m_use);
            denom += w * pl[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] += finite_f(po[i][e]) ? w * po[i][e] : po[i][e];
        }
    }
    const int rho = 32 * tile + row, node = rho / a.G;
    if (node >= n) return;
    const float inv = denom == 0.0f ? 0.0f : 1.0f / denom;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = denom == 0.0f ? 0.0f : t[e] * inv;
    tree_store<KIND>(a, (size_t)r0 + node, kvh * a.G + rho - node * a.G, a.c.hd, j, t);
}
template <int KIND> inline void launch_tree_combine(hipStream_t st, const TreeArgs &a) {
    const unsigned grid = (unsigned)((size_t)a.c.n_seqs * a.c.n_kv * a.tiles * ceil_div(8 * a.c.hd, 256));
    if (a.n_splits <= 4) tree_combine_kernel<KIND, 4><<<grid, 256, 0, st>>>(a);
    else tree_combine_kernel<KIND, 16><<<grid, 256, 0, st>>>(a);
}
