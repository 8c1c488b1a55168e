// Attention of packed prompts: causal, grouped heads, ragged sequences, keys and values as they come from a projection or from a cache that was read back.
//
// Rows (i, h) of one kv head of a sequence are cut into tiles (prompt_layout.h), so that the query heads of a group share keys and values.  Per block
// of keys a wavefront computes, for 32 of its tile's rows,
//   S^T (keys x rows) = K Q^T,   online softmax per row = per accumulator column,   O^T (dimensions x rows) += V^T P^T,
// and P^T needs no data movement: the accumulator registers of S^T are the B operand of the second product, if the keys of V^T are taken in their order.
// Keys and values go through LDS, straight from memory, for all four wavefronts of a workgroup; a block's products come from there while the next one arrives.
//
// What bounds it: matrix and vector units, and, before either is full, the card's power (bf16, 16 001 rows of 32 heads of 128 in 8 groups: 1 880 - 1 980 us, 1.06 - 1.12 PFLOP/s, where a large library
// product reaches 1.22 - 1.4; matrix units busy for 58 % of the cycles, vector units for 47, at 1.5 - 1.7 GHz).  A block's 16 products of 32 rows are 512 cycles of a SIMD, its exponentials and what
// belongs to them some 75 instructions, which other wavefronts' products hide; there are two to five of them a SIMD.  Short prompts pay for a tile's beginning and end, some 9 us with waiting, of
// which the CU's other workgroups hide a part (12 prompts of 61 to 2 352 rows, 32 heads of 128: 248 - 259 us, 0.75 - 0.78 PFLOP/s; 38 % and 39 %).  With heads of 32 and 64 the products of
// a block are fewer and its 75 instructions are not: 8 192 rows of 16 heads 520 - 540 and 780 - 818 TFLOP/s.  fp32: a block's chain from products to exponentials to products, which the CU's other
// workgroups hide where there are some: of the matrix units' 154 TFLOP/s 118 - 127 over 8 192 rows of 16 heads of 64, 128 and 256, 78 - 88 over 2 048, which are one workgroup a CU.
// Tried, and not here: workgroups of 8 wavefronts with four blocks in LDS (16 001 rows: the same; 12 prompts 3 % slower), parts of a block's products between another's exponentials in one wavefront (10 %
// slower), 64 rows a wavefront (registers), workgroups that stay and take one tile after the other with the next one's keys on their way (12 prompts 12 % slower: shares fixed beforehand come out uneven,
// and each block has more to keep track of), values on their way to registers before the exponentials (the same with heads of 128, 10 to 26 % slower with 64, 192 and 256).
#pragma once
#include <type_traits>

#include "common.hip.h"
#include "kernels_cache.hip.h"
#include "prompt_layout.h"

struct PromptArgs {
    const void *q, *k, *v;     // [n_rows][H][hd], [n_kv_rows][n_kv][hd] twice; rows a stride apart
    void *out;                 // [n_rows][H][hd]
    long q_stride, k_stride, v_stride, out_stride;
    const int32_t *row_start, *kv_start;   // kv_start NULL: row_start
    int n_rows, n_kv_rows, n_seqs, H, n_kv, G;
    int tiles;                 // upper bound, of all sequences
    int n_splits, per_split;   // of a tile's blocks of keys
    float scale_log2e;
    float *part_o;             // [tile][kv head][split][32-row tile][32 * hd]   unnormalised, order of prompt_part_index
    float *part_ml;            // [tile][kv head][split][32-row tile][2][32]     reference (base 2), sum
    bool q_wide, out_wide;     // rows 16-byte aligned
};

constexpr int kPromptWaves = 4;
// bf16: the products' operands have 16 bits, so probabilities are rounded to them, by 2^-8 of each at most; results are 1.9 - 2.3e-3 off (root mean square, relative; 120 to 16 001 rows of normal values),
// where their own rounding alone is 1.6e-3.  op_tree_attention does the same.

// Waves that the compiler leaves registers for, of a SIMD: two overlap one's products with the other's exponentials (fp32, 8 192 rows of 16 heads of 128 in 4 groups over themselves: 67 against 52 TFLOP/s);
// with heads of 192 and 256 in fp32 the queries and the output alone fill what one may have.  (bf16 with heads of 256 takes all 256 registers and keeps 3 more in memory; with heads of 96 and 128, and
// fp32 with 96, 43 to 47 scalars lie in lanes of a vector register.)
constexpr int prompt_waves_per_simd(int size, int hd) { return size == 2 || hd <= 128 ? 2 : 1; }
// Tokens of a block.  Of wide heads 32, which halves the scores, and with operands that are loaded as others are used up leaves room for a second wave or a third (bf16, as above, heads of 256: 1 120
// against 435 TFLOP/s, 192: 1 104 against 811, 128: 999 against 979; heads of 64: 772 against 784).
constexpr int prompt_block(int size, int hd) { return size == 2 && hd < 128 ? 64 : 32; }

// A workgroup's tile: sequence (-1: there is none), tile of it, first row and number of rows, first key and number of keys
struct PromptTile { int b, t, r0, n, k0, n_keys; };
struct PromptSeq { int r0, n, k0, n_keys; };
SJD_D PromptSeq prompt_seq(const PromptArgs &a, int b) {
    PromptSeq s{rows_first(a.row_start, b, a.n_rows), rows_count(a.row_start, b, a.n_rows), 0, 0};
    s.k0 = a.kv_start ? rows_first(a.kv_start, b, a.n_kv_rows) : s.r0;
    s.n_keys = a.kv_start ? rows_count(a.kv_start, b, a.n_kv_rows) : s.n;
    return s;
}
// The tile that a workgroup takes.  Workgroups begin in the order of their numbers, so those with many keys come first: the last tiles of a sequence, and of up to 64 sequences the longest
// (12 of 61 to 2 352 rows, 32 heads of 128: 277 -> 270 us against the last one first).  Of more, a tile's number says where to look, 64 places at a time (5 120 of 16 rows: 879 -> 290 us against adding up
// the tiles of all sequences before it).
SJD_D PromptTile prompt_find_tile(const PromptArgs &a, int rows, int index) {
    const int lane = threadIdx.x & 63;
    PromptSeq s{0, 0, 0, 0};
    int t, l, b = lane;
    if (a.n_seqs <= 64) {
        if (b < a.n_seqs) s = prompt_seq(a, b);
        const int tiles = prompt_tiles(s.n, a.G, rows);
        const uint32_t order = (uint32_t)min(s.n_keys, (1 << 26) - 1) << 6 | (63 - lane);
        int before = 0;
        for (int o = 0; o < a.n_seqs; ++o)
            before += (uint32_t)__builtin_amdgcn_readlane(order, o) > order ? __builtin_amdgcn_readlane(tiles, o) : 0;
        const unsigned long long mine = __ballot(before <= index && index < before + tiles);
        if (!mine) return PromptTile{-1, 0, 0, 0, 0, 0};
        l = __ffsll((long long)mine) - 1;
        t = __builtin_amdgcn_readlane(tiles, l) - 1 - (index - __builtin_amdgcn_readlane(before, l));
    } else {
        index = a.tiles - 1 - index;
        int lo = 0, n = a.n_seqs;          // it is one of [lo, lo + n)
        for (;;) {
            const int step = (n + 63) / 64;
            const bool in = lane * step < n;
            b = lo + lane * step;
            const int start = in ? prompt_place(rows_first(a.row_start, b, a.n_rows), b, a.G, rows) : 0;
            const unsigned long long upto = __ballot(in && start <= index);
            if (!upto) return PromptTile{-1, 0, 0, 0, 0, 0};
            l = 63 - __clzll((long long)upto);
            if (step == 1) {
                t = index - __builtin_amdgcn_readlane(start, l);
                break;
            }
            lo += l * step;
            n = min(step, n - l * step);
        }
        b = __builtin_amdgcn_readlane(b, l);
        s = prompt_seq(a, b);
        l = 0;
        if (t >= __builtin_amdgcn_readfirstlane(prompt_tiles(s.n, a.G, rows))) return PromptTile{-1, 0, 0, 0, 0, 0};
    }
    return PromptTile{__builtin_amdgcn_readlane(b, l), t, __builtin_amdgcn_readlane(s.r0, l), __builtin_amdgcn_readlane(s.n, l), __builtin_amdgcn_readlane(s.k0, l),
                      __builtin_amdgcn_readlane(s.n_keys, l)};
}

SJD_D size_t prompt_slot(const PromptArgs &a, int tile, int kvh, int split) { return ((size_t)tile * a.n_kv + kvh) * a.n_splits + split; }
// Partial results lie in the order in which the lanes hold them: a wavefront's store is 1 KiB
SJD_D int prompt_part_index(int row, int j) { return ((j >> 3) * 64 + ((j >> 2) & 1) * 32 + row) * 4; }

// four dimensions of an output row
template <typename T> SJD_D void prompt_store(const PromptArgs &a, size_t row, int h, int hd, int j, f32x4 t) {
    T *p = (T *)a.out + row * a.out_stride + (size_t)h * hd + j;
    if constexpr (sizeof(T) == 4) {
        if (a.out_wide) *reinterpret_cast<f32x4 *>(p) = t;
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = t[e];
        }
    } else {
        const uint2 w = {pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3])};
        if (a.out_wide) *reinterpret_cast<uint2 *>(p) = w;
        else {
            p[0] = (bf16_t)w.x; p[1] = (bf16_t)(w.x >> 16); p[2] = (bf16_t)w.y; p[3] = (bf16_t)(w.y >> 16);
        }
    }
}

// The query operand of 32 rows: lane's row = first + lane % 32.  Rows behind the last are zeros.
template <typename T, int HD>
SJD_D void prompt_load_q(const PromptArgs &a, const PromptTile &s, int kvh, int first, int lane, u32x4 (&q)[HD * sizeof(T) / 32]) {
    const int rho = first + (lane & 31), i = rho / a.G, g = rho - i * a.G;
    const bool live = i < s.n;
    constexpr int PIECE = 16 / sizeof(T);
    const T *src = (const T *)a.q + (size_t)(s.r0 + (live ? i : 0)) * a.q_stride + (size_t)(kvh * a.G + (live ? g : 0)) * HD;
#pragma unroll
    for (int n = 0; n < (int)(HD * sizeof(T) / 32); ++n) {
        const T *p = src + (n * 2 + (lane >> 5)) * PIECE;
        u32x4 x = {0u, 0u, 0u, 0u};
        if (live) {
            if (a.q_wide) x = *reinterpret_cast<const u32x4 *>(p);
            else if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = __builtin_bit_cast(uint32_t, p[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = p[2 * e] | (uint32_t)p[2 * e + 1] << 16;
            }
        }
        q[n] = x;
    }
}

typedef __attribute__((address_space(3))) void prompt_lds_t;
typedef const __attribute__((address_space(1))) void prompt_glb_t;
typedef short prompt_s16x4 __attribute__((ext_vector_type(4)));

// 16 bytes of each lane, `off` from base, to LDS, the lanes' one behind the other.  In the compiler's own form every read of what it cannot tell from the target would wait for the load, the reads
// of another buffer of the same array among them; here prompt_barrier is what waits.  M0 is named as written, so that the compiler sets it again where it needs it behind this (it warns that it
// does not keep a reserved register, which is what is meant).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
SJD_D void prompt_to_lds(const char *base, uint32_t off, unsigned char *lds) {
    const uint32_t to = (uint32_t)(uintptr_t)(prompt_lds_t *)lds;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// Keys or values of a block on their way to LDS.  WIDE: rows are 16-byte aligned and go there without passing through registers.  (Element by element, rows of one element more: 8 192 rows of 16 heads of 64,
// 128 and 256 in bf16 168 -> 225, 282 -> 418, 477 -> 661 us, 2 048 in fp32 108 -> 113, 198 -> 213, 441 -> 622.)  Tokens behind the last are
// copies of the last one: nobody sees them.
template <typename T, int HD, bool WIDE> struct PromptFetch {
    static constexpr int BLOCK = prompt_block(sizeof(T), HD), ROW = HD * sizeof(T), PIECES = BLOCK * ROW / 16, THREADS = kPromptWaves * 64, PER = PIECES / THREADS;
    static_assert(PIECES % THREADS == 0, "a block divides among the threads");
    // Pieces of a lane whose tokens are a multiple of 16 apart have the same places in their rows
    static constexpr int TOKENS = THREADS * 16 / ROW, DIFFERENT = THREADS * 16 % ROW == 0 && TOKENS % 16 == 0 ? 1 : PER;
    uint32_t at[DIFFERENT];    // bytes from the block's first token
    SJD_D static int token(int i, int wave, int lane) { return ((i * kPromptWaves + wave) * 64 + lane) / (ROW / 16); }
    SJD_D static int piece(int i, int wave, int lane) {
        const int n = (i * kPromptWaves + wave) * 64 + lane;
        return prompt_swizzle(n / (ROW / 16), n % (ROW / 16), ROW);
    }
    SJD_D PromptFetch(long stride, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < DIFFERENT; ++i) at[i] = (uint32_t)token(i, wave, lane) * (uint32_t)(stride * sizeof(T)) + piece(i, wave, lane) * 16;
    }
    SJD_D void run(const T *base, long stride, int t0, int n_keys, unsigned char *lds, int wave, int lane) const {
        const char *block = (const char *)base + (size_t)t0 * stride * sizeof(T);
        unsigned char *to = lds + wave * 1024;
        if (WIDE && t0 + BLOCK <= n_keys) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                prompt_to_lds(block + (DIFFERENT == 1 ? i * TOKENS * stride * (long)sizeof(T) : 0), at[DIFFERENT == 1 ? 0 : i], to + i * THREADS * 16);
            return;
        }
        asm volatile("" : "+v"(lane));       // (rare: nothing of it is kept in registers from block to block)
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t t = (uint32_t)min(token(i, wave, lane), n_keys - 1 - t0);
            if constexpr (WIDE) prompt_to_lds(block, t * (uint32_t)(stride * sizeof(T)) + piece(i, wave, lane) * 16, to + i * THREADS * 16);
            else {
                const T *e = (const T *)(block + t * (size_t)(stride * sizeof(T)) + piece(i, wave, lane) * 16);
                u32x4 x;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    if constexpr (sizeof(T) == 4) x[d] = __builtin_bit_cast(uint32_t, e[d]);
                    else x[d] = e[2 * d] | (uint32_t)e[2 * d + 1] << 16;
                }
                *reinterpret_cast<u32x4 *>(to + i * THREADS * 16 + lane * 16) = x;
            }
        }
    }
};

// What every thread has asked for is in LDS, and what was there has been read.  (A barrier by itself does not wait for loads to LDS.)
SJD_D void prompt_barrier() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Operands of the bf16 products in a block in LDS: places of a lane's 16 bytes of keys (rows of the operand = 32 keys, 16 dimensions at a time), and of the 8 bytes that it fetches for
// values (rows = dimensions 32 db + lane % 32; of 16 keys 16 i, the element e is key 16 i + 8 (e / 4) + 4 (lane / 32) + e % 4, as the scores have them).  Those come from the rows by the
// transposing loads: 16 lanes fetch 16 dimensions of 4 keys, and each gets the 4 keys of one.
template <int HD> struct PromptPlaces {
    static constexpr int ROW = HD * 2, AGAIN = ROW % 128 == 64 ? 64 : ROW % 256 == 128 ? 128 : 256, NK = AGAIN / 32, NV = AGAIN / 64;    // (places repeat after so many bytes)
    // Places within these differ from the first by an exclusive or of what their pieces differ in: where registers are short only the first is kept.
    static constexpr int KK = prompt_block(2, HD) == 32 ? 1 : NK, KV = prompt_block(2, HD) == 32 ? 1 : NV;
    int k[KK], v[2][KV];
    SJD_D explicit PromptPlaces(int lane) {
#pragma unroll
        for (int n = 0; n < KK; ++n) {
            k[n] = (lane & 31) * ROW + prompt_swizzle(lane & 31, 2 * n + (lane >> 5), ROW) * 16;
            asm volatile("" : "+v"(k[n]));       // (once: the compiler would keep them for each buffer)
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int db = 0; db < KV; ++db) {
                const int t = 8 * r + 4 * (lane >> 5) + ((lane >> 2) & 3), j = 32 * db + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
                v[r][db] = t * ROW + prompt_swizzle(t, j >> 3, ROW) * 16 + (j & 4) * 2;
                asm volatile("" : "+v"(v[r][db]));
            }
    }
    SJD_D void move(int bytes) {
#pragma unroll
        for (int n = 0; n < KK; ++n) k[n] += bytes;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int db = 0; db < KV; ++db) v[r][db] += bytes;
    }
    SJD_D u32x4 keys(const unsigned char *block, int half, int n) const {
        const int at = KK == 1 ? k[0] ^ n % NK * 32 : k[n % NK];
        return *reinterpret_cast<const u32x4 *>(block + at + n / NK * AGAIN + half * 32 * ROW);
    }
    SJD_D u32x4 values(const unsigned char *block, int i, int db) const {
        typedef __attribute__((address_space(3))) prompt_s16x4 lds4;
        u32x4 x;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int at = KV == 1 ? v[r][0] ^ db % NV * 64 : v[r][db % NV];
            const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(block + at + db / NV * AGAIN + 16 * i * ROW)));
            x[2 * r] = y.x;
            x[2 * r + 1] = y.y;
        }
        return x;
    }
};
// The same for fp32: a lane's 16 bytes of keys, and its value of token 8 (e / 4) + 4 (lane / 32) + e % 4.  All places differ from the first by an exclusive or and an offset.
template <int HD> struct PromptPlaces32 {
    static constexpr int ROW = HD * 4, AGAIN = ROW % 256 == 128 ? 128 : 256;
    int k, v;
    SJD_D explicit PromptPlaces32(int lane) {
        k = (lane & 31) * ROW + prompt_swizzle(lane & 31, lane >> 5, ROW) * 16;
        v = 4 * (lane >> 5) * ROW + prompt_swizzle(4 * (lane >> 5), (lane >> 2) & 7, ROW) * 16 + (lane & 3) * 4;
        asm volatile("" : "+v"(k), "+v"(v));
    }
    SJD_D void move(int bytes) { k += bytes; v += bytes; }
    SJD_D u32x4 keys(const unsigned char *block, int n) const { return *reinterpret_cast<const u32x4 *>(block + (k ^ n * 32 % AGAIN) + n * 32 / AGAIN * AGAIN); }
    SJD_D float value(const unsigned char *block, int e, int db) const {
        const int t = 8 * (e >> 2) + (e & 3);        // (its swizzle and that of 4 (lane / 32) have no bit in common)
        return *reinterpret_cast<const float *>(block + (v ^ prompt_swizzle(t, 0, ROW) * 16 ^ db * 128 % AGAIN) + t * ROW + db * 128 / AGAIN * AGAIN);
    }
};

// The running state of 32 rows: O^T, reference of the exponentials (base 2), this lane's half of the sums
template <int HD> struct PromptState {
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
// Probabilities are 2^(score - m).  A rescaling puts m 8 above the row's maximum, a whole number (it is exact), and the next one comes when the maximum has grown
// beyond m (bf16: also when a lane's probabilities of a block, that far from the reference, add up to more than 1): until then the largest probability is between 2^-9 and 1, so rescalings are rare,
// and no sum of products with finite values overflows that does not in the formula.
// It moves m wherever 8 above the block's maximum is higher: where it did not, a row of many scores between m - 5 and m was weighed twice in every block (8 192 rows of 16 heads of 128 over keys of which
// all but the first 32 score 5 above those: 348 us, 227 now, 225 where all score the same).
// From magnitudes of 2^24 on m, a float, may be far off the maximum, whose exponent is exact (score * scale_log2e, in one instruction with the difference).  There m is the next float at or below it, and exponents
// above 0, which are smaller than a rounding of the scores, are 0: the largest score has the weight 1, those of its rounding too, and whatever is below it less.
constexpr float kPromptAhead = 8.0f, kPromptFar = 0x1p24f;
template <int HD> SJD_D void prompt_rescale(PromptState<HD> &st, float score, float scale_log2e) {
    const float mx = score * scale_log2e;
    float ahead = __builtin_ceilf(mx) + kPromptAhead;
    if (fabsf(mx) >= kPromptFar) ahead = fmaf(score, scale_log2e, -mx) < 0.0f ? __builtin_bit_cast(float, __builtin_bit_cast(int, mx) + (mx < 0.0f ? 1 : -1)) : mx;
    const float m = ahead > st.m ? ahead : st.m;
    const float alpha = __builtin_amdgcn_exp2f(st.m - (m == -INFINITY ? 0.0f : m));     // (not (-inf) - (-inf))
    st.m = m;
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < HD / 32; ++db) {
#pragma unroll
        for (int v = 0; v < 16; ++v) st.o[db][v] *= alpha;
        __builtin_amdgcn_sched_barrier(0);
    }
}

// An exponent after a rescaling: at most 0 (NaN stays)
SJD_D float prompt_exponent(float score, float scale_log2e, float m) { return __builtin_elementwise_minimum(fmaf(score, scale_log2e, -m), 0.0f); }

// the larger of a lane's and its partner's in the other half
SJD_D float prompt_both_halves(float x) {
    const auto y = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (int)y[0]), __builtin_bit_cast(float, (int)y[1]));
}
// sum + the two bf16 numbers of a pair
SJD_D float prompt_add_pair(float sum, uint32_t pair) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(cache_bf16x2, pair), __builtin_bit_cast(cache_bf16x2, 0x3F803F80u), sum, false);
}

// is a value infinite or NaN
SJD_D bool prompt_wild(float x) { return !finite_f(x); }
// two bf16 numbers: infinite ones and NaN become 0, and are noted
SJD_D uint32_t prompt_tame2(uint32_t u, bool &wild) {
    const bool lo = (u & 0x7F80u) == 0x7F80u, hi = (u & 0x7F800000u) == 0x7F800000u;
    wild |= lo | hi;
    return u & ((lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u));
}
// Values that are infinite or NaN, of units that not every row sees: in O += V P their 0 * inf would reach rows that do not see them, so there they are
// taken as 0, and added here, behind the last block, to the rows that do: p * inf is inf.  (Rare: token by token, from memory.)  Tokens [from, to); `sees`: the last one that the lane's row sees.
template <typename T, int HD> SJD_D void prompt_add_wild(PromptState<HD> &st, const T *v, long stride, int from, int to, int sees, int lane) {
#pragma unroll 1
    for (int t = from; t < to; ++t)
#pragma unroll
        for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float x = to_float<T>(v[t * stride + 32 * db + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)]);
                if (t <= sees && prompt_wild(x)) st.o[db][e] += x;
            }
}

// N matrix products with M other pieces of work spread between them, in this order
template <int N, int M, typename A, typename B> SJD_D void prompt_spread(A product, B other) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        product(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = i * M / N; j < (i + 1) * M / N; ++j) other(j);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// A wavefront of the fp32 kernel: 32 rows, a block of 32 keys at a time.
template <int HD> struct PromptWave32 {
    // keys: 4 products from 16 bytes; values: one from 4.  Those that are loaded before their products begin
    static constexpr int NK = HD / 8, DB = HD / 32, NV = 16 * DB, AHEAD_K = 2, AHEAD_V = 8;
    PromptState<HD> st;
    u32x4 q[NK], k[2 * AHEAD_K];
    float v[2 * AHEAD_V];
    f32x16 s;
    bool wild = false;                                // values of blocks that were masked were infinite or NaN
    PromptPlaces32<HD> at;
    SJD_D explicit PromptWave32(int lane) : at(lane) { st.clear(); }
    // last: of the block's keys, the last one that the lane's row sees; masked: some row may not see all of them
    SJD_D void block(const unsigned char *keys, const unsigned char *values, int last, bool masked, float scale_log2e, int lane) {
        auto load_k = [&](int n) { k[n % (2 * AHEAD_K)] = at.keys(keys, n); };
        auto score = [&](int n) {
            const uint32_t ke = k[n / 4 % (2 * AHEAD_K)][n % 4], qe = q[n / 4][n % 4];
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, ke), __builtin_bit_cast(float, qe), s, 0, 0, 0);
        };
        auto load_v = [&](int n) { v[n % (2 * AHEAD_V)] = at.value(values, n / DB, n % DB); };
        auto product = [&](int n) { st.o[n % DB] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[n % (2 * AHEAD_V)], s[n / DB], st.o[n % DB], 0, 0, 0); };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < AHEAD_K; ++n) load_k(n);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.0f;
        prompt_spread<4 * (NK - AHEAD_K), NK - AHEAD_K>([&](int n) { score(n); }, [&](int n) { load_k(n + AHEAD_K); });
        prompt_spread<4 * AHEAD_K, 0>([&](int n) { score(4 * (NK - AHEAD_K) + n); }, [&](int) {});
#pragma unroll
        for (int n = 0; n < AHEAD_V; ++n) load_v(n);
        if (masked) {
            const int mine = last - 4 * (lane >> 5);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = 8 * (e >> 2) + (e & 3) <= mine ? s[e] : -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
        mx = prompt_both_halves(mx);
        if (__ballot(mx * scale_log2e > st.m)) prompt_rescale<HD>(st, mx, scale_log2e);
        const float m = st.m == -INFINITY ? 0.0f : st.m;        // a row that has seen nothing so far: not (-inf) - (-inf)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[e] = __builtin_amdgcn_exp2f(prompt_exponent(s[e], scale_log2e, m));
            st.l += s[e];
        }
#pragma unroll
        for (int n = 0; n < NV; n += AHEAD_V) {
            if (masked)
#pragma unroll
                for (int i = 0; i < AHEAD_V; ++i) {
                    float &x = v[(n + i) % (2 * AHEAD_V)];
                    if (prompt_wild(x)) { wild = true; x = 0.0f; }
                }
            if (n + AHEAD_V < NV) prompt_spread<AHEAD_V, AHEAD_V>([&](int i) { product(n + i); }, [&](int i) { load_v(n + i + AHEAD_V); });
            else prompt_spread<AHEAD_V, 0>([&](int i) { product(n + i); }, [&](int) {});
        }
    }
};

// What becomes of 32 rows (first: the first of them; node: the lane's row of the sequence): results, or parts of them
template <typename T, int HD>
SJD_D void prompt_finish(const PromptArgs &a, const PromptTile &s, const PromptState<HD> &st, int kvh, bool several, size_t slot, int first, int node, int lane) {
    if (first >= (long)s.n * a.G) return;
    const float sum = st.l + __shfl_xor(st.l, 32, 64);
    if (several) {
        if (lane < 32) {
            a.part_ml[slot * 64 + lane] = st.m;
            a.part_ml[slot * 64 + 32 + lane] = sum;
        }
        if (node >= s.n) return;
        float *part = a.part_o + slot * 32 * HD + prompt_part_index(lane & 31, 4 * (lane >> 5));
#pragma unroll
        for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                *reinterpret_cast<f32x4 *>(part + prompt_part_index(0, db * 32 + 8 * u)) = f32x4{st.o[db][4 * u], st.o[db][4 * u + 1], st.o[db][4 * u + 2], st.o[db][4 * u + 3]};
        return;
    }
    // (it is NaN, and so is the row, where a score is; it is 0 where the row saw nothing, and so is the output)
    const float norm = sum == 0.0f ? 0.0f : 1.0f / sum;
    const size_t row = (size_t)s.r0 + node;
    const int h = kvh * a.G + first + (lane & 31) - node * a.G;
    if (sizeof(T) == 4 || !a.out_wide) {
        if (node >= s.n) return;
#pragma unroll
        for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                prompt_store<T>(a, row, h, HD, db * 32 + 8 * u + 4 * (lane >> 5), f32x4{st.o[db][4 * u], st.o[db][4 * u + 1], st.o[db][4 * u + 2], st.o[db][4 * u + 3]} * norm);
        return;
    }
    // a lane holds 4 of 8 dimensions, and stores all 8 of one half of them
    const bool live = node < s.n;
    bf16_t *out = (bf16_t *)a.out + (live ? row * a.out_stride + (size_t)h * HD : 0) + 8 * (lane >> 5);
#pragma unroll
    for (int db = 0; db < HD / 32; ++db)
#pragma unroll
        for (int u = 0; u < 4; u += 2) {
            u32x4 x;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const auto y = __builtin_amdgcn_permlane32_swap(pack_bf16(st.o[db][4 * u + 2 * e] * norm, st.o[db][4 * u + 2 * e + 1] * norm),
                                                                pack_bf16(st.o[db][4 * u + 4 + 2 * e] * norm, st.o[db][4 * u + 4 + 2 * e + 1] * norm), false, false);
                x[e] = y[0];
                x[2 + e] = y[1];
            }
            if (live) *reinterpret_cast<u32x4 *>(out + db * 32 + 8 * u) = x;
        }
}

// A wavefront of the bf16 kernel: 32 rows, a block of keys at a time, 32 (HALVES: 1) or 64 (2).
template <int HD> struct PromptWave16 {
    static constexpr int NQ = HD / 16, DB = HD / 32, HALVES = prompt_block(2, HD) / 32, NK = HALVES * NQ, NV = HALVES * 2 * DB;
    // Operands of keys and values that are loaded before their products begin, and those held: the others replace those that have been used
    static constexpr int AHEAD = HALVES == 2 ? NQ : 4, HELD = 2 * AHEAD;
    static_assert(NQ == 2 * DB && NK % AHEAD == 0, "as many for keys as for values");
    PromptState<HD> st;
    u32x4 q[NQ], k[HELD], v[HELD], p[HALVES][2];      // operands: queries, keys, values, probabilities
    f32x16 s[HALVES];
    float m, sum, e0, e1;
    float unset;                                      // NaN as long as m is nothing yet, of a row that sees something; else 0
    bool wild = false;                                // values of blocks that were masked were infinite or NaN
    PromptPlaces<HD> at;
    SJD_D explicit PromptWave16(int lane) : at(lane) { st.clear(); m = 0.0f; }
    SJD_D void begin(bool sees) { unset = sees ? NAN : 0.0f; }
    SJD_D void load_k(const unsigned char *block, int n) { k[n % HELD] = at.keys(block, n / NQ, n % NQ); }
    SJD_D void load_v(const unsigned char *block, int n) { v[n % HELD] = at.values(block, n / DB, n % DB); }
    SJD_D void score(int n) {
        if (n % NQ == 0)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[n / NQ][e] = 0.0f;
        s[n / NQ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[n % HELD]), __builtin_bit_cast(bf16x8, q[n % NQ]), s[n / NQ], 0, 0, 0);
    }
    // last: of the block's keys, the last one that the lane's row sees
    SJD_D void mask(int last) {
        const int mine = last - 4 * (int)((threadIdx.x >> 5) & 1);
#pragma unroll
        for (int i = 0; i < HALVES; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] = 32 * i + 8 * (e >> 2) + (e & 3) <= mine ? s[i][e] : -INFINITY;
    }
    // Probabilities are 2^(score - m).  As long as a lane's of a block add up to at most 1 none is above 1, and m stays; else, and until there is a score above -inf, it is put ahead of the largest score.
    SJD_D void settle(float scale_log2e) {
        float mx = s[0][0];
#pragma unroll
        for (int i = 0; i < HALVES; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[i][e]);
        prompt_rescale<HD>(st, prompt_both_halves(mx), scale_log2e);
        m = st.m == -INFINITY ? 0.0f : st.m;           // a row that has seen nothing: not (-inf) - (-inf)
        unset = st.m == -INFINITY ? unset : 0.0f;
    }
    // probabilities 2 n and 2 n + 1; those of n - 1 as operands.  What the products take is what the sum adds, so that a row's weights add up to 1 whatever their rounding to bf16 (a row
    // that sees one key gives its value, exactly).  SETTLED: after a rescaling.
    template <bool SETTLED, int I> SJD_D void weigh(int n, float scale_log2e) {
        if (n > 0) {
            const uint32_t both = pack_bf16(e0, e1);
            p[I][(n - 1) / 4][(n - 1) % 4] = both;
            sum = prompt_add_pair(sum, both);
        }
        if (n < 8) {
            auto exponent = [&](float x) { return SETTLED ? prompt_exponent(x, scale_log2e, m) : fmaf(x, scale_log2e, -m); };
            e0 = __builtin_amdgcn_exp2f(exponent(s[I][2 * n]));
            e1 = __builtin_amdgcn_exp2f(exponent(s[I][2 * n + 1]));
        }
    }
    template <bool SETTLED> SJD_D void weigh_all(float scale_log2e, float from) {
        sum = from;
#pragma unroll
        for (int n = 0; n < 9; ++n) weigh<SETTLED, 0>(n, scale_log2e);
        if constexpr (HALVES == 2)
#pragma unroll
            for (int n = 0; n < 9; ++n) weigh<SETTLED, 1>(n, scale_log2e);
    }
    SJD_D void product(int n) {
        st.o[n % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[n % HELD]), __builtin_bit_cast(bf16x8, p[n / (2 * DB)][n / DB % 2]), st.o[n % DB], 0, 0, 0);
    }
    // Are there values in N operands that are infinite or NaN (0 times them is NaN)?  They become 0.
    template <int N> static SJD_D bool tame(u32x4 *x) {
        float sum = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const uint32_t w = x[n][d];
                sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(cache_bf16x2, w), __builtin_bit_cast(cache_bf16x2, 0u), sum, false);
            }
        const bool found = __ballot(sum != 0.0f);
        if (found) {
            bool any = false;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int d = 0; d < 4; ++d) x[n][d] = prompt_tame2(x[n][d], any);
        }
        return found;
    }
    // Who has products goes first (8 192 rows of 16 heads of 192 and 256 1 089 and 1 158 TFLOP/s, 1 022 and 1 048 without; of 128 the same; of 64 and 96 785 and 964, 808 and 978 without).
    template <int P> static SJD_D void priority() {
        if constexpr (HALVES == 1) __builtin_amdgcn_s_setprio(P);
    }
    // A block.  last: of its keys, the last one that the lane's row sees; masked: some row may not see all of it.
    SJD_D void block(const unsigned char *keys, const unsigned char *values, int last, bool masked, float scale_log2e) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) load_k(keys, n);
        priority<1>();
        prompt_spread<NK - AHEAD, NK - AHEAD>([&](int n) { score(n); }, [&](int n) { load_k(keys, n + AHEAD); });
        prompt_spread<AHEAD, 0>([&](int n) { score(NK - AHEAD + n); }, [&](int) {});
        priority<0>();
        if (masked) mask(last);
        weigh_all<false>(scale_log2e, unset);
        if (__ballot(!(sum <= 1.0f))) {
            settle(scale_log2e);
            weigh_all<true>(scale_log2e, 0.0f);
        }
        st.l += sum;
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) load_v(values, n);
#pragma unroll
        for (int n = 0; n < NV; n += AHEAD) {           // (those of a masked block are looked at while the next ones are not yet there)
            if (masked) wild |= tame<AHEAD>(v + n % HELD);
            priority<1>();
            if (n + AHEAD < NV) prompt_spread<AHEAD, AHEAD>([&](int i) { product(n + i); }, [&](int i) { load_v(values, n + i + AHEAD); });
            else prompt_spread<AHEAD, 0>([&](int i) { product(n + i); }, [&](int) {});
        }
        priority<0>();
    }
};

// Workgroup = four wavefronts of 32 rows each, of a split.
template <int HD, bool WIDE>
__global__ __launch_bounds__(kPromptWaves * 64, prompt_waves_per_simd(2, HD)) void prompt_attention16_kernel(PromptArgs a) {
    constexpr int BLOCK = prompt_block(2, HD), BYTES = BLOCK * HD * 2, ROWS = kPromptWaves * 32;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * BYTES];      // keys and values of a block, and of the next one
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kvh = blockIdx.x % a.n_kv, tile = blockIdx.x / a.n_kv % a.tiles, split = blockIdx.x / a.n_kv / a.tiles;
    const PromptTile s = prompt_find_tile(a, ROWS, tile);
    if (s.b < 0) return;
    const PromptBlocks range = prompt_blocks(prompt_keys(s.t, s.n, s.n_keys, a.G, ROWS), BLOCK, split, a.n_splits, a.per_split);
    if (!range.any) return;
    const bf16_t *k = (const bf16_t *)a.k + (size_t)s.k0 * a.k_stride + (size_t)kvh * HD, *v = (const bf16_t *)a.v + (size_t)s.k0 * a.v_stride + (size_t)kvh * HD;
    PromptWave16<HD> w(lane);
    const int row0 = s.t * ROWS + wave * 32, offset = prompt_offset(s.n, s.n_keys), node = (row0 + (lane & 31)) / a.G;
    prompt_load_q<bf16_t, HD>(a, s, kvh, row0, lane, w.q);
    // last key that the lane's row sees; the least such key of the wavefront's rows, and the blocks that one of them sees something of
    const int sees = node < s.n ? node + offset : -1, low = __builtin_amdgcn_readfirstlane(row0 / a.G + offset);
    const int mine = row0 / a.G < s.n ? __builtin_amdgcn_readfirstlane(min(range.last, (min((row0 + 31) / a.G, s.n - 1) + offset + BLOCK) / BLOCK)) : 0;
    const PromptFetch<bf16_t, HD, WIDE> fetch_k(a.k_stride, wave, lane), fetch_v(a.v_stride, wave, lane);
    auto get_k = [&](int blk, unsigned char *to) {
        if (blk < range.last) fetch_k.run(k, a.k_stride, blk * BLOCK, s.n_keys, to, wave, lane);
    };
    auto get_v = [&](int blk, unsigned char *to) {
        if (blk < range.last) fetch_v.run(v, a.v_stride, blk * BLOCK, s.n_keys, to, wave, lane);
    };
    int blk = range.first, buf = 0;
    get_k(blk, lds);
    get_v(blk, lds + BYTES);
    auto turn = [&]() {
        prompt_barrier();     // this block is there, and everybody is done with the last one
        buf = 2 * BYTES - buf;
        get_k(blk + 1, lds + buf);
        get_v(blk + 1, lds + buf + BYTES);
    };
    // (queries: waited for here; at their first use, in the loop, it would be a wait for everything, every time)
#pragma unroll
    for (int n = 0; n < HD / 16; ++n) asm volatile("" : "+v"(w.q[n]));
    w.begin(sees >= blk * BLOCK);
    for (; blk < mine; ++blk) {
        turn();
        w.block(lds, lds + BYTES, sees - blk * BLOCK, blk * BLOCK + BLOCK - 1 > low, a.scale_log2e);
        w.at.move(buf ? 2 * BYTES : -2 * BYTES);
    }
    // what is left the other wavefronts see: this one helps to fetch (in a loop of its own: with a branch around the block above the output would be copied every time)
    for (; blk < range.last; ++blk) turn();
    if (w.wild) prompt_add_wild<bf16_t, HD>(w.st, v, a.v_stride, max(range.first, (low + 1) / BLOCK) * BLOCK, min(mine * BLOCK, s.n_keys), sees, lane);
    prompt_finish<bf16_t, HD>(a, s, w.st, kvh, range.several, prompt_slot(a, tile, kvh, split) * (ROWS / 32) + wave, row0, node, lane);
}

// fp32, the same.
template <int HD, bool WIDE>
__global__ __launch_bounds__(kPromptWaves * 64, prompt_waves_per_simd(4, HD)) void prompt_attention32_kernel(PromptArgs a) {
    constexpr int BLOCK = prompt_block(4, HD), BYTES = BLOCK * HD * 4, ROWS = kPromptWaves * 32;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kvh = blockIdx.x % a.n_kv, tile = blockIdx.x / a.n_kv % a.tiles, split = blockIdx.x / a.n_kv / a.tiles;
    const PromptTile s = prompt_find_tile(a, ROWS, tile);
    if (s.b < 0) return;
    const PromptBlocks range = prompt_blocks(prompt_keys(s.t, s.n, s.n_keys, a.G, ROWS), BLOCK, split, a.n_splits, a.per_split);
    if (!range.any) return;
    const float *k = (const float *)a.k + (size_t)s.k0 * a.k_stride + (size_t)kvh * HD, *v = (const float *)a.v + (size_t)s.k0 * a.v_stride + (size_t)kvh * HD;
    const int row0 = s.t * ROWS + wave * 32, offset = prompt_offset(s.n, s.n_keys), node = (row0 + (lane & 31)) / a.G;
    PromptWave32<HD> w(lane);
    prompt_load_q<float, HD>(a, s, kvh, row0, lane, w.q);
    const int sees = node < s.n ? node + offset : -1, low = __builtin_amdgcn_readfirstlane(row0 / a.G + offset);
    const int mine = row0 / a.G < s.n ? __builtin_amdgcn_readfirstlane(min(range.last, (min((row0 + 31) / a.G, s.n - 1) + offset + BLOCK) / BLOCK)) : 0;
    const PromptFetch<float, HD, WIDE> fetch_k(a.k_stride, wave, lane), fetch_v(a.v_stride, wave, lane);
    auto fetch = [&](int blk, unsigned char *to) {
        if (blk >= range.last) return;
        fetch_k.run(k, a.k_stride, blk * BLOCK, s.n_keys, to, wave, lane);
        fetch_v.run(v, a.v_stride, blk * BLOCK, s.n_keys, to + BYTES, wave, lane);
    };
    int blk = range.first, buf = 0;
    fetch(blk, lds);
    auto turn = [&]() {
        prompt_barrier();     // this block is there, and everybody is done with the last one
        buf = 2 * BYTES - buf;
        fetch(blk + 1, lds + buf);
    };
#pragma unroll
    for (int n = 0; n < HD / 8; ++n) asm volatile("" : "+v"(w.q[n]));        // (as above)
    for (; blk < mine; ++blk) {
        turn();
        w.block(lds, lds + BYTES, sees - blk * BLOCK, blk * BLOCK + BLOCK - 1 > low, a.scale_log2e, lane);
        w.at.move(buf ? 2 * BYTES : -2 * BYTES);
    }
    for (; blk < range.last; ++blk) turn();
    if (__ballot(w.wild)) prompt_add_wild<float, HD>(w.st, v, a.v_stride, max(range.first, (low + 1) / BLOCK) * BLOCK, min(mine * BLOCK, s.n_keys), sees, lane);
    prompt_finish<float, HD>(a, s, w.st, kvh, range.several, prompt_slot(a, tile, kvh, split) * (ROWS / 32) + wave, row0, node, lane);
}

// Joins the splits of every row that has several: out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  A thread owns four dimensions of a row, of every WAYS-th few splits, which are on their
// way together; WAYS wavefronts share a row.  Where a split saw nothing of a row l = 0.
// CAREFUL: infinities stay what they are when their weight is 0 (a result that is NaN without is computed once more so).
struct PromptJoin { float m, denom; f32x4 t; };
template <bool CAREFUL> SJD_D f32x4 prompt_weighted(f32x4 t, float w) {
    if constexpr (!CAREFUL) return t * w;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = finite_f(t[e]) ? t[e] * w : t[e];
    return t;
}
// a and b, about the larger reference
template <bool CAREFUL> SJD_D PromptJoin prompt_join(PromptJoin a, PromptJoin b) {
    const float m = fmaxf(a.m, b.m), m_use = m == -INFINITY ? 0.0f : m, x = __builtin_amdgcn_exp2f(a.m - m_use), y = __builtin_amdgcn_exp2f(b.m - m_use);
    return {m, a.denom * x + b.denom * y, prompt_weighted<CAREFUL>(a.t, x) + prompt_weighted<CAREFUL>(b.t, y)};
}
template <typename T, int HD, int WAYS>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a) {
    constexpr int ROWS = kPromptWaves * 32, QUADS = ROWS * (HD / 4), EACH = 256 / WAYS, WGS = QUADS / EACH, N = WAYS == 1 ? 8 : 4;
    __shared__ PromptJoin other[WAYS][EACH];
    const int part = blockIdx.x % WGS, kvh = blockIdx.x / WGS % a.n_kv, tile = blockIdx.x / WGS / a.n_kv;
    const PromptTile s = prompt_find_tile(a, ROWS, tile);
    if (s.b < 0) return;
    const int splits = prompt_splits(prompt_keys(s.t, s.n, s.n_keys, a.G, ROWS), prompt_block(sizeof(T), HD), a.n_splits, a.per_split);
    const int u = part * EACH + threadIdx.x % EACH, way = threadIdx.x / EACH, row = u & 31, j = (u >> 5) % (HD / 4) * 4, sub = (u >> 5) / (HD / 4);
    const int rho = s.t * ROWS + sub * 32 + row, node = rho / a.G;
    if (splits == 1) return;
    auto sum = [&](auto careful) {
        PromptJoin x{-INFINITY, 0.0f, {0.0f, 0.0f, 0.0f, 0.0f}};
        for (int i0 = way * N; i0 < splits && node < s.n; i0 += WAYS * N) {
            PromptJoin y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const size_t slot = prompt_slot(a, tile, kvh, min(i0 + i, splits - 1)) * (ROWS / 32) + sub;
                y[i].m = a.part_ml[slot * 64 + row];
                y[i].denom = i0 + i < splits ? a.part_ml[slot * 64 + 32 + row] : 0.0f;
                y[i].t = *reinterpret_cast<const f32x4 *>(a.part_o + slot * 32 * HD + prompt_part_index(row, j));
            }
            float m = x.m;
#pragma unroll
            for (int i = 0; i < N; ++i) m = fmaxf(m, y[i].m);
            const float m_use = m == -INFINITY ? 0.0f : m, alpha = __builtin_amdgcn_exp2f(x.m - m_use);
            x.m = m;
            x.denom *= alpha;
            x.t = prompt_weighted<decltype(careful)::value>(x.t, alpha);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float w = y[i].denom == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(y[i].m - m_use);
                x.denom += w * y[i].denom;
                x.t += prompt_weighted<decltype(careful)::value>(y[i].t, w);
            }
        }
        return x;
    };
    PromptJoin x = sum(std::false_type());
    if (__ballot(!(x.t[0] + x.t[1] + x.t[2] + x.t[3] == x.t[0] + x.t[1] + x.t[2] + x.t[3]))) x = sum(std::true_type());
    if constexpr (WAYS > 1) {
        if (way) other[way][threadIdx.x % EACH] = x;
        __syncthreads();
        if (way) return;
#pragma unroll
        for (int i = 1; i < WAYS; ++i) x = prompt_join<true>(x, other[i][threadIdx.x]);
    }
    if (node >= s.n) return;
    const float inv = x.denom == 0.0f ? 0.0f : 1.0f / x.denom;
#pragma unroll
    for (int e = 0; e < 4; ++e) x.t[e] = x.denom == 0.0f ? 0.0f : x.t[e] * inv;
    prompt_store<T>(a, (size_t)s.r0 + node, kvh * a.G + rho - node * a.G, HD, j, x.t);
}
