// Attention of packed prompts: causal, grouped heads, ragged sequences, keys and values as they come from a projection or from a cache that was read back.
//
// Rows (i, h) of one kv head of a sequence are cut into tiles (prompt_layout.h), so that the query heads of a group share keys and values.  Per block
// of keys a wavefront computes, for each of its tiles of 32 rows,
//   S^T (keys x rows) = K Q^T,   online softmax per row = per accumulator column,   O^T (dimensions x rows) += V^T P^T,
// and P^T needs no data movement: the accumulator registers of S^T are the B operand of the second product, if the keys of V^T are taken in their order.
// Keys and values go through LDS, straight from memory, for all wavefronts of a workgroup.
#pragma once
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
    bool q_wide, out_wide;     // rows 16-byte (out: 4 elements) aligned
};

constexpr int kPromptWaves = 4;
constexpr int prompt_waves_per_simd(int size, int hd) { return size * hd <= 256 ? 2 : 1; }
// tokens of a block
template <typename T> constexpr int kPromptBlock = sizeof(T) == 2 ? 64 : 32;

// A workgroup's tile: sequence (-1: there is none), tile of it, first row and number of rows, first key and number of keys
struct PromptTile { int b, t, r0, n, k0, n_keys; };
SJD_D PromptTile prompt_find_tile(const PromptArgs &a, int rows, int index) {
    const int lane = threadIdx.x & 63;
    long before = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
        const int b = s0 + lane;
        int r0 = 0, n = 0, k0 = 0, n_keys = 0;
        if (b < a.n_seqs) {
            r0 = k0 = rows_first(a.row_start, b, a.n_rows);
            n = n_keys = rows_count(a.row_start, b, a.n_rows);
            if (a.kv_start) {
                k0 = rows_first(a.kv_start, b, a.n_kv_rows);
                n_keys = rows_count(a.kv_start, b, a.n_kv_rows);
            }
        }
        const int tiles = prompt_tiles(n, a.G, rows);
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
        const unsigned long long mine = __ballot(before + upto > index);
        if (mine) {
            const int l = __ffsll((long long)mine) - 1;
            PromptTile f;
            f.b = s0 + l;
            f.t = (int)(index - before) - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(tiles, l));
            f.r0 = __builtin_amdgcn_readlane(r0, l);
            f.n = __builtin_amdgcn_readlane(n, l);
            f.k0 = __builtin_amdgcn_readlane(k0, l);
            f.n_keys = __builtin_amdgcn_readlane(n_keys, l);
            return f;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return PromptTile{-1, 0, 0, 0, 0, 0};
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

// Keys or values of a block on their way to LDS.  WIDE: rows are 16-byte aligned and go there without passing through registers.  Tokens behind the last are
// copies of the last one: nobody sees them.
template <typename T, int HD, bool WIDE> struct PromptFetch {
    static constexpr int BLOCK = kPromptBlock<T>, ROW = HD * sizeof(T), PIECES = BLOCK * ROW / 16, THREADS = kPromptWaves * 64, PER = PIECES / THREADS;
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
        const bool whole = t0 + BLOCK <= n_keys;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            unsigned char *to = lds + (i * kPromptWaves + wave) * 1024;
            if constexpr (WIDE) {
                const char *from = block + (DIFFERENT == 1 ? i * TOKENS * stride * (long)sizeof(T) : 0);
                uint32_t off = at[DIFFERENT == 1 ? 0 : i];
                if (!whole) {
                    const int t = min(token(i, wave, lane), n_keys - 1 - t0);
                    from = block;
                    off = (uint32_t)t * (uint32_t)(stride * sizeof(T)) + piece(i, wave, lane) * 16;
                }
                __builtin_amdgcn_global_load_lds((prompt_glb_t *)(from + off), (prompt_lds_t *)to, 16, 0, 0);
            } else {
                const T *p = base + (size_t)min(t0 + token(i, wave, lane), n_keys - 1) * stride + piece(i, wave, lane) * (16 / sizeof(T));
                u32x4 x;
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = __builtin_bit_cast(uint32_t, p[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = p[2 * e] | (uint32_t)p[2 * e + 1] << 16;
                }
                *reinterpret_cast<u32x4 *>(to + lane * 16) = x;
            }
        }
    }
};

// What every thread has asked for is in LDS, and read from there.  (A barrier by itself waits for neither: loads to LDS are not stores to it in the compiler's eyes.)
SJD_D void prompt_barrier() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// S^T of 32 keys (from token `sub` * 32 of the block) and 32 rows
template <typename T, int HD> SJD_D f32x16 prompt_scores(const unsigned char *k, int sub, const u32x4 (&q)[HD * sizeof(T) / 32], int lane) {
    f32x16 s;
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = 0.0f;
    constexpr int ROW = HD * sizeof(T);
    const int t = sub * 32 + (lane & 31);
#pragma unroll
    for (int n = 0; n < ROW / 32; ++n) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(k + t * ROW + prompt_swizzle(t, 2 * n + (lane >> 5), ROW) * 16);
        if constexpr (sizeof(T) == 2) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, q[n]), s, 0, 0, 0);
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t xe = x[e], qe = q[n][e];
                s = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, xe), __builtin_bit_cast(float, qe), s, 0, 0, 0);
            }
        }
    }
    return s;
}

// A operand of the second product, dimensions 32 db + lane % 32.  bf16: 16 tokens, 16 i + 8 (e / 4) + 4 (lane / 32) + e % 4 for its element e, read from
// their rows by the transposing loads (16 lanes fetch 16 dimensions of 4 tokens, and each gets the 4 tokens of one).
template <int HD> SJD_D u32x4 prompt_values16(const unsigned char *v, int i, int db, int lane) {
    constexpr int ROW = HD * 2;
    u32x4 x;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int t = 16 * i + 8 * r + 4 * (lane >> 5) + ((lane >> 2) & 3), j = 32 * db + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        typedef __attribute__((address_space(3))) prompt_s16x4 lds4;
        const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(v + t * ROW + prompt_swizzle(t, j >> 3, ROW) * 16 + (j & 4) * 2)));
        x[2 * r] = y.x;
        x[2 * r + 1] = y.y;
    }
    return x;
}
// fp32: a token, 8 (v / 4) + 4 (lane / 32) + v % 4
template <int HD> SJD_D float prompt_value32(const unsigned char *l, int v, int db, int lane) {
    constexpr int ROW = HD * 4;
    const int t = 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3), j = 32 * db + (lane & 31);
    return *reinterpret_cast<const float *>(l + t * ROW + prompt_swizzle(t, j >> 2, ROW) * 16 + (j & 3) * 4);
}

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
// beyond m: until then the largest probability is between 2^-9 and 1, so rescalings are rare, and no sum of products with finite values overflows that does not in
// the formula.
constexpr float kPromptAhead = 8.0f;
template <int HD> SJD_D void prompt_rescale(PromptState<HD> &st, float mx) {
    if (!__ballot(mx > st.m)) return;
    const float m = fmaxf(st.m, __builtin_ceilf(mx) + kPromptAhead);
    const float alpha = __builtin_amdgcn_exp2f(st.m - (m == -INFINITY ? 0.0f : m));     // (not (-inf) - (-inf))
    st.m = m;
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < HD / 32; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) st.o[db][v] *= alpha;
}

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
// Values that are infinite or NaN, of a block that not every row sees as a whole: in O += V P their 0 * inf would reach rows that do not see them, so there they are
// taken as 0, and added here to the rows that do: p * inf is inf.  (Rare: token by token.)  `last`: the last token of the block that the lane's row sees.
template <typename T, int HD> SJD_D void prompt_add_wild(PromptState<HD> &st, const unsigned char *v, int last, int lane) {
    constexpr int ROW = HD * sizeof(T);
#pragma unroll 1
    for (int t = 0; t < kPromptBlock<T>; ++t)
#pragma unroll
        for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                int at = t;
                asm volatile("" : "+v"(at));      // (an address at a time: kept ahead of the loop they would take the registers of the caller's)
                const int j = 32 * db + 8 * u + 4 * (lane >> 5);
                const T *p = reinterpret_cast<const T *>(v + at * ROW + prompt_swizzle(at, j * (int)sizeof(T) / 16, ROW) * 16 + (j * sizeof(T)) % 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = to_float<T>(p[e]);
                    if (t <= last && prompt_wild(x)) st.o[db][4 * u + e] += x;
                }
            }
}

// One block of 32 rows.  `last`: of the block's tokens, the last one that the lane's row sees.  MASKED: some row may not see all of them.
template <typename T, int HD, bool MASKED>
SJD_D void prompt_block(PromptState<HD> &st, const unsigned char *k, const unsigned char *v, const u32x4 (&q)[HD * sizeof(T) / 32], int last, float scale_log2e, int lane) {
    constexpr int SUB = kPromptBlock<T> / 32;
    f32x16 s[SUB];
    const int mine = last - 4 * (lane >> 5);
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
        s[u] = prompt_scores<T, HD>(k, u, q, lane);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            if (MASKED) s[u][e] = 32 * u + 8 * (e >> 2) + (e & 3) <= mine ? s[u][e] : -INFINITY;
            mx = fmaxf(mx, s[u][e]);
        }
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * scale_log2e;
    prompt_rescale<HD>(st, mx);
    const float m_use = st.m == -INFINITY ? 0.0f : st.m;    // a row that has seen nothing so far: not (-inf) - (-inf)
    float sum = 0.0f;
    bool wild = false;
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[u][e] = __builtin_amdgcn_exp2f(fmaf(s[u][e], scale_log2e, -m_use));
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sum += s[u][e];
#pragma unroll
                for (int db = 0; db < HD / 32; ++db) {
                    float x = prompt_value32<HD>(v, e, db, lane);
                    if (MASKED && prompt_wild(x)) { wild = true; x = 0.0f; }
                    st.o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[u][e], st.o[db], 0, 0, 0);
                }
            }
        } else {
            // What the products take is what the sum adds, so that a row's weights add up to 1 whatever their rounding to bf16 (a row that sees one token
            // gives its value, exactly); one instruction for two of them.
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                u32x4 p;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    p[d] = pack_bf16(s[u][8 * i + 2 * d], s[u][8 * i + 2 * d + 1]);
                    const uint32_t pd = p[d];
                    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(cache_bf16x2, pd), __builtin_bit_cast(cache_bf16x2, 0x3F803F80u), sum, false);
                }
#pragma unroll
                for (int db = 0; db < HD / 32; ++db) {
                    u32x4 x = prompt_values16<HD>(v, 2 * u + i, db, lane);
                    if (MASKED)
#pragma unroll
                        for (int d = 0; d < 4; ++d) x[d] = prompt_tame2(x[d], wild);
                    st.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, p), st.o[db], 0, 0, 0);
                }
            }
        }
    }
    st.l += sum;
    if (MASKED && __ballot(wild)) prompt_add_wild<T, HD>(st, v, last, lane);
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

// One block of 64 keys, of one or two tiles of 32 rows, bf16.  With two tiles the exponentials of one are spread between the matrix products of the other.  last[r]: of the
// block's tokens, the last one that the lane's row sees; masked: some row may not see all of them.
template <int HD, int RT>
SJD_D void prompt_block16(PromptState<HD> (&st)[RT], const unsigned char *k, const unsigned char *v, const u32x4 (&q)[RT][HD / 16], const int (&sees)[RT], int t0, bool masked, float scale_log2e,
                          int lane) {
    constexpr int NQ = HD / 16, DB = HD / 32;
    f32x16 s[RT][2];
    u32x4 kf[2][NQ], vf[2][2 * DB], p[RT][4];
    float m_use[RT], mx[RT];
    bool wild[2] = {false, false};
    const int t = lane & 31;
    auto load_k = [&](int u, int n) { kf[u][n] = *reinterpret_cast<const u32x4 *>(k + (32 * u + t) * HD * 2 + prompt_swizzle(t, 2 * n + (lane >> 5), HD * 2) * 16); };
    auto load_v = [&](int u, int n) { vf[u][n] = prompt_values16<HD>(v, 2 * u + n / DB, n % DB, lane); };
    auto score = [&](int r, int u, int n) {
        if (n == 0)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[r][u][e] = 0.0f;
        s[r][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[u][n]), __builtin_bit_cast(bf16x8, q[r][n]), s[r][u], 0, 0, 0);
    };
    auto mask = [&](int r) {
        const int mine = sees[r] - t0 - 4 * (lane >> 5);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[r][u][e] = 32 * u + 8 * (e >> 2) + (e & 3) <= mine ? s[r][u][e] : -INFINITY;
    };
    auto largest = [&](int r, int n) {       // n-th of 8
        if (n == 0) mx[r] = s[r][0][0];
#pragma unroll
        for (int e = 0; e < 4; ++e) mx[r] = fmaxf(mx[r], s[r][n >> 2][4 * (n & 3) + e]);
    };
    auto settle = [&](int r) {
        prompt_rescale<HD>(st[r], prompt_both_halves(mx[r]) * scale_log2e);
        m_use[r] = st[r].m == -INFINITY ? 0.0f : st[r].m;
    };
    // probabilities 2 n and 2 n + 1 of 32 keys; those of n - 1 as operands
    auto weigh = [&](int r, int u, int n) {
        if (n < 8) {
            s[r][u][2 * n] = __builtin_amdgcn_exp2f(fmaf(s[r][u][2 * n], scale_log2e, -m_use[r]));
            s[r][u][2 * n + 1] = __builtin_amdgcn_exp2f(fmaf(s[r][u][2 * n + 1], scale_log2e, -m_use[r]));
        }
        if (n > 0) {
            const uint32_t both = pack_bf16(s[r][u][2 * n - 2], s[r][u][2 * n - 1]);
            p[r][2 * u + (n - 1) / 4][(n - 1) % 4] = both;
            st[r].l = prompt_add_pair(st[r].l, both);
        }
    };
    auto product = [&](int r, int u, int n) {      // n-th of 2 DB
        st[r].o[n % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[u][n]), __builtin_bit_cast(bf16x8, p[r][2 * u + n / DB]), st[r].o[n % DB], 0, 0, 0);
    };
    // values that are infinite or NaN: 0 times them is NaN
    auto look = [&](int u) {
        float x = 0.0f;
#pragma unroll
        for (int n = 0; n < 2 * DB; ++n)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const uint32_t w = vf[u][n][d];
                x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(cache_bf16x2, w), __builtin_bit_cast(cache_bf16x2, 0u), x, false);
            }
        wild[u] = __ballot(x != 0.0f);
        if (wild[u]) {
            bool any = false;
#pragma unroll
            for (int n = 0; n < 2 * DB; ++n)
#pragma unroll
                for (int d = 0; d < 4; ++d) vf[u][n][d] = prompt_tame2(vf[u][n][d], any);
        }
    };
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < NQ; ++n) load_k(0, n);
    __builtin_amdgcn_s_setprio(1);
    prompt_spread<NQ, NQ>([&](int n) { score(0, 0, n); }, [&](int n) { load_k(1, n); });
    prompt_spread<NQ, 0>([&](int n) { score(0, 1, n); }, [&](int) {});
    __builtin_amdgcn_s_setprio(0);
    if (masked) mask(0);
    if constexpr (RT == 2) {
        prompt_spread<NQ, 8>([&](int n) { score(1, 0, n); }, [&](int n) { largest(0, n); });
        settle(0);
        prompt_spread<NQ, 9 + 2 * DB>([&](int n) { score(1, 1, n); }, [&](int n) { n < 9 ? weigh(0, 0, n) : load_v(0, n - 9); });
        if (masked) {
            mask(1);
            look(0);
        }
        prompt_spread<2 * DB, 17 + 2 * DB>([&](int n) { product(0, 0, n); }, [&](int n) { n < 9 ? weigh(0, 1, n) : n < 17 ? largest(1, n - 9) : load_v(1, n - 17); });
        settle(1);
        if (masked) look(1);
        prompt_spread<2 * DB, 9>([&](int n) { product(0, 1, n); }, [&](int n) { weigh(1, 0, n); });
        prompt_spread<2 * DB, 9>([&](int n) { product(1, 0, n); }, [&](int n) { weigh(1, 1, n); });
        prompt_spread<2 * DB, 0>([&](int n) { product(1, 1, n); }, [&](int) {});
    } else {
#pragma unroll
        for (int n = 0; n < 8; ++n) largest(0, n);
        settle(0);
#pragma unroll
        for (int n = 0; n < 2 * DB; ++n) load_v(0, n);
#pragma unroll
        for (int n = 0; n < 9; ++n) weigh(0, 0, n);
        if (masked) look(0);
    __builtin_amdgcn_s_setprio(1);
        prompt_spread<2 * DB, 9 + 2 * DB>([&](int n) { product(0, 0, n); }, [&](int n) { n < 2 * DB ? load_v(1, n) : weigh(0, 1, n - 2 * DB); });
        if (masked) look(1);
        prompt_spread<2 * DB, 0>([&](int n) { product(0, 1, n); }, [&](int) {});
    __builtin_amdgcn_s_setprio(0);
    }
    if (wild[0] || wild[1])
#pragma unroll
        for (int r = 0; r < RT; ++r) prompt_add_wild<bf16_t, HD>(st[r], v, sees[r] - t0, lane);
}

// Workgroup = four wavefronts of RT tiles of 32 rows each, of a split.
template <typename T, int HD, int RT, bool WIDE>
__global__ __launch_bounds__(kPromptWaves * 64, prompt_waves_per_simd(sizeof(T), HD)) void prompt_attention_kernel(PromptArgs a) {
    constexpr int BLOCK = kPromptBlock<T>, BYTES = BLOCK * HD * sizeof(T), ROWS = kPromptWaves * 32 * RT;
    // (arrays of their own, so that the compiler knows that what is on its way to one is not read from the other)
    __shared__ __attribute__((aligned(16))) unsigned char k_even[BYTES], v_even[BYTES], k_odd[BYTES], v_odd[BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kvh = blockIdx.x % a.n_kv, tile = blockIdx.x / a.n_kv % a.tiles, split = blockIdx.x / a.n_kv / a.tiles;
    const PromptTile s = prompt_find_tile(a, ROWS, tile);
    if (s.b < 0) return;
    const PromptBlocks range = prompt_blocks(prompt_keys(s.t, s.n, s.n_keys, a.G, ROWS), BLOCK, split, a.n_splits, a.per_split);
    if (!range.any) return;
    const T *k = (const T *)a.k + (size_t)s.k0 * a.k_stride + (size_t)kvh * HD, *v = (const T *)a.v + (size_t)s.k0 * a.v_stride + (size_t)kvh * HD;
    PromptState<HD> st[RT];
    u32x4 q[RT][HD * sizeof(T) / 32];
    int sees[RT], low = 0, high = -1;    // last key that the lane's row sees; the least and the largest such key of the wavefront's rows
    const int row0 = s.t * ROWS + wave * 32 * RT, offset = prompt_offset(s.n, s.n_keys);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int first = row0 + 32 * r, node = (first + (lane & 31)) / a.G;
        st[r].clear();
        prompt_load_q<T, HD>(a, s, kvh, first, lane, q[r]);
        sees[r] = node < s.n ? node + offset : -1;
    }
    low = __builtin_amdgcn_readfirstlane(row0 / a.G + offset);
    if (row0 / a.G < s.n) high = __builtin_amdgcn_readfirstlane(min((row0 + 32 * RT - 1) / a.G, s.n - 1) + offset);
    const PromptFetch<T, HD, WIDE> fetch_k(a.k_stride, wave, lane), fetch_v(a.v_stride, wave, lane);
    auto fetch = [&](int blk, unsigned char *lk, unsigned char *lv) {
        fetch_k.run(k, a.k_stride, blk * BLOCK, s.n_keys, lk, wave, lane);
        fetch_v.run(v, a.v_stride, blk * BLOCK, s.n_keys, lv, wave, lane);
    };
    auto block = [&](int blk, const unsigned char *lk, const unsigned char *lv) {
        const int t0 = blk * BLOCK;
        if (t0 > high) return;
        if constexpr (sizeof(T) == 2) prompt_block16<HD, RT>(st, lk, lv, q, sees, t0, t0 + BLOCK - 1 > low, a.scale_log2e, lane);
        else {
#pragma unroll
            for (int r = 0; r < RT; ++r) prompt_block<T, HD, true>(st[r], lk, lv, q[r], sees[r] - t0, a.scale_log2e, lane);
        }
    };
    if (range.first < range.last) fetch(range.first, k_even, v_even);
    for (int blk = range.first; blk < range.last; blk += 2) {
        prompt_barrier();     // this block is there, and everybody is done with the last one
        if (blk + 1 < range.last) fetch(blk + 1, k_odd, v_odd);
        block(blk, k_even, v_even);
        if (blk + 1 >= range.last) break;
        prompt_barrier();
        if (blk + 2 < range.last) fetch(blk + 2, k_even, v_even);
        block(blk + 1, k_odd, v_odd);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int rho = row0 + 32 * r + (lane & 31), node = rho / a.G;
        if (row0 + 32 * r >= (long)s.n * a.G) continue;
        const float sum = st[r].l + __shfl_xor(st[r].l, 32, 64);
        // (it is NaN, and so is the row, where a score is; it is 0 where the row saw nothing)
        const float norm = range.several ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum;
        const size_t slot = prompt_slot(a, tile, kvh, split) * (ROWS / 32) + wave * RT + r;
        if (range.several && lane < 32) {
            a.part_ml[slot * 64 + lane] = st[r].m;
            a.part_ml[slot * 64 + 32 + lane] = sum;
        }
        if (node >= s.n) continue;
#pragma unroll
        for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int j = db * 32 + 8 * u + 4 * (lane >> 5);
                f32x4 t;
#pragma unroll
                for (int e = 0; e < 4; ++e) t[e] = norm == 0.0f ? 0.0f : st[r].o[db][4 * u + e] * norm;
                if (range.several) *reinterpret_cast<f32x4 *>(a.part_o + slot * 32 * HD + prompt_part_index(lane & 31, j)) = t;
                else prompt_store<T>(a, (size_t)s.r0 + node, kvh * a.G + rho - node * a.G, HD, j, t);
            }
    }
}

// Joins the splits of every row that has several: out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  A thread owns four dimensions of a row.
template <typename T, int HD, int RT>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a) {
    constexpr int ROWS = kPromptWaves * 32 * RT, QUADS = ROWS * (HD / 4), WGS = QUADS / 256;
    const int part = blockIdx.x % WGS, kvh = blockIdx.x / WGS % a.n_kv, tile = blockIdx.x / WGS / a.n_kv;
    const PromptTile s = prompt_find_tile(a, ROWS, tile);
    if (s.b < 0) return;
    const int keys = prompt_keys(s.t, s.n, s.n_keys, a.G, ROWS);
    if (!prompt_blocks(keys, kPromptBlock<T>, 0, a.n_splits, a.per_split).several) return;
    const int u = part * 256 + threadIdx.x, row = u & 31, j = (u >> 5) % (HD / 4) * 4, sub = (u >> 5) / (HD / 4);
    const int rho = s.t * ROWS + sub * 32 + row, node = rho / a.G;
    if (node >= s.n) return;
    float m = -INFINITY, denom = 0.0f;
    f32x4 t = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = 0; i < a.n_splits && prompt_blocks(keys, kPromptBlock<T>, i, a.n_splits, a.per_split).any; ++i) {
        const size_t slot = prompt_slot(a, tile, kvh, i) * (ROWS / 32) + sub;
        const float pm = a.part_ml[slot * 64 + row], pl = a.part_ml[slot * 64 + 32 + row];
        const f32x4 po = *reinterpret_cast<const f32x4 *>(a.part_o + slot * 32 * HD + prompt_part_index(row, j));
        if (pl == 0.0f) continue;
        const float m_new = fmaxf(m, pm), m_use = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - m_use), w = __builtin_amdgcn_exp2f(pm - m_use);
        m = m_new;
        denom = denom * alpha + w * pl;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = (finite_f(t[e]) ? t[e] * alpha : t[e]) + (finite_f(po[e]) ? w * po[e] : po[e]);      // (alpha may be 0: not 0 * inf)
    }
    const float inv = denom == 0.0f ? 0.0f : 1.0f / denom;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = denom == 0.0f ? 0.0f : t[e] * inv;
    prompt_store<T>(a, (size_t)s.r0 + node, kvh * a.G + rho - node * a.G, HD, j, t);
}
