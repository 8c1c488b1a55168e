// Entry points of the operators of scoring and prefilling prompts: norms of queries and keys with their rotary positions, attention of packed prompts, log probabilities.
#include <float.h>
#include <math.h>

#include "kernels_logprobs.hip.h"
#include "kernels_norm_rotary.hip.h"
#include "kernels_prompt.hip.h"
#include "rotary_args.h"
#include "tree_ops.h"

namespace {

template <typename T, int TEAM, bool LAYER> void run_norm_rotary_team(hipStream_t st, dim3 grid, const NormRotaryArgs &a) {
    if (a.r.hd == 16 * TEAM) norm_rotary_kernel<T, TEAM, LAYER, true><<<grid, 256, 0, st>>>(a);
    else norm_rotary_kernel<T, TEAM, LAYER, false><<<grid, 256, 0, st>>>(a);
}
template <typename T, bool LAYER> void run_norm_rotary(hipStream_t st, dim3 grid, int team, const NormRotaryArgs &a) {
    switch (team) {
    case 0: norm_rotary_any_kernel<T, LAYER><<<grid, 256, 0, st>>>(a); break;
    case 1: run_norm_rotary_team<T, 1, LAYER>(st, grid, a); break;
    case 2: run_norm_rotary_team<T, 2, LAYER>(st, grid, a); break;
    case 4: run_norm_rotary_team<T, 4, LAYER>(st, grid, a); break;
    case 8: run_norm_rotary_team<T, 8, LAYER>(st, grid, a); break;
    case 16: run_norm_rotary_team<T, 16, LAYER>(st, grid, a); break;
    default: run_norm_rotary_team<T, 32, LAYER>(st, grid, a); break;
    }
}
template <typename T> void run_norm_rotary_type(hipStream_t st, dim3 grid, int team, bool layer, const NormRotaryArgs &a) {
    layer ? run_norm_rotary<T, true>(st, grid, team, a) : run_norm_rotary<T, false>(st, grid, team, a);
}

// ------------------------------------------------------------------------------------------------------------- attention
struct PromptPlan { int tiles, n_splits, per_split; size_t part_o, part_ml; };

// How many ways the keys of a tile are split: in bf16 not at all where there is a workgroup for every place without (what is split is written and read once more); else from an estimate of what that
// takes, in us.  A block takes `alone`, and `each` of every workgroup of the CU where that is more.  If all workgroups have their places at once, a split's blocks take that, one behind the other; if
// not, all blocks keep all CUs busy (71 % of them, as sequences differ, and causal prompts see half of their own rows), and the last splits a part of them.  5.5 us are a workgroup's beginning and end,
// each time that all places are taken; several splits are written, read, and joined by a launch more.
// (Its numbers are those that come nearest to what 1 to 96 ways took for 37 shapes of both types, from one row behind 3 000 keys and 16 behind 100 000 to 16 001 over themselves: its choice is the best
// for 24 of them, and at most 13 % slower than that.  Three times as many workgroups as there are places took 82 % more at 4 x 300 rows behind 700, no splits 27 times as long at 16 behind 100 000.)
// No more of them than workgroups for kPromptRounds times the places: then the last ones' part, which is all that splits take off, is at most 1 / kPromptRounds, and the workspace does not grow without
// bound with what max_kv expects (fp32, 2^20 rows of 16 heads behind as many keys: 49 GiB of partial results for 0.4 % of the time), nor the launch beyond what one holds.
constexpr size_t kPromptRounds = 32;
int prompt_n_splits(int size, int hd, long rows, size_t work, size_t blocks) {
    const double keys = prompt_block(size, hd) / 32 * (size == 4 ? hd / 64.0 : hd / 128.0), alone = (size == 4 ? 4.7 : 0.84) * keys, each = (size == 4 ? 1.6 : 0.54) * keys;
    const size_t cus = 256, slots = cus * prompt_resident(size, hd);
    if (size == 2 && work >= slots) return 1;
    double best = 0;
    int n = 1;
    for (size_t s = 1; s <= blocks && s <= 256 && (s == 1 || work * s <= kPromptRounds * slots); s += s < 4 ? 1 : s & (s - 1) ? s / 3 : s / 2) {       // 1, 2, 3, 4, 6, 8, 12 ..
        const size_t per = ceil_div_sz(blocks, s), splits = ceil_div_sz(blocks, per), rounds = ceil_div_sz(work * splits, slots);
        const double shared = each * ceil_div_sz(work * splits, cus);
        const double us = (rounds <= 1 ? per * (shared > alone ? shared : alone) : 0.71 * each * work * blocks / cus + 0.67 * per * each * slots / cus) + 5.5 * rounds +
                          (splits > 1 ? 7 + 0.06 * splits + 1.4e-6 * rows * hd * splits : 0);
        if (s == 1 || us < best) { best = us; n = (int)splits; }
    }
    return n;
}
PromptPlan prompt_plan(int dtype, int n_rows, int n_seqs, int n_heads, int n_kv, int hd, int max_kv) {
    PromptPlan p;
    const int G = n_heads / n_kv, rows = kPromptWaves * 32, block = prompt_block(dtype == SJD_F32 ? 4 : 2, hd);
    p.tiles = (int)prompt_max_tiles(n_rows, n_seqs, G, rows);
    const size_t work = (size_t)p.tiles * n_kv, blocks = ceil_div_sz((size_t)max_kv, block);
    p.n_splits = prompt_n_splits(dtype == SJD_F32 ? 4 : 2, hd, (long)n_rows * n_heads, work, blocks);
    p.per_split = (int)ceil_div_sz(blocks ? blocks : 1, p.n_splits);
    const size_t slots = p.n_splits > 1 ? work * p.n_splits * (rows / 32) : 0;
    p.part_o = slots * 32 * hd * sizeof(float);
    p.part_ml = slots * 64 * sizeof(float);
    return p;
}

int check_prompt(int32_t dtype, int32_t n_rows, int32_t n_seqs, int32_t n_heads, int32_t n_kv, int32_t hd, int32_t max_rows, int32_t max_kv, PromptPlan &p) {
    if (dtype != SJD_F32 && dtype != SJD_BF16) TREE_FAIL(SJD_EINVAL, "rows are SJD_F32 or SJD_BF16");
    switch (hd) {
    case 32: case 64: case 96: case 128: case 192: case 256: break;
    default: TREE_FAIL(SJD_EINVAL, "head_dim must be 32, 64, 96, 128, 192 or 256");
    }
    if (n_kv < 1 || n_kv > 65535 || n_heads < 1 || n_heads % n_kv || n_heads > 1 << 20) TREE_FAIL(SJD_EINVAL, "n_kv_heads must be 1 .. 65535, n_heads a multiple of it");
    if (n_seqs < 1 || n_seqs > 1 << 30 || n_rows < 0 || n_rows > 1 << 29) TREE_FAIL(SJD_EINVAL, "n_seqs must be 1 .. 2^30, n_rows 0 .. 2^29");
    if (max_rows < 0 || max_rows > 1 << 29 || max_kv < 0 || max_kv > 1 << 30) TREE_FAIL(SJD_EINVAL, "max_rows must be 0 .. 2^29, max_kv 0 .. 2^30");
    // (and what follows stays within its integers)
    const long G = n_heads / n_kv;
    if (n_rows * G > 1l << 30 || prompt_max_tiles(n_rows, n_seqs, (int)G, 32 * kPromptWaves) * n_kv > (long)kMaxWorkgroups) TREE_FAIL(SJD_EINVAL, "too many rows for one launch");
    p = prompt_plan(dtype, n_rows, n_seqs, n_heads, n_kv, hd, max_kv);
    return SJD_OK;
}

template <typename T, int HD> void run_prompt(hipStream_t st, const PromptArgs &a, bool wide_kv) {
    const unsigned grid = (unsigned)((size_t)a.tiles * a.n_kv * a.n_splits);
    if constexpr (sizeof(T) == 2) {
        if (wide_kv) prompt_attention16_kernel<HD, true><<<grid, kPromptWaves * 64, 0, st>>>(a);
        else prompt_attention16_kernel<HD, false><<<grid, kPromptWaves * 64, 0, st>>>(a);
    } else {
        if (wide_kv) prompt_attention32_kernel<HD, true><<<grid, kPromptWaves * 64, 0, st>>>(a);
        else prompt_attention32_kernel<HD, false><<<grid, kPromptWaves * 64, 0, st>>>(a);
    }
    if (a.n_splits > 1) {
        const unsigned quads = (unsigned)((size_t)a.tiles * a.n_kv * (kPromptWaves * 32 * HD / 1024));
        // (One wavefront a row, four: 4 splits 25.9 and 29.5 us the call, 5 in fp32 14.9 and 15.4, 8 101 and 104, 12 427 and 435, 16 in fp32 123 and 125, 32 15.5 and 13.3, 63 31.4 and 27.4.)
        if (a.n_splits > 8) prompt_join_kernel<T, HD, 4><<<4 * quads, 256, 0, st>>>(a);
        else prompt_join_kernel<T, HD, 1><<<quads, 256, 0, st>>>(a);
    }
}
template <typename T> void run_prompt_type(hipStream_t st, int hd, const PromptArgs &a, bool wide_kv) {
    switch (hd) {
    case 32: run_prompt<T, 32>(st, a, wide_kv); break;
    case 64: run_prompt<T, 64>(st, a, wide_kv); break;
    case 96: run_prompt<T, 96>(st, a, wide_kv); break;
    case 128: run_prompt<T, 128>(st, a, wide_kv); break;
    case 192: run_prompt<T, 192>(st, a, wide_kv); break;
    default: run_prompt<T, 256>(st, a, wide_kv); break;
    }
}

// ------------------------------------------------------------------------------------------------------ log probabilities
// How many workgroups a row is split over: as many as the card holds at once, four a CU, but none with less than one step a wavefront, and no more than one joining workgroup holds.
// (512, 768, 1024, 2048 workgroups: 256 rows of 65 536 with 20 ids 30.7, 30.7, 28.7, 37.8 us, 33 masked rows of 184 621 25.3, 21.9, 20.3, 22.0.)
// Up to four steps a wavefront a row is not split: up to three (12 000) the launch that joins takes longer, in a graph and call by call; from five (20 000) on a split row with ids is faster in a graph and as
// fast call by call, where the second launch costs the host 4 us.  At four it is 3 us slower call by call and 2 to 3 faster in a graph.  (8 rows, fp32, us in a graph, unsplit and split, and call by call:
//            no ids                        5 ids                          20 ids
//    8 192   5.3   7.1    12.2 16.0    9.8 10.5    12.7 16.7    13.3 12.7    13.5 16.7
//   12 000   7.2   8.6    12.2 16.1   12.4 12.8    12.7 16.8    16.1 15.9    16.2 17.0
//   16 384   7.0   7.0    12.3 16.1   12.9 10.7    13.2 16.9    16.1 13.3    16.3 16.7
//   20 000   9.0   8.4    12.1 16.1   16.0 12.5    16.3 16.7    18.6 15.8    18.8 17.2
//   32 768  10.4   7.1    12.3 16.4   21.9 10.8    21.9 16.9    23.1 14.5    23.3 16.8
//   48 000  14.8   8.3    15.1 16.3   28.1 12.6    28.3 16.7    30.8 16.9    31.0 17.2
// one row, 64 rows and bf16 the same but for 1 or 2 us; 256 rows gain less.)
int logprob_splits(int n_rows, int vocab, int n_top) {
    if (vocab <= 4 * kLogprobWaves * kLogprobStep) return 1;
    const int want = 1024 / (n_rows > 0 ? n_rows : 1), most = vocab / (kLogprobWaves * kLogprobStep), held = n_top ? kLogprobJoin / n_top : 64;
    int n = want < most ? want : most;
    if (n > held) n = held;
    if (n > 64) n = 64;
    return n > 1 ? n : 1;
}

int check_logprobs(int32_t n_rows, int32_t vocab, int32_t n_top) {
    if (n_rows < 0 || vocab < 1 || vocab > 1 << 24) TREE_FAIL(SJD_EINVAL, "n_rows must not be negative, vocab 1 .. 2^24");
    if (n_top < 0 || n_top > kTopMax) TREE_FAIL(SJD_EINVAL, "n_top must be 0 .. %d", kTopMax);
    if ((size_t)n_rows * logprob_splits(n_rows, vocab, n_top) > kMaxWorkgroups) TREE_FAIL(SJD_EINVAL, "too many rows for one launch");
    return SJD_OK;
}

}  // namespace

extern "C" {

int sjd_op_norm_rotary(void *hip_stream, int32_t dtype, int32_t norm, float eps, int32_t per_head, int32_t interleaved, const uint64_t *table,
                       int32_t rotary_dim, float magnitude, const int32_t *positions, int32_t n_rows, int32_t head_dim, const void *q, int64_t q_stride,
                       const void *q_gain, const void *q_bias, void *q_out, int64_t q_out_stride, int32_t n_heads, const void *k, int64_t k_stride,
                       const void *k_gain, const void *k_bias, void *k_out, int64_t k_out_stride, int32_t n_kv_heads) {
    NormRotaryArgs a = {{table, positions, {q, k}, {q_out, k_out}, {(long)q_stride, (long)k_stride}, {(long)q_out_stride, (long)k_out_stride},
                         {n_heads, n_kv_heads}, n_rows, head_dim, rotary_dim / 2, interleaved ? 1 : 0, 1, magnitude},
                        {q_gain, k_gain}, {q_bias, k_bias}, per_head ? 1 : 0, eps};
    bool w;
    const int rc = rotary_check(a.r, dtype, rotary_dim, w);
    if (rc) return rc;
    if (norm != SJD_NORM_RMS && norm != SJD_NORM_LAYER) TREE_FAIL(SJD_EINVAL, "unknown norm %d", norm);
    if (!(eps >= 1e-30f) || !(eps < INFINITY)) TREE_FAIL(SJD_EINVAL, "eps must be at least 1e-30");
    if (!q_gain || (n_kv_heads && !k_gain)) TREE_FAIL(SJD_EINVAL, "a gain is missing");
    const int size = dtype == SJD_F32 ? 4 : 2;
    for (int s = 0; s < 2; ++s) {
        if (!a.r.heads[s]) continue;
        const long n = (long)(per_head ? a.r.heads[s] : 1) * head_dim;
        for (const void *g : {a.gain[s], a.bias[s]}) {
            if (!g) continue;
            if ((uintptr_t)g % size) TREE_FAIL(SJD_EINVAL, "gains and biases are not aligned to their elements");
            w = w && (uintptr_t)g % 16 == 0;
            for (int o = 0; o < 2 && n_rows; ++o)
                if (a.r.heads[o] && !rows_apart(g, n, n, 1, a.r.y[o], a.r.y_stride[o], (long)a.r.heads[o] * head_dim, n_rows, size))
                    TREE_FAIL(SJD_EINVAL, "an output overlaps a gain or a bias");
        }
    }
    if (!n_rows) return SJD_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    const int heads = n_heads + n_kv_heads;
    int team = 0;            // lanes a head: one for 16 elements, 0: any rows
    dim3 grid;
    if (w) {
        const int need = a.r.interleaved ? (head_dim + 15) / 16 : a.r.half / 8 + (head_dim - rotary_dim + 15) / 16;
        for (team = 1; team < need;) team *= 2;
        // (2 rows a workgroup at most, 4, 8: 9 408 rows of 64 heads of 128 with means, gains and biases 61.9, 65.3, 68.7 us, 12 000 rows of 40 heads 40.4, 40.0, 43.0)
        if (!rotary_grid(a.r, 2, (long)heads * team, grid)) TREE_FAIL(SJD_EINVAL, "too many rows for one launch");
    } else {
        if ((size_t)n_rows > kMaxWorkgroups) TREE_FAIL(SJD_EINVAL, "too many rows for one launch");
        grid = dim3(n_rows, n_rows >= 512 ? 1 : ceil_div(heads, 4) < 512 / n_rows + 1 ? ceil_div(heads, 4) : 512 / n_rows + 1);
    }
    const bool layer = norm == SJD_NORM_LAYER;
    dtype == SJD_F32 ? run_norm_rotary_type<float>(st, grid, team, layer, a) : run_norm_rotary_type<bf16_t>(st, grid, team, layer, a);
    TREE_TRY(hipGetLastError());
    return SJD_OK;
}

int sjd_op_prompt_attention_workspace(int32_t dtype, int32_t n_rows, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_rows,
                                      int32_t max_kv, uint64_t *bytes) {
    if (!bytes) TREE_FAIL(SJD_EINVAL, "null argument");
    PromptPlan p;
    const int rc = check_prompt(dtype, n_rows, n_seqs, n_heads, n_kv_heads, head_dim, max_rows, max_kv, p);
    if (rc) return rc;
    *bytes = p.part_o + p.part_ml;
    return SJD_OK;
}

int sjd_op_prompt_attention(void *hip_stream, int32_t dtype, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                            void *out, int64_t out_stride, const int32_t *row_start, const int32_t *kv_start, int32_t n_rows, int32_t n_kv_rows, int32_t n_seqs,
                            int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale, int32_t max_rows, int32_t max_kv, void *workspace,
                            uint64_t workspace_bytes) {
    PromptPlan p;
    const int rc = check_prompt(dtype, n_rows, n_seqs, n_heads, n_kv_heads, head_dim, max_rows, max_kv, p);
    if (rc) return rc;
    if (!kv_start) n_kv_rows = n_rows;
    if (n_kv_rows < 0 || n_kv_rows > 1 << 30) TREE_FAIL(SJD_EINVAL, "n_kv_rows must be 0 .. 2^30");
    if (!row_start || (n_rows && (!q || !out)) || (n_rows && n_kv_rows && (!k || !v))) TREE_FAIL(SJD_EINVAL, "null argument");
    if (!(scale >= 0.0f) || !(scale < INFINITY)) TREE_FAIL(SJD_EINVAL, "scale must be positive, or 0 for 1 / sqrt(head_dim)");
    const int size = dtype == SJD_F32 ? 4 : 2;
    if ((uintptr_t)q % size || (uintptr_t)k % size || (uintptr_t)v % size || (uintptr_t)out % size) TREE_FAIL(SJD_EINVAL, "rows are not aligned to their elements");
    const long row = (long)n_heads * head_dim, kv_row = (long)n_kv_heads * head_dim;
    if (n_rows > 1 && out_stride < row) TREE_FAIL(SJD_EINVAL, "output rows overlap");
    if ((n_rows > 1 && q_stride < 0) || (n_kv_rows > 1 && (k_stride < 0 || v_stride < 0))) TREE_FAIL(SJD_EINVAL, "negative stride");
    if (!n_rows) return SJD_OK;
    // in place: a workgroup has read its queries when it writes their results, and nobody else reads them
    if (!(q == out && (q_stride == out_stride || n_rows == 1)) && !rows_apart(q, q_stride, row, n_rows, out, out_stride, row, n_rows, size))
        TREE_FAIL(SJD_EINVAL, "the output overlaps the queries");
    if (n_kv_rows && (!rows_apart(k, k_stride, kv_row, n_kv_rows, out, out_stride, row, n_rows, size) ||
                      !rows_apart(v, v_stride, kv_row, n_kv_rows, out, out_stride, row, n_rows, size)))
        TREE_FAIL(SJD_EINVAL, "the output overlaps keys or values");
    if (p.part_o + p.part_ml > workspace_bytes)
        TREE_FAIL(SJD_ECAPACITY, "the workspace holds %llu bytes, %zu are needed", (unsigned long long)workspace_bytes, p.part_o + p.part_ml);
    if (p.part_o && (!workspace || (uintptr_t)workspace % 16)) TREE_FAIL(SJD_EINVAL, "the workspace must be 16-byte aligned");
    PromptArgs a;
    a.q = q; a.k = k; a.v = v; a.out = out;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = out_stride;
    a.row_start = row_start; a.kv_start = kv_start;
    a.n_rows = n_rows; a.n_kv_rows = n_kv_rows; a.n_seqs = n_seqs; a.H = n_heads; a.n_kv = n_kv_heads; a.G = n_heads / n_kv_heads;
    a.tiles = p.tiles; a.n_splits = p.n_splits; a.per_split = p.per_split;
    a.scale_log2e = (float)(1.4426950408889634 * (scale > 0.0f ? (double)scale : 1.0 / sqrt((double)head_dim)));
    a.part_o = (float *)workspace;
    a.part_ml = (float *)((char *)workspace + p.part_o);
    a.q_wide = wide(q, q_stride, size, 16);
    a.out_wide = wide(out, out_stride, size, 16);
    // (their places within a block are 32-bit offsets)
    auto near = [&](long stride) { return n_kv_rows < 2 || stride < (1l << 31) / (64 * size); };
    const bool wide_kv = wide(k, k_stride, size, 16) && wide(v, v_stride, size, 16) && near(k_stride) && near(v_stride);
    hipStream_t st = (hipStream_t)hip_stream;
    dtype == SJD_F32 ? run_prompt_type<float>(st, head_dim, a, wide_kv) : run_prompt_type<bf16_t>(st, head_dim, a, wide_kv);
    TREE_TRY(hipGetLastError());
    return SJD_OK;
}

int sjd_op_token_logprobs_workspace(int32_t n_rows, int32_t vocab, int32_t n_top, uint64_t *bytes) {
    if (!bytes) TREE_FAIL(SJD_EINVAL, "null argument");
    const int rc = check_logprobs(n_rows, vocab, n_top);
    if (rc) return rc;
    const int splits = logprob_splits(n_rows, vocab, n_top);
    *bytes = splits > 1 ? (uint64_t)n_rows * splits * logprob_part_bytes(n_top) : 0;
    return SJD_OK;
}

int sjd_op_token_logprobs(void *hip_stream, int32_t dtype, const void *logits, int64_t stride, const int32_t *tokens, float *logprob, int32_t *rank, float *entropy,
                          int32_t *top_ids, float *top_logprobs, int32_t n_rows, int32_t vocab, int32_t n_top, void *workspace, uint64_t workspace_bytes) {
    if (dtype != SJD_F32 && dtype != SJD_BF16) TREE_FAIL(SJD_EINVAL, "logits are SJD_F32 or SJD_BF16");
    const int rc = check_logprobs(n_rows, vocab, n_top);
    if (rc) return rc;
    if (n_rows && (!logits || !tokens || !logprob || !rank || !entropy || (n_top && (!top_ids || !top_logprobs)))) TREE_FAIL(SJD_EINVAL, "null argument");
    const int size = dtype == SJD_F32 ? 4 : 2;
    if ((uintptr_t)logits % size) TREE_FAIL(SJD_EINVAL, "logits are not aligned to their elements");
    if (n_rows > 1 && stride < 0) TREE_FAIL(SJD_EINVAL, "negative stride");
    if (!n_rows) return SJD_OK;
    struct { void *p; long n; } out[5] = {{logprob, n_rows}, {rank, n_rows}, {entropy, n_rows}, {top_ids, (long)n_rows * n_top}, {top_logprobs, (long)n_rows * n_top}};
    for (int i = 0; i < 5; ++i) {
        if (!out[i].n) continue;
        if ((uintptr_t)out[i].p % 4) TREE_FAIL(SJD_EINVAL, "an output is not aligned to its elements");
        for (int j = 0; j < i; ++j)
            if (out[j].n && !rows_apart(out[i].p, out[i].n, out[i].n, 1, out[j].p, out[j].n, out[j].n, 1, 4)) TREE_FAIL(SJD_EINVAL, "outputs overlap");
        // (the logits' last row ends with its vocabulary; in bytes, as their elements may be smaller)
        if (!rows_apart(out[i].p, 4 * out[i].n, 4 * out[i].n, 1, logits, stride * size, (long)vocab * size, n_rows, 1) ||
            !rows_apart(out[i].p, out[i].n, out[i].n, 1, tokens, n_rows, n_rows, 1, 4)) TREE_FAIL(SJD_EINVAL, "an output overlaps an input");
    }
    LogprobArgs a = {logits, (long)stride, tokens, n_rows, vocab, n_top, logprob_splits(n_rows, vocab, n_top), logprob, entropy, top_logprobs, rank, top_ids,
                     (unsigned char *)workspace};
    const uint64_t need = a.n_splits > 1 ? (uint64_t)n_rows * a.n_splits * logprob_part_bytes(n_top) : 0;
    if (need > workspace_bytes) TREE_FAIL(SJD_ECAPACITY, "the workspace holds %llu bytes, %llu are needed", (unsigned long long)workspace_bytes, (unsigned long long)need);
    if (need && (!workspace || (uintptr_t)workspace % 16)) TREE_FAIL(SJD_EINVAL, "the workspace must be 16-byte aligned");
    hipStream_t st = (hipStream_t)hip_stream;
    const unsigned grid = (unsigned)n_rows * a.n_splits;
    if (dtype == SJD_F32) n_top ? logprob_kernel<float, true><<<grid, 256, 0, st>>>(a) : logprob_kernel<float, false><<<grid, 256, 0, st>>>(a);
    else n_top ? logprob_kernel<bf16_t, true><<<grid, 256, 0, st>>>(a) : logprob_kernel<bf16_t, false><<<grid, 256, 0, st>>>(a);
    TREE_TRY(hipGetLastError());
    if (a.n_splits > 1) {
        if (dtype == SJD_F32) logprob_join_kernel<float><<<n_rows, 256, 0, st>>>(a);
        else logprob_join_kernel<bf16_t><<<n_rows, 256, 0, st>>>(a);
        TREE_TRY(hipGetLastError());
    }
    return SJD_OK;
}

}  // extern "C"
