/*
 * sjd -- speculative Jacobi decoding (SJD++) of a discrete autoregressive
 * image-token transformer on one AMD MI355X (gfx950).  C ABI.
 *
 * The library decodes image tokens after a text prompt with the iteration of
 * Sec. 4.1 of the paper (the speculative Jacobi iteration): a window of L tokens
 * (the last final token followed by L-1 drafts) is run through ONE causal
 * forward of the transformer against a paged KV cache, as a conditional /
 * unconditional pair for classifier-free guidance (Sec. 5.1: guidance weight,
 * top-K); drafts are accepted left to right with probability min(1, p/q)
 * (Eq. 2), the first unaccepted position is redrawn from the residual
 * normalise(max(0, p - q)) (Eq. 3), and each later draft is kept when its
 * confidence p/q exceeds tau and redrawn from p otherwise (Eq. 4-5; tau = +inf
 * is the rule without reuse, Eq. 6).
 *
 * Conventions
 *  - every function returns SJD_OK (0) or a negative sjd_status and never
 *    throws or aborts; sjd_last_error() gives a text for the last failure of a
 *    context (or of sjd_create when passed NULL);
 *  - "device" pointers are HIP device pointers on the current device, "host"
 *    pointers are ordinary process memory;
 *  - hip_stream is a hipStream_t passed as void* (NULL = the default stream);
 *    it is borrowed and must outlive the context; all work of a context is
 *    enqueued on it.  On an ordinary stream sjd_step records its launches
 *    beside its first run (stream capture, thread-local mode) and replays them
 *    as a HIP graph from then on; on the default stream, which cannot be
 *    captured, or where the recording fails, it launches them one by one;
 *  - a context is not thread-safe; different contexts are independent.
 */
#ifndef SJD_H
#define SJD_H
#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sjd_ctx sjd_ctx;

enum sjd_status {
    SJD_OK = 0,
    SJD_EINVAL = -1,    /* bad argument or unsupported shape          */
    SJD_ENOMEM = -2,    /* device or host allocation failed           */
    SJD_ESTATE = -3,    /* call order violated                        */
    SJD_EDEVICE = -4,   /* a HIP call failed                          */
    SJD_ECAPACITY = -5  /* more sequences / context than created for  */
};

enum sjd_dtype {
    SJD_F32 = 0,
    SJD_BF16 = 1,
    SJD_FP8 = 2  /* caches of the tree operators only: e4m3 codes, one power of two a token and key/value head as their scale */
};

/* kernel_flags bits */
enum {
    SJD_KERNELS_REFERENCE = 1, /* use the plain (non-MFMA) GEMM and attention kernels */
    SJD_NO_GRAPH = 2,          /* never capture the step into a HIP graph: launch its
                                * kernels one by one                                   */
    SJD_KERNELS_ROWGROUPS = 4, /* bf16, > 64 rows: keep the 64-row-group streaming projection
                                * kernels instead of the LDS-staged tile kernels       */
    SJD_ATTENTION_CHUNKED = 8, /* bf16: always split the context over workgroups and merge
                                * in a second kernel, also where one workgroup per head
                                * would do (short contexts); a prefill then runs window by
                                * window instead of packing the prompts' rows          */
    SJD_KERNELS_TILES = 16,    /* bf16, >= 256 rows: the tile kernels also where smaller
                                * tiles or row groups are expected to be faster        */
    SJD_NO_L2_WARM = 32,       /* bf16, <= 64 rows: projection launches carry no extra
                                * workgroups that touch the next launch's weights and
                                * key/value pages into L2 (same results either way)    */
    SJD_TILES_256_ROWS = 64,   /* bf16, >= 256 rows: every tile kernel launch uses 256-row
                                * workgroup tiles (default: 128-row tiles where they
                                * balance the CUs better)                              */
    SJD_NO_ROW_SPLIT = 128,    /* bf16, up to 64 rows: projections of so few column groups
                                * that their rows are split as well, with all rows in one
                                * workgroup (default: 16 or 32 rows each);
                                * more rows: 64-row groups also for projections of so few
                                * column groups that 32-row groups would each get a CU     */
    SJD_NO_MIXED_WIDTH = 256,  /* bf16: no launch mixes workgroup shapes.  <= 64 rows: gate/up and
                                * head projections of more than 256 column groups with one
                                * workgroup per group (default: one workgroup per CU, some of
                                * them two groups wide); >= 256 rows: one tile height per launch
                                * (default: 256-row tiles on every CU with the remaining column
                                * tiles as 128-row tiles beside them, where the 256-row tiles
                                * number between one and two per CU)                    */
    SJD_KEEP_LOGITS = 1024,    /* keep the fp32 logits of every step for sjd_debug_copy_logits.  Without it the
                                * vocabulary head of the fused bf16 path writes only the guided logits
                                * z = (l_u + s (l_c - l_u)) / T of each position (windows of 32, or one sequence
                                * with a window of 16), which is all the sampling stage reads            */
    SJD_NO_HEAD_FUSION = 2048, /* the vocabulary head always writes the logits and the sampling kernel combines the
                                * two branches (same results either way)                                 */
    SJD_NO_K_ROTATION = 512    /* bf16, row-group projection kernels: every workgroup walks K
                                * from 0 (default: each starts at its own offset and wraps,
                                * so that they do not all ask for the same activation lines
                                * at the same time; sums differ in the last bits only)  */
};

/* Architecture and capacities; plain data, copied by sjd_create.
 * Pre-norm decoder blocks: RMSNorm, rotary embedding on q and k (rotate-half
 * pairing (i, i + hd/2), angle pos * rope_theta^(-2i/hd)), grouped-query
 * attention with scale 1/sqrt(hd), SwiGLU MLP, final RMSNorm, untied head.
 * The paper fixes none of this (Sec. 3.1 only asks for a transformer that
 * predicts a categorical distribution); it is the shape of the workloads. */
typedef struct {
    int32_t n_layers, d_model, n_heads, n_kv_heads, d_ff;
    int32_t vocab, sample_lo, sample_hi; /* token ids in [sample_lo, sample_hi) are sampled */
    float rms_eps, rope_theta;
    int32_t dtype;           /* sjd_dtype: storage of weights, activations fed to GEMMs, KV cache */
    int32_t max_seqs;        /* prompts decoded together (each is a cond + uncond pair) */
    int32_t max_ctx;         /* positions per branch: prompt + image tokens             */
    int32_t window;          /* L >= 1: the last final token + L-1 drafts              */
    int32_t kv_page_tokens;  /* tokens per KV page; multiple of 32; 0 = 64              */
    int32_t kernel_flags;
} sjd_model_desc;

/* DEVICE pointers to weights of type `dtype`.  Linear weights are
 * [out_features][in_features] row-major (y = W x); per-layer members are HOST
 * arrays of n_layers device pointers.  sjd_create copies (and re-lays-out)
 * everything it needs: nothing is referenced after it returns. */
typedef struct {
    const void *tok_emb;    /* [vocab][d_model] */
    const void *final_norm; /* [d_model]        */
    const void *lm_head;    /* [vocab][d_model] */
    const void *const *attn_norm; /* [d_model]                     */
    const void *const *wq;        /* [n_heads*hd][d_model]         */
    const void *const *wk;        /* [n_kv_heads*hd][d_model]      */
    const void *const *wv;        /* [n_kv_heads*hd][d_model]      */
    const void *const *wo;        /* [d_model][n_heads*hd]         */
    const void *const *mlp_norm;  /* [d_model]                     */
    const void *const *w_gate;    /* [d_ff][d_model]               */
    const void *const *w_up;      /* [d_ff][d_model]               */
    const void *const *w_down;    /* [d_model][d_ff]               */
} sjd_weights;

/* Sampling distribution and decoding rule (Sec. 5.1).
 * p = softmax over the top_k largest of z = (l_u + cfg_scale (l_c - l_u)) /
 * temperature (ties at the k-th value kept).  Randomness is Philox4x32-10 keyed
 * by `seed` with counter (step, row, sequence, 0). */
typedef struct {
    float cfg_scale, temperature;
    int32_t top_k;
    float reuse_tau;  /* 0.5 in the paper; +INF disables reuse (Eq. 6) */
    uint64_t seed;
    /* Sec. 4.2, how a window slot that has never had a draft is filled (slots of the first window, before any image
     * token exists, are always uniform):
     *   0  drawn uniformly over the sampled ids (reference: uniform);
     *   1  copy of the token to its left (reference: one-hot at that token);
     *   2  copy of the token one image row above, row_width tokens back (one-hot; uniform in the first row);
     *   3  drawn from the distribution its left neighbour was drawn from, i.e. the last row of the step
     *      (reference: that row);
     *   4  drawn from the distribution of the token one image row above: the row under which that token became
     *      final (the context keeps the last row_width of them per sequence), or the reference of the draft at
     *      that place if it is still in the window (reference: the same; uniform in the first image row). */
    int32_t init_mode;
    int32_t row_width; /* tokens per image row; used by init_mode 2 and 4 (>= 1 there) */
} sjd_sampling;

typedef struct {
    int32_t n_accepted;   /* drafts accepted this step (Eq. 2)                          */
    int32_t n_finalized;  /* tokens made final this step = n_accepted + 1, 0 if done    */
    int32_t reject_index; /* window slot of the first rejected draft, -1 if none        */
    int32_t done;         /* 1 once all image tokens of the sequence are final          */
} sjd_step_result;

/* Creates a context on the current device: allocates KV pages for
 * max_seqs * 2 * max_ctx positions, workspaces and decoding state; copies the
 * weights.  Errors: SJD_EINVAL (null pointer, unsupported shape: bf16 needs
 * hd % 32 == 0, d_model % 16 == 0, d_ff % 16 == 0), SJD_ENOMEM, SJD_EDEVICE. */
int sjd_create(const sjd_model_desc *desc, const sjd_weights *weights, const sjd_sampling *sampling,
               void *hip_stream, sjd_ctx **out);

/* Starts n_seqs decodes (Sec. 4.1: the text prompt is run through the model first).  All
 * arrays are HOST arrays of length n_seqs, read during the call only.  Every
 * prompt token but the last is run through the model into the KV cache; the
 * last one becomes the first window input; the L-1 drafts are drawn uniformly.
 * May be called again to start new decodes.
 * Which kernels run the rows, and so the order of bf16 sums, follows from how
 * many rows a forward has (the batch size; in a prefill the prompts' total
 * length) and from the longest cached context: in bf16 a sequence's logits agree
 * to rounding, not bit for bit, between batches of other sizes or prompt
 * lengths, and with a fixed seed its tokens may differ.  In fp32 they do not
 * depend on its neighbours.  Errors: SJD_EINVAL (null, length
 * < 1, id outside the vocabulary), SJD_ECAPACITY (n_seqs > max_seqs or
 * prompt + image tokens > max_ctx; nothing is enqueued), SJD_EDEVICE. */
int sjd_prefill(sjd_ctx *ctx, int32_t n_seqs, const int32_t *const *cond_ids, const int32_t *cond_len,
                const int32_t *const *uncond_ids, const int32_t *uncond_len, const int32_t *n_image_tokens);

/* One speculative Jacobi iteration for every unfinished sequence (Sec. 4.1
 * Steps 1-4).  out is a HOST array of n_seqs results.  The call returns after
 * the step has completed on the device.  Sequences that are done are left
 * untouched (n_finalized = 0, done = 1).  Errors: SJD_ESTATE (no prefill) and
 * SJD_EINVAL (null argument), before anything ran; SJD_EDEVICE: a launch or
 * the device failed, and the step may have run in part or whole: go on from sjd_prefill or sjd_snapshot_restore. */
int sjd_step(sjd_ctx *ctx, sjd_step_result *out);

/* Frees everything the context owns.  NULL is allowed. */
void sjd_destroy(sjd_ctx *ctx);

/* Copies the image tokens of sequence `seq` that are final so far into dst
 * (HOST, capacity cap, may be NULL when cap == 0); *n_out receives their count. */
int sjd_get_tokens(sjd_ctx *ctx, int32_t seq, int32_t *dst, int32_t cap, int32_t *n_out);

/* Current window of sequence `seq` (HOST arrays of length `window`): tokens
 * (slot 0 = last final token) and per slot the output row of the previous step
 * that is its reference distribution (-1 = uniform); *n_slots = slots in use. */
int sjd_get_window(sjd_ctx *ctx, int32_t seq, int32_t *tokens, int32_t *ref_rows, int32_t *n_slots);

/* Forced tokens (structure tokens of an image grammar, such as the end-of-row
 * token that closes every row of a 48 x 49 token image): image position i of
 * sequence `seq` may only take ids in [first_id[i], end_id[i]), i < n_positions
 * (HOST arrays; absolute ids inside [sample_lo, sample_hi)).  Ids outside the
 * range get probability 0 at that position before top-K (Sec. 3.1) is applied,
 * so a range of one id forces that token.  Drafts are still initialised over all
 * sampled ids; one that falls outside its position's range has p = 0 and is
 * rejected by Eq. 2 with certainty.  Call after sjd_prefill (which resets every
 * position to the whole sampled range); positions >= n_positions keep theirs.
 * Errors: SJD_ESTATE (no prefill), SJD_EINVAL (bad index, empty range, range
 * outside the sampled ids, n_positions > image tokens of the sequence). */
int sjd_set_token_ranges(sjd_ctx *ctx, int32_t seq, const int32_t *first_id, const int32_t *end_id, int32_t n_positions);

const char *sjd_last_error(const sjd_ctx *ctx);

/* fp32 logits of the last step, [n_seqs][2 (cond, uncond)][window][V_s],
 * V_s = sample_hi - sample_lo, to HOST memory.  SJD_ESTATE when the context does
 * not keep them (created without SJD_KEEP_LOGITS and its head writes guided
 * logits only). */
int sjd_debug_copy_logits(sjd_ctx *ctx, float *dst_host);

/* Runs Steps 3-4 on caller-provided logits (HOST, layout as above) instead of
 * the forward: the KV cache is not written, its length advances as usual. */
int sjd_debug_step_from_logits(sjd_ctx *ctx, const float *logits_host, sjd_step_result *out);

/* Snapshot of the decoding state of the current batch, to HOST memory and back.
 * What Sec. 4.1 carries from one iteration to the next is small and explicit:
 * the accepted tokens, the window's drafts with the distributions they were
 * drawn from (the previous iteration's rows), the step counter that indexes the
 * random stream, and the cache of the accepted prefix.  A snapshot holds exactly
 * that (cache pages of accepted positions only), so a half-decoded batch can be
 * parked and resumed, or rolled back: after sjd_snapshot_restore the following
 * sjd_step calls return what they returned after sjd_snapshot_save, bit for bit.
 *   sjd_snapshot_size     *bytes = size a save would write now (it grows with
 *                         the accepted prefix).
 *   sjd_snapshot_save     writes the snapshot to dst_host (cap bytes available);
 *                         *written = its size.  SJD_ECAPACITY if cap is too small.
 *   sjd_snapshot_restore  src_host / bytes as written by a save on a context
 *                         created with the same model description and sampling
 *                         parameters (anything else, a truncated or altered
 *                         buffer: SJD_EINVAL, context unchanged).  Replaces
 *                         whatever batch the context held; no prefill needed.
 * All three return after the copies completed; SJD_ESTATE before the first
 * prefill (size, save).  The buffer is plain bytes owned by the caller; its
 * format is private to the library version that wrote it. */
int sjd_snapshot_size(sjd_ctx *ctx, uint64_t *bytes);
int sjd_snapshot_save(sjd_ctx *ctx, void *dst_host, uint64_t cap, uint64_t *written);
int sjd_snapshot_restore(sjd_ctx *ctx, const void *src_host, uint64_t bytes);

/* Per-kernel timing.  With tracing on, sjd_step brackets every kernel launch
 * with HIP events on the context's stream and accumulates their durations.
 * sjd_trace_read copies up to cap entries: name (static string), number of
 * launches, total milliseconds; *n_out = number of kernel classes. */
typedef struct {
    const char *name;
    int64_t launches;
    double total_ms;
} sjd_trace_entry;
int sjd_trace_enable(sjd_ctx *ctx, int32_t on);
int sjd_trace_reset(sjd_ctx *ctx);
int sjd_trace_read(sjd_ctx *ctx, sjd_trace_entry *dst, int32_t cap, int32_t *n_out);

/* ---- single operations, for kernel-level tests and microbenchmarks.
 * All pointers are DEVICE pointers in plain row-major layouts; the calls
 * allocate temporaries, run on `hip_stream` and return after completion. */

/* C[M][N] (fp32) = A[M][K] * W[N][K]^T with the GEMM kernel the decoder uses
 * for `dtype` (reference kernel if flags has SJD_KERNELS_REFERENCE).
 * splits <= 0 lets the library choose the split-K factor.  `repeat` >= 1
 * launches the kernel that many times; *avg_ms (HOST, may be NULL) receives the
 * mean kernel time measured with HIP events. */
int sjd_op_gemm(void *hip_stream, int32_t dtype, int32_t flags, const void *A, const void *W, float *C, int32_t M,
                int32_t N, int32_t K, int32_t splits, int32_t repeat, float *avg_ms);

/* sjd_op_gemm for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same kernels,
 * with the temporaries (both operands re-laid-out for the kernels and the split-K
 * partial sums) in a 32 MiB workspace that is part of the library image on every
 * device.  The call allocates nothing, creates no events and returns after completion.
 * SJD_ECAPACITY when the temporaries of M x N x K exceed the workspace
 * (bf16: 2 (ceil32(M) + ceil32(N)) K + 4 splits M N bytes, each part rounded up to 256).
 * All calls on one device share the workspace: calls that overlap on one device
 * (different streams or threads) race; serialise them. */
int sjd_op_gemm_static(void *hip_stream, int32_t dtype, int32_t flags, const void *A, const void *W, float *C, int32_t M,
                       int32_t N, int32_t K, int32_t splits);

/* Window attention of one (sequence, branch): q [n][H][hd], k and v
 * [ctx + n][Hkv][hd] of `dtype` (the first ctx positions are the cache, the
 * last n the window), out [n][H][hd] fp32.  Query i sees positions
 * 0 .. ctx + i. */
int sjd_op_window_attention(void *hip_stream, int32_t dtype, int32_t flags, const void *q, const void *k,
                            const void *v, float *out, int32_t n, int32_t ctx, int32_t n_heads,
                            int32_t n_kv_heads, int32_t head_dim, int32_t page_tokens, int32_t repeat,
                            float *avg_ms);

/* Sampling distribution of `rows` positions (Sec. 3.1 top-K sampling with the
 * guidance weight of Sec. 5.1): logits_c / logits_u [rows][V] fp32 -> e [rows][V]
 * fp32 softmax weights (0 outside the top-k set) and Z [rows] uint64 integer
 * normalisers.  allow_lo / allow_hi (DEVICE [rows], both or neither NULL): row r
 * may only keep ids in [allow_lo[r], allow_hi[r]).  kept_ids [rows][V] and
 * kept_cnt [rows] (DEVICE, may be NULL) receive the form in which the decoder
 * stores a row: the ids with a weight, ascending, and their number. */
int sjd_op_sampling_rows(void *hip_stream, const float *logits_c, const float *logits_u, float *e, uint64_t *Z,
                         int32_t rows, int32_t V, float cfg_scale, float temperature, int32_t top_k,
                         const int32_t *allow_lo, const int32_t *allow_hi, int32_t *kept_ids, int32_t *kept_cnt,
                         int32_t repeat, float *avg_ms);

/* out[4*i .. 4*i+3] = Philox4x32-10(counter = (i, row, seq, 0), key = seed), i < n. */
int sjd_op_philox(void *hip_stream, uint64_t seed, uint32_t row, uint32_t seq, uint32_t *out, int32_t n);

/* ---- operators of a step of tree speculation: rotary positions, the paged key/value cache (plain or quantised), attention of
 * a tree of drafts over it, verification of the tree.  A window of drafts is a tree without branches, and a single token a
 * tree of one node.
 *
 * Unlike the single operations above these allocate nothing, enqueue their kernels on `hip_stream` and return at once;
 * they can be captured into a HIP graph, and a graph that is replayed reads the lengths, tables and positions that are in device
 * memory then.  Pointers are DEVICE pointers on the stream's device, which is the current one, unless HOST is said; strides are in
 * elements.  Calls that may run at the same time need workspaces of their own and must not write what the other reads.
 *
 * Ragged rows: rows [row_start[b], row_start[b + 1]) of the arrays are sequence b's, b < n_seqs (row_start has n_seqs + 1
 * entries, ascending; what lies outside [0, n_rows] is cut off), and row row_start[b] + i belongs to position
 * first_pos[b] + i of its cache.  Outputs of rows of no sequence are left as they were.  A sequence whose first_pos is negative or above
 * 2^30 lies outside its cache as a whole, whichever of its rows would come to stand inside.
 *
 * Sizes and pointers are checked on the host (SJD_EINVAL, nothing enqueued; so is a call of more workgroups than a launch has
 * room for, 2^24 - 1: of the order of 2^24 tiles of rows, or of sequences).  What is in device memory is checked by the kernels:
 * a page table entry outside [0, n_pages), or a position outside [0, pages_per_seq * page_tokens), is never
 * followed: writes to it are dropped, reads of it give zeros, attention does not see it. */

/* A paged cache: plain data; the caller owns both allocations.  Pages of one sequence are listed in its row of the page
 * table; an unused entry is any value outside [0, n_pages).  Sequences may share pages that nobody writes.  The layout inside a
 * page is private: it is written by sjd_op_cache_write and sjd_op_cache_compact. */
typedef struct {
    void *pages;               /* n_pages * sjd_cache_page_bytes() bytes, 16-byte aligned                       */
    const int32_t *page_table; /* [n_seqs][pages_per_seq]                                                       */
    int32_t n_pages, page_tokens; /* page_tokens: a multiple of 32                                              */
    int32_t n_kv_heads, head_dim; /* head_dim: 32, 64, 96, 128, 192 or 256                                      */
    int32_t dtype;             /* sjd_dtype of what is stored                                                   */
    int32_t n_seqs, pages_per_seq;
} sjd_kv_cache;

/* *bytes (HOST) of one page.  Only page_tokens, n_kv_heads, head_dim and dtype of `cache` are read. */
int sjd_cache_page_bytes(const sjd_kv_cache *cache, uint64_t *bytes);

/* Writes rows of keys and values, k and v [n_rows][n_kv_heads][head_dim] of src_dtype (SJD_F32 or SJD_BF16; a row's heads are
 * contiguous, rows k_stride / v_stride apart), to positions first_pos[b] + i.
 * SJD_FP8: a token's keys of one head share the scale 2^e, and so do its values, with the smallest e in [-100, 119] for which
 * max |x| <= 448 * 2^e over the finite elements; the code of x is the e4m3 number nearest to x * 2^-e, ties to even, at most
 * 448 in magnitude.  Infinities and NaN become NaN.  SJD_BF16 rounds to nearest even, SJD_F32 keeps the value.
 * Nothing else in the pages changes. */
int sjd_op_cache_write(void *hip_stream, const sjd_kv_cache *cache, int32_t src_dtype, const void *k, int64_t k_stride, const void *v,
                       int64_t v_stride, const int32_t *row_start, const int32_t *first_pos, int32_t n_rows);

/* The way back: k and v [n_rows][n_kv_heads][head_dim] (contiguous, apart) of dst_dtype receive what is stored at positions first_pos[b] + i:
 * for SJD_FP8 code * 2^e, exact in either type. */
int sjd_op_cache_read(void *hip_stream, const sjd_kv_cache *cache, int32_t dst_dtype, void *k, void *v, const int32_t *row_start,
                      const int32_t *first_pos, int32_t n_rows);

/* Keeps a path of a tree: of the rows at positions first_pos[b] + 0, 1, ..., those of nodes path[b][0 .. path_len[b] - 1] move to
 * positions first_pos[b] + 0 .. path_len[b] - 1, bit for bit.  path [n_seqs][max_path]; its nodes ascend, and what comes
 * from the first that does not (or is negative) is ignored.  Where the old or the new position is outside nothing moves. */
int sjd_op_cache_compact(void *hip_stream, const sjd_kv_cache *cache, const int32_t *first_pos, const int32_t *path,
                         const int32_t *path_len, int32_t max_path);

/* Frequencies of a rotary embedding for sjd_op_rotary: table [rotary_dim / 2] (HOST; the caller copies it to the device), entry i =
 * f_i / (2 pi) in units of 2^-64 turns, f_i = theta^(-2i / rotary_dim) radians a position, scaled for contexts `factor` times
 * as long as the trained_ctx positions that a model was trained on:
 *   SJD_ROPE_PLAIN   not at all;
 *   SJD_ROPE_LINEAR  f_i / factor;
 *   SJD_ROPE_BASE    theta * factor^(rotary_dim / (rotary_dim - 2)) in place of theta (rotary_dim > 2);
 *   SJD_ROPE_PARTS   by how many turns n_i = trained_ctx * f_i / (2 pi) the pair makes: f_i from high_turns on, f_i / factor
 *                    up to low_turns, and between them f_i * (g + (1 - g) / factor), g = (n_i - low_turns) / (high_turns - low_turns).
 * rotary_dim: even, >= 2; theta > 1, factor >= 1 (LINEAR and on), trained_ctx > 0 and 0 <= low_turns < high_turns (PARTS). */
enum sjd_rope_scaling { SJD_ROPE_PLAIN = 0, SJD_ROPE_LINEAR = 1, SJD_ROPE_BASE = 2, SJD_ROPE_PARTS = 3 };
int sjd_rope_table(int32_t rotary_dim, double theta, int32_t scaling, double factor, double trained_ctx, double low_turns,
                   double high_turns, uint64_t *table);

/* Turns pairs of the first rotary_dim dimensions of every head by positions[row] * f_i and multiplies them by `magnitude`; the
 * other dimensions are copied.  Pairs are (i, i + rotary_dim / 2), or (2i, 2i + 1) with `interleaved`.  x and y [n_rows][heads][head_dim]
 * of `dtype` (heads contiguous, rows a stride apart), in one call for queries (n_heads) and keys (n_kv_heads; 0: none).  y may
 * be x with the same stride, and may not overlap it otherwise, nor the outputs each other (parts of one buffer's rows may lie between each
 * other).  Angles are less than 2^-32 turns off at any position; a negative position turns back.  head_dim <= 512. */
int sjd_op_rotary(void *hip_stream, int32_t dtype, int32_t interleaved, const uint64_t *table, int32_t rotary_dim, float magnitude,
                  const int32_t *positions, int32_t n_rows, int32_t head_dim, const void *q, int64_t q_stride, void *q_out,
                  int64_t q_out_stride, int32_t n_heads, const void *k, int64_t k_stride, void *k_out, int64_t k_out_stride,
                  int32_t n_kv_heads);

/* Masks and depths of a tree from its parents (all HOST): node i < n has parent parents[i] < i (negative: a root); bit j of
 * mask[i][j / 32] is set where node j is i or one of its ancestors, mask [n][mask_words]; depth[i] (may be NULL) = number
 * of ancestors.  SJD_EINVAL: a parent that does not come first, or mask_words * 32 < n. */
int sjd_tree_masks(const int32_t *parents, int32_t n, int32_t mask_words, uint32_t *mask, int32_t *depth);

/* Attention of the rows of trees over a cache that holds them already: node i of sequence b (row row_start[b] + i, position
 * ctx_len[b] + i) attends to positions [0, ctx_len[b]) and to those nodes j of its own tree whose bit j % 32 of
 * mask[row][j / 32] is set; with mask NULL to nodes 0 .. i (a window).  Row by row out = softmax(scale * q k) v with one kv head to
 * n_heads / n_kv_heads query heads; a row that sees nothing gets zeros, and so do the rows of a sequence whose ctx_len is negative.  Keys and values that a row does not see do not touch it,
 * infinities and NaN included; an infinite value that it does see makes its result infinite, and may make it NaN where its weight is below what fp32 holds.
 * q and out [n_rows][n_heads][head_dim] of `dtype`: SJD_F32 for an SJD_F32 cache, SJD_BF16 for the others.  Probabilities are rounded
 * to bf16 there, for the products with values and for the sum that divides, so that weights add up to 1; the sums are fp32.  (The mean error against 64
 * bits is up to 1.4 times that of a result that is only rounded to bf16 at the end.)  out may be q with the same stride, and may not
 * overlap it otherwise.  scale > 0, or 0 for 1 / sqrt(head_dim).
 * max_rows: no tree has more rows (those behind are left as they were).  max_ctx: what ctx_len is expected to reach; it only
 * chooses how the work is divided, and with it the order of sums.  The workspace (16-byte aligned) has at least the bytes that
 * sjd_op_tree_attention_workspace writes to *bytes (HOST; may be 0, then it may be NULL) for the same arguments.  SJD_ECAPACITY: it is smaller. */
int sjd_op_tree_attention_workspace(const sjd_kv_cache *cache, int32_t n_heads, int32_t max_rows, int32_t max_ctx, uint64_t *bytes);
int sjd_op_tree_attention(void *hip_stream, const sjd_kv_cache *cache, int32_t dtype, const void *q, int64_t q_stride, void *out,
                          int64_t out_stride, const int32_t *row_start, const int32_t *ctx_len, const uint32_t *mask, int32_t mask_words,
                          int32_t n_rows, int32_t n_heads, float scale, int32_t max_rows, int32_t max_ctx, void *workspace,
                          uint64_t workspace_bytes);

/* Verification of trees of drafted tokens: Eq. 2 and 3 of the paper for a node's drafted successors one after the other, from given
 * random words.  tokens and parents [n_rows]: node i of a sequence (row row_start[b] + i) carries a token and the index of its
 * parent, which is smaller; node 0 is the root (the last final token, which is not tested).  Row i of p [n_rows][vocab], p_stride apart: the
 * target's probabilities of what follows node i.  Row i of q: the draft model's, from which i's children were drawn; q NULL: they were
 * not drawn but chosen (a model's likeliest tokens), each a proposal of probability 1.
 * From node 0 on, the children x of the node reached, in the order of their indices:  with rho_0 = p and S_0 = 1, child k is
 * accepted where r q(x) S_k < rho_k(x), r = (accept_words[its row] + 1/2) 2^-32; if not, rho_{k+1} = max(0, rho_k - S_k q) and
 * S_{k+1} = sum rho_{k+1}.  Where no child is accepted next_token is drawn from the last rho (from p, where that is all 0).  Where
 * max_path nodes are reached it is drawn from the last one's p, and that node's children are not tested.  Drawn is the first id
 * whose cumulated weight exceeds the share draw_words[b] / 2^64 of all.  In distribution the accepted tokens and the
 * next one are what the target alone would have produced, whatever max_path is.  All of it is specified bit for bit: double
 * precision, the products in the order (r q) S and S q, sums of trunc(min(rho, 1) 2^44); a p that is negative or NaN is 0, and so is rho
 * from the rejection on that a NaN of q takes part in.  A token outside [0, vocab) is rejected.
 * Outputs: path [n_seqs][max_path], the nodes reached, node 0 first, -1 behind them; path_len [n_seqs] (accepted drafts + 1; 0 for a
 * sequence without rows); next_token [n_seqs] (-1 without rows, or where p is all 0).  path and path_len are what
 * sjd_op_cache_compact takes.  max_rows <= 1024, vocab <= 524288; rows of a tree behind max_rows are ignored.  With q, every rejected child of a node
 * costs a pass over the vocabulary, with a step an id for each one rejected before it.  The workspace
 * (16-byte aligned) as in sjd_op_tree_attention. */
int sjd_op_tree_verify_workspace(int32_t n_rows, int32_t n_seqs, int32_t vocab, uint64_t *bytes);
int sjd_op_tree_verify(void *hip_stream, const int32_t *tokens, const int32_t *parents, const int32_t *row_start, const float *p,
                       int64_t p_stride, const float *q, int64_t q_stride, const uint32_t *accept_words, const uint64_t *draw_words,
                       int32_t *path, int32_t *path_len, int32_t *next_token, int32_t n_rows, int32_t n_seqs, int32_t vocab,
                       int32_t max_rows, int32_t max_path, void *workspace, uint64_t workspace_bytes);

/* ---- operators of scoring and prefilling prompts: norms of queries and keys with their rotary positions, attention of packed prompts, log
 * probabilities of their tokens.  They are called as those of tree speculation above are: nothing is allocated, work is enqueued on `hip_stream`, pointers are DEVICE
 * pointers on its device, which is the current one, sizes and pointers are checked on the host, and what is in device memory by the kernels. */

/* sjd_op_rotary of heads that are normalised first, in one pass: y = (x - c) / sqrt(mean((x - c)^2) + eps) * gain + bias over the head_dim
 * elements of a head, c = 0 (SJD_NORM_RMS) or their mean (SJD_NORM_LAYER); then pairs of y are turned, and multiplied by `magnitude`, the other
 * dimensions are y.  Gains and biases of `dtype`: [head_dim] for all heads, or, with per_head, [heads][head_dim]; a bias may be NULL.  All of it is in fp32, rounded
 * once at the end; any finite x is right, also where its square is beyond fp32 (eps then counts as nothing); a head with an infinity or NaN has NaN in it.  1e-30 <= eps.  The other arguments and
 * conditions are those of sjd_op_rotary (in place included); outputs may not overlap gains and biases. */
enum sjd_head_norm { SJD_NORM_RMS = 0, SJD_NORM_LAYER = 1 };
int sjd_op_norm_rotary(void *hip_stream, int32_t dtype, int32_t norm, float eps, int32_t per_head, int32_t interleaved, const uint64_t *table,
                       int32_t rotary_dim, float magnitude, const int32_t *positions, int32_t n_rows, int32_t head_dim, const void *q, int64_t q_stride,
                       const void *q_gain, const void *q_bias, void *q_out, int64_t q_out_stride, int32_t n_heads, const void *k, int64_t k_stride,
                       const void *k_gain, const void *k_bias, void *k_out, int64_t k_out_stride, int32_t n_kv_heads);

/* Causal attention of packed prompts.  Sequence b's queries are rows [row_start[b], row_start[b + 1]) of q, its keys and values rows
 * [kv_start[b], kv_start[b + 1]) of k and v (kv_start NULL: the same rows, and n_kv_rows is not read), of which the last are its queries' own: of n queries and t
 * keys query i sees keys 0 .. i + t - n, so that a prompt may go on behind what is cached.  (row_start and kv_start have n_seqs + 1 entries, ascending; what lies outside [0, n_rows]
 * or [0, n_kv_rows] is cut off.)  Row by row out = softmax(scale * q k) v with one kv head to n_heads / n_kv_heads query heads; a query that sees nothing (t < n) gets
 * zeros.  Keys and values that a query does not see do not touch it, infinities and NaN included; an infinite value that it does see makes its result
 * infinite, and may make it NaN where its weight is below what fp32 holds.  Rows of no sequence are left as they were.
 * q and out [n_rows][n_heads][head_dim], k and v [n_kv_rows][n_kv_heads][head_dim] of `dtype` (SJD_F32 or SJD_BF16; a row's heads are contiguous, rows a stride
 * apart: parts of a fused projection); head_dim 32, 64, 96, 128, 192 or 256.  Sums are fp32; for SJD_BF16 probabilities are rounded to bf16 for the products
 * with values and for the sum that divides.  out may be q with the same stride, and may not overlap it otherwise, nor k and v.  scale > 0, or 0 for 1 / sqrt(head_dim).
 * max_kv: what a sequence's keys are expected to reach; it only chooses how the work is divided, and with it the order of sums and the workspace.  max_rows, the same of its
 * queries, is checked, and changes nothing.  Workspace (16-byte aligned): the bytes that sjd_op_prompt_attention_workspace writes to *bytes (HOST; may be 0) for the same
 * arguments.  SJD_ECAPACITY: it is smaller. */
int sjd_op_prompt_attention_workspace(int32_t dtype, int32_t n_rows, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_rows,
                                      int32_t max_kv, uint64_t *bytes);
int sjd_op_prompt_attention(void *hip_stream, int32_t dtype, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                            void *out, int64_t out_stride, const int32_t *row_start, const int32_t *kv_start, int32_t n_rows, int32_t n_kv_rows, int32_t n_seqs,
                            int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale, int32_t max_rows, int32_t max_kv, void *workspace,
                            uint64_t workspace_bytes);

/* Log probabilities.  Row r of logits [n_rows][vocab] (SJD_F32 or SJD_BF16, rows `stride` elements apart), p = softmax of it:
 *   logprob[r] = ln p(tokens[r]), rank[r] = number of ids that are likelier, or as likely and lower; for a token outside [0, vocab) -inf and -1;
 *   entropy[r] = - sum p ln p;
 *   top_ids, top_logprobs [n_rows][n_top]: the likeliest ids, the lower one first where they are as likely, and their ln p; -1 and -inf behind the last id whose logit
 *   is above -inf.
 * Logits may be -inf (masked ids); of a row that is -inf altogether every ln p is -inf and the entropy is 0.  A row that holds a NaN or +inf has NaN for its numbers, -1 for
 * its top_ids, and no meaning in its rank.  Sums are fp32; no ln p is above 0.  n_top 0 .. 64 (0: top_ids and top_logprobs may be NULL); vocab <= 2^24.  Outputs may not overlap each
 * other or an input.  Workspace as in sjd_op_prompt_attention. */
int sjd_op_token_logprobs_workspace(int32_t n_rows, int32_t vocab, int32_t n_top, uint64_t *bytes);
int sjd_op_token_logprobs(void *hip_stream, int32_t dtype, const void *logits, int64_t stride, const int32_t *tokens, float *logprob, int32_t *rank, float *entropy,
                          int32_t *top_ids, float *top_logprobs, int32_t n_rows, int32_t vocab, int32_t n_top, void *workspace, uint64_t workspace_bytes);

#ifdef __cplusplus
}
#endif
#endif
