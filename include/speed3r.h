/*
 * speed3r.h -- C ABI of the MI355X (gfx950) implementation of Speed3R's Global
 * Sparse Attention (GSA), Sec. 3.2 of the paper, forward pass, one scene
 * (batch omitted as in the paper), one GPU.
 *
 * The path (Sec. 3.2, eqs. 3-8; supplementary Alg. 1 and Alg. 2):
 *   1. pool      Q, K, V are mean-pooled over blocks of `block` tokens: runs of
 *                consecutive tokens (the last block may be short and is averaged
 *                over its valid tokens) or, on request, the paper's s x s spatial
 *                windows of every view's patch grid.
 *   2. scores    S_guide[h,i,j] = Qc[h,i] . Kc[h,j]                  (eq. 4)
 *   3. compress  Oc'[h,i] = softmax_j(scale * S_guide[h,i,:]) Vc[h]  (eq. 3)
 *   4. topk      per (h,i): the k = min(topk, n_blk) key blocks with the
 *                largest S_guide[h,i,:] ("Selection Branch"); all queries of a
 *                block share the set; stored ascending.
 *   5. select    O_sel[t,h] = softmax over the valid tokens of the selected
 *                blocks of (scale * q[t,h] . k[u,h]), times v      (eq. 6, Alg. 2)
 *   6. merge     out = g * Oc'[h, t / block] + (1 - g) * O_sel,
 *                g = sigmoid(gate_logits) or 1/2                   (eqs. 5, 7, 8)
 * and, as the comparison point, plain dense softmax attention (eq. 2 form).
 * Optional parts of the layer (fields of s3r_params): special tokens, which get
 * dense attention over all tokens (eqs. 1-2), a fixed set of key blocks every
 * query block attends besides its TopK (Sec. 3.3), spatial pooling windows,
 * unpooled queries in the compression branch.
 *
 * General conventions
 *   - Every data pointer is a DEVICE pointer unless stated otherwise; the
 *     caller owns all of them; the library never frees caller memory.
 *   - q, k, v, out, gate_logits, o_sel: layout [n_tok][heads][head_dim],
 *     contiguous, element type given by `dtype`, 16-byte aligned (q, k, v of
 *     speed3r_sparse_global_attn_ex may instead be strided, see stride_tok).
 *     Inputs are read-only and must not alias outputs.
 *   - n_blk = ceil(n_tok / block).  head_dim must be 64, block one of
 *     16, 32, 64, 128 (else S3R_ERR_UNSUPPORTED).  topk > n_blk is clamped.
 *     n_tok need not be a multiple of block.
 *   - All work is enqueued on `stream` (a hipStream_t passed as void*, NULL =
 *     the default stream); no call synchronises the host except where noted.
 *   - Every function returns a status code; speed3r_last_error() gives a
 *     message for the last failure on the calling thread.  Nothing is thrown.
 *   - Entry points that say "library-held scratch" keep one grow-only device
 *     buffer per process (allocated with hipMalloc on first use or growth;
 *     growth synchronises the device); calls using it must not overlap.
 */
#ifndef SPEED3R_H
#define SPEED3R_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    S3R_OK = 0,
    S3R_ERR_INVALID_ARG = 1, /* null / misaligned pointer, non-positive size ...   */
    S3R_ERR_UNSUPPORTED = 2, /* head_dim != 64, block not in {16,32,64,128}, dtype */
    S3R_ERR_WORKSPACE = 3,   /* caller workspace too small / allocation failed     */
    S3R_ERR_HIP = 4          /* a HIP runtime call or kernel launch failed         */
} s3r_status;

typedef enum { S3R_F32 = 0, S3R_BF16 = 1 } s3r_dtype;

/* Bits of the device status word (s3r_params.status). */
enum { S3R_DIAG_FORCED_RANGE = 1, S3R_DIAG_FORCED_ORDER = 2 };
/* Bits of the status word of the cache and cross attention calls: a page number outside [0, n_pages); a list of row
 * starts that is out of range or not ascending; a length outside the page table (for append and read also one below the
 * sequence's rows); a position outside the tables.  Asking for it is one more launch, which takes the cache calls half a microsecond for each
 * sequence. */
enum { S3R_DIAG_PAGE = 4, S3R_DIAG_SPANS = 8, S3R_DIAG_LENGTH = 16, S3R_DIAG_POSITION = 32 };

/* Stages of the path, for speed3r_get_stage_ms(). */
enum {
    S3R_STAGE_POOL = 0,     /* block pooling (+ K/V tile re-layout for the MFMA path); cache rows in and out; rotary positions and
                             * the residual stream's norms, forward and gradient      */
    S3R_STAGE_SPLIT = 1,    /* pooled fp32 -> operand tiles (+ their per-head statistics) */
    S3R_STAGE_COMPRESS = 2, /* S_guide + compressed attention (short sequences: + TopK) */
    S3R_STAGE_TOPK = 3,     /* per-query-block TopK (incl. its filter sweep)          */
    S3R_STAGE_SELECT = 4,   /* block-sparse attention + merge                         */
    S3R_STAGE_DENSE = 5,    /* dense, cross, causal and cache attention, and the gradients of cross and causal attention */
    S3R_N_STAGES = 6
};

typedef struct s3r_params {
    const void *q, *k, *v;   /* in   [n_tok][heads][head_dim] (or stride_tok, stride_head below)  */
    void *out;               /* out  [n_tok][heads][head_dim], merged result (eq. 8)            */
    const void *gate_logits; /* in, optional (NULL: g = 1/2), same layout and dtype as q        */
    /* Forced blocks (Sec. 3.3: the fixed global context of the VGGT variant, e.g. all blocks of the
     * reference view): n_forced block indices in DEVICE memory that every query block attends in
     * addition to its TopK, which then runs over the other blocks only.  The list must be strictly
     * ascending and within [0, n_blk).  The library cannot look at device memory without a host
     * synchronisation, which it never does: a list that breaks this is reported through `status`
     * below; the call itself then runs on the list with its entries clamped into range (memory-safe;
     * a block listed twice is attended twice, so the result is not the paper's). */
    const int32_t *forced_blocks; /* in, optional (NULL: none)                                   */
    int n_forced;            /* 0 when forced_blocks is NULL                                    */
    /* out, optional: one device word, written by the call (stream-ordered like every output): 0, or
     * S3R_DIAG_FORCED_RANGE | S3R_DIAG_FORCED_ORDER for a forced_blocks list with an entry outside
     * [0, n_blk) / not strictly ascending.  4-byte aligned. */
    int32_t *status;
    /* Special tokens (Sec. 3.2 eqs. 1-2 and "Final Output"): the n_tok rows come in views of
     * tokens_per_view rows, the first special_per_view of each being special (camera / register)
     * tokens.  Those rows get plain softmax attention over ALL n_tok rows; the remaining image rows,
     * taken in order, form the sequence the sparse path works on (blocks, TopK, forced blocks and the
     * optional block-level outputs all refer to that image-only sequence); every result is written to
     * the row it belongs to.  Both 0: no special tokens.  tokens_per_view = n_tok with the special
     * tokens first is the paper's own [X_spec; X_img] arrangement. */
    int tokens_per_view;     /* 0, or a divisor of n_tok                                        */
    int special_per_view;    /* 0 <= special_per_view < tokens_per_view                         */
    /* Spatial pooling windows (Sec. 3.2: non-overlapping s x s average pooling on each image's patch
     * grid).  The tokens_per_view - special_per_view image rows of a view are a row-major grid_h x
     * grid_w grid; blocks are its window x window windows (block must equal window * window), taken in
     * row-major order over the grid, views one after another: n_blk = views * ceil(grid_h / window) *
     * ceil(grid_w / window).  Windows on the right and bottom edges are cut where the grid ends and hold
     * fewer tokens.  All 0: blocks are runs of `block` consecutive image rows. */
    int grid_h, grid_w, window;
    /* Queries of the compression branch.  0: pooled like the keys (Q_comp, eq. 3; the paper's form): one
     * compressed output per block, upsampled to its tokens (eq. 5).  1: every image row's own query
     * attends the pooled keys, O_comp[t] = softmax_j(scale * q[t] . Kc[j]) Vc, and that row's result is
     * merged (eq. 8); block scores and TopK remain those of the pooled queries, and the optional
     * output o_comp remains the per-block result.  bf16 data: Kc and Vc enter this product rounded to
     * bf16.  Costs n_tok x n_blk attention (at 1000 views several times the rest of the path). */
    int compress_queries;
    int64_t n_tok;
    /* Layout of q, k and v (all three alike; Sec. 3.2 takes Q, K, V as given, e.g. as three views of one
     * packed projection output): elements between consecutive rows and between heads; the head_dim
     * channels of a head are contiguous.  0: the packed default (stride_tok = heads * head_dim,
     * stride_head = head_dim).  Multiples of 8 elements.  out, gate_logits and o_sel are always packed. */
    int64_t stride_tok, stride_head;
    int heads, head_dim, block, topk;
    s3r_dtype dtype;
    float softmax_scale;     /* <= 0: 1/sqrt(head_dim).  Used by both branches.                 */
    /* w = speed3r_selected_per_row(n_tok, block, topk, n_forced) blocks per row: */
    int32_t *topk_idx;       /* out, optional: [heads][n_blk][w] ascending block indices        */
    float *lse_sel;          /* out, optional: [heads][n_tok], Alg. 2's L (natural log); special
                                rows are left untouched, and so are theirs in o_sel               */
    float *o_comp;           /* out, optional: [heads][n_blk][head_dim] fp32, Oc' of eq. 3      */
    void *o_sel;             /* out, optional: [n_tok][heads][head_dim], O_sel of eq. 6         */
    void *workspace;         /* caller-owned device scratch, 256-byte aligned                   */
    size_t workspace_bytes;  /* >= speed3r_workspace_bytes(...) for the same problem            */
    void *stream;            /* hipStream_t                                                     */
} s3r_params;

/* Bytes of device scratch speed3r_sparse_global_attn_ex needs (0 on invalid arguments) for
 * the given n_forced (0 without forced blocks). */
size_t speed3r_workspace_bytes(int64_t n_tok, int heads, int head_dim, int block, int topk, int n_forced,
                               s3r_dtype dtype);

/* The same from a filled-in parameter block (only its shape fields are read: n_tok, heads, head_dim,
 * block, topk, dtype, n_forced, tokens_per_view, special_per_view); needed with special tokens.
 * Special rows run in key splits, whose partial results take room here; they are more than the time alone asks for,
 * for their precision, and a workspace that holds only the leaner number is accepted too: the call then runs in that many. */
size_t speed3r_workspace_bytes_ex(const s3r_params *p);

/* Number of blocks n_blk of the sequence the sparse path works on, for a filled-in parameter block
 * (shape fields only); -1 on invalid arguments. */
int64_t speed3r_num_blocks(const s3r_params *p);

/* Key blocks each query block attends: n_forced + min(topk, n_blk - n_forced) (Sec. 3.3), or
 * min(topk, n_blk) without forced blocks; -1 on invalid arguments. */
int speed3r_selected_per_row(int64_t n_tok, int block, int topk, int n_forced);

/* The whole GSA path (steps 1-6 above; Sec. 3.2, eqs. 3-8).  Re-entrant across streams when each
 * call has its own workspace.  Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, HIP. */
s3r_status speed3r_sparse_global_attn_ex(const s3r_params *params);

/* Short form of the above: bf16, scale 1/sqrt(head_dim), no gate (g = 1/2), library-held scratch.
 * Returns an s3r_status as int. */
int speed3r_sparse_global_attn(const void *q, const void *k, const void *v, void *out,
                               int64_t n_tok, int heads, int head_dim, int block, int topk,
                               void *stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc): the short form above with its scratch in a fixed device array of
 * S3R_STATIC_SCRATCH_BYTES that is part of the library's code object, so the call performs no hipMalloc,
 * hipFree, event creation or any other allocating call; every GPU the library runs on holds its own copy of
 * that array until the process ends.  Same arguments, same kernels and bit-identical results as
 * speed3r_sparse_global_attn.  Problems whose speed3r_workspace_bytes(..., n_forced = 0, S3R_BF16) exceeds
 * S3R_STATIC_SCRATCH_BYTES are refused with S3R_ERR_WORKSPACE before anything is enqueued (8 views x 1374
 * tokens x 16 heads, block 64, top-16 needs 57 MiB and fits).  All calls on one GPU share that GPU's array:
 * calls that overlap in time on one GPU (different streams or threads) race; calls ordered on one stream are
 * fine, and no call depends on what an earlier one left in the array. */
#define S3R_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
int speed3r_sparse_global_attn_noalloc(const void *q, const void *k, const void *v, void *out,
                                       int64_t n_tok, int heads, int head_dim, int block, int topk,
                                       void *stream);

/* Dense softmax attention over all n_tok keys (eq. 2 form): out[t,h] = softmax_u(scale q.k) v.
 * The speed-up denominator.  lse (optional) is [heads][n_tok].  Library-held scratch. */
s3r_status speed3r_dense_attn(const void *q, const void *k, const void *v, void *out, float *lse,
                              int64_t n_tok, int heads, int head_dim, s3r_dtype dtype,
                              float softmax_scale, void *stream);

/* ---- stage entry points (per-kernel parity tests and profiling) ---------------------------- */

/* Step 1 (Sec. 3.2 "Compression Branch"): block means of q, k, v.
 * qc, kc, vc: out, fp32 [heads][n_blk][head_dim]. */
s3r_status speed3r_pool_blocks(const void *q, const void *k, const void *v, float *qc, float *kc,
                               float *vc, int64_t n_tok, int heads, int head_dim, int block,
                               s3r_dtype dtype, void *stream);

/* Steps 2-3 (eqs. 3-4; Alg. 1 without its TopK part) on pooled fp32 tensors.
 *   qc, kc, vc : in  fp32 [heads][n_blk][head_dim]
 *   s_guide    : out fp32 [heads][n_blk][ld_s], unscaled scores; ld_s >= n_blk, ld_s % 4 == 0;
 *                columns n_blk..ld_s-1 of a row are scratch (unspecified values)
 *   o_comp     : out fp32 [heads][n_blk][head_dim]
 *   accurate_pv: nonzero computes P.Vc with bf16 hi+lo operand pairs (fp32-level accuracy,
 *                used for S3R_F32 problems); zero uses single bf16 operands.
 * Library-held scratch. */
s3r_status speed3r_compress_attn_scores(const float *qc, const float *kc, const float *vc,
                                        float *s_guide, int64_t ld_s, float *o_comp, int64_t n_blk,
                                        int heads, int head_dim, float softmax_scale,
                                        int accurate_pv, void *stream);

/* Steps 2-4 in one go, without S_guide in memory (Sec. 3.2 "Efficient Kernel Implementation",
 * supplementary Sec. 1): compressed attention and, for every query block, the ascending indices of the
 * k = min(topk, n_blk) pooled keys with the largest scores; equal scores go to the smaller index.
 *   qc, kc, vc : in  fp32 [heads][n_blk][head_dim]
 *   o_comp     : out fp32 [heads][n_blk][head_dim]
 *   idx        : out int32 [heads][n_blk][k]
 *   accurate_pv: nonzero keeps the logits of the compressed softmax and the P.Vc product at fp32
 *                accuracy (bf16 hi+lo operand pairs; used for S3R_F32 problems); zero computes them
 *                from single fp16 / bf16 operands (logits good to 2^-10 |q||k|).  The index sets do
 *                not depend on it: they are decided by fp32 dot products either way.
 * Requires k <= 64 (S3R_ERR_UNSUPPORTED otherwise: use the two entry points around this one).
 * Should the scores of a row tie so massively that its candidate lists run over, the call falls back,
 * on the device, to scores written to library scratch; the result is the same.  Library-held scratch. */
s3r_status speed3r_compress_attn_topk(const float *qc, const float *kc, const float *vc, float *o_comp,
                                      int32_t *idx, int64_t n_blk, int heads, int head_dim, int topk,
                                      float softmax_scale, int accurate_pv, void *stream);

/* Step 4 (TopKSelect): idx[h][i][0..k) = ascending indices of the k = min(topk, n_blk) largest
 * entries of s_guide[h][i][0..n_blk); equal scores go to the smaller index.  Deterministic.
 * s_guide must hold no NaN. */
s3r_status speed3r_topk_blocks(const float *s_guide, int64_t ld_s, int32_t *idx, int64_t n_blk,
                               int heads, int topk, void *stream);

/* Steps 5-6 (eq. 6 / Alg. 2, then eqs. 5, 7, 8) with a given index tensor.
 *   idx     : in  [heads][n_blk][kk] block indices in [0, n_blk), distinct per row; 1 <= kk <= n_blk
 *             (entries outside the range are held into it, so that a broken list stays memory-safe; a
 *             block listed twice is attended twice)
 *   o_comp  : in, optional fp32 [heads][n_blk][head_dim]; NULL: `out` receives O_sel unmerged
 *   gate_logits, o_sel, lse: as in s3r_params (all optional)
 * Library-held scratch. */
s3r_status speed3r_select_attn(const void *q, const void *k, const void *v, const int32_t *idx,
                               const float *o_comp, const void *gate_logits, void *out, void *o_sel,
                               float *lse, int64_t n_tok, int heads, int head_dim, int block, int kk,
                               s3r_dtype dtype, float softmax_scale, void *stream);

/* ---- cross attention and its gradient --------------------------------------------------------- */

/* out[i,h] = softmax_j(scale q[i,h] . k[j,h']) v[j,h'] with keys of another length than the queries: a decoder's rows over the
 * states of a scene (dense attention, eq. 2 form, is the case q, k, v of one length).  heads is a multiple of kv_heads; query head h
 * reads head h' = h / (heads / kv_heads) of k and v.
 *   Batches: sequences lie one behind the other; sequence b has query rows q_start[b] .. q_start[b+1] - 1 and keys kv_start[b] ..
 *   kv_start[b+1] - 1 (both may be none).  The starts are in DEVICE memory, ascending, within [0, n_q] and [0, n_kv].  A list that breaks
 *   this is reported through `status`; the call then runs on entries held into range (memory-safe).  Rows outside all sequences are
 *   left as they were, in outputs and gradients alike.
 *   Mask: keys with key_mask 0 take no part, whatever their k and v hold (padding, invalid patches); their gradients are 0.
 *   A query row without any key, or whose scores are all -inf, gets out = 0 and lse = -inf; without any key its gradient is 0.
 *   Limits: 65536 sequences, batch * kv_heads 2^19, rows * heads 2^28 (the cache calls: rows * (heads + 2 kv_heads)).
 *   Sums, maxima and log-sums are fp32.  bf16 data: probabilities (and dS, in the gradient) enter the second product rounded to
 *   bf16 (errors of the results up to about 1.4 times that of rounding them); those of few rows in two bf16 parts (errors of the rounding
 *   alone): in the forward call of up to 64 (keys and values of up to 16 MiB together), 32 (48 MiB) or 16 rows, in the gradient of up to 64,
 *   counting those of all heads that share one, on average over the batch; in the gradient of causal rows the last 64 of a sequence, in what they give
 *   to the last keys.  A sequence's last bits thus depend on the lengths in its batch.  accurate_pv: two parts for all rows (causal or not; a fifth to a half more
 *   time where there are many).
 *   fp32 data: products in bf16 parts, each off by up to 2^-21 of its magnitude (operands below 2^-102 keep fewer bits).
 *   Infinities: bf16 v and d_out: one in v reaches out, and one in d_out reaches dv, as an infinity, where its weight is above 2^-100; dq
 *   and dk are then infinities or NaN.  fp32 v and d_out: it may come out as NaN.
 *   The gradient takes out and lse as the forward call left them; the gradients of shared heads are summed.  Its results do not
 *   depend on the order in which workgroups run. */
typedef struct s3r_cross_params {
    const void *q;           /* in  [n_q][heads][64] (or q_stride_*)                                    */
    const void *k, *v;       /* in  [n_kv][kv_heads][64] (or kv_stride_*)                               */
    void *out;               /* out [n_q][heads][64]; the gradient reads it                              */
    float *lse;              /* out, optional [heads][n_q], natural log; the gradient reads it (required) */
    const void *d_out;       /* gradient: in [n_q][heads][64]                                            */
    void *dq, *dk, *dv;      /* gradient: out [n_q][heads][64], [n_kv][kv_heads][64] twice               */
    const int32_t *q_start, *kv_start; /* in, optional [batch + 1] (both NULL: one sequence of all rows) */
    const uint8_t *key_mask; /* in, optional [n_kv]                                                      */
    int32_t *status;         /* out, optional: one device word, 0 or S3R_DIAG_SPANS                      */
    int64_t n_q, n_kv;       /* rows of the tensors; 0 is allowed (their pointers are then not read)     */
    int64_t q_stride_tok, q_stride_head;   /* elements between rows and heads of q (0: packed), multiples of 8 */
    int64_t kv_stride_tok, kv_stride_head; /* of k and of v                                               */
    int batch;               /* sequences; 1 (or 0) without starts                                       */
    int heads, kv_heads, head_dim;
    s3r_dtype dtype;
    float softmax_scale;     /* <= 0: 1/sqrt(head_dim)                                                   */
    void *workspace;         /* caller-owned device scratch, 256-byte aligned                            */
    size_t workspace_bytes;  /* >= speed3r_cross_workspace_bytes(...)                                    */
    void *stream;
    int accurate_pv;         /* nonzero: bf16 probabilities and dS in two parts, however many rows       */
} s3r_cross_params;

/* Bytes of device scratch that the forward call (backward 0) or the gradient (1) needs; only the shape fields are read.  May be 0;
 * SIZE_MAX on invalid arguments. */
size_t speed3r_cross_workspace_bytes(const s3r_cross_params *p, int backward);
s3r_status speed3r_cross_attn(const s3r_cross_params *p);
s3r_status speed3r_cross_attn_backward(const s3r_cross_params *p);

/* The same over packed sequences whose rows are their LAST tokens (of n rows and m keys, row i is token m - n + i; all m are those of the
 * sequence, n = m: a prompt over itself, n < m: new tokens over earlier ones): a row sees the tokens of its own view of tokens_per_view
 * tokens and of the views before.  tokens_per_view 1: causal by token, up to the row itself; a view's tokens see one another otherwise, as views that arrive
 * one after another do.  Everything else, p's fields, masks, broken lists, workspaces and arithmetic, is as above.  A row before the first key (n > m)
 * sees none.  What stands in k and v of tokens that a row does not see, or in q and d_out of rows that do not see a key, takes no part in its
 * results, infinities and NaN included; their last bits may differ with it, within the errors above (32 rows decide together when to look for a larger
 * maximum, which is the unit that probabilities are rounded in).  bf16: an infinity in v stays one in the rows that see it, whatever its weight, where some of a
 * tile's 128 rows (those of all heads that share keys count; of few rows 16) do not see all of its unit of 64 keys; elsewhere as above. */
size_t speed3r_causal_workspace_bytes(const s3r_cross_params *p, int tokens_per_view, int backward);
s3r_status speed3r_causal_attn(const s3r_cross_params *p, int tokens_per_view);
s3r_status speed3r_causal_attn_backward(const s3r_cross_params *p, int tokens_per_view);

/* ---- a cache of keys and values in 4 bits ------------------------------------------------------ */

/* Views (or tokens) that arrive one after another: keys and values of earlier rows are kept in pages, 34 bytes for the 64 channels of a
 * head.  The form is that of the microscaling formats (MXFP4): 32 channels share a power of two 2^e, the smallest in [-100, 125] with
 * max |x| < 7 * 2^e, and each is the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} * 2^e, ties to the even code.  Magnitudes from
 * 6 * 2^125 on are held as 6 * 2^125, those below 2^-102 as 0; a block of 32 with a NaN or an infinity reads as NaN.
 *   Pages: `page` tokens each (16, 32, 64 or 128; many rows attend up to a tenth faster over pages of 128 than of 32).  Token t of sequence b is token t % page of page page_table[b][t / page].
 *   A sequence has kv_len[b] tokens.  page_table and kv_len are in DEVICE memory, so that a captured graph may be replayed with other contents;
 *   a broken entry is reported through `status`, and memory-safe: lengths are held into the table, and tokens on a page outside
 *   [0, n_pages) are not written, read as 0 and are not attended.
 *   Rows: those of sequence b are row_start[b] .. row_start[b+1] - 1 (as in s3r_cross_params) and are its LAST tokens: of n rows,
 *   row i is token kv_len[b] - n + i.  kv_len counts the rows of the call.  Rows outside all sequences are left as they were.  */
typedef struct s3r_cache_params {
    uint8_t *k_codes, *v_codes;   /* [n_pages][kv_heads][page][32], channels 2 i (low half) and 2 i + 1 in byte i; 16-byte aligned */
    uint8_t *k_scales, *v_scales; /* [n_pages][kv_heads][page][2], e + 127 of channels 0..31 and 32..63; 255: NaN                   */
    const int32_t *page_table;    /* [batch][max_pages]                                                  */
    const int32_t *kv_len;        /* [batch]                                                             */
    const int32_t *row_start;     /* [batch + 1], NULL: one sequence of all n_rows rows                  */
    int64_t n_pages, n_rows;      /* n_rows may be 0                                                     */
    int page, max_pages, batch;
    int heads, kv_heads, head_dim;
    s3r_dtype dtype;              /* of q, k, v and out                                                  */
    const void *q;                /* append: in, optional, rotated into out; attention: in [n_rows][heads][64] */
    void *out;                    /* [n_rows][heads][64]: q rotated; attention                           */
    void *k, *v;                  /* append: in; read: out [n_rows][kv_heads][64] (or kv_stride_*)       */
    int64_t q_stride_tok, q_stride_head, kv_stride_tok, kv_stride_head; /* 0: packed; multiples of 8 elements */
    /* append: rotation of k and q, or NULL: none.  The 64 channels of a head are rot_axes (1 or 2) groups, each with a position of
     * its own (2: row and column of a patch); a group's channels are turned in pairs, i and i + half a group (rot_neighbours 0) or 2 i and
     * 2 i + 1 (1), by the angle with cosine cos[position][i].  Computed in 64 bits and rounded once. */
    const float *cos, *sin;       /* [n_positions][32 / rot_axes], 16-byte aligned                       */
    const int32_t *positions;     /* [n_rows][rot_axes]; NULL (rot_axes 1): the row's token number.  Held into [0, n_positions) */
    int64_t n_positions;
    int rot_axes, rot_neighbours;
    /* attention */
    int causal;                   /* 1: row i of n sees tokens 0 .. kv_len - n + i; 0: all kv_len        */
    float softmax_scale;          /* <= 0: 1/sqrt(head_dim)                                              */
    float *lse;                   /* out, optional [heads][n_rows], natural log                          */
    int32_t *status;              /* out, optional: one device word, 0 or S3R_DIAG_* bits                */
    void *workspace;              /* attention: caller-owned device scratch, 256-byte aligned            */
    size_t workspace_bytes;       /* >= speed3r_cache_workspace_bytes(...)                               */
    void *stream;
} s3r_cache_params;

/* Keys and values of the rows go to the cache, k rotated; q rotated goes to out, which must not be q, k or v.  One launch.  Two rows of a call must not be the
 * same token of the same page (which of them is kept is not specified). */
s3r_status speed3r_cache_append(const s3r_cache_params *p);
/* The rows' tokens as values: what the cache holds for them, exactly (to k and v). */
s3r_status speed3r_cache_read(const s3r_cache_params *p);
/* out = softmax(scale q . k) v over the cached tokens that a row sees; a row that sees none (or only scores of -inf) gets out = 0,
 * lse = -inf.  q is taken as it is (rotated by append).  NaNs in the cache reach only the rows that see them.  Sums, maxima and log-sums are fp32; cached values enter
 * exactly; bf16 rows: probabilities enter the second product rounded to bf16. */
s3r_status speed3r_cache_attn(const s3r_cache_params *p);
/* Bytes of device scratch of speed3r_cache_attn; only the shape fields are read.  May be 0; SIZE_MAX on invalid arguments. */
size_t speed3r_cache_workspace_bytes(const s3r_cache_params *p);

/* ---- rotary positions with the norm of a head ------------------------------------------------- */

typedef enum { S3R_NORM_NONE = 0, S3R_NORM_RMS = 1, S3R_NORM_LAYER = 2 } s3r_norm;
typedef enum { S3R_PAIRS_HALVES = 0, S3R_PAIRS_NEIGHBOURS = 1, S3R_PAIRS_WHOLE = 2 } s3r_pairs;

/* What q and k go through before any of the attentions: every head's 64 channels are normed (or not), n = norm(x) weight + bias, and
 * pairs of channels turned by the angles of the row's positions, one for each axis (time or view, row, column):
 *   out_a = n_a cos - n_b sin,  out_b = n_b cos + n_a sin.
 *   Axes: axis x has axis_pairs[x] pairs, P = their sum <= 32; pair p of all (those of axis 0 first) takes
 *   cos[position of its axis][p].  Channels that are in no pair are not turned.
 *   Pairs: S3R_PAIRS_HALVES: the channels of an axis are a group of 2 axis_pairs[x], of which i and i + axis_pairs[x] are a pair;
 *   S3R_PAIRS_NEIGHBOURS: channels 2 p and 2 p + 1;  S3R_PAIRS_WHOLE: channels p and P + p.
 *   Norm: over a head's channels, S3R_NORM_LAYER (x - mean) / sqrt(variance + eps) or S3R_NORM_RMS x / sqrt(mean of squares + eps), for
 *   magnitudes up to 2^56; everything is computed in fp32 and rounded once.
 * Either of q and k may be absent (heads or kv_heads 0); heads need not be a multiple of kv_heads.
 * The gradient takes those of q_out and k_out and, with a norm, q and k again.  The gradients of weights are sums over all rows and heads, in
 * an order that does not depend on that of the workgroups, up to 16 terms and then four sums in fp32, the rest in 64 bits.  Without a norm q, k, and weights are not read. */
typedef struct s3r_rotary_params {
    const void *q, *k;            /* in  [n_rows][heads][64], [n_rows][kv_heads][64] (or *_stride_*)     */
    void *q_out, *k_out;          /* out, packed; must not alias inputs                                  */
    const void *d_q_out, *d_k_out; /* gradient: in, packed                                               */
    void *dq, *dk;                /* gradient: out (or d*_stride_*: parts of one gradient of a projection) */
    const void *q_weight, *q_bias, *k_weight, *k_bias;     /* in, optional [64] of weight_dtype (1 and 0) */
    void *dq_weight, *dq_bias, *dk_weight, *dk_bias;       /* gradient: out, optional, of weight_dtype    */
    const float *cos, *sin;       /* [n_positions][P], 16-byte aligned; NULL with axes 0: no rotation    */
    const int32_t *positions;     /* [n_rows][axes]; NULL (axes 1): the row's number.  Held into [0, n_positions) */
    int32_t *status;              /* out, optional: one device word, 0 or S3R_DIAG_POSITION              */
    int64_t n_rows, n_positions;  /* n_rows may be 0; rows * (heads + kv_heads) at most 2^28             */
    int64_t q_stride_tok, q_stride_head, k_stride_tok, k_stride_head;     /* elements, 0: packed; multiples of 8 */
    int64_t dq_stride_tok, dq_stride_head, dk_stride_tok, dk_stride_head;
    int heads, kv_heads, head_dim;
    s3r_dtype dtype, weight_dtype;
    int axes;                     /* 0 .. 3                                                              */
    int axis_pairs[3];
    s3r_pairs pairs;
    s3r_norm norm;
    float eps;                    /* with a norm: positive                                               */
    void *workspace;              /* gradient: caller-owned device scratch, 256-byte aligned             */
    size_t workspace_bytes;       /* >= speed3r_rotary_workspace_bytes(...)                              */
    void *stream;
} s3r_rotary_params;

s3r_status speed3r_rotary(const s3r_rotary_params *p);
s3r_status speed3r_rotary_backward(const s3r_rotary_params *p);
/* Bytes of device scratch of the gradient.  May be 0; SIZE_MAX on invalid arguments. */
size_t speed3r_rotary_workspace_bytes(const s3r_rotary_params *p);

/* ---- the residual stream with the norms around a block ------------------------------------------ */

/* The end of one block and the start of the next:
 *   r = x + residual_scale * scale * gate * u,  u = post-norm(f) post_weight + post_bias (or f);   y = norm(r) weight + bias
 * for rows of `width` channels: x is the residual stream, f what the block adds to it, scale a learned factor for each channel, gate one
 * for each channel of each sequence.  Only x is required: without f, r is x; y, r, and every weight may be absent (NULL).
 *   Norms: as in s3r_rotary_params, over the `width` channels, for magnitudes up to 2^56.  Everything is computed in fp32 and rounded once:
 *   y is the norm of r before its rounding.
 *   Sequences: with gates, those of sequence b are the rows row_start[b] .. row_start[b+1] - 1 (DEVICE memory; broken lists as in
 *   s3r_cross_params); rows outside all sequences are left as they were, in r, y, dx and df.  row_start NULL: one sequence of all rows.
 *   Types: the stream (x, r and their gradients) is of x_dtype: dtype, or fp32 with everything else in bf16.  weights, biases and scale
 *   are of weight_dtype, gates of dtype.
 * The gradient takes those of y and r (either may be NULL: 0), x and f again, and gives
 * those of x, f and of every weight that is asked for, sums in an order that does not depend on that of the workgroups, of which at most
 * 256 terms and 32 sums of these are added one after the other in fp32, and all beyond that in 64 bits. */
typedef struct s3r_residual_params {
    const void *x, *f;            /* in  [n_rows][width] (or *_stride)                                   */
    void *r, *y;                  /* out, packed; r may be x itself where x is packed                    */
    const void *weight, *bias, *post_weight, *post_bias, *scale;   /* in, optional [width]               */
    const void *gate;             /* in, optional [batch][width] (or gate_stride)                        */
    const int32_t *row_start;     /* in, optional [batch + 1]; with gates                                */
    const void *d_r, *d_y;        /* gradient: in, packed                                                */
    void *dx, *df;                /* gradient: out, packed; df with f                                    */
    void *d_weight, *d_bias, *d_post_weight, *d_post_bias, *d_scale; /* gradient: out, optional [width]  */
    void *d_gate;                 /* gradient: out, optional [batch][width], packed                      */
    int32_t *status;              /* out, optional: one device word, 0 or S3R_DIAG_SPANS                 */
    int64_t n_rows;               /* 0 .. 2^28                                                           */
    int64_t x_stride, f_stride, gate_stride; /* elements between rows, 0: packed; multiples of 8         */
    int width;                    /* a multiple of 8 up to 8192                                          */
    int batch;                    /* sequences; 1 (or 0) without row_start; at most 65536                */
    s3r_dtype x_dtype, dtype, weight_dtype;
    s3r_norm norm, post_norm;     /* of r (needed for y), and of f                                       */
    float eps;                    /* with a norm: positive                                               */
    float residual_scale;         /* finite; 0: 1                                                        */
    void *workspace;              /* gradient: caller-owned device scratch, 256-byte aligned             */
    size_t workspace_bytes;       /* >= speed3r_residual_workspace_bytes(...)                            */
    void *stream;
} s3r_residual_params;

s3r_status speed3r_residual_norm(const s3r_residual_params *p);
s3r_status speed3r_residual_norm_backward(const s3r_residual_params *p);
/* Bytes of device scratch of the gradient (those of weights count where their pointers are given).  May be 0; SIZE_MAX on invalid arguments. */
size_t speed3r_residual_workspace_bytes(const s3r_residual_params *p);

/* ---- utilities ------------------------------------------------------------------------------ */

/* Measurement of what the data movement of the selection stage (eq. 6 / Alg. 2) costs by itself: the
 * selection kernel for bf16 blocks of 64 or 128 tokens with its arithmetic taken out.  It walks idx
 * ([heads][n_blk][kk], as in speed3r_select_attn) with the same work mapping, brings every selected K/V
 * unit into LDS through the same ring with the same waits and barriers, reads Q and writes `out` (which
 * receives a copy of q).  Time it with speed3r_set_profiling / speed3r_get_stage_ms (stage SELECT): the
 * real kernel cannot be faster than this on the same index lists.
 *   ring_stages: 0 or 2 = the real kernels' two-stage LDS ring; 3, 4 = deeper rings (more units on their
 *                way per workgroup);
 *   wg_per_cu  : 0 = as many workgroups per CU as fit (the real kernels' five); 1..5 = at most that many
 *                (fewer query blocks in progress per XCD: more of the units neighbouring query blocks share
 *                are still in that XCD's L2 when the second one asks).
 * Library-held scratch. */
s3r_status speed3r_probe_select_loads(const void *q, const void *k, const void *v, const int32_t *idx,
                                      void *out, int64_t n_tok, int heads, int head_dim, int block, int kk,
                                      int ring_stages, int wg_per_cu, void *stream);

/* When enabled, every entry point brackets each kernel launch with HIP events on the call's own
 * stream and keeps them until speed3r_get_stage_ms reads them (process-wide switch; default off). */
s3r_status speed3r_set_profiling(int enable);

/* Host arrays of S3R_N_STAGES entries: summed kernel milliseconds and number of launches per
 * stage over all profiled calls since the previous speed3r_get_stage_ms (or since profiling was
 * switched on); the record is cleared.  Waits for the recorded events, so call it after the work. */
s3r_status speed3r_get_stage_ms(float *ms, int *launches);

/* Selects kernel families, process-wide.  0 = automatic: MFMA attention kernels (fp32 problems in bf16
 * operand parts), and for up to 64 TopK blocks per row the TopK that runs
 * inside the compression sweep, or with it in one launch, without writing
 * S_guide to memory (supplementary Sec. 1).  1 = always
 * the generic attention kernel.  2 = like 0 but TopK always from S_guide written to memory. */
s3r_status speed3r_set_kernel_choice(int choice);

/* Frees the library-held scratch (synchronises the device). */
s3r_status speed3r_release_scratch(void);

/* Message for the last non-OK status on this thread (static storage, never NULL). */
const char *speed3r_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SPEED3R_H */
