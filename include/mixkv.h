/*
 * mixkv.h -- C ABI of libmixkv: MixKV's prefill-time KV-cache compression step
 * on one MI355X (gfx950).
 *
 * For every layer l and KV head h the library scores each cached key, mixes an
 * importance score with a diversity score according to the head's redundancy,
 * keeps the top-B entries and gathers the kept K/V rows into a compacted cache
 * (paper: Sec. 3.1 "KV Cache Compression" for the operator; Sec. 3.2 for the
 * importance and diversity scores; Sec. 3.3, Eq. 3-5 for the redundancy and the
 * head-wise mix; Appendix Algorithm 1 for the whole loop).
 *
 * Conventions
 *   Pointers   Members of mixkv_layer_in / mixkv_layer_out and `workspace` are
 *              DEVICE pointers owned by the caller.  The params struct and the
 *              arrays of layer structs are HOST memory, read during the call only.
 *   Ownership  The library allocates no device memory and keeps no state between
 *              calls.  Two calls may run concurrently on different streams if they
 *              use different workspaces and outputs.
 *   Ordering   All work is enqueued on `hip_stream` (a hipStream_t, NULL = the
 *              default stream).  Calls return without synchronising; outputs are
 *              valid once the stream has been synchronised.
 *   Errors     Every entry point returns a mixkv_status.  Arguments are validated
 *              on the host before anything is launched; on an argument error no
 *              output is touched.  HIP launch failures map to MIXKV_ERR_HIP.
 *   Notation   N cached tokens (the paper's T), D head dim, W window length,
 *              B budget per head (window included), B' = B - W (Algorithm 1),
 *              Nc = N - W candidates, G = n_q_heads / n_kv_heads.
 *   Layout     K, V: [batch, n_kv_heads, N, D], D contiguous, strides in elements.
 *              Qwin: [batch, n_q_heads, W, D] contiguous; query head g serves KV
 *              head g / G.  Row starts must be 16-byte aligned.
 */
#ifndef MIXKV_H
#define MIXKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MIXKV_VERSION 12
#define MIXKV_MAX_LAYERS 128      /* layers per call */
#define MIXKV_MAX_WINDOW 64
#define MIXKV_MAX_GROUP_ROWS 512  /* G * W */

typedef enum {
  MIXKV_OK = 0,
  MIXKV_ERR_INVALID_ARG = 1,
  MIXKV_ERR_UNSUPPORTED = 2,
  MIXKV_ERR_WORKSPACE_TOO_SMALL = 3,
  MIXKV_ERR_HIP = 4
} mixkv_status;

typedef enum { MIXKV_F32 = 0, MIXKV_BF16 = 1 } mixkv_dtype;
typedef enum { MIXKV_POOL_NONE = 0, MIXKV_POOL_AVG = 1, MIXKV_POOL_MAX = 2 } mixkv_pool;
/* How many rows a head keeps (Sec. 3.1: the budget B; Algorithm 1, budget line).
 *   FIXED          every head of every layer keeps params->budget rows
 *   HEAD_ADAPTIVE  the heads of one (layer, batch item) share a pool of n_kv_heads * budget rows, split by score
 *   PER_HEAD       the caller gives the rows kept by every (layer, KV head) in params->head_budgets: layer-wise
 *                  (pyramid) and static head-wise allocation schemes (Sec. 4.1, Table 1) compute such tables */
typedef enum { MIXKV_BUDGET_FIXED = 0, MIXKV_BUDGET_HEAD_ADAPTIVE = 1, MIXKV_BUDGET_PER_HEAD = 2 } mixkv_budget_mode;
/* Intrinsic importance (Sec. 3.2): none, the value norm |V_i| (the method's choice), or the negative
 * key norm -|K_i| (the KNorm alternative of the ablation, Sec. 4.3 / Table 4). */
typedef enum { MIXKV_INTRINSIC_NONE = 0, MIXKV_INTRINSIC_VNORM = 1, MIXKV_INTRINSIC_KNORM = 2 } mixkv_intrinsic;
/* How importance and diversity are combined into s_comp (Sec. 3.3, Eq. 5 and the ablation rows of
 * Table 4).  s_div_scaled is the diversity after min-max and mean matching in every mode.
 *   HEAD_ADAPTIVE  (1 - r) s_imp + r s_div_scaled with the head's own redundancy r (Eq. 4, Eq. 5)
 *   SUM            s_imp + s_div_scaled, no head weights
 *   DIV_ONLY       s_div_scaled
 *   IMP_ONLY       s_imp
 *   GIVEN_R        Eq. 5 with the caller's weight mixkv_layer_in.r_given in place of r (head weights
 *                  measured offline and shared by all samples) */
typedef enum {
  MIXKV_MIX_HEAD_ADAPTIVE = 0, MIXKV_MIX_SUM = 1, MIXKV_MIX_DIV_ONLY = 2, MIXKV_MIX_IMP_ONLY = 3, MIXKV_MIX_GIVEN_R = 4
} mixkv_mix;

typedef struct {
  mixkv_dtype dtype;         /* element type of K, V, Qwin and of K_out, V_out */
  int32_t batch;
  int32_t n_q_heads;         /* multiple of n_kv_heads */
  int32_t n_kv_heads;
  int32_t head_dim;          /* D: 64 or 128 */
  int32_t seq_len;           /* N >= 2, window included */
  int32_t window;            /* 1 <= W <= MIXKV_MAX_WINDOW and W < N; the queries are the last W positions */
  int32_t budget;            /* W <= B <= N rows kept per head (fixed mode) / on average (adaptive mode) / on average
                                at most (per-head mode: n_kv_heads * B rows is the capacity of one batch item's outputs) */
  mixkv_pool pool;           /* 1-D pooling of the window attention over candidates */
  int32_t pool_kernel;       /* odd, 1..63; ignored for MIXKV_POOL_NONE */
  int32_t causal_window;     /* 1: window query w (position Nc+w) attends to keys 0..Nc+w; 0: to all N keys */
  float softmax_scale;       /* multiplies Q.K before the softmax; the library never rescales Q itself */
  float eps;                 /* the epsilon of the paper's min-max and mean-matching formulas, > 0 */
  mixkv_intrinsic intrinsic; /* VNORM: importance = attention + scaled value norm (Sec. 3.2, Eq. 2); see the enum */
  mixkv_mix mix;             /* HEAD_ADAPTIVE: (1 - r) * importance + r * diversity (Sec. 3.3, Eq. 5); see the enum */
  mixkv_budget_mode budget_mode;
  int32_t budget_floor;      /* adaptive mode: minimum non-window rows per head, 0 <= floor <= B - W */
  const int32_t *head_budgets; /* HOST, per-head mode only (else ignored, may be NULL): [n_layers, n_kv_heads], rows
                                kept by KV head h of layer l (the l-th layer struct of the call), window included,
                                the same for every batch item; W <= b <= N and sum_h b[l][h] <= n_kv_heads * B */
} mixkv_params;

/* One layer of the cache to compress. */
typedef struct {
  const void *K;             /* [batch, n_kv_heads, N, D] */
  const void *V;             /* same shape and strides as K */
  int64_t kv_stride_b, kv_stride_h, kv_stride_n;   /* in elements; kv_stride_n >= D */
  const void *Qwin;          /* [batch, n_q_heads, W, D] contiguous, post-RoPE observation-window queries */
  const float *r_given;      /* [batch, n_kv_heads] head weights for MIXKV_MIX_GIVEN_R, finite; ignored (may be
                                NULL) in every other mix mode */
  const float *window_lse;   /* optional [batch, n_q_heads, W]: for every window query row the natural logarithm of
                                sum_i exp(softmax_scale * Q.K_i) over the keys the row attends to (all N, or 0..Nc+w
                                with causal_window), as the prefill attention kernel already produced it for these
                                rows.  When given (then for every layer of the call) the first pass computes no
                                window logits and the softmax is normalised by these values; NULL: computed here */
} mixkv_layer_in;

/* Outputs for one layer.  Which members are required is stated per entry point. */
typedef struct {
  float *scores;             /* [batch, n_kv_heads, N]: the mixed score s_comp at candidates, +inf at the W window slots */
  float *redundancy;         /* [batch, n_kv_heads]: the head's redundancy r (Eq. 4) */
  int32_t *indices;          /* kept positions, ascending per head, the W window positions last.
                                fixed: [batch, n_kv_heads, B]; adaptive and per-head: [batch, n_kv_heads * B], heads packed
                                back to back (per-head mode may leave the tail of a batch item's slots untouched) */
  int32_t *counts;           /* [batch, n_kv_heads] rows kept per head (B in fixed mode) */
  int32_t *offsets;          /* adaptive and per-head: [batch, n_kv_heads + 1] exclusive prefix sums of counts; may be
                                NULL in fixed mode */
  void *K_out, *V_out;       /* rows of K / V at `indices`, copied bit for bit, D contiguous.
                                fixed: [batch, n_kv_heads, B, D]; adaptive and per-head: [batch, n_kv_heads * B, D] packed
                                like indices */
} mixkv_layer_out;

/*
 * Bytes of device workspace mixkv_score / mixkv_compress need for `n_layers`
 * layers of this shape.  mixkv_select needs none and accepts NULL, except in
 * per-head budget mode, where it stages the budget table there and needs
 * n_layers * n_kv_heads * 4 bytes.  With more it ranks in more workgroups, with
 * the same results; whatever it is given is scratch that the call may write, in
 * every budget mode:
 *   n_layers * batch * n_kv_heads * 8192 bytes (two 1024-entry candidate lists
 *     per head): in head-adaptive mode, with up to 32 768 candidates and
 *     M = min(floor + n_kv_heads * (budget - window - floor), Nc) <= 1024, every
 *     head is ranked by a workgroup of its own and a small kernel splits the pool;
 *   this function's figure: the same for any M, and beyond 32 768 candidates (up
 *     to 524 288), in every mode, a head's row is cut into segments with a
 *     workgroup each, as long as a segment's list (of up to M entries, or in
 *     fixed and per-head mode as many as the largest budget keeps beside the
 *     window) has at most 16 384 entries, or all of a head's together 32 768.
 * In all other cases one workgroup ranks the whole rows of a head (fixed and
 * per-head mode) or of all heads of a batch item (head-adaptive mode), several
 * to some tens of times slower on long rows.
 * Host only; touches no GPU (head_budgets is not read).  The workspace needs no
 * initialisation and 256-byte alignment.
 */
mixkv_status mixkv_workspace_size(const mixkv_params *params, int32_t n_layers, size_t *bytes);

/*
 * Score every cached key (Algorithm 1, step 1 and the mixing half of step 2).
 * Per (layer, batch item, KV head):
 *   s_ex   mean over the G*W window queries of softmax attention on key i (Sec. 3.2,
 *          extrinsic importance), pooled over candidates; the rows' normalisers are computed
 *          here or taken from in[l].window_lse;
 *   s_imp  s_ex + min-max normalised value norm scaled to mean(s_ex) (Sec. 3.2, Eq. 2);
 *   s_div  -Khat_i . mean_j Khat_j with Khat the L2-normalised keys, all N keys in the mean
 *          (Sec. 3.2, diversity metrics), min-max normalised and scaled to mean(s_imp) (Sec. 3.3);
 *   r      (N^2 |mean Khat|^2 - N) / (N (N-1))   (Sec. 3.3, Eq. 3-4);
 *   s_comp (1 - r) s_imp + r s_div_scaled         (Sec. 3.3, Eq. 5).
 * All minima, maxima and means are over the Nc candidates.  params->intrinsic and params->mix
 * switch to the ablation's variants (Sec. 4.3, Table 4): with KNORM, -|K_i| takes the place of
 * |V_i| in s_imp; the mix modes change the last line only.
 * Writes out[l].scores (required) and out[l].redundancy (optional, may be NULL; always the head's
 * own r of Eq. 4, whatever the mix mode).
 */
mixkv_status mixkv_score(const mixkv_params *params, const mixkv_layer_in *in, mixkv_layer_out *out,
                         int32_t n_layers, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * TopB on caller-provided scores (Sec. 3.1; Algorithm 1, TopB step with B' = B - W and the
 * window excluded from ranking and always kept).  Reads out[l].scores (only the Nc candidate
 * slots are read); writes out[l].indices, out[l].counts and, if non-NULL, out[l].offsets
 * (required in adaptive mode).  Ties go to the smaller position.  NaN scores are not supported.
 * Fixed mode: each head keeps its B' best candidates.  Head-adaptive mode, per (layer, batch
 * item): every head keeps its budget_floor best candidates, then the remaining
 * n_kv_heads * (B' - budget_floor) slots go to the best remaining candidates of all heads
 * together (ties: smaller head, then smaller position).  Per-head mode: head h of layer l keeps its
 * head_budgets[l][h] - W best candidates.
 * The workspace is optional in fixed and head-adaptive mode, and so is its size (mixkv_workspace_size says what each
 * size brings); like every workspace it belongs to the call until the call's work is done.
 */
mixkv_status mixkv_select(const mixkv_params *params, mixkv_layer_out *out, int32_t n_layers,
                          void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The whole step (Algorithm 1): score, select, and gather the kept K/V rows (Sec. 3.1,
 * Khat, Vhat = TopB(K, V, {s_i})).  Writes indices, counts, K_out, V_out (all required),
 * offsets (required in adaptive mode), and scores / redundancy when non-NULL.
 * K_out / V_out must not overlap K / V.
 */
mixkv_status mixkv_compress(const mixkv_params *params, const mixkv_layer_in *in, mixkv_layer_out *out,
                            int32_t n_layers, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * mixkv_compress for callers that can neither allocate device memory nor hand over a workspace:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  The
 * workspace is an array of MIXKV_STATIC_SCRATCH_BYTES inside the library's own device data (every
 * GPU the library runs on holds one from load until the process ends); inputs and outputs are the
 * caller's as in mixkv_compress, and so are the results, bit for bit.  The call allocates and
 * frees nothing.  Shapes whose workspace (mixkv_workspace_size) exceeds the array return
 * MIXKV_ERR_WORKSPACE_TOO_SMALL and touch nothing: 32 MiB hold the whole 28-layer 8K cache of the
 * 28Q/4KV shape in one call; larger caches go layer group by layer group.  Nothing in the array has
 * to start at zero (every word is written before it is read within a call) and it keeps the last
 * call's contents.  All calls on one GPU share the array: calls that overlap in time on one GPU
 * (different streams, or different host threads) race; serialise them or use mixkv_compress with
 * separate workspaces.  The first call on a device looks the array's address up once
 * (hipGetSymbolAddress); make that call outside a graph capture.
 */
#define MIXKV_STATIC_SCRATCH_BYTES (32u << 20)
mixkv_status mixkv_compress_static(const mixkv_params *params, const mixkv_layer_in *in, mixkv_layer_out *out,
                                   int32_t n_layers, void *hip_stream);

/*
 * Profiling aid: mixkv_compress with every kernel launch bracketed by a pair of HIP events on
 * `hip_stream`.  Synchronises the stream before returning and writes the milliseconds each
 * pipeline stage took to the HOST array stage_ms[MIXKV_N_STAGES] (summed over launch groups when
 * n_layers exceeds one group).  Stage names come from mixkv_stage_name.  Outputs are those of
 * mixkv_compress (Algorithm 1).
 */
#define MIXKV_N_STAGES 5
mixkv_status mixkv_compress_profiled(const mixkv_params *params, const mixkv_layer_in *in, mixkv_layer_out *out,
                                     int32_t n_layers, void *workspace, size_t workspace_bytes, void *hip_stream,
                                     float *stage_ms);
const char *mixkv_stage_name(int32_t stage);

/*
 * Redundancy analysis of cached keys or values (Sec. 1, the figures that show the cosine similarity
 * of keys inside one head, and the average similarity of keys and of values per layer and head;
 * Sec. 3.3, Eq. 3-4 for the similarity matrix and its off-diagonal mean).  For every (batch item,
 * head) of every layer, with R the N x N matrix of cosine similarities between the rows of X
 * (a row of norm below 1e-30 counts as the zero vector):
 *   redundancy  the mean of the off-diagonal entries of R (for X = K this is the r of mixkv_score);
 *   block_map   [nb, nb], nb = ceil(N / block): the mean of R over the rows of block a and the
 *               columns of block b, blocks being `block` consecutive positions (the last one may be
 *               shorter; diagonal entries belong to the diagonal blocks): the heat-map of R at a
 *               resolution of `block` tokens.
 * Only dtype, batch, n_kv_heads (the number of heads of X), head_dim and seq_len of `params` are
 * used; the rest must merely be valid.  1 <= block <= N.  Either output may be NULL, not both.
 * Workspace: mixkv_similarity_workspace_size bytes, 256-byte aligned, no initialisation.
 */
typedef struct {
  const void *X;             /* DEVICE [batch, n_kv_heads, N, D], D contiguous: keys or values */
  int64_t stride_b, stride_h, stride_n;   /* in elements; stride_n >= D; row starts 16-byte aligned */
} mixkv_rows_in;
typedef struct {
  float *redundancy;         /* DEVICE [batch, n_kv_heads] */
  float *block_map;          /* DEVICE [batch, n_kv_heads, nb, nb] */
} mixkv_similarity_out;
mixkv_status mixkv_similarity_workspace_size(const mixkv_params *params, int32_t n_layers, int32_t block, size_t *bytes);
mixkv_status mixkv_similarity(const mixkv_params *params, const mixkv_rows_in *in, const mixkv_similarity_out *out,
                              int32_t n_layers, int32_t block, void *workspace, size_t workspace_bytes,
                              void *hip_stream);

/*
 * Attention of one new token over the compacted cache (Sec. 3.1: the compressed K, V are what the
 * attention of the decoding phase reads).  Per layer, batch item and query head g (KV head
 * h = g / G): out_g = sum_j softmax_j(softmax_scale * Q_g . k_j) v_j over the rows of head h: the
 * counts[b][h] kept rows in K_cache / V_cache, laid out as mixkv_compress wrote them for
 * params->budget_mode and params->budget (fixed: [batch, n_kv_heads, B, D]; otherwise packed
 * [batch, n_kv_heads * B, D] with `offsets`), followed by the first tail_len rows of K_tail / V_tail
 * ([batch, n_kv_heads, tail_capacity, D]: the rows appended since the compression, the new token's
 * own row included; the caller's projection kernel writes them there).  fp32 accumulation; `out` has
 * the dtype of the inputs (bf16: rounded to nearest even).  All pointers are DEVICE pointers, rows
 * 16-byte aligned; K_tail / V_tail may be NULL when tail_len is 0, offsets when the layout is fixed.
 * counts / offsets are clamped to the capacity of the layout before use.
 * Workspace: long caches (by the rows per head, params->budget + tail_len: more than 384 in fp32, 512 or
 * more in bf16 if few heads share the GPU) are split over several workgroups per head whose partial
 * results pass through `workspace`: mixkv_decode_workspace_size bytes (0 for caches that are not split,
 * then NULL is accepted), 256-byte aligned, no initialisation.  In bf16 a smaller workspace may be
 * accepted (MIXKV_ERR_WORKSPACE_TOO_SMALL if not): the rows are then split into fewer ranges, which
 * takes longer and sums in another order, so that outputs may differ in their last bit from those
 * with the full workspace.  With the same arguments, sizes included, outputs repeat bit for bit.
 */
typedef struct {
  const void *K_cache, *V_cache;
  const int32_t *counts;     /* [batch, n_kv_heads] */
  const int32_t *offsets;    /* [batch, n_kv_heads + 1], packed layouts */
  const void *K_tail, *V_tail;
  const void *Q;             /* [batch, n_q_heads, D] the new token's queries */
  void *out;                 /* [batch, n_q_heads, D] */
} mixkv_decode_layer;
mixkv_status mixkv_decode_workspace_size(const mixkv_params *params, int32_t n_layers, int32_t tail_len, size_t *bytes);
mixkv_status mixkv_decode_attention(const mixkv_params *params, const mixkv_decode_layer *layers, int32_t n_layers,
                                    int32_t tail_len, int32_t tail_capacity, void *workspace, size_t workspace_bytes,
                                    void *hip_stream);

/*
 * Appends one token to the tails that mixkv_decode_attention reads (Sec. 3.1: the compressed cache
 * is what decoding continues on, so it grows again by one row per decoded token).  Per layer,
 * batch item b and KV head h: K_tail[b][h][position][:] = K_new[b][h][:], and the same for V:
 * verbatim copies in the dtype of params.  K_new / V_new are [batch, n_kv_heads, D] contiguous (the
 * new token's post-RoPE key and value rows), K_tail / V_tail [batch, n_kv_heads, tail_capacity, D]
 * contiguous; DEVICE pointers owned by the caller, 16-byte aligned; a tail may not overlap the new
 * rows.  0 <= position < tail_capacity, else MIXKV_ERR_INVALID_ARG (nothing is launched); the rows
 * before `position` are not touched.  After the call on the same stream,
 * mixkv_decode_attention with tail_len = position + 1 sees the new row.  No workspace.
 */
typedef struct {
  const void *K_new, *V_new;
  void *K_tail, *V_tail;
} mixkv_append_layer;
mixkv_status mixkv_append(const mixkv_params *params, const mixkv_append_layer *layers, int32_t n_layers,
                          int32_t position, int32_t tail_capacity, void *hip_stream);

/*
 * The paged cache: a compacted (or full) cache that decoding continues on, held in pages.
 *
 * A page holds page_rows rows of one KV head, keys and values apart.  page_table[b][h][i] is the page with the rows
 * [i * page_rows, (i + 1) * page_rows) of KV head h of sequence b; heads of one sequence may have different lengths, as
 * head-adaptive budgets give them (Sec. 3.1, Sec. 4.1), and a sequence of length 0 is padding.  An entry outside
 * [0, n_pages) is no page: rows that would go there are dropped, rows that would come from there do not exist.
 *
 * MIXKV_PAGE_ROWS: a page is page_rows rows of head_dim elements in the dtype of the params.
 * MIXKV_PAGE_4BIT (bf16 only): 32 neighbouring elements of a row share a step S and a base B, both fp16, and an element is
 * stored as a code of 4 bits that stands for B + S (1 + code / 16): 5 bits an element in all.  With lo and hi the smallest and
 * largest of the 32 elements x, each first brought into [-16384, 16384],
 *     S = fp16((hi - lo) 16 / 15),  B = fp16(lo - S),  code = min(max(round(16 (x - B - S) / S), 0), 15)  (0 where S = 0),
 * the differences in 64 bits, each fp16 rounded to nearest even through fp32, the code to nearest even.  An element is off by at
 * most S / 32, where fp16 resolves B and S.  D = head_dim, P = page_rows, code e of a word in its bits [4 n, 4 n + 4),
 * n = e / 2 + 4 (e % 2); a page of keys or values has P D 5 / 8 bytes, the codes first:
 *   keys    word r D/8 + s D/32 + g' of the page: the codes of the elements 32 g + 8 s + e of row r; then (S, B) of (r, g) at fp16
 *           2 (r D/32 + g').  g' is 0, 2, 1, 3 for g = 0 ... 3 if D = 128, g if D = 64.
 *   values  strip q of the 32 rows from row 32 t: the rows 32 t + 4 q + i and 32 t + 16 + 4 q + i, i = 0 ... 3, as e = 2 i and 2 i + 1.
 *           Word (4 t + q) D + 64 j + 4 m + w: the codes of the element 64 j + 16 w + m of the strip's rows; then S of the strip's
 *           row e and group g at fp16 ((4 t + q) D/32 + g) 16 + e, B eight further.
 * NaN is not supported in rows that go into 4-bit pages, nor in keys where K_bounds are kept.
 * A program that builds pages itself may write them in this form.  Pages need no initialisation; rows of a page that have not
 * been written are never used.  A page that a call writes to must be written to for one place of one (sequence, head) only.
 * Pages, bounds, dense rows and outputs of a call may not overlap one another where any of them is written.
 *
 * lengths[b][h] counts the rows of a head, those that a call appends among them: a program adds the new rows to the
 * lengths first.  Lengths are clamped to [0, max_pages * page_rows].
 */
typedef enum { MIXKV_PAGE_ROWS = 0, MIXKV_PAGE_4BIT = 1 } mixkv_page_format;

typedef struct {
  mixkv_dtype dtype;         /* element type of rows, queries, outputs and key bounds */
  mixkv_page_format format;  /* of the pages; 4BIT needs MIXKV_BF16 */
  int32_t batch;
  int32_t n_q_heads;         /* multiple of n_kv_heads; batch * n_q_heads <= 2^18 */
  int32_t n_kv_heads;
  int32_t head_dim;          /* 64 or 128 */
  int32_t page_rows;         /* 32, 64 or 128 */
  int32_t max_pages;         /* entries of a head in the page table; max_pages * page_rows <= 2^30 */
  int32_t n_pages;           /* pages in a layer's K_pages and V_pages */
  float softmax_scale;       /* > 0, at most 2^127 */
} mixkv_paged_params;

/* One layer's pages.  DEVICE pointers owned by the caller, K_pages, V_pages and K_bounds 16-byte aligned. */
typedef struct {
  void *K_pages, *V_pages;   /* n_pages pages each, back to back */
  void *K_bounds;            /* [n_pages, 2, D], dtype of the params: per element the smallest and the largest key that was written to
                                the page since its first row was; NULL where no call needs it */
  const int32_t *page_table; /* [batch, n_kv_heads, max_pages] */
  const int32_t *lengths;    /* [batch, n_kv_heads] */
} mixkv_paged_cache;

/* Bytes of a page of keys (or values).  Host only. */
mixkv_status mixkv_page_bytes(const mixkv_paged_params *params, size_t *bytes);

/* Dense rows of one layer that go into pages or come out of them.  Row r of KV head h starts at element r * stride_n + h * stride_h of K
 * (and of V); stride_n >= D, stride_h >= 0 (0: the heads' rows lie among one another, as in packed caches), row starts 16-byte
 * aligned.  The rows of (b, h) are [row_start[b][h], row_start[b][h] + row_count[b][h]); those outside [0, n_rows) are left out. */
typedef struct {
  void *K, *V;               /* read by mixkv_paged_append, written by mixkv_paged_read */
  int64_t stride_n, stride_h;
  const int32_t *row_start, *row_count;  /* DEVICE [batch, n_kv_heads] */
  const void *Q;             /* append only, may be NULL: queries of the same rows, head g of row r at r * q_stride_n + g * q_stride_h;
                                for a KV head's rows the G query heads that it serves; for every layer of a call or none */
  int64_t q_stride_n, q_stride_h;
  void *Q_out;               /* [n_rows, n_q_heads, D] contiguous: the rotated queries; required with Q, may not overlap K, V or Q */
} mixkv_paged_rows;

/* Rotation of keys and queries to their positions: with the elements i and i + D/2 of a row as a pair (a, b), c and s the cosine and
 * sine of its angle, (a c - b s, b c + a s), in 64 bits, rounded to fp32 and from there to the dtype.  The angle of pair i is that of
 * positions[axis][r] for the row's index r: axis 0 everywhere (n_axes 1), or (n_axes 3) axis 0 for the first sections[0] pairs, 1 for
 * the next sections[1], 2 for the last sections[2] (time, height and width of vision-language models).  Positions are
 * clamped to the tables.  Shared by the layers of a call. */
typedef struct {
  const float *cos, *sin;    /* DEVICE [n_positions, D / 2] */
  int32_t n_positions;
  const int32_t *positions;  /* DEVICE [n_axes, n_rows] */
  int32_t n_axes;            /* 1 or 3 */
  int32_t sections[3];       /* n_axes 3: each >= 0, sum D / 2; else ignored */
} mixkv_rope;

/*
 * Appends rows to the paged caches of `n_layers` layers (Sec. 3.1: decoding continues on the compressed cache): row t of
 * the row_count[b][h] rows of (b, h) becomes row lengths[b][h] - row_count[b][h] + t of the head.  Keys and queries are
 * rotated (rope, or NULL: not; keys that mixkv_compress kept are rotated already), values are stored as they are; pages
 * hold them in params->format.  K_bounds, where given, take in the new keys as stored rows of the dtype; a page whose first row is
 * written forgets what it bounded.  One call serves a decoding step (a row per sequence), prompts (ragged rows, one after
 * another, with unused rows behind them) and a cache that mixkv_compress has written (row_start from its offsets, stride_h 0).  Rows of
 * pages, queries and bounds that no row goes to keep their contents; a repeated call stores the same again.
 * max_count: the largest row_count, as far as the host knows it (>= 1): it sizes the launch; larger counts are served, slower.
 */
mixkv_status mixkv_paged_append(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_rows *rows,
                                int32_t n_layers, const mixkv_rope *rope, int32_t n_rows, int32_t max_count, void *hip_stream);

/*
 * The way back: the newest row_count[b][h] rows of every head (all of them with row_count = lengths) into dense rows of the
 * dtype (4-bit elements rounded to it), for a cache that is to be compressed again with mixkv_compress, moved, or looked
 * at.  Dense rows that nothing comes to keep their contents.  Q, Q_out and K_bounds are not used.
 */
mixkv_status mixkv_paged_read(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_rows *rows,
                              int32_t n_layers, int32_t n_rows, int32_t max_count, void *hip_stream);

/*
 * Pages worth attending to: for the new token of every sequence and every KV head, the max_selected pages with the largest score
 *     s_p = fp32(sum_d (Q+_d hi_pd + Q-_d lo_pd)),  Q+_d = sum_g max(q_gd, 0),  Q-_d = sum_g min(q_gd, 0)  over the head's G queries,
 * in 64 bits, with lo and hi the page's K_bounds: the sum over the queries of the largest dot product that any key within
 * the bounds can have (a bound that meets a zero counts nothing, infinite ones too).  The bounds are those of the rows as
 * appended: elements of 4-bit pages, which attention takes, lie up to half a code and the fp16 rounding of their base outside them.  The first keep_first and
 * the last keep_last pages are always among them (keep_first + keep_last <=
 * max_selected, and max_selected * page_rows <= 2^30 here and in mixkv_paged_attention); equal scores go to the earlier page, a place without a
 * page scores -infinity, and so does one whose score is NaN (queries hold none); a head with no more pages than max_selected keeps all.
 * Writes selected [batch, n_kv_heads, max_selected] (places in the head's page table, ascending, then -1) and n_selected
 * [batch, n_kv_heads].  K_pages and V_pages are not used and may be NULL; softmax_scale is not used.
 * Workspace: mixkv_paged_select_workspace_size bytes, 256-byte aligned, no initialisation.
 */
typedef struct {
  const void *Q;             /* [batch, n_q_heads, D] contiguous, 16-byte aligned */
  int32_t *selected;         /* [batch, n_kv_heads, max_selected] */
  int32_t *n_selected;       /* [batch, n_kv_heads] */
} mixkv_paged_select_layer;
mixkv_status mixkv_paged_select_workspace_size(const mixkv_paged_params *params, int32_t n_layers, size_t *bytes);
mixkv_status mixkv_paged_select(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_select_layer *layers,
                                int32_t n_layers, int32_t max_selected, int32_t keep_first, int32_t keep_last, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/*
 * Attention of one new token per sequence over its pages (Sec. 3.1, as mixkv_decode_attention): out_g = sum_j
 * softmax_j(softmax_scale * Q_g . k_j) v_j over the rows of KV head g / G, all lengths[b][h] of them or (selected given, for every
 * layer or none) those in the pages selected[b][h][0 .. n_selected[b][h]): places in the page table, in any order; one that is no place
 * in the table is passed over, a page that is listed twice counts twice.  A head without rows gets zeros.  fp32
 * accumulation, out in the dtype.  With 4-bit pages, values and weights enter the second product as fp16.
 * Logits are to stay below 2^25 in magnitude, beyond which fp32 has no differences of one left between them, values below 2^100.
 * max_rows: the largest number of rows of a head (of selected pages, whole), as far as the host knows it (>= 1): with it the
 * rows are dealt to workgroups; longer heads are served, slower.  Outputs repeat bit for bit for the same arguments, max_rows included.
 * Workspace: mixkv_paged_attention_workspace_size bytes (0: NULL is accepted), 256-byte aligned, no initialisation.
 */
typedef struct {
  const void *Q;             /* [batch, n_q_heads, D] contiguous, rows 16-byte aligned */
  void *out;                 /* [batch, n_q_heads, D], 16-byte aligned */
  const int32_t *selected;   /* [batch, n_kv_heads, max_selected] or NULL */
  const int32_t *n_selected; /* [batch, n_kv_heads], with selected */
} mixkv_paged_attention_layer;
mixkv_status mixkv_paged_attention_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t max_rows, size_t *bytes);
mixkv_status mixkv_paged_attention(const mixkv_paged_params *params, const mixkv_paged_cache *caches,
                                   const mixkv_paged_attention_layer *layers, int32_t n_layers, int32_t max_selected, int32_t max_rows,
                                   void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Queries of new rows: a prompt's, a few drafted tokens', a step's single ones, of ragged sequences one after another with unused rows
 * behind them.  The rows of (b, h) are [row_start[b][h], row_start[b][h] + row_count[b][h]), for each the G query heads that KV head h
 * serves; those outside [0, n_rows) are left out, and a row belongs to one sequence only.  Their keys and values are in the cache already (mixkv_paged_append, which takes the same
 * row_start and row_count, and whose Q_out is Q here): row t of a head's row_count[b][h] rows has the place p = lengths[b][h] - row_count[b][h] + t,
 * and sees the places j <= p with
 *     j > p - window   or   j < keep_first:
 * the newest `window` rows, its own among them, and the first keep_first ones (sinks).  A window of max_pages * page_rows or more
 * leaves nothing out.  A row whose p is below 0 sees nothing.  Places are counted in rows of the cache; heads of one sequence may have different lengths.
 * What a place that a row does not see holds, infinities and NaN too, does not reach that row's results.
 */
typedef struct {
  const void *Q;             /* head g of row r at element r * q_stride_n + g * q_stride_h; 16-byte aligned, rows and heads too */
  int64_t q_stride_n, q_stride_h;
  const int32_t *row_start, *row_count;  /* DEVICE [batch, n_kv_heads] */
  void *out;                 /* mixkv_paged_window_attention only: [n_rows, n_q_heads, D] contiguous, 16-byte aligned, may not overlap Q */
  float *lse;                /* [n_rows, n_q_heads]: written by mixkv_paged_window_attention (may be NULL there), read by mixkv_paged_weights */
} mixkv_paged_queries;

/*
 * Attention of new rows over the rows that each of them sees (Sec. 3.1: the prefill in front of the compression, and decoding behind it):
 * out = sum_j softmax_j(softmax_scale * q . k_j) v_j, and lse = log sum_j exp(softmax_scale * q . k_j), the natural logarithm (for the last
 * W rows of a prompt what mixkv_layer_in.window_lse asks for, with causal_window and a window that leaves nothing out).  A row that sees nothing gets zeros
 * and -infinity.  Rows of out and lse that belong to no (sequence, head) keep their contents.  fp32 accumulation, out in the dtype.  With
 * many new rows of bf16 the weights enter the second product as bf16; with 4-bit pages values and weights enter it as fp16.  Logits and values as for mixkv_paged_attention.
 * max_count: the largest row_count; a head's rows beyond max_count are not served (their outputs keep their contents).  max_rows: the largest length, as
 * far as the host knows it (>= 1): longer heads are served, slower.  Outputs repeat bit for bit for the same arguments, max_count and max_rows
 * included.  n_rows * n_q_heads <= 2^31 - 1.  Workspace: mixkv_paged_window_attention_workspace_size bytes (0: NULL is accepted), 256-byte
 * aligned, no initialisation.
 */
mixkv_status mixkv_paged_window_attention_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t n_rows, int32_t window,
                                                         int32_t keep_first, int32_t max_count, int32_t max_rows, size_t *bytes);
mixkv_status mixkv_paged_window_attention(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_queries *queries,
                                          int32_t n_layers, int32_t n_rows, int32_t window, int32_t keep_first, int32_t max_count, int32_t max_rows,
                                          void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The attention that cached rows have been given, summed up: with the lse that mixkv_paged_window_attention left for the same queries, window and
 * keep_first (or any other normaliser), row j of KV head h has its weight raised by
 *     sum over the new rows that see j, and over the G query heads, of exp(softmax_scale * q . k_j - lse),
 * in fp32; the weights of the new rows themselves begin at zero.  A place's weight lies beside its page: weights[l][page][row of the page], 16-byte aligned.  It is read,
 * raised and written without atomics, as pages are: a page may be listed for one place of one (sequence, head) only here, also where it is shared for reading (a
 * common prefix), since each of two heads would lose what the other adds.  Rows
 * whose lse is -infinity give nothing.  Weights of rows that do not exist, and of old rows that no new row sees, keep their contents.  A head's
 * rows beyond max_count are not served; max_rows as above.  n_rows * n_q_heads <= 2^30.  V_pages are not used and may be NULL.  Sums repeat bit for bit for the same
 * arguments.  Workspace: mixkv_paged_weights_workspace_size bytes (0: NULL is accepted), 256-byte aligned, no initialisation.
 */
mixkv_status mixkv_paged_weights_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t n_rows, int32_t window, int32_t keep_first,
                                                int32_t max_count, int32_t max_rows, size_t *bytes);
mixkv_status mixkv_paged_weights(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_queries *queries, float *const *weights,
                                 int32_t n_layers, int32_t n_rows, int32_t window, int32_t keep_first, int32_t max_count, int32_t max_rows, void *workspace,
                                 size_t workspace_bytes, void *hip_stream);

/*
 * Eviction by weight: head (b, h) keeps min(lengths[b][h], keep[b][h]) of its rows, those with the largest weight (equal ones: the earlier
 * row; NaN counts as -infinity); the first keep_first and the last keep_last rows of a head count as infinite.  Rows whose page is none do not
 * exist: they are not kept.  The kept rows move in order, bit for bit, into the pages of `into` (whose page table has the same shape, and
 * whose pools may be the caches' own), with their weights; a place of `into` without a page is left out.  kept receives the places they
 * come from, n_kept how many they are: the lengths of `into` from then on (into[l].lengths is not used).  K_bounds, if both have them, become the bounds of the rows that a page
 * of `into` now holds (4-bit elements rounded to the dtype).  The pages that `into` lists may be none of those that the caches list; these are not
 * written, and free afterwards.
 * max_keep: the largest keep, and the width of kept; larger ones are taken as it.  max_rows: the largest length, as far as the host knows
 * it (>= 1): longer heads are served, slower.  Workspace: mixkv_paged_evict_workspace_size bytes (0: NULL is accepted), 256-byte aligned, no initialisation.
 */
typedef struct {
  const float *weights;      /* [n_pages, page_rows], of the caches' pages; 16-byte aligned */
  float *weights_into;       /* the same of the pages of `into` (may be the same array), or NULL */
  const int32_t *keep;       /* [batch, n_kv_heads]; below 0: none */
  int32_t *kept;             /* [batch, n_kv_heads, max_keep] places, ascending, then -1 */
  int32_t *n_kept;           /* [batch, n_kv_heads] */
} mixkv_paged_evict_layer;
mixkv_status mixkv_paged_evict_workspace_size(const mixkv_paged_params *params, int32_t n_layers, int32_t max_rows, size_t *bytes);
mixkv_status mixkv_paged_evict(const mixkv_paged_params *params, const mixkv_paged_cache *caches, const mixkv_paged_cache *into,
                               const mixkv_paged_evict_layer *layers, int32_t n_layers, int32_t max_keep, int32_t keep_first, int32_t keep_last,
                               int32_t max_rows, void *workspace, size_t workspace_bytes, void *hip_stream);

const char *mixkv_status_string(mixkv_status status);
int32_t mixkv_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MIXKV_H */
