/*
 * last.h -- C ABI of the MI355X (gfx950) LAST token-selection library.
 *
 * LAST (arXiv 2607.27952) prunes visual tokens before edge-to-cloud
 * transmission. This library implements the data-parallel hot path:
 *
 *   last_token_scores  Sec. 3.3, Eq. 6-8: the attention row of the last query
 *                      token against every key of the guidance model's prefill
 *                      (softmax over the whole visual + text context), its
 *                      visual columns summed over guidance layers and heads,
 *                      normalised over the visual tokens.
 *   last_rows_scores   Sec. 4.3, Table 4: the same scores from other causal
 *                      query rows (first, middle or every query token).
 *   last_prefill_attention  Sec. 3.3: the guidance model's causal prefill
 *                      attention, with the same scores read from its last row.
 *   diverse_select     Sec. 3.4, Eq. 9-12: importance-weighted greedy k-center
 *                      over unit-normalised encoder features under a budget
 *                      K = ceil(rho N) (Eq. 2); or the Top-k ablation of
 *                      Sec. 4.3, Table 5. Kept indices come out ascending.
 *   diverse_select_similarity, diverse_select_pick  the k-center of
 *                      diverse_select in two calls (distances, then greedy),
 *                      so the distances can overlap the score pass.
 *   gather_kept        Sec. 3.4, Eq. 12: the kept rows X_S, in original order,
 *                      copied byte for byte for transmission.
 *   last_rotary, last_rotary_append  rotary positions with several axes; the
 *                      same with keys and values put into a paged cache.
 *   last_decode_attention  attention of one new token over a paged cache.
 *   last_cache_prune, last_cache_copy  Eq. 12 on a cache (the kept tokens
 *                      compacted into new pages); pages copied.
 *
 * Conventions shared by every call
 *   - Pointers without a suffix are device pointers; pointers suffixed _h are
 *     host copies of the same small arrays, used for validation and launch
 *     planning. Each _h array must hold exactly what its device twin holds.
 *   - The caller owns every buffer, including the workspace (size it with the
 *     matching *_workspace query). The library never allocates device memory,
 *     never synchronises, and only enqueues work on `stream` (a hipStream_t;
 *     NULL is the default stream).
 *   - Every argument is validated on the host, from the _h copies, before any
 *     HIP call. On error nothing is enqueued, outputs are left untouched, and
 *     a non-zero last_status is returned. A failed kernel launch returns
 *     LAST_ERR_DEVICE (possibly after earlier kernels of the same call have
 *     been enqueued).
 *   - Ragged batches of R requests are packed with CSR offsets (int32, length
 *     R+1, starting at 0, non-decreasing). Indices into a request's visual
 *     tokens are request-local int32 in [0, N_r).
 *   - Results are deterministic: the same inputs give bitwise-identical
 *     outputs on every run (fixed reduction orders, ties to the lowest index).
 *   - Calls on different streams are independent if their workspaces and
 *     outputs do not overlap.
 */
#ifndef LAST_H
#define LAST_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LAST_OK = 0,
  LAST_ERR_INVALID = 1,     /* malformed arguments (shapes, CSR, budgets, NULLs) */
  LAST_ERR_UNSUPPORTED = 2, /* valid but outside what the kernels implement */
  LAST_ERR_WORKSPACE = 3,   /* workspace pointer NULL or smaller than required */
  LAST_ERR_DEVICE = 4       /* a HIP call failed; see last_status_string */
} last_status;

typedef enum { LAST_F32 = 0, LAST_BF16 = 1 } last_dtype;

typedef enum {
  LAST_SEL_KCENTER = 0, /* Eq. 9-11: greedy argmax of w_i * delta_i */
  LAST_SEL_TOPK = 1     /* Table 5 "LAST (Top-k)": the K largest w_i */
} last_sel_mode;

/*
 * Batch description for last_token_scores.
 *   R          number of requests (>= 1)
 *   G          guidance layers whose rows are summed (Eq. 7 sums over layers;
 *              any subset of a model's layers can be passed, G >= 1)
 *   Hq, Hkv    query and key heads; Hq % Hkv == 0. Query head h reads KV head
 *              h / (Hq / Hkv) (grouped-query attention). Eq. 7 sums over all
 *              Hq query heads.
 *   Dh         head dimension, 64 or 128 (others: LAST_ERR_UNSUPPORTED)
 *   qk_dtype   storage type of q and k (LAST_F32 or LAST_BF16)
 *   softmax_scale  sigma in softmax(sigma q.k); <= 0 selects 1/sqrt(Dh)
 *   cu_seqlens [R+1] token offsets into k; P_r = cu_seqlens[r+1]-cu_seqlens[r]
 *              is the prefill length of request r (>= 2). Its last token,
 *              position P_r - 1, is the query token whose row is scored.
 *   vis_start  [R] start of request r's visual span within its sequence
 *   cu_vis     [R+1] offsets into scores (and into the features given to
 *              diverse_select); N_r = cu_vis[r+1]-cu_vis[r] >= 1 visual tokens
 *              occupy positions [vis_start[r], vis_start[r] + N_r), which must
 *              end before the last token: vis_start[r] + N_r <= P_r - 1.
 */
typedef struct last_batch {
  int32_t R, G, Hq, Hkv, Dh;
  last_dtype qk_dtype;
  float softmax_scale;
  const int32_t *cu_seqlens, *cu_seqlens_h;
  const int32_t *vis_start, *vis_start_h;
  const int32_t *cu_vis, *cu_vis_h;
} last_batch;

/* Workspace bytes last_token_scores needs for this batch (0 if invalid). */
size_t last_token_scores_workspace(const last_batch *b);

/*
 * Sec. 3.3, Eq. 6-8.
 *   q          [G][R][Hq][Dh] the last query token of each request, per layer
 *              (after rotary embedding, as the attention sees it)
 *   k          [G][T_total][Hkv][Dh] keys of every prefill token (after rotary
 *              embedding), T_total = cu_seqlens[R]
 *   scores     [N_total] out: w~ per visual token; each request's entries are
 *              >= 0 and sum to 1 (Eq. 8)
 *   attn_rows  optional [G][Hq][T_total] out (NULL to skip): the full softmax
 *              rows A^(l,h)[p*, :] of every request, for inspection
 *   ws         device workspace of at least last_token_scores_workspace(b)
 *              bytes, 256-byte aligned
 */
last_status last_token_scores(const last_batch *b, const void *q, const void *k,
                              float *scores, float *attn_rows, void *ws,
                              size_t ws_bytes, void *stream);

/*
 * last_token_scores without a workspace argument, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation). Same arguments, kernels and results as
 * last_token_scores; its scratch is a static device array of
 * LAST_STATIC_SCRATCH_BYTES that every device running the library holds until
 * the process ends. The call itself allocates nothing: the array's address is
 * looked up once per device, on that device's first call.
 *   - A batch whose workspace (last_token_scores_workspace) exceeds
 *     LAST_STATIC_SCRATCH_BYTES is rejected with LAST_ERR_WORKSPACE before any
 *     HIP call.
 *   - The current device must be the one `stream` belongs to.
 *   - All calls on one device share its array: calls that overlap in time on
 *     one device (different streams, or different host threads) race and give
 *     undefined results. Nothing in the array needs to start at zero; each call
 *     writes every part it reads.
 */
#define LAST_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
last_status last_token_scores_static(const last_batch *b, const void *q,
                                     const void *k, float *scores,
                                     float *attn_rows, void *stream);

/*
 * Sec. 4.3, Table 4 (attention-source ablation): the sources compared there,
 * for a text query of M tokens q_1 .. q_M at positions q_begin .. q_end - 1
 * of a request (M = q_end - q_begin; q_M is the last query token p*).
 *   LAST_SRC_LAST      q_M            (the method's choice, Eq. 7)
 *   LAST_SRC_FIRST     q_1
 *   LAST_SRC_MIDDLE    q_ceil(M/2)    (indices count query tokens)
 *   LAST_SRC_ALL_MEAN  q_1 .. q_M     (rows averaged; the average and the sum
 *                                      give the same scores after Eq. 8)
 */
typedef enum {
  LAST_SRC_LAST = 0,
  LAST_SRC_FIRST = 1,
  LAST_SRC_MIDDLE = 2,
  LAST_SRC_ALL_MEAN = 3
} last_source;

/* Host helper: writes the request-local positions of source `src`'s rows to
 * pos_h (room for q_end - q_begin entries) in increasing order and returns
 * how many; -1 for q_begin < 0, q_end <= q_begin or an unknown source. */
int32_t last_source_rows(last_source src, int32_t q_begin, int32_t q_end, int32_t *pos_h);

/* Workspace bytes last_rows_scores needs (0 if the arguments are invalid). */
size_t last_rows_scores_workspace(const last_batch *b, const int32_t *cu_rows_h,
                                  const int32_t *row_pos_h);

/*
 * Sec. 4.3, Table 4, generalising Eq. 6-8 from the last query token's row to
 * any set of query rows per request:
 *   s_i = sum_l sum_h sum_{m in rows(r)} A^(l,h)[p_m, v_r + i],  w~ = s / sum s
 * Under the causal mask the row at position p attends to keys 0 .. p only:
 * its softmax runs over those p + 1 keys and visual tokens after p get
 * nothing from it.
 *   b          as for last_token_scores
 *   cu_rows    [R+1] CSR offsets of each request's rows; M_r >= 1
 *   row_pos    [M_total] request-local position of each row, with
 *              vis_start[r] <= p < P_r (every row sees a visual token)
 *   q          [G][M_total][Hq][Dh] the queries of those rows (after rotary
 *              embedding), same dtype as k
 *   k, scores, ws, stream   as for last_token_scores
 * One row per request (Last, First, Middle) runs the streamed single-row
 * kernels; several rows (All Mean) run two matrix-core passes over the keys:
 * row statistics, then the visual probabilities summed over rows and heads.
 * The result with one row per request at P_r - 1 equals last_token_scores.
 */
last_status last_rows_scores(const last_batch *b, const int32_t *cu_rows,
                             const int32_t *cu_rows_h, const int32_t *row_pos,
                             const int32_t *row_pos_h, const void *q, const void *k,
                             float *scores, void *ws, size_t ws_bytes, void *stream);

/* Workspace bytes last_prefill_attention needs (0 if invalid). */
size_t last_prefill_attention_workspace(const last_batch *b);

/*
 * Sec. 3.3: the guidance model's causal prefill attention, whose attention
 * tensors LAST reads, with the relevance of Eq. 6-8 taken from the same pass
 * (no second pass over the keys):
 *   out_p = sum_{j <= p} softmax_j(sigma q_p . k_j) v_j   for every position p
 *   scores = w~ from the rows of the last position of each request, exactly
 *            as last_token_scores computes them.
 *   b          as for last_token_scores; qk_dtype must be LAST_BF16 (others:
 *              LAST_ERR_UNSUPPORTED)
 *   q          [G][T_total][Hq][Dh] queries of every prefill position (after
 *              rotary embedding); each request's last position is its last
 *              query token
 *   k, v       [G][T_total][Hkv][Dh] keys and values
 *   out        [G][T_total][Hq][Dh] out, bf16 (rounded to nearest even)
 *   scores     [N_total] out, as for last_token_scores
 * The products use bf16 inputs with fp32 accumulation; the probabilities
 * enter the value product rounded to bf16 (relative error <= 2^-8 each).
 */
last_status last_prefill_attention(const last_batch *b, const void *q, const void *k,
                                   const void *v, void *out, float *scores, void *ws,
                                   size_t ws_bytes, void *stream);

/* Workspace bytes diverse_select needs (0 if the arguments are invalid):
 * for the k-center, those of the form it will take (see diverse_select),
 * which LAST_KCENTER_FORM, read at every call, can change. */
size_t diverse_select_workspace(int32_t R, const int32_t *cu_vis_h, int32_t Dv,
                                last_dtype fdtype, last_sel_mode mode);

/*
 * Sec. 3.4, Eq. 9-12 (mode LAST_SEL_KCENTER) or Sec. 4.3, Table 5
 * (mode LAST_SEL_TOPK).
 *   scores     [N_total] non-negative, finite fp32 relevance per visual token
 *              (normally the output of last_token_scores; any source works;
 *              negative or NaN entries are treated as 0)
 *   feats      [N_total][Dv] encoder features X of the visual tokens,
 *              row-major, fdtype (LAST_F32 or LAST_BF16); 1 <= Dv <= 65536
 *   cu_vis     [R+1] as in last_batch; N_r <= 131072 per request. The
 *              k-center takes one of two forms with the same results, bit
 *              for bit:
 *              - the matrix: all coverage distances of each request at once
 *                (4 ceil(N_r/128)^2 128^2 bytes of workspace per request:
 *                17 GB at 65536 tokens, 69 GB at 131072), then the greedy;
 *              - the rounds (bf16 features, Dv a multiple of 256 up to 4096,
 *                N_r <= 32768): only the distances to the tokens picked (the
 *                paper's O(K N d_v) form, about 28 bytes of workspace per
 *                token and 1.3 KB per request), computed for up to 128 picks at
 *                a time; the picks of a round are certified exact against
 *                every token outside its 192 candidates.
 *              By default the rounds take batches whose every request has
 *              8192 tokens or more and the shapes above, and other batches
 *              of those shapes where an estimate from the sizes and budgets
 *              says they are faster, whatever the relevance or, with the
 *              choice made on the device, unless a request's relevance is
 *              even (the workspace is then still the matrix's, as the query,
 *              which knows no budgets, says); the environment
 *              variable LAST_KCENTER_FORM=gram or =rounds forces one (rounds
 *              only where those shapes allow). The rounds run as a queue of
 *              tasks on one block per compute unit in which no block waits
 *              for one that has not started; a wait longer than 10 s (the
 *              device kept busy by other work) fills every unfinished
 *              request's kept and order with -1 and its gains with NaN.
 *              In the matrix form, requests longer than 32768 tokens (and longer than
 *              8192 when the batch is small) run the greedy on several
 *              compute units that exchange their candidates every step; if
 *              they cannot all run at once for 10 s (the device kept full
 *              by other work), the request's kept and order are filled
 *              with -1 and its gains with NaN (blocks that time out at the
 *              very end may leave some of the request's valid indices
 *              beside the -1 entries; either way the request is invalid).
 *              The environment variable LAST_MC_WAIT_US, read at every
 *              call, replaces the 10 s of either form (in microseconds)
 *   cu_keep    [R+1] budgets: K_r = cu_keep[r+1]-cu_keep[r], 1 <= K_r <= N_r
 *              (use last_budget for K = ceil(rho N), Eq. 2)
 *   kept       [K_total] out: the selected request-local indices, ascending
 *              within each request (Eq. 12)
 *   order      optional [K_total] out: the pick sequence j_1..j_K (k-center),
 *              or the kept indices by decreasing score (Top-k)
 *   gains      optional [K_total] out: w_j1 at t = 1 and w_jt * delta_jt at
 *              t >= 2 (k-center), or the scores in pick order (Top-k)
 * Ties in every argmax go to the lowest index. The coverage distance of
 * Eq. 10 is 1 - cos clamped at 0; a zero-norm feature has cosine 0 with
 * every token; bitwise-identical features are at distance exactly 0.
 */
last_status diverse_select(int32_t R, int32_t Dv, last_dtype fdtype,
                           last_sel_mode mode, const float *scores,
                           const void *feats, const int32_t *cu_vis,
                           const int32_t *cu_vis_h, const int32_t *cu_keep,
                           const int32_t *cu_keep_h, int32_t *kept,
                           int32_t *order, float *gains, void *ws,
                           size_t ws_bytes, void *stream);

/*
 * diverse_select in mode LAST_SEL_KCENTER, as two calls (Sec. 3.4): the
 * pairwise coverage distances of Eq. 10 depend only on the features, the
 * greedy of Eq. 9-11 also on the relevance scores. Splitting them lets a
 * caller compute the distances on a second stream while the scores of the
 * same batch are still being computed (Eq. 6-8), and join the streams before
 * the pick call. Together the two calls enqueue the same kernels as one
 * diverse_select call and give bit-identical kept, order and gains.
 *   ws         the diverse_select_similarity_workspace(R, cu_vis_h, Dv,
 *              fdtype) bytes, 256-byte aligned. The two calls always take the
 *              matrix form (the pick call has no features to fold rounds
 *              with). The similarity
 *              call writes the distances there; the pick call reads them, so
 *              both calls take the same workspace and the same R, Dv, fdtype
 *              and cu_vis (checked only for shape; distances of other
 *              features give a selection over those features).
 *   ordering   the pick call must run after the similarity call has
 *              finished (same stream, or an event the pick stream waits on),
 *              and no other call may reuse the workspace in between.
 * Arguments, errors and outputs are otherwise those of diverse_select; the
 * similarity call does not need the scores, the pick call not the features.
 */
size_t diverse_select_similarity_workspace(int32_t R, const int32_t *cu_vis_h,
                                           int32_t Dv, last_dtype fdtype);
last_status diverse_select_similarity(int32_t R, int32_t Dv, last_dtype fdtype,
                                      const void *feats, const int32_t *cu_vis,
                                      const int32_t *cu_vis_h, void *ws,
                                      size_t ws_bytes, void *stream);
last_status diverse_select_pick(int32_t R, int32_t Dv, last_dtype fdtype,
                                const float *scores, const int32_t *cu_vis,
                                const int32_t *cu_vis_h, const int32_t *cu_keep,
                                const int32_t *cu_keep_h, int32_t *kept,
                                int32_t *order, float *gains, void *ws,
                                size_t ws_bytes, void *stream);

/*
 * Sec. 3.4, Eq. 12: out[t] = feats[cu_vis[r] + kept[t]] for every kept slot
 * t of request r, copied byte for byte (row_bytes = Dv * elem_bytes).
 *   kept       [K_total] request-local indices (e.g. from diverse_select);
 *              an index outside [0, N_r) yields a zero-filled row
 *   out        [K_total][Dv] out, same element type as feats
 */
last_status gather_kept(int32_t R, int32_t Dv, size_t elem_bytes,
                        const void *feats, const int32_t *cu_vis,
                        const int32_t *cu_vis_h, const int32_t *kept,
                        const int32_t *cu_keep, const int32_t *cu_keep_h,
                        void *out, void *stream);

/* Workspace bytes last_connector needs for K rows: the normalised rows and
 * the hidden activations, bf16 (0 if the arguments are invalid). */
size_t last_connector_workspace(int64_t K, int32_t Dv, int32_t Dh);

/*
 * Sec. 3.4 after Eq. 12 (H_S = phi_c(X_S)) and Sec. 3.2: the cloud connector
 * applied token by token to the K rows the edge transmitted. The paper names
 * phi_c without a formula; this is the token-wise connector of the model
 * family it builds on:
 *   xhat = (x - mean(x)) / sqrt(var(x) + eps) * gamma + beta   (biased var)
 *   h    = GELU(W1 xhat + b1),  GELU(u) = u (1 + erf(u / sqrt 2)) / 2
 *   y    = W2 h + b2
 *   dtype      LAST_BF16 (others: LAST_ERR_UNSUPPORTED)
 *   K          rows, 0 <= K < 2^31 (0: nothing to do)
 *   x          [K][Dv] transmitted rows X_S (normally gather_kept's out)
 *   gamma,beta [Dv] fp32 LayerNorm scale and shift
 *   w1, b1     [Dh][Dv] (one hidden feature per row, dtype) and [Dh] fp32
 *   w2, b2     [Do][Dh] (one output feature per row, dtype) and [Do] fp32
 *   out        [K][Do] out, dtype (rounded to nearest even)
 *   eps        > 0 and finite (LAST_ERR_INVALID otherwise)
 * Dv and Dh must be multiples of 64 and Do of 4, each in [64, 65536], and
 * ceil(K / 256) ceil(max(Dh, Do) / 256) below 2^31 (LAST_ERR_UNSUPPORTED
 * otherwise). Every pointer must be 16-byte aligned (LAST_ERR_INVALID).
 * xhat and h are rounded to bf16 before the products, which accumulate in
 * fp32; GELU's erf is evaluated to within 1e-6 (1 + |u|). The workspace (256-byte aligned,
 * last_connector_workspace bytes) holds xhat and h; the caller owns every
 * buffer.
 */
last_status last_connector(last_dtype dtype, int64_t K, int32_t Dv, int32_t Dh, int32_t Do,
                           float eps, const void *x, const float *gamma, const float *beta,
                           const void *w1, const float *b1, const void *w2, const float *b2,
                           void *out, void *ws, size_t ws_bytes, void *stream);

/*
 * The paged cache of keys and values that answers are decoded from (Sec. 3.2,
 * 3.4: the cloud model reads the transmitted tokens, then produces its answer
 * token by token). G layers, each n_pages pages of page_size tokens:
 *   element (layer l, page p, head h, token t, d) of k lies at
 *   k[l layer_stride + p page_stride + h head_stride + t token_stride + d],
 *   strides in elements; v has the same layout.
 * Any order of layer, page, head and token is accepted as long as no two rows
 * of Dh elements overlap (the strides nest) and every row is 16-byte aligned.
 * page_size is a power of two in [8, 1024], Dh 64 or 128 and Hkv at most 65536
 * (others: LAST_ERR_UNSUPPORTED). k and v must not overlap each other.
 */
typedef struct last_cache {
  int32_t G, n_pages, page_size, Hkv, Dh;
  last_dtype dtype;
  int64_t layer_stride, page_stride, head_stride, token_stride;
  void *k, *v;
} last_cache;

/*
 * The sequences of a cache.
 *   R          sequences (>= 1)
 *   max_pages  entries of a page table row; max_pages * page_size <= 2^30
 *              (LAST_ERR_UNSUPPORTED otherwise)
 *   table      [R][max_pages] device: token t of sequence r lies in page
 *              table[r][t / page_size], the same page in every layer. Entries
 *              behind the last page of lens[r] tokens are never read.
 *   table_h    host copy, or NULL where the call allows it; where it is given,
 *              the entries of lens_h[r] tokens must name pages of the cache
 *              (LAST_ERR_INVALID)
 *   lens       [R] device: tokens of each sequence, 0 allowed
 *   lens_h     [R] host: what lens holds, or (calls that say so) a bound of it
 * The page table and the lengths may change between the replays of a captured
 * call, so the kernels check them too: a page outside [0, n_pages) is never
 * followed, and lengths are cut to [0, max(lens_h)]. That is the longest bound
 * of the call: a length above its own sequence's bound but not above that is
 * taken as it stands, through entries of table that the host did not check.
 */
typedef struct last_pages {
  int32_t R, max_pages;
  const int32_t *table, *table_h;
  const int32_t *lens, *lens_h;
} last_pages;

/*
 * A rotation of heads by positions with one to four axes (for visual tokens
 * time, height and width; for text all axes hold the same position):
 *   a_i = pos[axis[i]] * inv_freq[i],  i = 0 .. n_freqs - 1
 *   (x, y) -> (x cos a_i - y sin a_i, y cos a_i + x sin a_i)
 * for the pairs (x, y) = elements (i, i + n_freqs) of a head, or (2i, 2i + 1)
 * with adjacent != 0. Elements from 2 n_freqs on pass unchanged. inverse != 0
 * turns by -a_i: the inverse, which is also the gradient (the rotation is
 * orthogonal: dx = R^T dy), a call of its own.
 *   inv_freq   [n_freqs] device fp32, taken as they are: the angle is their
 *              product with the position in 64 bits
 *   axis       [n_freqs] device, and axis_h its host copy: each in [0, n_axes)
 * n_freqs is a positive multiple of 8 with 2 n_freqs <= Dh (others:
 * LAST_ERR_UNSUPPORTED), 1 <= n_axes <= 4.
 */
typedef struct last_rotation {
  int32_t n_axes, n_freqs, adjacent, inverse;
  const float *inv_freq;
  const int32_t *axis, *axis_h;
} last_rotation;

/*
 * Rows of heads, [G][T][heads][Dh]: element (g, t, h, d) lies at
 * data[g layer_stride + t token_stride + h Dh + d] (strides in elements), so
 * that q, k and v may be parts of one projection's output. Rows are 16-byte
 * aligned. What is only read may repeat (stride 0); what is written may not.
 */
typedef struct last_heads {
  void *data;
  int64_t layer_stride, token_stride;
} last_heads;

/*
 * The rotary embedding that last_prefill_attention and the score calls expect
 * their q and k to carry: q_out = rot(q), k_out = rot(k).
 *   G, T       layers and tokens (T >= 0); every layer has the same positions.
 *              G T below 2^24 is always taken; past that
 *              LAST_ERR_UNSUPPORTED may be returned
 *   Hq, Hkv    heads of q and k, at most 65536 each (LAST_ERR_UNSUPPORTED
 *              otherwise); one of them may be 0, its rows are then not read
 *              and may be NULL
 *   Dh         64 or 128 (others: LAST_ERR_UNSUPPORTED)
 *   dtype      of all rows (LAST_F32 or LAST_BF16); turned in fp32, rounded
 *              once, to nearest even
 *   pos        [n_axes][T] int32 positions, any value
 * In place (q_out the same rows as q, k_out as k) is allowed; other overlaps
 * of what is written with what is read are not.
 */
last_status last_rotary(const last_rotation *rot, last_dtype dtype, int32_t G, int32_t T,
                        int32_t Hq, int32_t Hkv, int32_t Dh, const int32_t *pos,
                        const last_heads *q, const last_heads *k, const last_heads *q_out,
                        const last_heads *k_out, void *stream);

/*
 * last_rotary with the turned keys, and the values, written into a cache:
 * the new tokens of sequence r become its last ones, at positions
 * lens[r] - n_r .. lens[r] - 1 of the sequence, where n_r is their number. So
 * lens counts them already, and the same last_pages serve the decoding step
 * that follows.
 *   rot        NULL: nothing is turned (keys are stored as they are, q and
 *              pos are not read, and Hq must be 0)
 *   c          the cache; layers [layer, layer + G) are written, row g of k
 *              and v into layer + g
 *   p          sequences; lens_h bounds lens from above, table_h may be NULL
 *   G, T       layers and new tokens of all sequences, limited as in
 *              last_rotary
 *   cu_new     [R+1] CSR offsets of each sequence's new tokens, which end at
 *              T (device and host copy); both NULL: one token per sequence, T = R
 *   pos        [n_axes][T] positions of the rotation (not of the cache)
 *   q, q_out   [G][T][Hq][Dh]; Hq may be 0 (not read then)
 *   k, v       [G][T][Hkv][Dh], the cache's dtype; not part of the cache
 * A token whose place lies before the sequence's start, behind the bound
 * max(lens_h), or in a page outside the cache is not stored (its q_out is
 * still written): a padded batch gives its empty slots lens[r] = 0.
 * No two sequences may write the same page.
 */
last_status last_rotary_append(const last_rotation *rot, const last_cache *c, int32_t layer,
                               int32_t G, const last_pages *p, int32_t T, const int32_t *cu_new,
                               const int32_t *cu_new_h, int32_t Hq, const int32_t *pos,
                               const last_heads *q, const last_heads *q_out, const last_heads *k,
                               const last_heads *v, void *stream);

/* Workspace bytes last_decode_attention needs (0 if the arguments are invalid,
 * at least 256 otherwise): a function of the cache's shape, Hq, the number of
 * sequences and lens_h, which need not be exact. It does not fall as sequences
 * or longer bounds are added, so a workspace for the most sequences and the
 * longest bounds serves every call below them. */
size_t last_decode_attention_workspace(const last_cache *c, const last_pages *p, int32_t Hq);

/*
 * Attention of one new token per sequence over its cached keys and values,
 * the decoding counterpart of last_prefill_attention:
 *   s_j = sigma q_r . k_j,  j = 0 .. lens[r] - 1
 *   out_r = sum_j e^(s_j - lse) v_j,  lse = ln sum_j e^(s_j)
 * per query head; query head h reads KV head h / (Hq / Hkv). A sequence of
 * length 0 gives out 0 and lse -inf; one whose page table names a page outside
 * the cache (within its length) gives NaN in both.
 *   layer      the layer read
 *   p          lens_h bounds lens from above (it shapes the launch; a captured
 *              call may be replayed with any lens up to its maximum); table_h
 *              may be NULL
 *   Hq         query heads, a multiple of the cache's Hkv. R Hq below 2^22 with
 *              R Hq times the longest bound below 2^35 is always taken; past
 *              that LAST_ERR_UNSUPPORTED may be returned
 *   scale      sigma; <= 0 selects 1/sqrt(Dh)
 *   q          [R][Hq][Dh] after the rotary embedding, row r at r * q_stride
 *              elements, 16-byte aligned
 *   out        [R][Hq][Dh] out, the cache's dtype, rounded to nearest even
 *   lse        optional [R][Hq] fp32 out (NULL to skip)
 *   ws         last_decode_attention_workspace bytes, 256-byte aligned; calls
 *              that may overlap in time need their own
 * Logits, softmax statistics, probabilities and sums are held in fp32 (for
 * bf16 caches a probability enters the value product as the sum of three bf16
 * numbers, exactly; as some of them may be 0, an infinite value may give NaN
 * instead of infinity). A long cache is split over blocks whose partial
 * results are joined in a fixed order.
 */
last_status last_decode_attention(const last_cache *c, int32_t layer, const last_pages *p,
                                  int32_t Hq, float scale, const void *q, int64_t q_stride,
                                  void *out, float *lse, void *ws, size_t ws_bytes, void *stream);

/*
 * Sec. 3.4, Eq. 12 on a cache: after the selection, a prompt's cache keeps its
 * text and the kept visual tokens only, in their order, in every layer:
 *   new token i comes from token  i                          i < vis_start
 *                                 vis_start + kept[i - vis_start]   the K_r next
 *                                 i - K_r + N_r              the rest
 *   src        the sequences as they are; lens_h exact, table_h required;
 *              vis_start + N_r <= lens
 *   dst        where they go, R and max_pages of its own, table_h required;
 *              lens_h[r] >= the new length lens - N_r + K_r; lens is not read
 *   vis_start, cu_vis  the visual spans as in last_batch (N_r >= 0)
 *   kept, cu_keep      as from diverse_select (0 <= K_r <= N_r): an index
 *              outside [0, N_r) yields a zero-filled row
 *   new_lens   optional [R] device out: the new lengths; not src->lens
 * R below 2^23 and R times the longest new length below 2^28 are always
 * taken; past that LAST_ERR_UNSUPPORTED may be returned.
 * Pages that dst writes must be listed once and not by src (LAST_ERR_INVALID):
 * the source stays whole, so other sequences may share its pages. The
 * exception is a page wholly before vis_start that both tables name at the
 * same place: it is shared and not copied.
 */
last_status last_cache_prune(const last_cache *c, const last_pages *src, const last_pages *dst,
                             const int32_t *vis_start, const int32_t *vis_start_h,
                             const int32_t *cu_vis, const int32_t *cu_vis_h, const int32_t *kept,
                             const int32_t *cu_keep, const int32_t *cu_keep_h, int32_t *new_lens,
                             void *stream);

/*
 * Copies n pages, keys and values of every layer, byte for byte: page src[i]
 * to page dst[i] (a forked sequence's last, partly filled page; pages moved
 * together). No page may be a target twice, or both source and target
 * (LAST_ERR_INVALID). src and dst: [n] device arrays with host copies, n >= 0.
 * Hkv page_size is at most 2^24 and 2 G n ceil(Hkv page_size Dh elt / 4096), elt
 * an element's bytes, below 2^24 (some 64 GiB; LAST_ERR_UNSUPPORTED otherwise).
 */
last_status last_cache_copy(const last_cache *c, int32_t n, const int32_t *src, const int32_t *src_h,
                            const int32_t *dst, const int32_t *dst_h, void *stream);

/* Sec. 3.2, Eq. 2: K = ceil(N * rho_num / rho_den), integer-exact, clamped
 * to [1, N]; returns -1 for N < 1 or a ratio outside (0, 1]. */
int32_t last_budget(int32_t N, int32_t rho_num, int32_t rho_den);

/* Human-readable text for a status (static storage). For LAST_ERR_DEVICE it
 * includes the most recent HIP error message seen by this thread. */
const char *last_status_string(last_status s);

/* Library version, as major * 10000 + minor * 100 + patch. */
int32_t last_version(void);

/*
 * Optional per-kernel timing, for benchmarking. While enabled, every kernel
 * the library launches is bracketed by a pair of HIP events on its stream
 * (event creation happens on first use; no device memory is allocated).
 * After the caller has synchronised the streams, last_profile_collect()
 * folds the finished pairs into per-kernel totals, which
 * last_profile_kernel() reports. The totals are process-wide and guarded by a
 * lock; with timing off (the default) a launch only reads an atomic flag, so
 * the compute calls stay free of shared mutable state. Event pairs beyond the
 * internal pool of 8192 are not recorded. A name returned by
 * last_profile_kernel() stays valid until the process ends.
 */
last_status last_profile_enable(int32_t on);
last_status last_profile_collect(void);
void last_profile_reset(void);
int32_t last_profile_count(void);
/* i-th kernel's name, launch count and total milliseconds; returns 0 if
 * there is no such entry. */
int32_t last_profile_kernel(int32_t i, const char **name, int64_t *launches,
                            double *total_ms);

#ifdef __cplusplus
}
#endif

#endif /* LAST_H */
