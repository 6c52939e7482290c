/*
 * restkv.h -- C ABI of the ReST-KV eviction path for AMD MI355X (gfx950).
 *
 * One call sequence compresses the KV cache of ONE transformer layer at prefill
 * time (the paper evicts once, after prefill; App. B):
 *
 *     restkv_prepare_wo   (once per layer's weights, not per request)
 *     restkv_score   ->  restkv_smooth  ->  restkv_select  ->  restkv_compact
 *
 * Notation (0-indexed): Hq query heads, Hkv KV heads, G = Hq/Hkv, d head_dim,
 * L cached tokens, W observation-window queries (the last W positions),
 * P = L - W evictable prefix tokens, B per-KV-head budget (the W window tokens
 * are always kept and count towards B).
 *
 * Pointers: every pointer argument except the parameter block is a DEVICE
 * pointer owned by the caller; the parameter block is a HOST pointer that is
 * read before the call returns.  The library allocates nothing, frees nothing
 * and never synchronises: each call validates its arguments on the host,
 * enqueues kernels on `stream` (a hipStream_t; NULL = the default stream) and
 * returns.  Scratch memory comes from the caller as `workspace` of at least
 * restkv_workspace_bytes() bytes, 256-byte aligned; its contents are undefined
 * between calls and calls that share a workspace must be ordered on one stream.
 *
 * Errors: every entry point returns RESTKV_OK (0) or a negative code; nothing is
 * enqueued when an error is returned, except RESTKV_EHIP, which reports a launch
 * failure of the HIP runtime and may leave earlier kernels of that call queued.
 * No entry point throws, aborts or prints.
 *
 * Design readings that the paper leaves open and no independent check can pin
 * ("parity unpinned"): the mean over the G query heads of a KV head (score), and
 * the way the fixed kernel size k widens under the adaptive window (smooth).
 */
#ifndef RESTKV_H_
#define RESTKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RESTKV_OK            0
#define RESTKV_EINVAL       (-1)  /* null pointer, inconsistent shape, budget outside (W, L], ... */
#define RESTKV_EUNSUPPORTED (-2)  /* head_dim not in {64,128}, unknown dtype, G*W too large ...   */
#define RESTKV_EWORKSPACE   (-3)  /* workspace missing, misaligned or too small                   */
#define RESTKV_EHIP         (-4)  /* the HIP runtime refused a launch                             */

#define RESTKV_F32  0   /* q, k, v and the compacted cache are IEEE binary32 */
#define RESTKV_BF16 1   /* ... are bfloat16                                   */

/*
 * Ablation variants (Sec. 4, ablation table; App. on the ablation study), selected through
 * restkv_params.variant.  0 is the method itself.
 *   indicator (restkv_score):  RESTKV_IND_ATTENTION   A[n], the attention weight alone
 *                              RESTKV_IND_VALUE_NORM  A[n] * ||v_n||_2  (gram is ignored by both)
 *   group reduction:           RESTKV_GROUP_MAX       largest indicator among the G query heads
 *                                                     of a KV head instead of their mean
 *   temporal (restkv_smooth):  RESTKV_TEMPORAL_MEAN   plain mean over the W window queries
 *                              RESTKV_TEMPORAL_INV_EMA the EMA recursion run from the newest
 *                                                     query to the oldest (oldest weighs alpha)
 *   spatial pooling:           RESTKV_POOL_MAX        maximum over the window instead of the mean
 * "No temporal smoothing" is ema_alpha = 1, "no spatial smoothing" base_window = 1 with
 * adaptive = 0, fixed average pooling adaptive = 0.
 */
#define RESTKV_IND_RECONSTRUCTION 0
#define RESTKV_IND_ATTENTION      1
#define RESTKV_IND_VALUE_NORM     2
#define RESTKV_GROUP_MAX          (1 << 2)
#define RESTKV_TEMPORAL_MEAN      (1 << 4)
#define RESTKV_TEMPORAL_INV_EMA   (2 << 4)
#define RESTKV_POOL_MAX           (1 << 6)

typedef void* restkv_stream_t;    /* a hipStream_t */

/*
 * Problem statement of one layer (Sec. 3.2, Definition 3.1: the layer's cache
 * <K_T, V_T>, the recent queries, the head's output projection and the budget B).
 */
typedef struct restkv_params {
  int32_t n_q_heads;     /* Hq                                                         */
  int32_t n_kv_heads;    /* Hkv, divides Hq                                            */
  int32_t head_dim;      /* d: 64 or 128                                               */
  int32_t seq_len;       /* L                                                          */
  int32_t window;        /* W = S_w, 1 <= W < L                                        */
  int32_t budget;        /* B, W < B <= L                                              */
  int32_t dtype;         /* RESTKV_F32 or RESTKV_BF16                                  */
  int32_t causal;        /* 1: window query i sees keys 0 .. L-W+i ; 0: all L keys     */
  float   scale;         /* logit scale; 0 selects 1/sqrt(d) (Eq. softmax)             */
  float   ema_alpha;     /* alpha of the EMA recursion: weight of the newest query     */
  int32_t base_window;   /* k: odd >= 1, the fixed kernel size of App. B               */
  int32_t adaptive;      /* 1: W_s and gamma_shift from D_front/D_rear ; 0: W_s=k, 0   */
  float   beta;          /* scaling factor of the adaptive window (> L / 2^30 when adaptive) */
  int32_t variant;       /* 0: the method; else a sum of RESTKV_IND_*, RESTKV_GROUP_MAX,
                            RESTKV_TEMPORAL_*, RESTKV_POOL_MAX (ablation variants, see below) */
  int64_t q_stride_h;    /* elements between query heads  (0: W*d)                     */
  int64_t q_stride_t;    /* elements between window queries (0: d)                     */
  int64_t kv_stride_h;   /* elements between KV heads     (0: L*d)                     */
  int64_t kv_stride_t;   /* elements between tokens       (0: d); rows are d-contiguous*/
  int64_t ld_score;      /* row stride (floats) of score / ema / final (0: P; >= P)    */
} restkv_params;

/*
 * Bytes of scratch the four calls below need for these parameters (0 if invalid).  The number differs between
 * builds of the library: ask the one that is loaded, keep none.  It covers both score paths, so bf16 layers
 * hold room for the FP32 one too.
 */
size_t restkv_workspace_bytes(const restkv_params* p);

/*
 * Gram matrices of the per-head output projection (Eq. mha: MHA = z W_O, with W_O
 * the head's rows of the layer's projection).  The indicator only needs
 * ||x W_O^h||_2, which depends on M_h = W_O^h W_O^hT alone.
 *   w_o   [Hq*d, d_model] float32, row-major, "z @ W_O" orientation: rows
 *         h*d .. (h+1)*d-1 belong to query head h (a framework weight stored
 *         [out,in] must be passed transposed).
 *   gram  [Hq, d, d] float32 out; symmetric by construction (restkv_score relies
 *         on M_h[i][j] == M_h[j][i]: some kernels read one triangle, some all).
 * Weight-only: run once per layer, not per request.  Accumulates in float64.
 */
int restkv_prepare_wo(const restkv_params* p, const float* w_o, int64_t d_model,
                      float* gram, restkv_stream_t stream);

/*
 * Layer-wise reconstruction indicator (Sec. 3.2, Eq. rec_ei; derivation App. A):
 * for every query head h, window query i and prefix token n
 *     I[h,i,n] = A[n] / (1 - A[n]) * || (z_{h,i} - v_n) W_O^h ||_2 ,
 * A = softmax(scale * q_{h,i} K^T) over the visible keys (Eq. softmax), z = A V.
 * The token holding the largest weight of a query is evaluated by the equivalent
 * leave-one-out form (Eq. ori with Eq. relation), which stays finite as A -> 1 (matrix-core kernels:
 * if it held more than half of the weight its key split had seen when it came, as every token with
 * A > 1/2 does).
 * Output is the mean over the G query heads of each KV head:
 *     score[g,i,n] = (1/G) sum_{h in g} I[h,i,n]          [Hkv, W, ld_score] float32
 *   q     [Hq, W, d]  (strides q_stride_*),  k, v  [Hkv, L, d] (strides kv_stride_*)
 *   gram  [Hq, d, d] from restkv_prepare_wo (any symmetric matrices), or NULL for
 *         W_O W_O^T = identity.
 * Columns n >= P of `score` are not written.
 * The squared distance is evaluated as z M z^T - 2 (z M) v_n^T + v_n M v_n^T in FP32; when the
 * three terms cancel (v_n W_O within a few 1e-3 of z W_O, relative to their norms) the rounding
 * residue of that sum enters by its magnitude (matrix-core kernels) or clamped at zero (FP32
 * kernels): the result then is a small non-negative number where the exact one is near zero.
 * The kernels for float32 inputs form their products from three bf16 parts of each value, to
 * the accuracy of FP32 products.  Inputs may be any FP32 values: what bf16 parts do not hold
 * (infinities, magnitudes near either end of the range) is found on the way and goes through
 * the FP32 instruction, which costs the part concerned (32 keys of a head, or a key split in the attention
 * pass) two to three times the time.  A key whose logits are -inf, as of a row of -FLT_MAX, has weight and score 0.
 */
int restkv_score(const restkv_params* p, const void* q, const void* k, const void* v,
                 const float* gram, float* score, void* workspace, size_t workspace_bytes,
                 restkv_stream_t stream);

/*
 * restkv_score with the attention statistics of the window queries taken from the caller's
 * own attention kernel instead of a pass over the cache (App. B: at prefill the statistics the
 * method needs are already there; Sec. 5: only the attention output of a small query window
 * is needed).  The usual pair a fused attention kernel returns:
 *   attn_out [Hq, W, d] float32, contiguous: softmax(scale q K^T) V of the W window queries over
 *            exactly the keys restkv_score would let them see (query i: keys 0 .. L-W+i when
 *            causal), same scale;
 *   lse      [Hq, W] float32: natural logarithm of each row's softmax denominator.
 * Everything else as restkv_score; the attention pass and its merge are replaced by a pass
 * over [Hq, W, d].  Without the unnormalised sums of a pass of its own the library cannot
 * evaluate a dominant key by the leave-one-out form: a key that holds more than about 0.9 of a
 * query's attention is scored through Eq. rec_ei in FP32 and loses accuracy as 1 - A
 * vanishes (relative error about 4e-6 / (1 - A)^2); every other key meets the same bound as
 * restkv_score.
 */
int restkv_score_from_attention(const restkv_params* p, const void* q, const void* k, const void* v,
                                const float* gram, const float* attn_out, const float* lse, float* score,
                                void* workspace, size_t workspace_bytes, restkv_stream_t stream);

/*
 * Spatial-temporal smoothing (Sec. 3.3).
 *   ema[g,n]   = EMA over the W window queries of score[g,:,n] (newest weighs alpha)
 *   D_front/D_rear = mean index of the per-query top-min(B,P) tokens of the raw
 *                score, over the first floor(W/2) / the remaining queries
 *   W_s   = k + 2 floor(|D_rear - D_front| / beta)
 *   gamma = floor((D_front - D_rear)/beta) (+1 unless D_front - D_rear > 0)
 *   final[g,n] = (1/W_s) sum_{j=-floor(W_s/2)+gamma}^{floor(W_s/2)+gamma} ema[g,n+j]
 *                (Eq. final_ei; terms outside [0,P) are zero)
 * adaptive = 0 or W = 1 gives W_s = k, gamma = 0.
 *   score [Hkv, W, ld] in;  ema [Hkv, ld] out (may be NULL: kept in workspace);
 *   final [Hkv, ld] out;  aws_info [Hkv, 2] int32 out = {W_s, gamma} (may be NULL);
 *   aws_d [Hkv, 2] float64 out = {D_front, D_rear} (may be NULL).
 */
int restkv_smooth(const restkv_params* p, const float* score, float* ema, float* final_score,
                  int32_t* aws_info, double* aws_d, void* workspace, size_t workspace_bytes,
                  restkv_stream_t stream);

/*
 * restkv_score followed by restkv_smooth as ONE call, with the same outputs (score included).
 * Workspace as reported by restkv_workspace_bytes.
 */
int restkv_score_smooth(const restkv_params* p, const void* q, const void* k, const void* v,
                        const float* gram, float* score, float* ema, float* final_score,
                        int32_t* aws_info, double* aws_d, void* workspace, size_t workspace_bytes,
                        restkv_stream_t stream);

/*
 * Per-head selection (Sec. 3.3, Eq. topk): the B - W prefix tokens with the
 * largest final[g, 0..P) (equal values: lower index wins), written in ascending
 * position order and followed by the window tokens P .. L-1.
 *   final [Hkv, ld] in;  idx [Hkv, B] int32 out.
 * Uses the workspace (samples, per-chunk counters, candidates); like every call
 * here it allocates nothing and returns RESTKV_EWORKSPACE if the workspace is
 * NULL, misaligned or smaller than restkv_workspace_bytes().
 */
int restkv_select(const restkv_params* p, const float* final_score, int32_t* idx,
                  void* workspace, size_t workspace_bytes, restkv_stream_t stream);

/*
 * Non-uniform budgets (App. C of the paper pairs the indicator with layer-wise and head-wise
 * allocation).  A layer-wise budget is just `budget` of that layer's parameter block; the
 * two calls below take a budget per KV head instead:
 *   head_budget [Hkv] int32 on the device; entry g is used as min(max(b, W + 1), budget), so
 *   `budget` of the parameter block is the largest budget and stays the row stride of idx,
 *   k_out and v_out.
 * restkv_smooth_b uses min(head_budget[g], P) in place of min(B, P) for the per-query top-B
 * statistics of head g; restkv_select_b keeps head_budget[g] - W prefix tokens of head g,
 * appends the W window tokens, and fills idx[g, head_budget[g] .. B) with -1, which
 * restkv_compact turns into zero rows.  Everything else as restkv_smooth / restkv_select.
 */
int restkv_smooth_b(const restkv_params* p, const float* score, const int32_t* head_budget, float* ema,
                    float* final_score, int32_t* aws_info, double* aws_d, void* workspace,
                    size_t workspace_bytes, restkv_stream_t stream);
int restkv_select_b(const restkv_params* p, const float* final_score, const int32_t* head_budget,
                    int32_t* idx, void* workspace, size_t workspace_bytes, restkv_stream_t stream);

/*
 * restkv_select for callers that cannot allocate device memory or hand over a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same result as
 * restkv_select (same kernels); the scratch is an array inside the library's device image, one
 * copy per GPU that lives until the process ends (restkv_select_static_capacity() bytes, 4 MiB).
 * Returns RESTKV_EWORKSPACE, with nothing enqueued, when the shape needs more than that: about
 * 0.5 KiB per 4096 prefix positions and KV head (250 KV heads fit at 128k tokens).  The call
 * allocates nothing and frees nothing (the first call on a GPU looks up the array's address
 * once).  Every call on a GPU uses that GPU's one array: calls that overlap in time on one GPU
 * (different streams or host threads) race; calls ordered on one stream are safe, and each call
 * clears what it needs cleared itself.
 */
int restkv_select_static(const restkv_params* p, const float* final_score, int32_t* idx,
                         restkv_stream_t stream);
size_t restkv_select_static_capacity(void);

/*
 * Gather of the kept rows (Eq. topk): k_out[g,j,:] = k[g, idx[g,j], :], same for v.
 *   idx [Hkv, B] int32 in, entries in [0, L) (an entry outside is written as zeros);
 *   k_out, v_out [Hkv, B, d] out, contiguous, dtype of the inputs.
 */
int restkv_compact(const restkv_params* p, const void* k, const void* v, const int32_t* idx,
                   void* k_out, void* v_out, restkv_stream_t stream);

/*
 * The four calls of a layer as one: restkv_score, restkv_smooth, restkv_select, restkv_compact with the same arguments and
 * the same results, bit for bit.  For short layers the smoothing over positions, the selection and the gather are one
 * launch (its time is stage "select"; "box" and "compact" then have none).  Every argument of every stage is checked
 * before anything is enqueued; ema, aws_info and aws_d may be NULL.
 */
int restkv_evict(const restkv_params* p, const void* q, const void* k, const void* v, const float* gram,
                 float* score, float* ema, float* final_score, int32_t* aws_info, double* aws_d, int32_t* idx,
                 void* k_out, void* v_out, void* workspace, size_t workspace_bytes, restkv_stream_t stream);

/*
 * ---- Paged cache -------------------------------------------------------------
 * What follows an eviction: the kept rows go into pages, decoding appends to them and attends to them, and the
 * rows come back as dense tensors when the cache is evicted again:
 *
 *     restkv_evict -> restkv_append (k_out, v_out, no rotation)
 *     each step:      restkv_append (new keys and values, rotated)  ->  restkv_attend
 *     re-eviction:    restkv_attend (window queries) -> restkv_fetch -> restkv_score_from_attention -> ...
 *
 * Pages.  A page holds page_size cache positions; `table` names, for each sequence (and, if told so, each KV head), the
 * page of positions 0 .. page_size-1, of the next page_size, and so on.  Keys and values lie in two arrays of rows, a
 * row the d channels of one position of one KV head.  The row of position t is row
 *     table[...][t / page_size] * page_stride + head * head_stride + (t % page_size) * token_stride .
 * Formats of a row: RESTKV_F32 and RESTKV_BF16, d values of that type; RESTKV_Q4, d/2 bytes of codes, and in a second
 * array (k_scale, v_scale) d/32 pairs {step, zero} of bfloat16.  Channel c of a 4-bit row is in byte c/2, the even one in
 * the low half; it belongs to group (c mod (d/16)) / 2, and stands for zero + step * code.  restkv_append makes them so,
 * in float32, each operation rounded to nearest:
 *     zero = least of the group, rounded down to bfloat16;  step = (greatest - zero) / 15, rounded up to bfloat16, and at
 *     least 2^-100 (0 if greatest = zero);  code = (x - zero) * (1 / step), rounded to the nearest integer (even).
 * So no value is further off than half a step (and float32 rounding).  A group that holds a NaN or an infinity, or
 * spans more than float32 does, comes back as NaN.
 *
 * Lengths.  `lens` says how many positions each sequence (or each KV head of it, after an eviction with
 * budgets per head) holds INCLUDING the new tokens of the call: new token i of n goes to position len - n + i, and as a
 * query it sees positions 0 .. len - n + i (all len with causal = 0).  The calls only read `lens`.
 * New tokens are packed: those of sequence s are rows new_start[s] .. new_start[s+1]-1 of the token tensors
 * (new_start NULL: max_new of each sequence).  Rows outside all sequences are left as they are.
 *
 * Values on the device cannot be refused.  A length below 0 counts as 0; of one beyond the room (max_len) the places of the new
 * tokens follow, and what they see, but no position from max_len on is written or seen.  A new_start outside [0, n_tokens], or
 * below the one before it, counts as brought inside (a row that two sequences then claim belongs to either); a sequence takes
 * part with its first max_new new tokens at most, and its places follow from the number that does; a position without a page
 * (its table entry outside [0, n_pages)) is neither written nor seen.  Table entries behind the last position in use are not
 * read as pages.  Two positions of one call must not share a slot.
 *
 * Limits beside those at the fields: an array of pages has fewer than 2^32 - 1 rows from its first to its last; values are of
 * magnitude 2^80 at most (sums are not divided before the end, so larger ones may pass float32); restkv_attend may refuse
 * max_new * n_q_heads of 2^24 and more (RESTKV_EUNSUPPORTED).  Strides by which rows of out, lse or q_out overlap are refused.  A call
 * without a sequence, a token or a row does nothing and looks at no array.
 */
#define RESTKV_Q4 4   /* restkv_cache.format: 4-bit codes with a step and a zero for every 32 channels */

typedef struct restkv_cache {
  int32_t n_seqs;        /* sequences, up to 16384 (0: nothing is done)                          */
  int32_t n_q_heads;     /* Hq                                                                   */
  int32_t n_kv_heads;    /* Hkv, divides Hq                                                      */
  int32_t head_dim;      /* d: 64 or 128                                                         */
  int32_t dtype;         /* tokens, queries, fetched rows: RESTKV_F32 or RESTKV_BF16             */
  int32_t format;        /* pages: the same, or RESTKV_Q4                                        */
  int32_t page_size;     /* positions of a page: a power of two, 16 .. 65536                     */
  int32_t n_pages;       /* pages there are                                                      */
  int32_t max_pages;     /* table entries of a sequence; max_pages * page_size <= 2^30           */
  int32_t max_len;       /* no length is above this (0: max_pages * page_size); a tight one spares launches */
  int32_t max_new;       /* most new tokens of one sequence in a call                            */
  int32_t n_tokens;      /* rows of the packed token tensors                                     */
  int32_t causal;        /* 1: a query sees positions up to its own; 0: all                      */
  int32_t rotary_dim;    /* channels that are rotated: 0 (none) or a multiple of 16 up to d      */
  int32_t rotary_pairs;  /* 0: channel c turns with c + rotary_dim/2; 1: channel 2c with 2c + 1  */
  int32_t n_positions;   /* rows of the tables of cosines and sines                              */
  int32_t out_dtype;     /* attention output: dtype, or RESTKV_F32                               */
  float   scale;         /* logit scale, below 2^127; 0 selects 1/sqrt(d)                        */
  int64_t page_stride, head_stride, token_stride;   /* rows; token_stride 0: [page][Hkv][page_size];
                            with tables per head head_stride may be 0.  token_stride <= 2^16     */
  int64_t table_stride_s, table_stride_h;   /* int32 entries; 0, 0: max_pages, 0 (heads share)   */
  int64_t lens_stride_s, lens_stride_h;     /* int32 entries; 0, 0: 1, 0 (heads share)           */
  int64_t q_stride_t, q_stride_h;           /* elements; 0: Hq*d, 0: d                           */
  int64_t kv_stride_t, kv_stride_h;         /* elements; 0: Hkv*d, 0: d                          */
  int64_t out_stride_t, out_stride_h;       /* elements; 0: Hq*d, 0: d                           */
  int64_t lse_stride_t, lse_stride_h;       /* floats;   0: Hq, 0: 1                             */
} restkv_cache;

/*
 * New tokens into the pages, keys rotated by their position on the way, and new queries rotated beside them.
 *   k, v    [n_tokens, Hkv, d] (strides kv_stride_*);  q  [n_tokens, Hq, d] (q_stride_*) or NULL;
 *   q_out   with q's strides; may be q itself
 *   k_pages, v_pages (and k_scale, v_scale with RESTKV_Q4): 16-byte aligned
 *   positions [n_tokens] int32: where each token stands in its text (an evicted cache is shorter than the text);
 *           NULL: its cache position (not with lens per head).  A token whose position lies outside [0, n_positions)
 *           is left out: nothing of it is written
 *   cos, sin [n_positions, rotary_dim/2] float32;  with rotary_dim = 0 none of the three is looked at
 * y[a] = x[a] cos - x[b] sin, y[b] = x[b] cos + x[a] sin for the channels a, b that turn together, in float32 with
 * each product and each sum rounded, then rounded once to the type of the pages (4-bit: the codes are made from float32).
 */
int restkv_append(const restkv_cache* c, const void* k, const void* v, void* k_pages, void* v_pages, void* k_scale,
                  void* v_scale, const int32_t* table, const int32_t* lens, const int32_t* new_start,
                  const int32_t* positions, const float* cos, const float* sin, const void* q, void* q_out,
                  restkv_stream_t stream);

/*
 * Attention of the new tokens' queries over the pages, which hold their keys and values already (restkv_append):
 *   out  [n_tokens, Hq, d] out_dtype (out_stride_*):  softmax(scale q K^T) V over the positions a query sees
 *   lse  [n_tokens, Hq] float32 (lse_stride_*), may be NULL: natural logarithm of the softmax denominator
 * A query that sees nothing, or only keys of logit -inf, gets 0 and -inf.  What a query does not see has no influence,
 * whatever it holds (infinities and NaN included); what it sees and is not finite gives an output that is not finite
 * (with bf16 and 4-bit pages an infinity may come out as NaN).  With out_dtype RESTKV_F32, out_stride_h = W*d, out_stride_t = d,
 * lse_stride_h = W and lse_stride_t = 1 one sequence's W queries give what restkv_score_from_attention takes.
 * Logits, statistics and sums are float32 (bf16 products are exact in it); softmax weights enter the products with
 * values to 2^-17, with float32 output to 2^-24 (of 4-bit pages with 16 + code, or code - 8, steps; what is between these and the value
 * is added in float32).  Results do not depend on timing: no atomics.
 * Workspace: restkv_attend_workspace_bytes(c), 256-byte aligned, whatever it holds; none where that returns 0.  Calls, or
 * replays of captured ones, that run at the same time need one each.
 */
size_t restkv_attend_workspace_bytes(const restkv_cache* c);
int restkv_attend(const restkv_cache* c, const void* q, const void* k_pages, const void* v_pages, const void* k_scale,
                  const void* v_scale, const int32_t* table, const int32_t* lens, const int32_t* new_start, void* out,
                  float* lse, void* workspace, size_t workspace_bytes, restkv_stream_t stream);

/*
 * Rows of the pages as dense tensors, 4-bit rows as the values they stand for (the paged sibling of restkv_compact):
 *   k_out, v_out [n_seqs, Hkv, n_rows, d] dtype, contiguous, 16-byte aligned
 *   idx  [n_seqs, Hkv, n_rows] int32 positions, or NULL: positions first .. first + n_rows - 1
 * A position outside [0, len) or without a page gives a row of zeros.
 */
int restkv_fetch(const restkv_cache* c, const void* k_pages, const void* v_pages, const void* k_scale, const void* v_scale,
                 const int32_t* table, const int32_t* lens, const int32_t* idx, int32_t first, int32_t n_rows, void* k_out,
                 void* v_out, restkv_stream_t stream);

/*
 * ---- Beams -------------------------------------------------------------------
 * Requests that are decoded in several branches over one paged cache: the beams of a beam search, or conversations behind
 * one prompt.  A group of n_beams neighbouring sequences belongs to a request, and beam b of group g is sequence
 * g * n_beams + b of the cache.  One step:
 *
 *     restkv_append -> restkv_attend_beams   (each layer)   -> logits -> restkv_beam_select -> restkv_beam_reorder
 *
 * Pages of a beam search.  A page that is full may stand in the tables of all beams of a group; a page that is still
 * written to belongs to one beam.  Which page a beam writes to next is in its table from the start (n_beams pages for each
 * column that the search may reach), so a step allocates nothing: restkv_beam_reorder deals the pages of the open columns
 * anew.  After a prompt in beam 0's pages a reorder with parents 0, 0, .. makes the other beams.
 */
typedef struct restkv_beams {
  int32_t n_groups;      /* requests, up to 16384 (0: nothing is done)                          */
  int32_t n_beams;       /* beams of a request, 1 .. 64                                          */
  int32_t n_vocab;       /* logits of a beam, 1 .. 2^24                                          */
  int32_t n_out;         /* continuations taken of a request, 1 .. 64                            */
  int32_t dtype;         /* logits: RESTKV_F32 or RESTKV_BF16                                    */
  int32_t end_token;     /* ends a beam, and is what a beam that has ended goes on with          */
  int64_t logit_stride;  /* elements from a beam's logits to the next beam's; 0: n_vocab         */
} restkv_beams;

/*
 * The best continuations of each request's beams.  With logits x[b, v] and the score c[b] that beam b has so far,
 *     score(b, v) = c[b] + (x[b, v] - m_b) - ln(sum over v' of exp(x[b, v'] - m_b)),   m_b the largest logit of b,
 * and a beam that has ended has one continuation, (b, end_token) of score c[b].  The n_out largest are taken; of equal
 * scores the lower beam's is the larger, then the one of the larger logit, then the lower token's.  Only scores that are
 * finite as float32 are taken: a logit of -inf (a token that is masked out) is none, a beam with a score that is not finite has none, nor has one
 * with a NaN or +inf among its logits.  Places that are left get -inf, -1, -1 and 1.
 *   logits   [n_groups * n_beams, n_vocab] dtype (logit_stride), any alignment of that type
 *   scores   [n_groups, n_beams] float32;  finished [n_groups, n_beams] int32 (nonzero: ended) or NULL
 *   new_scores [n_groups, n_out] float32, parents (the beam, 0 .. n_beams-1), tokens [n_groups, n_out] int32 out, best first
 *   new_finished [n_groups, n_out] int32 out, may be NULL: 1 where the token is end_token or the beam had ended
 * new_scores may be scores, and new_finished may be finished, if n_out = n_beams.
 * Exponentials are float32, and summed in float32 up to 32 at a time (sums of these, logarithms and scores 64 bits); scores are ordered
 * in 64 bits and rounded once.  Results do not depend on timing: places follow from the order of the continuations (a counter only says where
 * in a list one is kept until then).
 * Workspace: restkv_beam_workspace_bytes(b), 256-byte aligned, whatever it holds; calls that run at the same time need one each.
 */
size_t restkv_beam_workspace_bytes(const restkv_beams* b);
int restkv_beam_select(const restkv_beams* b, const void* logits, const float* scores, const int32_t* finished,
                       float* new_scores, int32_t* parents, int32_t* tokens, int32_t* new_finished, void* workspace,
                       size_t workspace_bytes, restkv_stream_t stream);

/*
 * Beam b of each group goes on from beam parents[b] of the group: its table names the parent's pages where they are full, and
 * in the columns that are still written to it has pages of its own with the parent's rows in them.
 *   parents [n_groups] rows of n_beams int32, parents_stride entries apart (0: n_beams); n_groups = n_seqs / n_beams.  An entry
 *           outside [0, n_beams) counts as b itself
 *   lens    positions that are there (strides as ever; without new tokens); those of a group's first beam count for all of it
 *   table   the tables before, table_out after; table_out may be table itself, else they must not overlap.  Strides as ever
 *   layers  HOST array of n_layers (0 .. 256): the pages of each layer, all as the description says.  Read before the call returns
 * A column is full if every KV head that shares the table has filled its page, and open from there to the last page in use.  In
 * an open column the pages of the parents go to one child each (the parent itself where it is its own child, else its first
 * child), those of beams without a child to the other children, in order of the beams; into these the rows in use are
 * copied.  Columns behind the open ones stay as they are.  So in columns that are, or will be, written to no page is lost or doubled,
 * and a step needs none.  (In a full column the pages of beams that nobody goes on from are in no table any more.)
 * In open columns the beams of a group must have pages that differ.  An entry outside [0, n_pages) is dealt like any, and no row
 * of it is read or written.  Rows behind the lengths are left as they were.
 */
typedef struct restkv_layer_pages { void *k_pages, *v_pages, *k_scale, *v_scale; } restkv_layer_pages;
int restkv_beam_reorder(const restkv_cache* c, int32_t n_beams, const int32_t* parents, int64_t parents_stride,
                        const int32_t* lens, const int32_t* table, int32_t* table_out, const restkv_layer_pages* layers,
                        int32_t n_layers, restkv_stream_t stream);

/*
 * restkv_attend for beams whose tables begin with the same pages: these are read once for all beams of a group.
 *   shared [n_seqs / n_beams] int32: so many table entries in front are the same for all sequences of the group (of each KV
 *          head, with tables per head).  Values below 0 count as 0; pages beyond what every beam of the group with new tokens
 *          has seen before them are each beam's own.
 * Everything else, the result too, as restkv_attend says (n_beams 1 .. 64).  Where the tables differ after all, a beam sees its own
 * pages there or the first beam's, by sizes.  Workspace: restkv_attend_beams_workspace_bytes(c, n_beams).  Beside caches that are read as
 * restkv_attend does, it has room for two sums of d + 2 floats for every query row of n_seqs * max_new * n_q_heads, and some more: 1.05 GiB for
 * 64 sequences with 512 new tokens each and 32 heads of 128 (restkv_attend: 81 MiB), so long prompts of beams go through restkv_attend.  May be refused
 * (RESTKV_EUNSUPPORTED): n_beams * max_new * n_q_heads / n_kv_heads of 2^24 and more, n_seqs * max_new * n_q_heads of 2^29 and more.
 */
size_t restkv_attend_beams_workspace_bytes(const restkv_cache* c, int32_t n_beams);
int restkv_attend_beams(const restkv_cache* c, int32_t n_beams, const int32_t* shared, const void* q, const void* k_pages,
                        const void* v_pages, const void* k_scale, const void* v_scale, const int32_t* table, const int32_t* lens,
                        const int32_t* new_start, void* out, float* lse, void* workspace, size_t workspace_bytes,
                        restkv_stream_t stream);

/*
 * Profiling aid (not part of the method): every kernel launch of a selected stage
 * is bracketed by two HIP events on the caller's stream.  stage_mask: bit s selects
 * stage s (see restkv_stage_name), -1 selects all, 0 turns timing off.  A bracket
 * costs a few microseconds of idle GPU, so timing all stages slows a layer by
 * about a tenth; timing one stage is nearly free.
 * restkv_timing_read() blocks until those events have completed, adds the elapsed
 * milliseconds and the number of launches per stage into ms[] / launches[] (host
 * arrays of n_stages >= RESTKV_N_STAGES entries) and forgets them.  Disabled by
 * default; enabling or disabling also forgets pending records.  Not thread-safe
 * against concurrent launches on other host threads beyond a mutex on the records.
 * Stages "attn_partial" and "vv" (attention and value-Gram pass): on the bf16 matrix-core path, and on most layers of the
 * FP32 path, they are one launch, which "attn_partial" counts.  "vv" reports launches where there is no attention pass
 * (statistics handed in), for the value norms of the indicators without a projection, and on FP32 layers where few rows per KV
 * head keep two wavefronts per workgroup and their key splits fill the compute units (heads of 128).
 */
#define RESTKV_N_STAGES 10
int restkv_timing_enable(int stage_mask);
int restkv_timing_read(double* ms, int64_t* launches, int n_stages);
const char* restkv_stage_name(int stage);   /* "gram", "attn_partial", ... */

/*
 * Measurement aid, no part of the eviction path: one plain streaming kernel (16-byte loads
 * and stores, reads and writes interleaved step by step, no arithmetic beyond an XOR) that reads
 * read_bytes from src and writes write_bytes to dst, so that a kernel's HBM rate can be set
 * against what the part delivers for the same byte mix.
 * src, dst: DEVICE pointers (16-byte aligned), caller-owned, must not overlap; read_bytes and
 * write_bytes multiples of 16; either may be 0.  Result: 32-bit word i of dst = i XOR (all
 * words the writing thread read in earlier steps), i.e. dst[i] = i for an all-zero source.
 * Asynchronous on `stream`; RESTKV_EINVAL for null, misaligned or odd-sized arguments.
 */
int restkv_stream_reference(const void* src, size_t read_bytes, void* dst, size_t write_bytes,
                            void* stream);

/*
 * Debug aid: with on != 0 restkv_score runs bf16 inputs through the kernels for float32 inputs
 * (same stages, products as exact as FP32 ones).  Process-wide.
 */
int restkv_debug_force_fp32(int on);

/*
 * Debug aid: how restkv_score with Gram matrices runs the attention pass of these parameters on the bf16 matrix-core
 * path (aligned pointers assumed; RESTKV_EUNSUPPORTED where that path does not take them).  plan: HOST array of 4:
 * number of key splits, 64-key tiles of a split, 1 if the value-Gram pass runs beside it on a part of the compute units,
 * 1 if heavy attention weights enter the sums as two bf16 numbers.
 */
int restkv_debug_score_plan(const restkv_params* p, int32_t* plan);

/*
 * Debug aid: how restkv_score with Gram matrices launches the passes of a float32 layer (RESTKV_EUNSUPPORTED for other
 * inputs).  plan: HOST array of 4: number of key splits, 1 if the value-Gram pass is in the attention pass's launch,
 * wavefronts of a workgroup of the score pass, 1 if these divide the heads of the group (else the keys).
 */
int restkv_debug_fp32_plan(const restkv_params* p, int32_t* plan);

/*
 * Debug aid: with on != 0 restkv_attend_beams reads shared pages once for all beams however short the caches are (short ones are
 * otherwise read as restkv_attend does).  Process-wide; its workspace size follows.
 */
int restkv_debug_force_shared(int on);

/*
 * Debug aid: into how many chunks restkv_attend_beams would cut what these caches hold, where it works by a list of chunks
 * (RESTKV_EUNSUPPORTED elsewhere), and how many there is room for in its workspace.  tiles: HOST array of tiles of 64 positions, 0 .. 2^24 each: what
 * each group shares (of each KV head, with lengths per head), then what each sequence (and head) has behind it.  chunks: HOST array of 4:
 * chunks of shared positions, room for these, chunks of the rest, room for those.
 */
int restkv_debug_beams_list(const restkv_cache* c, int32_t n_beams, const int32_t* tiles, int32_t* chunks);

/* Static description of an error code. */
const char* restkv_strerror(int code);

/* Library version (major*10000 + minor*100 + patch). */
int restkv_version(void);

#ifdef __cplusplus
}
#endif
#endif /* RESTKV_H_ */
