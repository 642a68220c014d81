/*
 * avtp.h -- C ABI of libavtp.so, the MI355X (gfx950) pruning-layer operator of
 * "Multi-Image Visual Token Pruning in Large Visual Language Models" (AVTP).
 *
 * A pruning layer turns the n visual tokens of each sequence into a shorter
 * subsequence (Method, "Visual Token Pruning": E_pruned = p(E_v)).  The four
 * calls below are the four steps of that map:
 *
 *   avtp_score   importance of every visual token and its per-image sum
 *   avtp_budget  per-image keep counts from the image importances
 *   avtp_select  per-image top-k -> ascending list of kept token indices
 *   avtp_compact gather of hidden states, position ids and the layer's K/V
 *
 * Conventions shared by every call
 *   - Every data pointer is caller-owned DEVICE memory unless its name starts
 *     with h_ or the comment says "host".  The library allocates nothing.
 *   - Calls are asynchronous on `stream` (a hipStream_t; NULL = null stream).
 *     Argument errors are detected on the host, before anything is enqueued,
 *     and returned synchronously; nothing is launched in that case.
 *   - Return value: AVTP_OK or a negative avtp_status.  HIP launch errors map
 *     to AVTP_ERR_HIP.
 *   - Data-dependent conditions found on the device are OR-ed into the
 *     optional per-sequence status word (int32 [B], caller zero-fills it).
 *   - Outputs must not alias inputs.  No global mutable state (except the
 *     per-GPU scratch of avtp_score_noalloc, below): calls on different
 *     streams with different buffers may run concurrently.
 */
#ifndef AVTP_H
#define AVTP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef void *avtp_stream_t; /* a hipStream_t */

typedef enum {
  AVTP_OK = 0,
  AVTP_ERR_INVALID_ARG = -1, /* null pointer, inconsistent layout, bad size */
  AVTP_ERR_UNSUPPORTED = -2, /* head_dim, dtype, or a size beyond the limits below */
  AVTP_ERR_INFEASIBLE = -3,  /* keep_total outside [sum of lower, sum of upper bounds] */
  AVTP_ERR_WORKSPACE = -4,   /* workspace missing or smaller than *_workspace_size */
  AVTP_ERR_HIP = -5          /* a HIP launch failed */
} avtp_status;

typedef enum { AVTP_BF16 = 0, AVTP_FP32 = 1 } avtp_dtype;

typedef enum {
  AVTP_SCORE_ATTN = 0,      /* attention paid by the text rows to each visual token */
  AVTP_SCORE_VARIATION = 1  /* 1 - cos(h^l, h^prior), the hidden-state variation  */
} avtp_score_mode;

typedef enum {
  AVTP_BUDGET_PROPORTIONAL = 0, /* keep ratio scaled by importance / mean importance */
  AVTP_BUDGET_RAW = 1           /* keep ratio shifted by alpha (importance - mean)   */
} avtp_budget_mode;

/* per-sequence device status bits */
#define AVTP_FLAG_NAN_SCORE 1       /* a visual score was NaN (ranked last)           */
#define AVTP_FLAG_NO_TEXT_AFTER 2   /* an image has no text row after it (scores = 0) */
#define AVTP_FLAG_INFEASIBLE 4      /* budget bounds cannot meet keep_total           */
#define AVTP_FLAG_OUT_CAPACITY 8    /* kept list longer than keep_capacity (truncated), */
                                    /* or a full page stack (avtp_page_trim)            */
#define AVTP_FLAG_BAD_PAGE 16       /* a block table entry in use lies outside the pool */
#define AVTP_FLAG_NO_PAGES 32       /* avtp_page_tables, _fork: a request got no place  */
#define AVTP_FLAG_REFUSED 64        /* avtp_page_fork, avtp_page_release: the sequence  */
                                    /* could not be forked or cut so, and stays         */

/* Limits checked on the host (AVTP_ERR_UNSUPPORTED beyond them). */
#define AVTP_MAX_IMAGES_PER_SEQ 256
#define AVTP_MAX_IMAGES 8192
#define AVTP_MAX_IMAGE_LEN (1 << 20)
#define AVTP_MAX_TENSORS 8
#define AVTP_MAX_LAYERS 1024       /* avtp_layer_select: layers               */
#define AVTP_MAX_SAMPLES (1 << 20) /* avtp_layer_select: samples              */
#define AVTP_MAX_REQUESTS (1 << 16) /* avtp_page_*: sequences of a batch      */
#define AVTP_MAX_PLANES 4          /* planes of positions of a rotation       */
/* The attention score (avtp_score in attention mode, avtp_row_lse) addresses
 * one sequence's keys and text-row queries with 32-bit byte offsets: every
 * sequence must have (its tokens) * Hkv * d * elem and (its text rows) *
 * Hq * d * elem below AVTP_MAX_SEQ_BYTES (elem: 2 for bf16, 4 for fp32). */
#define AVTP_MAX_SEQ_BYTES (1ll << 32)

/*
 * Packed ("THD") description of one batch of B sequences, N_tok tokens.
 * Sequence b owns tokens [cu_seqlens[b], cu_seqlens[b+1]).  Every token is
 * either a text token or belongs to exactly one image:
 *   image i: tokens [img_start[i], img_start[i] + img_len[i]) (global
 *            indices); the images of sequence b are cu_img[b] .. cu_img[b+1]-1,
 *            in ascending position order;
 *   text t:  token text_pos[t]; the text rows of sequence b are
 *            cu_text[b] .. cu_text[b+1]-1, in ascending position order.
 * keep_total[b] is the number of visual tokens sequence b keeps.
 * Each int32 array is given twice: as device memory (read by the kernels)
 * and as a host mirror with identical contents (read by the host-side
 * validation and launch sizing; never dereferenced on the device).  Arrays
 * of length 0 may be NULL (img_start, img_len when n_img = 0; text_pos when
 * T_tot = 0).
 */
typedef struct {
  int32_t B, n_img, N_tok, T_tot;
  const int32_t *cu_seqlens, *img_start, *img_len, *cu_img, *text_pos, *cu_text, *keep_total;
  const int32_t *h_cu_seqlens, *h_img_start, *h_img_len, *h_cu_img, *h_text_pos, *h_cu_text,
      *h_keep_total;
} avtp_layout;

/*
 * One tensor to compact.  For every plane p < planes and output row r:
 *   dst + p*dst_plane_stride + r*dst_stride  <-  row_bytes bytes from
 *   src + p*src_plane_stride + keep_idx[r]*src_stride
 * (token-major [N_tok, ...] tensors use planes = 1; position ids [P, N_tok]
 * use planes = P; head-major K/V [Hkv, N_tok, d] use planes = Hkv).
 * All strides and offsets in bytes.  dst may be NULL when no row is kept.
 */
typedef struct {
  const void *src;
  void *dst;
  int64_t row_bytes, src_stride, dst_stride;
  int32_t planes;
  int64_t src_plane_stride, dst_plane_stride;
} avtp_tensor;

/* ------------------------------------------------------------------------
 * avtp_score -- importance of every visual token.
 *
 * AVTP_SCORE_ATTN (the attention a layer pays to visual tokens, the quantity
 * summed in Sec. 3.3.2, here kept per token).  With c = softmax_scale, query
 * head h using key head g = h / (Hq/Hkv) (grouped-query attention), text row t
 * at position p_t and the causal row normaliser
 *   lse[h,t] = log sum_{j <= p_t, j in seq} exp(c q_{t,h}.k_{j,g}),
 * the score of visual token j is
 *   s_j = 1/Hq sum_h 1/|T_j| sum_{t in T_j} exp(c q_{t,h}.k_{j,g} - lse[h,t])
 * where T_j are the text rows after j.  Computed in two tiled passes over
 * the keys (row statistics, then column sums) with bf16 MFMA and fp32
 * accumulation; the attention matrix is never stored.  fp32 inputs run as three
 * bf16 parts and six partial products (each product within 2^-24 of itself); over
 * the whole range of fp32, for logits that meet very small, very large or
 * infinite values the fp32 MFMA is used.  If row_lse is given
 * (e.g. the softmax LSE of the layer's own fused attention, natural log,
 * [Hq, T_tot] fp32) the first pass is skipped.
 *   q_text [T_tot, Hq, d]  queries of the text rows (dtype; may be NULL when
 *                          T_tot = 0: every image then has no text row after it)
 *   k      [N_tok, Hkv, d] the layer's keys (dtype)
 *   d in {64, 128}, Hq % Hkv == 0.
 *
 * AVTP_SCORE_VARIATION (Sec. 3.3.1, importance = 1 - Sim(h^l, h^prior),
 * Sim = cosine similarity with a 1e-8 norm guard):
 *   h_cur, h_prior [N_tok, hidden] (dtype); q_text, k, row_lse unused.
 *
 * Outputs: scores [N_tok] fp32 (+inf at text positions), img_sum [n_img]
 * fp32 = sum of the image's scores (Sec. 3.3.3 mean importance times |V_i|).
 * An image with no text row after it scores 0 and flags
 * AVTP_FLAG_NO_TEXT_AFTER.  Deterministic: bit-identical key rows in one
 * image give bit-identical scores, and reruns are bit-identical.
 * ws: device scratch of at least avtp_score_workspace_size() bytes (0 for an
 * invalid layout or arguments); its contents need no initialisation.
 * ---------------------------------------------------------------------- */
size_t avtp_score_workspace_size(const avtp_layout *layout, int mode, int dtype, int Hq, int Hkv,
                                 int d);
int avtp_score(avtp_stream_t stream, const avtp_layout *layout, int mode, int dtype,
               const void *q_text, const void *k, int Hq, int Hkv, int d, float softmax_scale,
               const float *row_lse, const void *h_cur, const void *h_prior, int hidden,
               float *scores, float *img_sum, int32_t *status, void *ws, size_t ws_bytes);

/* The first pass of AVTP_SCORE_ATTN alone: row_lse_out [Hq, T_tot] fp32,
 * natural-log LSE of each text row's causal attention logits (definition
 * above).  Same arguments and workspace as avtp_score; q_text and
 * row_lse_out may be NULL when T_tot = 0 (nothing is launched). */
int avtp_row_lse(avtp_stream_t stream, const avtp_layout *layout, int dtype, const void *q_text,
                 const void *k, int Hq, int Hkv, int d, float softmax_scale, float *row_lse_out,
                 void *ws, size_t ws_bytes);

/* ------------------------------------------------------------------------
 * avtp_budget -- per-image keep counts (Sec. 3.3.3 ratio rule, clamp of the
 * appendix on alpha).  For sequence b with images of n_i tokens and sums S_i,
 * M = sum n_i, S = sum S_i, K = keep_total[b]:
 *   PROPORTIONAL: quota share w_i = (1-alpha) n_i/M + alpha S_i/S
 *   RAW:          w_i = n_i/M + alpha (S_i - n_i S/M) / K
 * (each the ratio r_i = r_base + alpha (Ibar_i - Ibar_avg) of the paper with
 * r_base = K/M; PROPORTIONAL measures importance in units of its mean).
 * w_i < 0 -> 0; only the ratios of the shares matter, so with w_max the
 * largest share of the sequence W_i = max(1, rint((w_i / w_max) * 2^28))
 * (float64, one operation at a time, no FMA contraction); if S is not
 * positive and finite, w_i = n_i/M.  Bounds
 *   lo_i = min(n_i, max(ceil(lo_permille n_i / 1000), floor_abs)),
 *   hi_i = max(lo_i, floor(hi_permille n_i / 1000))
 * (paper: 5 % and 95 %, i.e. 50 and 950).  Exact integer water-filling finds
 * q_i = clamp(lam W_i, lo_i, hi_i) with sum q_i = K; largest-remainder
 * rounding (ties to the lowest image index) gives budget[i], sum = K.
 * alpha in [0, 32].  AVTP_ERR_INFEASIBLE (host check) if K is outside
 * [sum lo_i, sum hi_i].  budget: [n_img] int32 output.
 * ---------------------------------------------------------------------- */
int avtp_budget(avtp_stream_t stream, const avtp_layout *layout, const float *img_sum, int mode,
                float alpha, int lo_permille, int hi_permille, int floor_abs, int32_t *budget,
                int32_t *status);

/* ------------------------------------------------------------------------
 * avtp_select -- the pruned subsequence (Method, "Visual Token Pruning": the
 * pruning map keeps a subset of the visual tokens and every text token),
 * with the per-image keep counts of Sec. 3.3.3 (an image keeps budget[i]
 * tokens, so more important images keep more).  Inside every image the
 * budget[i] highest-scoring tokens are kept (score descending; an exact tie
 * keeps the lowest token index; -0.0 equals +0.0; NaN ranks last), plus
 * every text token.  Writes the kept global token indices of each sequence
 * in ascending order to keep_idx[cu_out[b] .. cu_out[b+1]), and cu_out [B+1].
 *   scores [N_tok] fp32 (device; text positions are not read), budget
 *   [n_img] int32 (device), keep_idx [keep_capacity] int32 and cu_out [B+1]
 *   int32 (device outputs).
 * keep_capacity: entries available in keep_idx; must be at least
 * T_tot + sum(keep_total) (checked on the host); writes past it are dropped
 * and flag AVTP_FLAG_OUT_CAPACITY (budgets not summing to keep_total).
 * No workspace: the selection of an image runs inside one block, from its
 * keys cached in LDS (or re-read from scores for images above 4096 tokens),
 * and each block knows its output offset from the budgets; so there is no
 * avtp_select_workspace_size.
 * ---------------------------------------------------------------------- */
int avtp_select(avtp_stream_t stream, const avtp_layout *layout, const float *scores,
                const int32_t *budget, int32_t *keep_idx, int64_t keep_capacity, int32_t *cu_out,
                int32_t *status);

/* ------------------------------------------------------------------------
 * avtp_compact -- the pruned sequence that the following layers run on
 * (Method, "Visual Token Pruning": E_pruned replaces E_v; Sec. 3.3.3: the
 * kept tokens of each image): stable gather out[r] = in[keep_idx[r]] for up
 * to AVTP_MAX_TENSORS tensors in one launch (hidden states, position ids with
 * their original values, K and V of the layer).  n_out = number of entries
 * of keep_idx to apply (normally T_tot + sum(keep_total)); every keep_idx
 * entry should lie in [0, N_tok): an entry outside it reads nothing and
 * leaves its output row as it was.  tensors: HOST array of n_tensors
 * descriptors.  Copies are bit-exact.
 * ---------------------------------------------------------------------- */
int avtp_compact(avtp_stream_t stream, const avtp_layout *layout, const int32_t *keep_idx,
                 int64_t n_out, const avtp_tensor *tensors, int n_tensors);

/* ------------------------------------------------------------------------
 * avtp_pruned_layout -- the layout of the kept tokens, for the next pruning
 * layer of a progressive schedule (Sec. 3.3.2: pruning at several selected
 * layers; Sec. 3.3.1: the next layer's h^prior is the hidden state after this
 * pruning, i.e. this layer's compacted hidden rows).  Pruning keeps a
 * subsequence of every sequence (Method, "Visual Token Pruning"): kept token
 * r of the batch (keep_idx[r], from avtp_select, ascending per sequence)
 * becomes token r of the next layer.  Writes, as device int32 arrays of the
 * next layer's avtp_layout:
 *   cu_seqlens_out [B+1] = cu_out;
 *   img_start_out, img_len_out [n_img]: image i's first new index and its
 *     number of kept tokens (an image that keeps none has length 0 and sits
 *     where its tokens were);
 *   text_pos_out [T_tot]: the new index of every text token (all are kept);
 *   cu_img_out, cu_text_out [B+1]: unchanged copies.
 * The next layer's keep totals (the schedule) are the caller's.  Host
 * mirrors of the next layout are the caller's copies of these arrays.
 * ---------------------------------------------------------------------- */
int avtp_pruned_layout(avtp_stream_t stream, const avtp_layout *layout, const int32_t *keep_idx,
                       const int32_t *cu_out, int32_t *cu_seqlens_out, int32_t *img_start_out,
                       int32_t *img_len_out, int32_t *cu_img_out, int32_t *text_pos_out,
                       int32_t *cu_text_out);

/* ------------------------------------------------------------------------
 * Architecture-aware pruning-layer selection (Sec. 3.3.2), computed from
 * calibration prefills.  For sample i and layer l the paper sums the
 * attention the layer pays to every visual token,
 *   A_l^(i) = sum_j Attention(l, v_j^(i)),
 * ranks the layers within each sample, averages the ranks over the N samples,
 *   R_l = 1/N sum_i Rank(A_l^(i)),
 * and prunes at the k layers of highest average attention.
 *
 * avtp_layer_attention -- A of one layer for every sequence of a batch (each
 * sequence is one sample): A_out[b] = sum of img_sum over the images of
 * sequence b (img_sum from avtp_score in AVTP_SCORE_ATTN mode, whose
 * per-token score stands for Attention(l, v_j)), accumulated in float64 in
 * image order and rounded once to fp32; 0 for a sequence without images.
 *   img_sum [n_img] fp32 (device), A_out [B] fp32 (device; typically row l
 *   of the caller's [L][N] table, at the batch's sample offset).
 *
 * avtp_layer_select -- ranks and selection from the whole table.
 *   A [L][N] fp32 (device, row-major: layer l, sample i at A[l*N + i]);
 *   1 <= L <= AVTP_MAX_LAYERS, 1 <= N <= AVTP_MAX_SAMPLES, 1 <= k <= L.
 *   Within each sample, rank 1 is the largest A; equal values rank the lower
 *   layer index first (each sample's ranks are a permutation of 1..L); NaN
 *   ranks as the smallest value; -0.0 equals +0.0.
 *   rank_sum [L] int32 (device, output): sum_i Rank(A_l^(i)) = N * R_l exactly.
 *   selected [k] int32 (device, output): the k layers with the smallest rank
 *   sums (equal sums: lower layer index first), in ascending layer order.
 * Both calls: AVTP_ERR_INVALID_ARG for null pointers or sizes out of range.
 * ---------------------------------------------------------------------- */
int avtp_layer_attention(avtp_stream_t stream, const avtp_layout *layout, const float *img_sum,
                         float *A_out);
int avtp_layer_select(avtp_stream_t stream, const float *A, int L, int N, int k,
                      int32_t *rank_sum, int32_t *selected);

/* ------------------------------------------------------------------------
 * avtp_select_compact -- avtp_select followed by avtp_compact of the same
 * tensors to n_out = T_tot + sum(keep_total) rows (the pruned subsequence of
 * Method, "Visual Token Pruning", gathered in one call).  Same arguments and
 * outputs as the two calls; the kept rows and keep_idx are bit-identical to
 * theirs.  When the compaction moves at most 4 MiB (reads plus writes) it is
 * one launch, for the small configurations where launches and the
 * selection's latency dominate: every image is handled by several blocks
 * that each redo its selection and copy an interleaved share of its output
 * rows, so no block waits for another.  Above that the two kernels run back
 * to back (one block's copies cannot start before its selection ends, so the
 * one-launch form is slower there).
 * ---------------------------------------------------------------------- */
int avtp_select_compact(avtp_stream_t stream, const avtp_layout *layout, const float *scores,
                        const int32_t *budget, int32_t *keep_idx, int64_t keep_capacity,
                        int32_t *cu_out, int32_t *status, const avtp_tensor *tensors,
                        int n_tensors);

/* ------------------------------------------------------------------------
 * avtp_budget_select_compact -- avtp_budget, then avtp_select_compact: the
 * per-image budgets of Sec. 3.3.3 (adaptive keep ratio, appendix clamp on
 * alpha), the top-budget selection of every image and the gather of the
 * pruned subsequence (Method, "Visual Token Pruning"), in one call.
 * Arguments: those of avtp_budget (img_sum, mode, alpha, lo/hi permille,
 * floor_abs; budget[n_img] is written) followed by those of
 * avtp_select_compact.  Every output (budget, keep_idx, cu_out, the compacted
 * tensors, status flags) is bit-identical to the separate calls'.  Errors: as
 * the separate calls, all checked on the host before any launch, including
 * AVTP_ERR_INFEASIBLE.  While no sequence has more than 64 images, the
 * selection blocks each run the budget rule for their own sequence (the
 * same integer arithmetic as the budget kernel), so no budget launch is
 * needed: one launch in all when the compaction moves at most 4 MiB, else
 * the selection and the compaction kernels.  With more images per sequence
 * the budget kernel runs first.
 * ---------------------------------------------------------------------- */
int avtp_budget_select_compact(avtp_stream_t stream, const avtp_layout *layout,
                               const float *img_sum, int mode, float alpha, int lo_permille,
                               int hi_permille, int floor_abs, const float *scores, int32_t *budget,
                               int32_t *keep_idx, int64_t keep_capacity, int32_t *cu_out,
                               int32_t *status, const avtp_tensor *tensors, int n_tensors);

/* ------------------------------------------------------------------------
 * avtp_score_noalloc -- avtp_score for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc).  Same arguments, outputs and results as avtp_score
 * (bit-identical: the same kernels run), but no workspace argument: the
 * scratch space lives in a device array of AVTP_NOALLOC_MAX_WORKSPACE bytes
 * inside the library, one per GPU, held until the process ends.  Its address
 * on a device is looked up on the first call with that device current (a
 * hipGetSymbolAddress, which allocates nothing); the stream must belong to the
 * calling thread's current device.  Nothing is allocated, on any call.
 * Returns AVTP_ERR_WORKSPACE when the layout needs more scratch than that
 * (avtp_score_workspace_size tells how much); every other argument error as
 * avtp_score, before any HIP call.  All calls on one GPU share its array:
 * calls that overlap on one GPU (other streams or threads) race; calls in
 * stream order do not.  No scratch contents need clearing between calls.
 * ---------------------------------------------------------------------- */
#define AVTP_NOALLOC_MAX_WORKSPACE (16 << 20) /* bytes of the library's scratch per GPU */
int avtp_score_noalloc(avtp_stream_t stream, const avtp_layout *layout, int mode, int dtype,
                       const void *q_text, const void *k, int Hq, int Hkv, int d,
                       float softmax_scale, const float *row_lse, const void *h_cur,
                       const void *h_prior, int hidden, float *scores, float *img_sum,
                       int32_t *status);

/* ------------------------------------------------------------------------
 * The paged K/V cache.  Pruning leaves every sequence of every layer with a
 * length of its own (Sec. 3.3.3: the keep count of each image; Sec. 3.3.2: a
 * progressive schedule shortens the sequence again at each pruning layer), so
 * a layer's K and V are kept in pages of page_size tokens that sequences take
 * and hand back one at a time:
 *   k, v  [n_pages][Hkv][page_size][d] (dtype), page_size a power of two in
 *         [16, 1024], d in {64, 128}; token t of sequence b lies at place
 *         t mod page_size of page block_table[b][t / page_size];
 *   block_table [B][max_pages] int32, in token order;
 *   free_pages  [n_pages] int32, a stack of page ids: the first free_count[0]
 *         entries are free, the next page taken is the last of them;
 *   slot  page * page_size + place, the place of one token (int32, so
 *         n_pages * page_size is below 2^31).
 * A model's layers may share one table (same lengths) or have one each.  All
 * of it lives on the device and no call reads it back, so a step of a serving
 * loop can be captured into a graph: tables, store, attention, trim.  Updated
 * lengths and counts go to buffers of their own (outputs must not alias
 * inputs; only block_table, free_pages and the pages are updated in place).
 * B is at most AVTP_MAX_REQUESTS, B * max_pages below 2^31, max_pages *
 * page_size (a sequence's most tokens) at most 2^30.
 * ---------------------------------------------------------------------- */
typedef struct {
  void *k, *v;
  int32_t dtype, n_pages, page_size, Hkv, d;
} avtp_pages;

/* ------------------------------------------------------------------------
 * avtp_page_tables -- room for the new tokens of every request: block tables
 * and slot map from the request lengths.  Sequence b holds seq_len[b] tokens
 * and gets the next cu_new[b+1] - cu_new[b] ones, whose index in this step's
 * batch starts at cu_new[b] (cu_new[0] = 0; e.g. cu_out of a selection).  The
 * pages it lacks are popped off the stack, sequences in order, and entered in
 * its row of the table; other entries stay as they were.
 *   slot_map [n_new] int32 (output): the slot of every new token; -1 for
 *     tokens without a place and for entries from cu_new[B] on (a padded
 *     batch).
 *   seq_len_out [B], free_count_out [1] int32 (outputs): the state afterwards.
 * A request has no place if its row of the table is too short, if its new
 * tokens reach past n_new, or (needing pages) if the pages that it and the
 * requests before it need are more than the stack holds: its length and row stay
 * as they were, its slots are -1 and it flags AVTP_FLAG_NO_PAGES.  A page id
 * outside [0, n_pages) gives slots of -1 and flags AVTP_FLAG_BAD_PAGE.
 * free_count is read as at most n_pages.
 * avtp_page_reserve is the same call and keeps kv_len [B], the lengths for
 * avtp_page_attention, which counts a sequence's queries back from its length and
 * would take those of a request without a place for its last cached tokens.
 * kv_len[b] becomes seq_len_out[b], or 0 for a request without a place, whose
 * queries then see nothing (out 0, lse -inf); sequences without new tokens keep
 * theirs, so that a refusal stands until the request gets its place.  (Behind
 * avtp_page_trim: the smaller of kv_len and its seq_len_out.)
 * ---------------------------------------------------------------------- */
int avtp_page_tables(avtp_stream_t stream, int B, int page_size, const int32_t *cu_new,
                     const int32_t *seq_len, const int32_t *free_pages, int n_pages,
                     const int32_t *free_count, int32_t *block_table, int max_pages,
                     int32_t *slot_map, int64_t n_new, int32_t *seq_len_out,
                     int32_t *free_count_out, int32_t *status);
int avtp_page_reserve(avtp_stream_t stream, int B, int page_size, const int32_t *cu_new,
                      const int32_t *seq_len, const int32_t *free_pages, int n_pages,
                      const int32_t *free_count, int32_t *block_table, int max_pages,
                      int32_t *slot_map, int64_t n_new, int32_t *seq_len_out,
                      int32_t *free_count_out, int32_t *kv_len, int32_t *status);

/* ------------------------------------------------------------------------
 * avtp_page_trim -- sequences are cut to their first keep_len[b] tokens (0: the
 * request has ended; seq_len[b] or more: nothing changes; less: tokens are
 * taken back, e.g. rejected drafts).  The pages that hold none of the kept
 * tokens are pushed onto the stack, sequences in order, each one's in token
 * order; the table is only read, and every page of a row counts as its
 * sequence's own (one that two rows name is handed back twice).  seq_len_out [B]
 * = min(keep_len, seq_len), free_count_out [1].  Pages beyond the stack's
 * n_pages entries (more pages handed back than the pool has) are dropped and
 * flag AVTP_FLAG_OUT_CAPACITY.
 * ---------------------------------------------------------------------- */
int avtp_page_trim(avtp_stream_t stream, int B, int page_size, const int32_t *keep_len,
                   const int32_t *seq_len, const int32_t *block_table, int max_pages,
                   int32_t *free_pages, int n_pages, const int32_t *free_count,
                   int32_t *seq_len_out, int32_t *free_count_out, int32_t *status);

/* ------------------------------------------------------------------------
 * avtp_page_store -- K and V rows into their pages: for every r < n with slot
 * s = slot_map[r], row keep_idx[r] (row r when keep_idx is NULL) of k and v
 * [n_src, Hkv, d] goes to place s of the pages.  With the keep_idx of a
 * selection and the slot map of its cu_out this is the compaction of a pruned
 * layer's K and V (avtp_compact), straight into the cache.  k_stride and
 * v_stride: elements from one token to the next (Hkv * d or more; slices of a
 * fused projection are read in place).  Rows and strides are 16-byte aligned.
 * A slot outside the pool or a keep_idx entry outside [0, n_src) writes
 * nothing.  Of two rows with one slot either may stay.  Bit-exact.
 * ---------------------------------------------------------------------- */
int avtp_page_store(avtp_stream_t stream, const avtp_pages *pages, const void *k, int64_t k_stride,
                    const void *v, int64_t v_stride, int64_t n_src, const int32_t *slot_map,
                    const int32_t *keep_idx, int64_t n);

/* ------------------------------------------------------------------------
 * avtp_page_attention -- the attention of a chunk of new tokens over the
 * paged cache, their own K and V included.  The queries of sequence b are rows
 * cu_q[b] .. cu_q[b+1]-1 of q, its last n_b = cu_q[b+1] - cu_q[b] tokens (which
 * must be in the cache: avtp_page_reserve for requests without a place); row t
 * of them sees the first kv_len[b] - n_b + t + 1 cached tokens.  With c =
 * softmax_scale and query head h using key head g = h / (Hq/Hkv):
 *   lse[h,t] = log sum_j exp(c q_{t,h}.k_{j,g}),
 *   out[t,h] = sum_j exp(c q_{t,h}.k_{j,g} - lse[h,t]) v_{j,g}
 * over the tokens j the row sees.  A row that sees none (kv_len[b] < n_b): out 0,
 * lse -inf.  Values of tokens a row does not see do not reach it, whatever they
 * are, infinities and NaN included.
 *   q, out  [N_q, Hq, d] (dtype of the pages), q_stride and out_stride elements
 *     from one token to the next (Hq * d or more), rows and strides 16-byte
 *     aligned; rows of out from cu_q[B] on stay as they were;
 *   lse     [Hq, N_q] fp32, natural log (may be NULL): the row_lse of
 *     avtp_score for the text rows of the layer;
 *   max_kv_len: a bound on kv_len, which sizes the launch and the workspace
 *     only.  Any value is right for all lengths; the speed is best with one
 *     near the longest (see Speed).
 * A single new token per sequence is the decode step.  Products of bf16 run on
 * the bf16 MFMA with fp32 accumulation, the probabilities rounded to bf16 before
 * they weigh V (2^-8 of each at most); fp32 runs in fp32.  Sums and
 * maxima are fp32.  A block table entry outside [0, n_pages) reads nothing: its
 * tokens count as zeros and flag AVTP_FLAG_BAD_PAGE; so does a kv_len above
 * max_pages * page_size, of which the tokens in the table remain; a negative
 * one is 0.  No atomics on results: reruns are bit-identical.  The running sums
 * refer to a maximum that may lag behind, and then hold up to 2^13 for every token
 * a row sees: |v| may be 2^114 over the number of those tokens (2^97 of 131,072);
 * beyond it an output may overflow where the formula's quotient does not.  A row
 * whose logits are all -inf gives 0.  An infinite value whose weight is below 2^-126 of
 * the row's largest gives infinity, as the formula does, or NaN (fp32's 0 times it).
 * ws: device scratch of avtp_page_attention_workspace_size() bytes (which may
 * be 0, and is for an invalid argument), 256-byte aligned, no initialisation;
 * it depends on the sizes alone, so that a call captured at the largest
 * max_kv_len serves all lengths below.  Calls that may run at the same time
 * need one each.  N_q * Hq is below 2^31, Hq at most 256, and with more than 32
 * rows per sequence N_q * Hq / 128 + B * Hkv below 2^24.
 * Speed: with at most 32 rows (tokens times Hq / Hkv) per sequence on average,
 * the call is bound by reading K and V once; with more, by the products, or by its
 * longest sequence where many differ much in length (64 of 300 to 16,000 tokens, 7
 * query heads per key head: 4 new tokens each 102 us, 5 of them 294).  A batch of
 * long chunks and single tokens is best issued as two calls.  A max_kv_len below the
 * lengths makes too few blocks; one far above them costs steps of few or short
 * requests time (one token over 794: 9 us up to 1,024, 16 at 32,768, 22 at 131,072;
 * 64 requests of 300 tokens 21 and 31; of 300 to 16,000 163 and 169).
 * ---------------------------------------------------------------------- */
size_t avtp_page_attention_workspace_size(const avtp_pages *pages, int Hq, int B, int64_t N_q,
                                          int64_t max_kv_len);
int avtp_page_attention(avtp_stream_t stream, const avtp_pages *pages, const void *q,
                        int64_t q_stride, int Hq, int B, int64_t N_q, const int32_t *cu_q,
                        const int32_t *kv_len, const int32_t *block_table, int max_pages,
                        int64_t max_kv_len, float softmax_scale, void *out, int64_t out_stride,
                        float *lse, int32_t *status, void *ws, size_t ws_bytes);

/* ------------------------------------------------------------------------
 * avtp_page_attention_window -- avtp_page_attention where a row sees a window of the
 * latest tokens and the first ones only: the token at position p (row t of sequence b:
 * p = kv_len[b] - n_b + t) sees the cached tokens j <= p with j > p - window or
 * j < sinks.  window is 1 or more (1: itself), sinks 0 or more.  Everything else as
 * there, the speed's rules with the tokens that a row sees in the place of kv_len.
 * Pages of which no row of the call sees a token are not looked at: what the table
 * says of them does not matter (avtp_page_release hands them back).  The workspace
 * depends on window and sinks too.
 * ---------------------------------------------------------------------- */
size_t avtp_page_attention_window_workspace_size(const avtp_pages *pages, int Hq, int B,
                                                 int64_t N_q, int64_t max_kv_len, int window,
                                                 int sinks);
int avtp_page_attention_window(avtp_stream_t stream, const avtp_pages *pages, const void *q,
                               int64_t q_stride, int Hq, int B, int64_t N_q, const int32_t *cu_q,
                               const int32_t *kv_len, const int32_t *block_table, int max_pages,
                               int64_t max_kv_len, int window, int sinks, float softmax_scale,
                               void *out, int64_t out_stride, float *lse, int32_t *status,
                               void *ws, size_t ws_bytes);

/* ------------------------------------------------------------------------
 * avtp_page_fork -- sequences that start from the tokens of others, e.g. more
 * questions about the same images.  Sequence b with parent[b] = p >= 0 gets the
 * first fork_len[b] tokens of sequence p: the pages that they fill are named by both
 * rows from then on, and a last one that they fill in part is replaced, in b's row,
 * by a page off the stack, dst_page[b], into which src_page[b] has to be copied in
 * every layer (avtp_page_copy; both are -1 where there is nothing to copy).  So
 * tokens that either sequence gets later lie in pages of its own.
 *   parent [B]: -1 where nothing happens; sequence b must be empty, p no fork of the
 *     same call, 0 <= fork_len[b] <= seq_len[p], and all of it where p has left tokens
 *     behind its window (gone[p] > 0): else b stays as it was and flags
 *     AVTP_FLAG_REFUSED.
 *   gone, gone_out [B] (both or neither): avtp_page_release's; a fork has its parent's.
 *     They may be NULL only while no release has let go behind a window: a fork without
 *     them would hold pages that have left, and hand them back a second time.
 *   seq_len_out [B], free_count_out [1], src_page, dst_page [B] (outputs, which share no
 *     memory with each other or with an input; so for avtp_page_release).
 * Pages are taken in the order of the sequences; one for which none is left stays as
 * it was and flags AVTP_FLAG_NO_PAGES (its later ones that need none are made).  Where
 * the page to be copied, or the one off the stack, lies outside the pool the fork is made
 * with nothing to copy and flags AVTP_FLAG_BAD_PAGE.
 * Behind forks sequences are cut and ended with avtp_page_release: avtp_page_trim
 * would hand a shared page back twice.
 *
 * avtp_page_copy -- pages src_page[i] of a layer's K and V copied to dst_page[i], for
 * every i < n with both inside the pool.  No page may be named as a destination and
 * again as a source or a destination.  Bit-exact.
 *
 * avtp_page_release -- sequences are cut to their first keep_len[b] tokens as by
 * avtp_page_trim (0: the request has ended), and with window > 0 they let go of the
 * pages whose tokens have left the window: gone_out[b] = keep - window + 1 (at least
 * gone[b]; 0 for one that has ended), and the pages of a row between those that hold
 * the first `sinks` tokens and page gone_out[b] / page_size are no longer its own,
 * whatever its entries say.  The next token's window starts at gone_out[b]: tokens that
 * are stored and still wait for attention see further back, and come first.  With no
 * window gone may be NULL (nothing has left), or is taken over.  A page goes onto the
 * stack when no sequence holds it any more; the pages freed by a call are pushed in
 * ascending order.  Pages beyond the stack's n_pages entries are dropped.
 *   A cut inside a page that another sequence held before the call would let it write
 *   into the other's tokens, and one to less than gone[b] + window - 1 tokens would
 *   leave tokens that have left the window missing: the sequence stays whole and flags
 *   AVTP_FLAG_REFUSED.  (Fork the tokens to be kept to an empty row, and end this one.)
 *   seq_len_out [B], free_count_out [1], gone_out [B] (with gone).  A block table entry
 *   in use outside the pool is left out and flags AVTP_FLAG_BAD_PAGE.
 * window is at most 2^30, sinks at most 2^30, and the same at every call.  ws: device
 * scratch of avtp_page_release_workspace_size(n_pages) bytes, 256-byte aligned, no
 * initialisation; calls that may run at the same time need one each.
 * ---------------------------------------------------------------------- */
int avtp_page_fork(avtp_stream_t stream, int B, int page_size, const int32_t *parent,
                   const int32_t *fork_len, const int32_t *seq_len, const int32_t *free_pages,
                   int n_pages, const int32_t *free_count, int32_t *block_table, int max_pages,
                   const int32_t *gone, int32_t *seq_len_out, int32_t *free_count_out,
                   int32_t *src_page, int32_t *dst_page, int32_t *gone_out, int32_t *status);
int avtp_page_copy(avtp_stream_t stream, const avtp_pages *pages, const int32_t *src_page,
                   const int32_t *dst_page, int64_t n);
size_t avtp_page_release_workspace_size(int n_pages);
int avtp_page_release(avtp_stream_t stream, int B, int page_size, const int32_t *keep_len,
                      const int32_t *seq_len, const int32_t *block_table, int max_pages,
                      int32_t *free_pages, int n_pages, const int32_t *free_count, int window,
                      int sinks, const int32_t *gone, int32_t *seq_len_out,
                      int32_t *free_count_out, int32_t *gone_out, int32_t *status, void *ws,
                      size_t ws_bytes);

/* ------------------------------------------------------------------------
 * avtp_norm_rotary -- queries and keys normalised head by head and rotated by
 * their tokens' positions, in one pass.  Of the d values x of a head
 *   y = x w / sqrt(mean(x^2) + eps)     (q_weight, k_weight [d] fp32; NULL: y = x)
 * and of the first rot_dim of them (a multiple of 16, at most d; the others stay y)
 * the pairs (a, b) = (y[i], y[i + rot_dim / 2]), or (y[2i], y[2i+1]) where
 * interleaved is not 0, with t = 2 pi turns[i] / 2^64 pos[plane[i], token], become
 *   scale (a cos t - b sin t),  scale (b cos t + a sin t).
 * turns [rot_dim/2]: what one position turns pair i by, 2^64 a whole turn, so that
 * positions of any size lose nothing (64-bit product, whole turns drop out); a
 * negative frequency wraps and turns back.  Any stretching of the frequencies for
 * long contexts is in turns and scale.  pos [planes, n] int64 (pos_stride from one
 * plane to the next): the position ids that avtp_compact leaves; plane [rot_dim/2]
 * names the plane of each pair (NULL: the first for all; an entry outside
 * [0, planes) counts as 0).  planes is at most AVTP_MAX_PLANES.
 * q, q_out [n, Hq, d], k, k_out [n, Hkv, d], d in {64, 128}; strides in elements from
 * one token to the next (slices of a fused projection are read in place), rows and
 * strides 16-byte aligned.  Hq or Hkv may be 0.  q_out may be q and k_out k, with the
 * same stride.  fp32 throughout, rounded once: a square sum above 2^128 (values of
 * about 2^60) is infinite, and gives zeros.  Infinities and NaN go through the formula.
 * avtp_page_store_rotary is the same for the rows of a step, with K and, as they are,
 * the rows of v on into the pages: row r to slot_map[r] (a slot outside the pool
 * stores nothing; of two rows with one slot either may stay).  q_out is written for
 * every row.
 * ---------------------------------------------------------------------- */
typedef struct {
  const uint64_t *turns; /* device */
  const int32_t *plane;  /* device, may be NULL */
  int32_t rot_dim, interleaved, planes;
  float scale;
} avtp_rotary;

int avtp_norm_rotary(avtp_stream_t stream, const avtp_rotary *rotary, int dtype, int d, int64_t n,
                     const int64_t *pos, int64_t pos_stride, const float *q_weight,
                     const float *k_weight, float eps, const void *q, int64_t q_stride, int Hq,
                     void *q_out, int64_t q_out_stride, const void *k, int64_t k_stride, int Hkv,
                     void *k_out, int64_t k_out_stride);
int avtp_page_store_rotary(avtp_stream_t stream, const avtp_pages *pages, const avtp_rotary *rotary,
                           int64_t n, const int64_t *pos, int64_t pos_stride,
                           const float *q_weight, const float *k_weight, float eps, const void *q,
                           int64_t q_stride, int Hq, void *q_out, int64_t q_out_stride,
                           const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                           const int32_t *slot_map);

/* Human-readable name of an avtp_status value (static string). */
const char *avtp_status_string(int status);

/* ABI version: (major << 16) | minor. */
int avtp_version(void);

#ifdef __cplusplus
}
#endif
#endif /* AVTP_H */
