/*
 * maskkv.h - C ABI of the MaskKV eviction hot path for AMD MI355X (gfx950).
 *
 * The library implements, for one transformer layer at a time, the data-parallel steps
 * of MaskKV (arXiv 2510.09309, Section 3.3 "The MaskKV Framework"):
 *
 *   maskkv_score    Stage 1 "Mask-Voting": A = softmax_row(Q_mask K_full^T / sqrt(d_k)),
 *                   I_j = sum_i A_ij for the prompt tokens j.
 *   maskkv_select   S_keep = argtopk(I, k_{l,h}) per (layer, head) with ragged budgets
 *                   (last equation of Stage 2), after an optional smoothing window.
 *   maskkv_compact  eviction: the cache keeps only the selected prompt K/V rows
 *                   (appendix "Prompt-state Exclusion": only prompt K/V are cached).
 *   maskkv_attend   bidirectional attention of the response span over
 *                   [kept prompt KV ; response KV] (layer forward equation, Section 3.1;
 *                   appendix proof: AttnOut_m = sum_j alpha_mj V_j).
 *   maskkv_attend_full   the same attention over the un-evicted sequence (the cost the
 *                   eviction removes; used for the speed-up figure).
 *   maskkv_head_budgets  Stage 2, head level: prompt preference P_h and
 *                   k_{l,h} = floor(alpha k_l + (1-alpha) N_h k_l P_h / sum_j P_j).
 *   maskkv_layer_importance, maskkv_layer_budgets   Stage 2, layer level: I^(l) = 1 - mean
 *                   cosine similarity of the attention sub-layer's input and output states, and
 *                   the boundary-aware split of the total budget over the layers.
 *   maskkv_compact_mx, maskkv_expand_mx, maskkv_attend_mx   the cache in 4 bits: eviction that stores the kept
 *                   rows so, the values that they stand for, and the attention that reads them.
 *   maskkv_accumulate, maskkv_evict (and _mx)   further eviction from the cache: the attention that each cached row has
 *                   got over the denoising steps, and the rows of each head that got most.
 *   maskkv_rotate   the positions of queries and keys, as rotations of pairs of their elements, before they are scored, cached or
 *                   attended to.
 *   maskkv_attend_tree   maskkv_attend where the response rows do not all see each other: trees of drafted tokens, blocks in
 *                   order; few rows over a long cache.  maskkv_tree_mask: who sees whom in a tree.
 *   maskkv_sample   a token for every row of logits, and the confidence in it by which a denoising step chooses what it keeps.
 *   maskkv_value_shift   Section 3.1 (feature-cache background): response tokens whose value
 *                   vector turned by more than a threshold between two denoising steps.
 *
 * Conventions
 *  - Every pointer marked DEVICE must be device memory reachable from the current HIP
 *    device; pointers marked HOST are ordinary host memory read during the call only.
 *  - The library never allocates, frees or synchronises.  All work is enqueued on the
 *    given stream (a hipStream_t passed as void*; NULL is the default stream).  The
 *    caller owns every buffer, including the workspace, and must keep it alive until the
 *    stream has drained.  Inputs are never modified; outputs are fully overwritten in
 *    their valid region.
 *  - Every function returns a maskkv_status.  On any status other than MASKKV_OK nothing
 *    has been enqueued.  maskkv_last_error() gives a per-thread detail string.
 *  - Sequences: batch item b has P_b prompt tokens followed by n_resp response-span
 *    tokens (N_b = P_b + n_resp keys).  Key/value heads are independent.
 *  - Grouped-query attention (the Dream-7B model of Section 4.1): desc->H counts KEY/VALUE
 *    heads and desc->q_per_kv = g > 1 says that query heads h*g .. h*g+g-1 read KV head h.
 *    Views of queries and outputs (Q_mask, Q_resp, O) then have H*g heads, lse has
 *    B*H*g*n_resp entries, and everything per head (scores, prompt_mass, budgets, cu_budget,
 *    the cache, K and V views) stays per KV head.  The paper does not say how votes map to a
 *    shared KV head; here every mask query of every query head in the group votes
 *    (scores = sum over the group of the per-head column sums).  g <= 64.
 */
#ifndef MASKKV_H
#define MASKKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MASKKV_VERSION 1
#define MASKKV_MAX_BATCH 64 /* per call; split larger batches */

typedef enum maskkv_status {
  MASKKV_OK = 0,
  MASKKV_EINVAL = 1,     /* null pointer, negative size, bad window, bad stride, ... */
  MASKKV_ESHAPE = 2,     /* unsupported head_dim (64 and 128 are supported) or batch too large */
  MASKKV_EDTYPE = 3,     /* dtype is neither MASKKV_F32 nor MASKKV_BF16 */
  MASKKV_EWORKSPACE = 4, /* workspace missing or smaller than maskkv_*_workspace_bytes */
  MASKKV_EHIP = 5,       /* a HIP launch failed; detail string carries hipGetErrorString */
  MASKKV_ECAPACITY = 6   /* (host-checkable) output capacity too small */
} maskkv_status;

typedef enum maskkv_dtype { MASKKV_F32 = 0, MASKKV_BF16 = 1 } maskkv_dtype;

typedef enum maskkv_pool_mode { MASKKV_POOL_MEAN = 0, MASKKV_POOL_MAX = 1 } maskkv_pool_mode;

/*
 * A 4-D view [B, H, T, d] of Q, K, V or O in DEVICE memory.  Element (b, h, t, e) lives at
 *   ptr + ((b*stride_b + h*stride_h + (seq_start[b] + t)*stride_t + e) * sizeof(element)),
 * strides in elements, the head_dim axis contiguous.  Rows must be 16-byte aligned
 * (ptr and all strides multiples of 16 bytes) and stride_t may not exceed 16 MiB in bytes
 * (MASKKV_EINVAL otherwise).  [B,H,T,d], [B,T,H,d] and packed
 * variable-length [T_total,H,d] (stride_b = 0 with seq_start) are all expressible.
 */
typedef struct maskkv_tensor {
  void* ptr;             /* DEVICE */
  int64_t stride_b;
  int64_t stride_h;
  int64_t stride_t;
  const int32_t* seq_start; /* HOST [B] token offset of each sequence on the T axis, or NULL for 0 */
} maskkv_tensor;

/* Problem description shared by all calls. */
typedef struct maskkv_desc {
  int32_t B;        /* sequences in the batch, 1..MASKKV_MAX_BATCH */
  int32_t H;        /* attention heads */
  int32_t d;        /* head_dim: 64 or 128 */
  int32_t dtype;    /* maskkv_dtype of Q, K, V, the cache and O */
  int32_t n_resp;   /* response-span length n_m: response keys per sequence; queries in attend */
  int32_t n_query;  /* mask queries per query head that vote in maskkv_score (normally n_resp; a sub-span,
                       e.g. only the late response positions of the position-aware voting study, is
                       expressed by pointing Q_mask at its first row) */
  int32_t P_max;    /* longest prompt in the batch */
  int32_t q_per_kv; /* grouped-query attention: query heads per key/value head; 0 or 1 = one each (MHA) */
  const int32_t* prompt_len; /* HOST [B] prompt lengths P_b in 0..P_max, or NULL: every P_b = P_max */
} maskkv_desc;

/* Library version (MASKKV_VERSION of the build). */
int maskkv_version(void);
/* Static string for a status code. */
const char* maskkv_strerror(int status);
/* Detail of the calling thread's most recent failure ("" if none). */
const char* maskkv_last_error(void);

/*
 * Workspace (DEVICE bytes) needed by maskkv_score for this description.  The workspace
 * holds the softmax row sums that the workgroups exchange (or per-key-segment row statistics
 * between two passes), a packed copy of the voting rows and, with more than 256 voting rows per
 * head, the column sums of every group of at most 256 rows, or for short fp32 prompts those of every
 * workgroup of 16 rows or more; contents are scratch.  The size depends on prompt_len: query it with
 * the description the call will use.  256-byte alignment is required.
 */
int maskkv_score_workspace_bytes(const maskkv_desc* desc, size_t* bytes);

/*
 * Stage 1, Mask-Voting.  For every (b, h):
 *   A = softmax over all N_b keys of (Q_mask[b,h] K_full[b,h]^T * scale)   (no mask)
 *   scores[(b*H + h)*score_stride + j] = sum_{i < n_query} A[i, j],  j in [0, P_b)
 *                          (summed over the g query heads of the group too when q_per_kv = g > 1)
 *   prompt_mass[b*H + h] = sum_{j < P_b} scores[..j]   (the mask-to-prompt attention sum
 *                          S_{m->p} of the prompt-preference metric), if not NULL.
 * Q_mask: view [B, H*g, n_query, d].  K_full: view [B, H, N_b, d], prompt rows then
 * response rows.  scale <= 0 selects 1/sqrt(d).  scores: DEVICE float, score_stride >=
 * P_max; entries j >= P_b are left untouched.  Accumulation is fp32 throughout.
 *
 * bf16 calls whose prompts have at most 128 tokens per compute unit are scored in one sweep over the keys where that
 * is the faster way.  Its workgroups, one per compute unit, wait for each other's row sums, so they all have to be
 * resident.  Calls on several streams of a process line up for that and take what they take on one stream.  Another
 * process that scores on the same GPU (or a second copy of this library) is not seen, nor is any other kernel
 * that leaves a compute unit less than 145 KB of LDS or not all of its registers for a long time: workgroups that have
 * waited for the others for 0.1 ms and about as long again as the sweep takes give up, and the call is done in two
 * passes by those that run, with the same results to fp32 rounding.  (Two processes that score 32 heads x 32k keys at
 * once: 0.45 ms a call of each, 0.12 ms alone.)
 */
int maskkv_score(const maskkv_desc* desc, const maskkv_tensor* Q_mask, const maskkv_tensor* K_full,
                 float scale, float* scores, int64_t score_stride, float* prompt_mass,
                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * Mask-Voting when the softmax normaliser of every voting row is already known.  At the initial inference step
 * (the step whose mask queries vote, Stage 1) the model's own attention over the un-evicted sequence forms the
 * same logits over the same keys, and a flash-style attention call returns each row's log-sum-exp: given those,
 * the scores need one sweep over the keys instead of two.
 *   row_lse[(b*H + h)*g*n_query + r] = log sum_j exp(q_r . k_j * scale)   (natural log, all N_b keys)
 * for voting row r of key/value head h (rows numbered as the rows of Q_mask: query head first, then query) - the
 * layout in which maskkv_attend_full writes `lse` when it is called with the same queries (n_query = n_resp) and
 * the same scale.  scores and prompt_mass as for maskkv_score; they equal its results up to the rounding of the
 * normalisers.  workspace: maskkv_score_workspace_bytes (only the part for more than 256 voting rows is used).
 */
int maskkv_score_given_lse(const maskkv_desc* desc, const maskkv_tensor* Q_mask, const maskkv_tensor* K_full,
                           float scale, const float* row_lse, float* scores, int64_t score_stride,
                           float* prompt_mass, void* workspace, size_t workspace_bytes, void* stream);

/*
 * maskkv_score for callers that cannot allocate device memory or carry a workspace: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same arguments and same result as maskkv_score, but the
 * scratch between the passes lives in an array of MASKKV_STATIC_SCRATCH_BYTES that is part of the library image
 * (every GPU the library runs on holds its own copy until the process ends).  The call allocates and frees
 * nothing.  Descriptions whose maskkv_score_workspace_bytes exceed MASKKV_STATIC_SCRATCH_BYTES are scored in
 * two passes, and rejected with MASKKV_EWORKSPACE (nothing enqueued) if these need more as well.  All calls on one GPU share that GPU's array: two calls that overlap in
 * time on one GPU (different streams, or different host threads) race; calls on one stream are ordered.  Every
 * scratch word a call reads is written by the same call first, so nothing needs clearing between calls.  The
 * first call on a device resolves the array's device address (hipGetSymbolAddress); make that call outside graph
 * capture.
 */
#define MASKKV_STATIC_SCRATCH_BYTES (16u << 20)
int maskkv_score_static(const maskkv_desc* desc, const maskkv_tensor* Q_mask, const maskkv_tensor* K_full,
                        float scale, float* scores, int64_t score_stride, float* prompt_mass, void* stream);

/* Workspace (DEVICE bytes) needed by maskkv_select: the candidates that the first
 * stage (one workgroup per 4096 prompt positions) hands to the per-head final stage, and their counts; 0 for
 * prompts of at most 16384 tokens (selected in one stage).  256-byte alignment. */
int maskkv_select_workspace_bytes(const maskkv_desc* desc, size_t* bytes);

/*
 * Smoothing + per-head top-k.  For every (b, h), with k = min(max(budgets[b*H+h], 0), P_b):
 *   pooled_j = mean (MASKKV_POOL_MEAN) or max (MASKKV_POOL_MAX) of scores over the window
 *              [max(0, j-r), min(P_b-1, j+r)], r = (pool_window-1)/2; the mean is evaluated
 *              in fp32 by adding the in-range terms from the lowest index upwards and
 *              dividing by their count.  pool_window must be odd, 1 (= no pooling) .. 63.
 *   keep     = the k positions with the largest pooled score, ties to the lower position,
 *              written in ascending order to idx[cu_budget[b*H+h] .. cu_budget[b*H+h+1]).
 *   cu_budget = exclusive prefix sum of the clamped budgets, B*H+1 entries.
 * budgets: DEVICE int32 [B*H] (device-resident so that maskkv_head_budgets can feed it
 * without a host round trip).  budgets_host: HOST int32 [B*H] copy of the same values, or
 * NULL.  With the copy the call checks them before anything is enqueued: a negative budget
 * is MASKKV_EINVAL, clamped budgets that sum to more than capacity are MASKKV_ECAPACITY.
 * Without it (budgets that only exist on the device) negative budgets count as 0, and if
 * the clamped budgets sum to more than capacity the rows beyond capacity are not written
 * while cu_budget still holds the unclipped prefix sums: size capacity as the sum of the
 * budgets, or B*H*k_l for budgets from maskkv_head_budgets (their sum never exceeds it).
 * idx: DEVICE int32 [capacity]; cu_budget: DEVICE int32 [B*H+1].  P_max may not exceed
 * 4 Mi tokens and B*H*P_max must fit 31 bits (MASKKV_ESHAPE).
 */
int maskkv_select(const maskkv_desc* desc, const float* scores, int64_t score_stride,
                  int pool_window, int pool_mode, const int32_t* budgets, const int32_t* budgets_host,
                  int32_t* idx, int32_t* cu_budget, int64_t capacity,
                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * Eviction as a gather.  Row r of the packed caches, r in [cu_budget[bh], cu_budget[bh+1]),
 * receives prompt row idx[r] of head bh:  Kc[r, :] = K[b, h, idx[r], :], same for V.
 * Kc, Vc: DEVICE [capacity, d] in desc->dtype, rows contiguous.  Rows >= min(capacity,
 * cu_budget[B*H]) are left untouched.  K, V: views whose first P_b rows are the prompt.
 */
int maskkv_compact(const maskkv_desc* desc, const maskkv_tensor* K, const maskkv_tensor* V,
                   const int32_t* idx, const int32_t* cu_budget, int64_t capacity,
                   void* Kc, void* Vc, void* stream);

/* Workspace (DEVICE bytes) for maskkv_attend (full = 0: the order in which the heads are processed, longest key
 * axis first; 0 where every workgroup starts at once) or maskkv_attend_full (full = 1: key-split partial results): what the
 * calls with this description ask for, and at most what they use (bf16 calls of up to 256 heads find the order without it, and
 * un-evicted calls over short prompts do not split the key axis).  256-byte alignment. */
int maskkv_attend_workspace_bytes(const maskkv_desc* desc, int full, size_t* bytes);

/*
 * Attention over the evicted cache.  For every (b, h), query head hq of h's group (hq = h when
 * q_per_kv <= 1) and response query i < n_resp:
 *   O[b,hq,i,:] = sum_j softmax_j(Q_resp[b,hq,i,:] . k_j * scale) v_j
 * with j over the cache rows [cu_budget[bh], cu_budget[bh+1]) of Kc/Vc (DEVICE [capacity, d];
 * row numbers are clipped to capacity) followed by the n_resp rows of K_resp/V_resp (views
 * [B, H, n_resp, d]).  No mask.  lse (DEVICE float
 * [B*H*g*n_resp], optional) receives the natural-log softmax normaliser of every row.
 * Inputs in desc->dtype, fp32 accumulation; probabilities are rounded to desc->dtype only
 * as the operand of the P.V product.  Q_resp, O: views [B, H*g, n_resp, d]; O is written in desc->dtype.
 */
int maskkv_attend(const maskkv_desc* desc, const maskkv_tensor* Q_resp,
                  const void* Kc, const void* Vc, const int32_t* cu_budget, int64_t capacity,
                  const maskkv_tensor* K_resp, const maskkv_tensor* V_resp, float scale,
                  const maskkv_tensor* O, float* lse,
                  void* workspace, size_t workspace_bytes, void* stream);

/* The same attention over all N_b = P_b + n_resp rows of K_full/V_full (nothing evicted). */
int maskkv_attend_full(const maskkv_desc* desc, const maskkv_tensor* Q_resp,
                       const maskkv_tensor* K_full, const maskkv_tensor* V_full, float scale,
                       const maskkv_tensor* O, float* lse,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * Rotary positions.  Pair i < width/2 of a row's first `width` elements is turned by the angle a = position * freq[i] and lengthened:
 *   (x, y) -> amplitude * (x cos a - y sin a,  y cos a + x sin a)
 * The pair is elements (i, i + width/2) with MASKKV_ROTARY_HALVES, (2i, 2i + 1) with MASKKV_ROTARY_PAIRS; elements from `width` on stay as they are.
 */
typedef enum maskkv_rotary_layout { MASKKV_ROTARY_HALVES = 0, MASKKV_ROTARY_PAIRS = 1 } maskkv_rotary_layout;

typedef struct maskkv_rotary {
  int32_t width;    /* even, 2 .. head_dim */
  int32_t layout;   /* a maskkv_rotary_layout */
  double amplitude; /* 1, or what a scaling for long contexts asks for */
  double freq[64];  /* radians a position, entries 0 .. width/2 - 1; 2^31 times each of them is finite */
} maskkv_rotary;

/* How frequencies are scaled for contexts `factor` times as long as the `trained` one (with f_i = base^(-2i/width)):
 *   PLAIN   f_i (factor, trained, slow and fast are not looked at)
 *   LINEAR  f_i / factor: positions are interpolated
 *   BASE    the same with base * factor^(width / (width - 2)) for base (width 2: as PLAIN): the fastest pair keeps its frequency, the slowest is divided by factor
 *   BANDS   by how often a pair turns within the trained length, r = trained * f_i / (2 pi): f_i where r >= fast, f_i / factor where
 *           r <= slow, and between them f_i * (w + (1 - w) / factor) with w = (r - slow) / (fast - slow);
 *           amplitude 1 + 0.1 ln(factor), for queries and for keys.
 * (The bands' ramp goes over how often a pair turns, not over the pair's number, and always comes with its amplitude.  A model that was trained with another
 * ramp, or with none but the frequencies, has its entries of maskkv_rotary set by the caller.) */
typedef enum maskkv_rotary_scaling {
  MASKKV_ROTARY_PLAIN = 0,
  MASKKV_ROTARY_LINEAR = 1,
  MASKKV_ROTARY_BASE = 2,
  MASKKV_ROTARY_BANDS = 3
} maskkv_rotary_scaling;

/*
 * Host arithmetic, no device work: fills *rotary (once, for all layers and steps of a model; a caller with frequencies of its own
 * fills it without this call).  width even, 2 .. 128; base > 0; and, where they are looked at, factor >= 1, trained > 0,
 * 0 <= slow < fast.
 */
int maskkv_rotary_frequencies(int32_t width, int32_t layout, double base, int32_t scaling, double factor, double trained,
                              double slow, double fast, maskkv_rotary* rotary);

/*
 * Rotates the rows of queries, of keys, or of both in one launch.  For b < B and t < token_len[b]:
 *   Q_out[b,h,t,:] = Q[b,h,t,:] turned by the position positions[b*n_tokens + t],  h < H*g;  K_out from K likewise, h < H.
 * Q, Q_out: views [B, H*g, n_tokens, d]; K, K_out: views [B, H, n_tokens, d]; a pair of them may be NULL, an output may be its own
 * input (the same view: in place), and outputs share no element with another view of the call (one that shares some with its own input is refused
 * where both have the same strides, or begin at the same row).  positions: DEVICE int32 [B, n_tokens],
 * any sign: rows turned by p and then by -p are (to rounding, with amplitude 1) what they were, so the rows of a cache can be moved to other
 * positions.  (A packed cache is a view of one sequence and one head.)  token_len: HOST int32 [B], 0 .. n_tokens, or NULL: n_tokens each; rows from token_len[b] on are left untouched.
 * 0 <= n_tokens <= 2^25.  Of the description B, H, d, dtype and q_per_kv count.  Angles are formed and reduced in 64 bits, sines and cosines and the
 * rotation in 32, rounded once to desc->dtype.
 */
int maskkv_rotate(const maskkv_desc* desc, const maskkv_rotary* rotary, const int32_t* positions, int32_t n_tokens,
                  const int32_t* token_len, const maskkv_tensor* Q, const maskkv_tensor* Q_out, const maskkv_tensor* K,
                  const maskkv_tensor* K_out, void* stream);

/*
 * Who sees whom among n rows of a sequence: bit j % 32 of word j / 32 of a row's W = (n + 31) / 32 words says whether row i sees row j.
 * mask: DEVICE uint32 [B, n, W].  For a drafted tree (or several next to each other) a row sees itself and the rows above it:
 *   parents[b*n + i] = the row that row i follows, less than i, or -1: row i follows the cache (a number of i or more counts as -1).
 *   -2 or less: there is no row i (a batch of trees of different sizes); it sees nothing and nothing follows it: a row that names it
 *   as its parent follows the cache.
 * parents: DEVICE int32 [B, n].  All words of every row are written.  B >= 0, 0 <= n <= 2^20, B <= 65535.
 */
int maskkv_tree_mask(const int32_t* parents, int32_t B, int32_t n, uint32_t* mask, void* stream);

/*
 * A cache in 4 bits (microscaling: one power of two for 32 neighbours along the head dimension).  All DEVICE, rows contiguous:
 * codes [capacity, d/2] bytes, scales [capacity, d/32] bytes.  Byte i of a row's codes holds element 2i in its low and element
 * 2i+1 in its high four bits: bit 3 is the sign, bits 0-2 number the sizes 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Scale byte s of a row
 * belongs to its elements 32s .. 32s+31, which stand for size * 2^(byte - 127); 255: for NaN, all of them.  maskkv_compact_mx
 * writes the bytes 3 .. 252 and 255 (above 252 the largest sizes would pass the range of fp32).
 * Pointers are multiples of 16 bytes.  A row takes 17/64 of what it takes in bf16.
 */
#define MASKKV_MX_MAX_ROWS 0x7FFF0000 /* capacity of the calls below, rows */
typedef struct maskkv_mx_cache {
  void* k_codes;
  void* k_scales;
  void* v_codes;
  void* v_scales;
} maskkv_mx_cache;

/*
 * Eviction as a gather into 4 bits: as maskkv_compact, but row r of the cache receives prompt row idx[r] of its head rounded to
 * 4 bits.  Of 32 neighbours x the scale is the smallest 2^e with max |x| <= 6 * 2^e, -124 <= e <= 125, and every x becomes the
 * nearest of the sizes times 2^e, a tie the one with the even number; what is beyond 6 * 2^125 becomes that.  32 neighbours with a NaN
 * or an infinity among them stand for NaN.  The result does not depend on anything but the row: equal rows give equal bytes.
 * Rows >= min(capacity, cu_budget[B*H]) are left untouched.
 */
int maskkv_compact_mx(const maskkv_desc* desc, const maskkv_tensor* K, const maskkv_tensor* V,
                      const int32_t* idx, const int32_t* cu_budget, int64_t capacity,
                      const maskkv_mx_cache* cache, void* stream);

/*
 * The values that a cache in 4 bits stands for, as packed rows Kc, Vc (DEVICE [capacity, d] in desc->dtype, exact in both
 * dtypes): what maskkv_attend and maskkv_accumulate read.  Rows >= min(capacity, cu_budget[B*H]) are left untouched.
 */
int maskkv_expand_mx(const maskkv_desc* desc, const maskkv_mx_cache* cache, const int32_t* cu_budget, int64_t capacity,
                     void* Kc, void* Vc, void* stream);

/* Workspace (DEVICE bytes) for maskkv_attend_mx with this description and capacity: partial results where the rows of a
 * head go to several workgroups: where few query rows attend to many rows, or where P_max and capacity leave room for a head that would
 * keep one workgroup busy for long; 0 where they do not.  256-byte alignment.  It is enough for every
 * smaller capacity too: a program that goes on evicting keeps the workspace of its first cache.  Nothing in it has to
 * be set before a call or outlives one; calls that may run at the same time (two streams, two captured graphs) need one each. */
int maskkv_attend_mx_workspace_bytes(const maskkv_desc* desc, int64_t capacity, size_t* bytes);

/*
 * maskkv_attend over a cache in 4 bits: the cached rows are the values that they stand for, the response rows K_resp/V_resp and the
 * queries are in desc->dtype, and everything else is as there (fp32 accumulation, probabilities rounded to desc->dtype only as
 * the operand of the P.V product, lse optional).  n_resp may be 1.
 */
int maskkv_attend_mx(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const maskkv_mx_cache* cache,
                     const int32_t* cu_budget, int64_t capacity, const maskkv_tensor* K_resp,
                     const maskkv_tensor* V_resp, float scale, const maskkv_tensor* O, float* lse,
                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * The attention that each cached row gets, added up over the denoising steps.  For row r of the cache of (b, h):
 *   weights_out[r] = decay * weights_in[r] + sum_i exp(q_i . k_r * scale - row_lse[i])
 * over all g * n_resp query rows i of the head's group (numbered as in Q_resp: query head first, then query), with the natural-log
 * normalisers that maskkv_attend or maskkv_attend_mx returned for the same queries, cache, response rows and scale
 * (row_lse[(b*H + h)*g*n_resp + i]).  A query row whose row_lse is +infinity adds nothing.  Kc: DEVICE [capacity, d] in
 * desc->dtype; weights: DEVICE float [capacity]; weights_in may be weights_out (but not
 * overlap it otherwise).  0 <= decay <= 1; with decay 0 weights_in is not
 * read and may be NULL.  fp32 accumulation in a fixed order: equal calls give equal bits.  Rows >= min(capacity,
 * cu_budget[B*H]) are left untouched.  _mx: the same over a cache in 4 bits, of which only the keys are read (v_codes and
 * v_scales may be NULL).
 */
int maskkv_accumulate(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const void* Kc, const int32_t* cu_budget,
                      int64_t capacity, float scale, const float* row_lse, float decay, const float* weights_in,
                      float* weights_out, void* stream);
int maskkv_accumulate_mx(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const maskkv_mx_cache* cache,
                         const int32_t* cu_budget, int64_t capacity, float scale, const float* row_lse, float decay,
                         const float* weights_in, float* weights_out, void* stream);

/*
 * Further eviction from the cache.  Of the n_h rows [cu_budget[bh], cu_budget[bh+1]) of every head (row numbers clipped to
 * capacity) the min(max(budgets[bh], 0), n_h) with the largest weights stay, ties to the lower row (a NaN counts as less than
 * every number, and -0 as 0), in their order:
 *   rows[r']   = the packed row that row r' of the smaller cache was,  r' in [cu_out[bh], cu_out[bh+1])
 *   Kc_out[r'] = Kc[rows[r']], and V, weights_out[r'] = weights[rows[r']] and idx_out[r'] = idx[rows[r']] likewise
 *   cu_out     = exclusive prefix sum of the rows that stay, B*H+1 entries.
 * rows, idx, idx_out: DEVICE int32 [capacity_out], [capacity], [capacity_out]; idx and idx_out (the rows' prompt positions)
 * may both be NULL, and so may weights_out; arrays of no rows (capacity or capacity_out 0) may be NULL too.  Where more than
 * capacity_out rows stay, those beyond it are not written while
 * cu_out holds the unclipped sums; sum_h budgets[bh] and capacity are always enough.  The smaller cache has buffers
 * of its own: an output that overlaps an input is MASKKV_EINVAL.  P_max may not exceed 4 Mi tokens, as in maskkv_select.  _mx: the same
 * for a cache in 4 bits, whose bytes are moved as they are.
 */
int maskkv_evict(const maskkv_desc* desc, const float* weights, const int32_t* cu_budget, int64_t capacity,
                 const int32_t* budgets, const void* Kc, const void* Vc, const int32_t* idx, void* Kc_out, void* Vc_out,
                 int32_t* idx_out, int32_t* rows, float* weights_out, int32_t* cu_out, int64_t capacity_out, void* stream);
int maskkv_evict_mx(const maskkv_desc* desc, const float* weights, const int32_t* cu_budget, int64_t capacity,
                    const int32_t* budgets, const maskkv_mx_cache* cache, const int32_t* idx,
                    const maskkv_mx_cache* cache_out, int32_t* idx_out, int32_t* rows, float* weights_out,
                    int32_t* cu_out, int64_t capacity_out, void* stream);

/* Workspace (DEVICE bytes) for maskkv_attend_tree with this description and capacity: partial results where the rows of a head go to
 * several workgroups; 0 where they do not.  256-byte alignment.  It is enough for every smaller capacity too.  Nothing in it has to be
 * set before a call or outlives one; calls that may run at the same time (two streams, two captured graphs) need one each. */
int maskkv_attend_tree_workspace_bytes(const maskkv_desc* desc, int64_t capacity, size_t* bytes);

/*
 * maskkv_attend where a response row i sees only the response rows j whose bit it has in `mask` (see maskkv_tree_mask; any bits are
 * allowed, in any order: blocks in order, windows, padded spans), and all cached rows of its head:
 *   O[b,hq,i,:] = sum_j softmax_j(Q_resp[b,hq,i,:] . k_j * scale) v_j,  j over the cache and the seen response rows.
 * mask: DEVICE uint32 [B, n_resp, (n_resp + 31) / 32], the same for all heads; bits from n_resp on are not looked at.  What a row does not see has no
 * part in its result, be it infinite or NaN.  A row that sees nothing (no bit, and no cached row) gets O = 0 and lse = -infinity.
 * The keys of a head are dealt to several workgroups where its query rows are few: single tokens and small trees over long caches.
 * capacity <= MASKKV_MX_MAX_ROWS.  A call that would launch 2^32 threads or more is MASKKV_ESHAPE: none of up to 2^27 query rows (B*H*g*n_resp) does.
 * Everything else as in maskkv_attend.
 */
int maskkv_attend_tree(const maskkv_desc* desc, const maskkv_tensor* Q_resp, const void* Kc, const void* Vc,
                       const int32_t* cu_budget, int64_t capacity, const maskkv_tensor* K_resp, const maskkv_tensor* V_resp,
                       const uint32_t* mask, float scale, const maskkv_tensor* O, float* lse, void* workspace,
                       size_t workspace_bytes, void* stream);

/* What maskkv_sample draws from: DEVICE arrays with an entry a row, 4-byte aligned (as token, prob and logprob), or NULL. */
typedef struct maskkv_sampling {
  const float* temperature; /* NULL: 1 each */
  const int32_t* top_k;     /* NULL, or an entry of 0 or less: no limit */
  const float* top_p;       /* NULL, or an entry of 1 or more: no limit */
  const float* min_p;       /* NULL, or an entry of 0 or less: no limit */
  const float* uniform;     /* random numbers, [0, 1) */
} maskkv_sampling;

/* Workspace (DEVICE bytes) for maskkv_sample of so many rows, and of fewer.  256-byte alignment.  Nothing in it has to be set before a
 * call or outlives one; calls that may run at the same time need one each. */
int maskkv_sample_workspace_bytes(int64_t rows, int32_t vocab, int32_t dtype, size_t* bytes);

/*
 * A token for every row of logits l, with given random numbers.  With m the row's largest logit, w_j = exp((l_j - m) / temperature):
 *   1. tokens are ranked by their logits, the largest first and equal ones by their number;
 *   2. top_k: the first top_k of them stay;
 *   3. top_p: of these, in that order, those before which less than top_p of their common mass (sum of w) lies; the first one always;
 *   4. min_p: of these, those with w_j >= min_p (at 1 and more: with the largest logit);
 *   token[r]   = in the order of their numbers, the first of the tokens that stay with  sum_{i <= j} w_i > uniform * (the sum of all that stay)
 *   prob[r]    = w_token / (the sum of all that stay): with which probability it was drawn
 *   logprob[r] = l_token - log sum_j exp(l_j): without temperature and limits, over all tokens.  Its exp is the confidence by which a
 *                denoising step chooses which positions it keeps.
 * A temperature of 0 or less (or NaN) takes the first of the largest logits, prob 1.  A NaN logit counts as -infinity; where +infinity occurs, its tokens share
 * all mass evenly.  A row without a finite or infinite logit above -infinity has token -1, prob 0 and logprob -infinity.  A random number below 0 counts
 * as 0, one of 1 and more (or NaN) as the largest below 1; limits that are NaN are none.
 * logits: DEVICE [rows, vocab] in `dtype` (a maskkv_dtype), rows row_stride >= vocab elements apart, aligned to an element; vocab 1 .. 2^24; 0 <= rows <= 2^20
 * (and rows times the stretches of 4 KB that a row, beginning anywhere in 16 bytes, may take fewer than 2^26 - 4, else MASKKV_ESHAPE).
 * token: DEVICE int32 [rows]; prob, logprob: DEVICE float [rows], or NULL.  Masses are held in 64 bits and summed up in a fixed order (or as whole
 * numbers): equal calls give equal bits, and a token is the definition's unless the random number or a limit lies within 1e-10 of the mass of where
 * another one would be.  (The terms of logprob's sum are 32-bit exponentials where the logits are bf16; the sum has 64 bits.)
 */
int maskkv_sample(const void* logits, int64_t rows, int32_t vocab, int32_t dtype, int64_t row_stride,
                  const maskkv_sampling* sampling, int32_t* token, float* prob, float* logprob, void* workspace,
                  size_t workspace_bytes, void* stream);

/*
 * Stage 2, head level, on the device.  For every b:
 *   P_h = prompt_mass[b*H+h] / (g*n_query)  (mask-to-prompt share of the voting rows' attention)
 *   budgets[b*H+h] = floor(alpha*k_l + (1-alpha) * H * k_l * P_h / sum_h' P_h')
 * prompt_mass: DEVICE float [B*H] as written by maskkv_score; budgets: DEVICE int32 [B*H].
 * k_l is the layer's per-head average budget; 0 <= alpha <= 1.  A sequence whose masses are all zero (empty
 * prompt) gets budgets[..] = k_l for every head.
 */
int maskkv_head_budgets(const maskkv_desc* desc, const float* prompt_mass, int32_t k_l, float alpha,
                        int32_t* budgets, void* stream);

/* Workspace (DEVICE bytes) needed by maskkv_layer_importance.  256-byte alignment. */
int maskkv_layer_importance_workspace_bytes(size_t* bytes);

/*
 * Stage 2, layer level, the layer importance metric:
 *   importance[0] = 1 - (1/n) sum_i cos_sim(h_in[i, :], h_out[i, :])
 * over the n_tokens rows of a layer's attention sub-layer input and output hidden states.
 * h_in, h_out: DEVICE [n_tokens, hidden] in `dtype` (a maskkv_dtype), rows row_stride elements apart
 * (row_stride >= hidden), pointers and row stride multiples of 16 bytes, hidden a multiple of 8
 * elements.  importance: DEVICE float [1].  fp32 accumulation.  n_tokens >= 1.
 */
int maskkv_layer_importance(const void* h_in, const void* h_out, int64_t n_tokens, int32_t hidden, int32_t dtype,
                            int64_t row_stride, float* importance, void* workspace, size_t workspace_bytes,
                            void* stream);

/*
 * Stage 2, layer level, the boundary-aware budget allocation (host arithmetic, no device work):
 *   k_base = floor(beta * k_p / L),  k_imp = k_p - L * k_base;
 *   k_imp is split between the boundary layers and the other (middle) layers in proportion to the sums
 *   of their importances; every layer receives k_base plus the floor of an equal share of its group's part.
 * importance: HOST float [n_layers]; boundary: HOST int32 [n_boundary] layer numbers, or NULL for
 * {first, last}; k_l: HOST int64 [n_layers] output.  k_p >= 0, 0 <= beta <= 1, importances >= 0 with a
 * positive sum.  The budget lost to the floors is left unallocated (sum k_l <= k_p).
 */
int maskkv_layer_budgets(const float* importance, int32_t n_layers, int64_t k_p, float beta,
                         const int32_t* boundary, int32_t n_boundary, int64_t* k_l);

/*
 * Response-token refresh criterion of the feature-cache background (Section 3.1, the set S_shift):
 *   cos[i]  = cos_sim(V_now[i, :], V_prev[i, :])  for the n_tokens response tokens of a layer
 *   refresh = ascending positions i with cos[i] < delta (strict), count[0] of them.
 * V_now, V_prev: DEVICE [n_tokens, width] in `dtype` (a maskkv_dtype; width = heads * head_dim), rows
 * row_stride elements apart, pointers and row stride multiples of 16 bytes, width a multiple of 8.
 * cos: DEVICE float [n_tokens]; refresh: DEVICE int32 [n_tokens] (entries >= count[0] untouched); count:
 * DEVICE int32 [1].  fp32 accumulation; the comparison is made on the fp32 cosine.  A row of zeros has no
 * cosine (NaN) and is not listed.  No workspace.
 */
int maskkv_value_shift(const void* V_now, const void* V_prev, int64_t n_tokens, int32_t width, int32_t dtype,
                       int64_t row_stride, float delta, float* cos, int32_t* refresh, int32_t* count, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MASKKV_H */
