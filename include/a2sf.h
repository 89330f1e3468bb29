/*
 * a2sf.h - C ABI of the MI355X (gfx950) A2SF hot path.
 *
 * A2SF = Accumulative Attention Score with Forgetting Factor (arxiv 2407.20485).
 * The library computes, for G independent heads (one head = one (layer, batch, head)
 * triple; the paper keeps a separate score per layer and per head, Section 2.2 and
 * Section 3.1 Eq.2):
 *
 *   prompt phase      masked self-attention (Section 1, Section 3.1 Eq.3), the forgotten
 *                     accumulated score of every prompt token (Section 3.3 Eq.5/Eq.6)
 *                     S_j = sum_{i>=j} alpha^(n-1-i) * softmax(Q K^T / sqrt(d))[i, j],
 *                     and one selection of the budgeted token set into a KV cache;
 *   generation step   attention of one new query over the retained tokens only
 *                     (Section 2.2: pruning changes the softmax denominator), the update
 *                     S <- alpha * S + a_t on every retained token (abstract, Section 3.3),
 *                     and eviction of the lowest-score tokens so that the budget holds
 *                     (Section 2.2, Section 3.1 after Eq.2, Section 4.1 for the split of
 *                     the budget into a score-selected and a most-recent part).
 *
 * Conventions shared by every call
 *  - All data pointers are DEVICE pointers owned by the caller; the library never
 *    allocates, frees or keeps them.  a2sf_cache itself is a small HOST struct.
 *  - Every call only enqueues work on `hip_stream` (a hipStream_t passed as void*;
 *    NULL = the default stream) and never synchronises.  Results are valid once the
 *    stream reaches the end of the enqueued work.
 *  - Arguments are validated on the host before anything is launched; an argument
 *    error returns its status and launches nothing (so it is testable without a GPU).
 *    A failed launch returns A2SF_EHIP.
 *  - Row-major everywhere, head dimension d contiguous.  d is 64 or 128.  dtype is
 *    fp32 or bf16 for Q/K/V/O; scores are always fp32, positions int32.
 *  - Data pointers must be 16-byte aligned.
 *  - 0 <= alpha <= 1 and finite.  The paper states 0 < alpha < 1 (Section 3.3) but
 *    evaluates alpha = 0 (Section 4.4) and alpha = 1 is the plain accumulated score of
 *    Section 3.1 Eq.4; both ends are accepted, with 0^0 = 1.
 *  - Budget B = select + recent >= 1.  recent = 0 is the paper's own A2SF setting and
 *    select = 0 is its local-attention baseline (Section 4.1).
 *  - "Position" is the 0-based index of a token in the sequence.  Ties between equal
 *    scores are resolved in favour of the lower position (the higher one is evicted).
 *  - Original positions stored in a cache must be distinct and >= 0.
 */
#ifndef A2SF_H
#define A2SF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  A2SF_OK = 0,
  A2SF_EINVAL = 1,     /* null pointer, misaligned pointer, alpha outside [0,1] or not finite,
                          negative count, unknown mode */
  A2SF_ESHAPE = 2,     /* d not in {64,128}, n < 1, G < 1, L < 1 ... */
  A2SF_EDTYPE = 3,     /* dtype not A2SF_F32 / A2SF_BF16 */
  A2SF_ECAPACITY = 4,  /* cache capacity too small for budget + 1, or above the supported maximum */
  A2SF_EWORKSPACE = 5, /* workspace missing or smaller than a2sf_workspace_bytes() */
  A2SF_EHIP = 6        /* the HIP runtime reported an error at launch */
} a2sf_status;

typedef enum { A2SF_F32 = 0, A2SF_BF16 = 1, A2SF_E4M3 = 2 /* pages only */ } a2sf_dtype;

/* How a generation step makes the cache dense again after an eviction. */
typedef enum {
  A2SF_EVICT_FAST = 0,   /* the new token's row is written into the evicted slot: no row
                            moves; slot order becomes arbitrary, the set of (pos, K, V, S)
                            tuples is what is defined */
  A2SF_EVICT_STABLE = 1  /* slots stay in ascending position (select + in-place compaction) */
} a2sf_evict_mode;

/* Section 4.1: the cache ratio is split into a score-selected and a most-recent part. */
typedef struct {
  int32_t select; /* tokens kept for their score, >= 0 */
  int32_t recent; /* newest tokens always kept, >= 0 */
} a2sf_budget;

/* The KV cache of G heads plus the A2SF bookkeeping (host struct, device pointers). */
typedef struct {
  void* k;        /* [G, capacity, d] dtype */
  void* v;        /* [G, capacity, d] dtype */
  float* scores;  /* [G, capacity] accumulated score of each slot */
  int32_t* pos;   /* [G, capacity] original position of each slot */
  int32_t* len;   /* [G] number of valid slots of each head */
  int32_t G;
  int32_t capacity; /* slots per head; needs >= select + recent + 1; at most A2SF_MAX_CAPACITY */
  int32_t d;
  int32_t dtype;  /* a2sf_dtype */
} a2sf_cache;

/* One float per slot is kept in the 160 KB of LDS of a compute unit by the generation step. */
#define A2SF_MAX_CAPACITY 36864

/* Bytes of device workspace that any of the calls below may need for these sizes
 * (n_max = longest prompt, 0 if a2sf_prefill is not used; capacity as in a2sf_cache).
 * Returns 0 on invalid arguments.  The content of the workspace need not be preserved
 * between calls; calls that share a workspace must not overlap in time. */
size_t a2sf_workspace_bytes(int32_t G, int32_t n_max, int32_t capacity, int32_t d,
                            int32_t dtype, a2sf_budget budget);

/* Prompt phase (Section 3.1 Eq.3, Section 3.3 Eq.5, one selection as in Section 2.2).
 *   q, k, v      [G, n, d] dtype, read only.
 *   cache        out: for every head the min(n, B) surviving tokens in ascending
 *                position: K, V rows, their Eq.5 score, their position; len = min(n, B).
 *                Survivors: the `recent` last positions, plus of the others the `select`
 *                with the largest score (tie -> lower position).
 *   o            out [G, n, d] dtype: attention output rows; may be NULL: then no P*V
 *                work is done, and rows whose weight alpha^(n-1-i) is
 *                exactly 0 in fp32 are not visited at all where the scores do not need them.
 *   scores_full  out [G, n] fp32: the Eq.5 score of every prompt token; may be NULL.
 * The n x n probability matrix is never written to memory.
 * Range of values: fp32 results have the precision of fp32 arithmetic for all normal numbers;
 * logits may take any finite value, and an infinity or NaN in a row of V reaches only the
 * rows that see it (such rows, and some of numbers beyond 2^100 or below 2^-110, take two to five
 * times as long).  bf16 works on tiles of 64 keys: an infinity or NaN in a row
 * of V may also reach earlier rows of its tile, as NaN, and a row whose logits (q . k / sqrt(d)) all
 * lie below about -7e29 comes out as NaN.  The same holds for a2sf_prefill_chunk. */
a2sf_status a2sf_prefill(const void* q, const void* k, const void* v, int32_t n, float alpha,
                         a2sf_budget budget, const a2sf_cache* cache, void* o,
                         float* scores_full, void* workspace, size_t workspace_bytes,
                         void* hip_stream);

/* a2sf_prefill with a relative tolerance on the Eq.5 scores (Section 3.3: the forgetting
 * factor sends the contribution of old rows to 0, so for alpha < 1 only the newest rows of
 * the prompt matter).  Rows whose whole remaining contribution to S_j is PROVABLY at most
 * score_rel_tol * S_j are not computed.  The bound needs nothing but the newest row: all rows
 * before n - W together add at most alpha^W / (1 - alpha) to any score (probabilities are
 * <= 1) while S_j >= P[n-1, j]; the kernel reads the smallest P[n-1, j] of each group of 64
 * keys off the newest row, which it processes first, and walks back W rows with
 * alpha^W <= score_rel_tol * (1 - alpha) * min_j P[n-1, j].
 *   score_rel_tol  in [0, 1); 0 = every row of nonzero fp32 weight, exactly a2sf_prefill.
 * Everything else as in a2sf_prefill.  The window is applied to bf16 prompts with d = 128 that are
 * longer than a few hundred rows; other shapes compute every row (the result is then a2sf_prefill's).  alpha = 1 has no
 * window, alpha = 0 only the newest row either way. */
a2sf_status a2sf_prefill_windowed(const void* q, const void* k, const void* v, int32_t n,
                                  float alpha, float score_rel_tol, a2sf_budget budget,
                                  const a2sf_cache* cache, void* o, float* scores_full,
                                  void* workspace, size_t workspace_bytes, void* hip_stream);

/* A further chunk of a prompt that is too long to be processed at once (beyond the paper,
 * which evicts once per generation step, Section 3.1): the chunk's m tokens are m generation
 * steps whose eviction is deferred to the end of the chunk, so that their rows go through the
 * matrix cores together.
 *   q, k, v   [G, m, d] dtype: the chunk's queries, keys and values; its tokens have
 *             positions pos0 .. pos0 + m - 1 (larger than every cached one).
 *   cache     in/out; requires len[g] + m <= capacity (so capacity > m).  Row i of the chunk
 *             attends the head's cached tokens and the chunk's tokens 0 .. i (softmax over
 *             exactly those, Section 2.2); o_i is that row's output; every cached token's score
 *             becomes alpha^m * S + sum_i alpha^(m-1-i) P[i, .] and a chunk token gets
 *             sum_{i >= its own row} alpha^(m-1-i) P[i, .] (Section 3.3 Eq.5 over the rows
 *             that exist); then ONE eviction as in a2sf_decode_step's stable mode brings the
 *             head down to min(len + m, B) tokens, slot order preserved.
 *             A head without room for the chunk is left untouched, its rows of o are NaN.
 *   o         out [G, m, d] dtype, may be NULL.
 * The first chunk of a prompt is a2sf_prefill (or this call on an empty cache, len = 0).
 * Workspace: a2sf_workspace_bytes(G, m, capacity, d, dtype, budget). */
a2sf_status a2sf_prefill_chunk(const void* q, const void* k, const void* v, int32_t m, int32_t pos0,
                               float alpha, a2sf_budget budget, const a2sf_cache* cache, void* o,
                               void* workspace, size_t workspace_bytes, void* hip_stream);

/* One generation step (abstract; Section 2.2; Section 3.3).
 *   q, k_new, v_new  [G, d] dtype: the new token's query, key and value.
 *   t_pos            original position of the new token (larger than every cached one).
 *   cache            in/out.  Requires 0 <= len[g] and len[g] + 1 <= capacity; a head that
 *                    violates this is left untouched and its row of o is filled with NaN
 *                    (the lengths live on the device, so the host cannot check them).
 *                    The new token joins with
 *                    score 0; a = softmax(K_c q / sqrt(d)) over the len+1 cached tokens;
 *                    o = a^T V_c; every score becomes alpha*S + a; then, if len+1 > B,
 *                    the len+1-B lowest-score tokens outside the `recent` newest
 *                    positions are evicted (tie -> the higher position goes) and
 *                    len = B; else len = len+1.
 *   mode             a2sf_evict_mode.
 *   o                out [G, d] dtype. */
a2sf_status a2sf_decode_step(const void* q, const void* k_new, const void* v_new, int32_t t_pos,
                             const a2sf_cache* cache, float alpha, a2sf_budget budget,
                             int32_t mode, void* o, void* workspace, size_t workspace_bytes,
                             void* hip_stream);

/* Grouped-query heads (beyond the paper, whose models are all multi-head): `group` query heads
 * share each of the G K/V heads of the cache, so a token is kept or evicted for the whole
 * group.  The group's score of a token is the SUM of its query heads' accumulated scores -- as
 * the paper's Eq.1 sums over the heads that one pruning decision serves.  Every query head has
 * its own softmax and its own output.
 *   group        1 .. 8 (1 = the plain calls).
 *   q            prefill: [G, group, n, d]; decode: [G, group, d].
 *   k, v / k_new, v_new   as in the plain calls: one row per K/V head.
 *   o            prefill: [G, group, n, d] (may be NULL); decode: [G, group, d].
 *   scores_full  [G, n] (prefill, may be NULL): the summed scores.
 * Workspace: a2sf_workspace_bytes(G * group, n, capacity, d, dtype, budget) for the prefill
 * (one log-sum-exp row per query head); the decode step needs one only in stable mode
 * (a2sf_workspace_bytes(G, 0, capacity, ...) is enough for that).  Given a larger one -- the
 * prefill's, or a2sf_workspace_bytes(G * group, 0, capacity, ...) plus
 * 4 * G * group * 64 * (d + 2) bytes -- a step over few K/V heads with long caches (bf16,
 * d = 128) splits each head's tokens over as many workgroups as its scratch
 * memory allows; results do not depend on that beyond fp32 summation order.  The decode step
 * holds group * capacity logits in LDS: group * capacity <= A2SF_GQA_MAX_LOGITS. */
#define A2SF_GQA_MAX_LOGITS 16384
a2sf_status a2sf_prefill_gqa(const void* q, const void* k, const void* v, int32_t n, int32_t group,
                             float alpha, a2sf_budget budget, const a2sf_cache* cache, void* o,
                             float* scores_full, void* workspace, size_t workspace_bytes,
                             void* hip_stream);
a2sf_status a2sf_decode_step_gqa(const void* q, const void* k_new, const void* v_new, int32_t t_pos,
                                 const a2sf_cache* cache, int32_t group, float alpha,
                                 a2sf_budget budget, int32_t mode, void* o, void* workspace,
                                 size_t workspace_bytes, void* hip_stream);

/* a2sf_prefill_chunk for grouped-query heads (the two extensions above together): a chunk of m
 * tokens of G K/V heads with `group` query heads each.  Every query head attends as a plain
 * head's chunk does, with its own softmax and output; a cached token's score becomes
 * alpha^m * S + the sum over the group's heads of sum_i alpha^(m-1-i) P_h[i, .]; one eviction
 * per K/V head.
 *   q, o      [G, group, m, d] (o may be NULL);  k, v  [G, m, d].
 * Everything else as in a2sf_prefill_chunk.
 * Workspace: a2sf_workspace_bytes(G * group, m, capacity, d, dtype, budget). */
a2sf_status a2sf_prefill_chunk_gqa(const void* q, const void* k, const void* v, int32_t m,
                                   int32_t pos0, int32_t group, float alpha, a2sf_budget budget,
                                   const a2sf_cache* cache, void* o, void* workspace,
                                   size_t workspace_bytes, void* hip_stream);

/* a2sf_decode_step for callers that cannot provide or allocate a workspace: code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation.  Identical in every
 * other respect (same kernels, same results); the scratch memory that a2sf_decode_step takes
 * as `workspace` is a fixed array of A2SF_STATIC_WS_BYTES inside the library instead, one per
 * GPU, held until the process ends.  Nothing is allocated or freed by this call.
 *  - Returns A2SF_EWORKSPACE, launching nothing, when
 *    a2sf_workspace_bytes(G, 0, capacity, d, dtype, budget) exceeds A2SF_STATIC_WS_BYTES.
 *  - Every call on one GPU uses the same array: calls that overlap in time on one GPU (on
 *    different streams) race.  The array keeps the previous call's content; every kernel
 *    writes what it later reads, so nothing has to be cleared.
 *  - The first call on a device looks the array's address up (hipGetSymbolAddress); make that
 *    first call outside any stream capture. */
#define A2SF_STATIC_WS_BYTES (16u << 20)
a2sf_status a2sf_decode_step_static_ws(const void* q, const void* k_new, const void* v_new,
                                       int32_t t_pos, const a2sf_cache* cache, float alpha,
                                       a2sf_budget budget, int32_t mode, void* o, void* hip_stream);

/* The same two calls with one forgetting factor per head (Section 6 of the paper names a
 * distinct factor per layer and head as the way to lift its limitation of a single one).
 *   alpha_heads  [G] fp32, device: head g uses alpha_heads[g], each in [0, 1].
 *   alpha_max    (prefill only) an upper bound of alpha_heads, checked like alpha; it sizes
 *                the row window of the score pass.  A head whose factor exceeds it is
 *                computed with alpha_max instead of its own factor.
 * Everything else as in a2sf_prefill / a2sf_decode_step. */
a2sf_status a2sf_prefill_alpha_per_head(const void* q, const void* k, const void* v, int32_t n,
                                        const float* alpha_heads, float alpha_max,
                                        a2sf_budget budget, const a2sf_cache* cache, void* o,
                                        float* scores_full, void* workspace,
                                        size_t workspace_bytes, void* hip_stream);
a2sf_status a2sf_decode_step_alpha_per_head(const void* q, const void* k_new, const void* v_new,
                                            int32_t t_pos, const a2sf_cache* cache,
                                            const float* alpha_heads, a2sf_budget budget,
                                            int32_t mode, void* o, void* workspace,
                                            size_t workspace_bytes, void* hip_stream);

/* Selection alone (Section 2.2, Section 4.1): which of the L tokens of each head survive.
 *   scores    [G, stride] fp32 (no NaN);  pos [G, stride] int32 or NULL (position = slot).
 *   len       [G] device, valid slots per head (<= L), or NULL: every head has L.
 *   keep_idx  out [G, B]: surviving slot indices in ascending slot order, first n_keep[g]
 *             entries valid;  n_keep out [G] = min(len, B).
 * Survivors: the `recent` largest positions plus the `select` best scores of the rest
 * (tie -> lower position); everything if len <= B. */
a2sf_status a2sf_select(const float* scores, const int32_t* pos, const int32_t* len, int32_t G,
                        int32_t L, int32_t stride, a2sf_budget budget, int32_t* keep_idx,
                        int32_t* n_keep, void* hip_stream);

/* Removal of the tokens that were not selected (Section 2.2: tokens with a small accumulated
 * score are removed from the KV cache; Section 3.1 after Eq.2), as an in-place stable
 * compaction: for every head, row keep_idx[g][r] of K, V, scores and pos moves to row r for
 * r < n_keep[g], and len[g] = n_keep[g].
 *   keep_idx  [G, keep_stride] strictly ascending indices of valid slots, i.e. below len[g]
 *             (as a2sf_select writes).
 *   n_keep    [G] device. */
a2sf_status a2sf_compact(const a2sf_cache* cache, const int32_t* keep_idx, int32_t keep_stride,
                         const int32_t* n_keep, void* hip_stream);

/* Diagnostic of Section 4.3 / Table 2: how close a pruning policy's attention row is to the
 * row of the Ideal mask, for one generation step of every head.  The Ideal attends ALL
 * tokens so far (nothing is ever removed) and keeps the entries of the tokens with the
 * largest attention score (tie -> lower position), as many as the policy's row has; the
 * policy's row has entries on the tokens in its cache and on the new token.  Either row is
 * the softmax over its own tokens (Section 2.2), zero elsewhere; the result is their cosine.
 *   q        [G, d] dtype: the step's query.
 *   k_all    [G, n_stride, d] dtype, read only: the keys of all tokens so far, row = position,
 *            rows 0 .. t_pos valid (row t_pos is the new token's key).
 *   t_pos    position of the new token; t_pos + 1 <= A2SF_SIM_MAX_ROWS, t_pos < n_stride.
 *   cache    the policy's cache BEFORE this step; only pos, len, capacity, G, d and dtype
 *            are read.  Cached positions must be < t_pos.
 *   cos_out  out [G] fp32, in [0, 1]; 1 when the two rows select the same tokens.
 * Call it right before the a2sf_decode_step of the same token. */
#define A2SF_SIM_MAX_ROWS 32768
a2sf_status a2sf_ideal_similarity(const void* q, const void* k_all, int32_t n_stride,
                                  int32_t t_pos, const a2sf_cache* cache, float* cos_out,
                                  void* hip_stream);

/* Average of the similarities over the steps from first_step on and over all heads: the
 * figure Table 2 reports (Section 4.3; steps before the budget is reached prune nothing and
 * are left out by the caller through first_step).
 *   cos       [steps, G] fp32, device, as successive a2sf_ideal_similarity calls wrote it.
 *   mean_out  out [1] fp32, device; 1 when no step is left to average. */
a2sf_status a2sf_similarity_mean(const float* cos, int32_t steps, int32_t G, int32_t first_step,
                                 float* mean_out, void* hip_stream);

/* How a2sf_decode_step will launch for these sizes (host only, launches nothing; for
 * benchmarks and profiles that have to name the kernels they measure).  Any out pointer may
 * be NULL.
 *   nsplit          workgroups per head; 1 = one fused kernel, > 1 = the tokens of a head are
 *                   split over that many workgroups and a second kernel combines them (reported
 *                   for bf16; few fp32 heads are split from fewer slots on).
 *   rows_per_split  cached tokens per workgroup when nsplit > 1.
 *   wave_slots      > 0: a wave works on a whole head (64 * wave_slots slots in registers).
 *   wave_heads      heads a wave works through in the fast eviction mode: 1, or more in the
 *                   form for launches with several times more heads than the chip holds waves
 *                   (persistent workgroups; a step's small writes are held back in LDS).
 * This is the fast eviction mode.  A step in A2SF_EVICT_STABLE differs: up to 4095 heads of at
 * most 512 slots (256 where a row has 512 bytes) take one kernel, whatever nsplit says; every
 * other step is the kernels reported here, one head per wave, and then selects and compacts. */
a2sf_status a2sf_decode_plan(int32_t G, int32_t capacity, int32_t d, int32_t* nsplit,
                             int32_t* rows_per_split, int32_t* wave_slots, int32_t* wave_heads);

/* ---- What a decoder layer computes around the attention ----------------------------------------------------------------
 * Root-mean-square norm, 8-bit rows and their products, rotary positions, sampling: the calls between one attention call
 * and the next.  The conventions above hold (device pointers, one stream, no allocation, no synchronisation); further:
 *  - Rows of a tensor lie `stride` elements apart, any stride >= their length (of a single row it is not looked at).
 *    Pointers need the alignment of their elements only, so rows may be parts of wider ones; 8-bit rows and the workspace:
 *    16 bytes.
 *  - Where an input and an output are the same rows, every element is read before it is written.  Other overlaps are
 *    not allowed.
 *  - A launch takes less than 2^32 lanes, and what needs more is refused with A2SF_ESHAPE: a row of a2sf_rms_norm takes 64 to 1024 by its
 *    length, a row of a2sf_sample or a2sf_log_probs 1024, 128 columns of a2sf_quantize 16, 128 x 128 weights 256, 64 bytes of a token's heads in a2sf_rotary 1.
 *  - Sums, norms and products are formed in 32 bits or more whatever the type (a2sf_matmul_scaled: where the caller does not leave that
 *    to the 8-bit matrix instruction; a2sf_paged_attention: the probabilities of bf16 calls, as stated there); results are rounded once. */
typedef struct {
  void* data;
  int64_t stride; /* elements from row to row */
} a2sf_rows;

/* Rows of 8-bit floats (e4m3: largest value 448, no infinities) with a scale for each 128 columns (for weights: for each
 * 128 x 128).  A scale is a power of two, held as its exponent plus 127 in a byte; 255 stands for "not a number".  The
 * values stand for q * 2^(scale - 127).  The calls that make them take the smallest scale, no smaller than 2^-127, that brings the
 * largest magnitude of its block to 448 or below, and round q to nearest, ties to even.  A block that holds an infinity
 * or a NaN becomes all NaN (scale 255). */
typedef struct {
  void* data;           /* rows start at multiples of 16 bytes */
  uint8_t* scales;      /* [rows (weights: ceil(rows / 128)), ceil(columns / 128)], rows start at multiples of 4 bytes */
  int64_t stride;       /* bytes from row to row, a multiple of 16 */
  int64_t scale_stride; /* bytes, a multiple of 4 */
} a2sf_rows8;

#define A2SF_MAX_ROW 65536 /* longest row of a2sf_rms_norm */

/* h = x + residual;  total = h;  y = h / sqrt(mean(h^2) + eps) * weight, row by row.
 *   x, residual  [rows, n] dtype; residual may be NULL (h = x).
 *   weight       [n] dtype.
 *   total        out [rows, n] dtype; may be NULL, and may be the rows of x or residual.  The norm is of h before its
 *                rounding to dtype, h being formed in 32 bits; its squares may leave their range at either end.
 *   out, out8    out: y in dtype, y in 8 bits; either may be NULL, not both.
 * n <= A2SF_MAX_ROW, eps >= 0 and finite. */
a2sf_status a2sf_rms_norm(const a2sf_rows* x, const a2sf_rows* residual, const void* weight, float eps, int32_t rows,
                          int32_t n, int32_t dtype, const a2sf_rows* total, const a2sf_rows* out,
                          const a2sf_rows8* out8, void* hip_stream);

/* Rows to 8 bits: y = x, or with a gate y = gate / (1 + exp(-gate)) * x (before its rounding within 12 * 2^-24 of its size; 0 for gates
 * below -87, where exp(-gate) leaves the range of 32 bits).
 *   x, gate    [rows, n] dtype; gate may be NULL.
 *   out, out8  out: y in dtype, y in 8 bits; either may be NULL, not both. */
a2sf_status a2sf_quantize(const a2sf_rows* x, const a2sf_rows* gate, int32_t rows, int32_t n, int32_t dtype,
                          const a2sf_rows* out, const a2sf_rows8* out8, void* hip_stream);

/* Weights [n, k] (n outputs of k inputs) to 8 bits with a scale for each 128 x 128; done once, when they are loaded. */
a2sf_status a2sf_quantize_weight(const a2sf_rows* w, int32_t n, int32_t k, int32_t dtype, const a2sf_rows8* out8,
                                 void* hip_stream);

/* C = A B^T of 8-bit rows: C[i, j] = sum over blocks of 128 of k: scale of A's block * scale of B's block * sum a b.
 *   a          [m, k] as a2sf_rms_norm and a2sf_quantize write them.
 *   b          [n, k] as a2sf_quantize_weight writes them.
 *   c          out [m, n], c_dtype (A2SF_F32 or A2SF_BF16).
 *   c_dtype    A2SF_F32, and A2SF_BF16 | A2SF_WIDE_SUMS: sums in 32 bits (within k * 2^-24 * sum |a b|, for scale bytes of 10 to 246: values are
 *              taken as bf16, whose subnormal numbers have fewer bits than those of smaller scales, and whose range ends before larger ones).  A2SF_BF16 alone: by the 8-bit matrix
 *              instruction, at about twice the rate where the rate counts; it cuts each of eight neighbouring products of k under 2^-13
 *              of the largest of them, so a sum is within 8 * 2^-13 * sum |a b| of the exact one before it is rounded to bf16 (for data
 *              like a model's 1.5e-5 of the result's size; a sum that cancels may lose all of it).
 *   workspace  may be NULL; with a2sf_matmul_workspace_bytes(m, n, k) bytes (0: none is of use; enough for either kind of sums) products
 *              that have too few tiles for the whole chip split their sums over k; with less, if their own parts fit.  The same sizes with
 *              the same choices give the same bits.
 * Bytes of the rows past k are not used.  k <= 2^20, rows of a and b and rows of scales at most 2^23 bytes apart. */
#define A2SF_WIDE_SUMS 0x100 /* or'ed to c_dtype, and to the dtype of a2sf_paged_attention */
size_t a2sf_matmul_workspace_bytes(int32_t m, int32_t n, int32_t k);
a2sf_status a2sf_matmul_scaled(const a2sf_rows8* a, const a2sf_rows8* b, int32_t m, int32_t n, int32_t k,
                               const a2sf_rows* c, int32_t c_dtype, void* workspace, size_t workspace_bytes,
                               void* hip_stream);

/* Rotary positions.  Each part is the heads [batch, length, heads, d] of one tensor, read and written through strides, so that a
 * QKV product [batch, length, (Hq + 2 Hkv) d] goes in one call to q [batch, Hq, length, d], k and v [batch, Hkv, length, d]
 * as a2sf_prefill takes them (length = 1: as a2sf_decode_step does), or turns in place.
 * Of a head's elements the first rotary_dims turn in pairs, the others are copied.  Pair i has the elements (i, i +
 * rotary_dims / 2) (A2SF_ROTARY_HALVES) or (2i, 2i + 1) (A2SF_ROTARY_NEIGHBOURS) and becomes
 * (x0 c - x1 s, x1 c + x0 s) with c, s of the token's position; inverse != 0: with -s, the rotation back, which is also
 * the gradient's. */
#define A2SF_MAX_ROTARY_PARTS 4
typedef enum { A2SF_ROTARY_HALVES = 0, A2SF_ROTARY_NEIGHBOURS = 1 } a2sf_rotary_pairs;
typedef struct {
  const void* x;
  void* y;             /* may be x with the same strides */
  int64_t x_stride[3]; /* elements from sequence to sequence, token to token, head to head; a head's are contiguous */
  int64_t y_stride[3];
  int32_t heads;
  int32_t rotate; /* 0: copied as they are (the heads of v) */
} a2sf_rotary_part;
/*   pos    [batch, length] int32, rows pos_stride apart.  A token whose position is not a row of the table gets NaN in
 *          the rotated parts' rotary_dims.
 *   table  [table_rows, rotary_dims] fp32: a position's cosines, then its sines (a2sf_rotary_table).
 * 1 to A2SF_MAX_ROTARY_PARTS parts, d <= 512, rotary_dims even and <= d. */
a2sf_status a2sf_rotary(const a2sf_rotary_part* parts, int32_t n_parts, int32_t batch, int32_t length, int32_t d,
                        int32_t dtype, const int32_t* pos, int64_t pos_stride, const float* table, int32_t table_rows,
                        int32_t rotary_dims, int32_t pairs, int32_t inverse, void* hip_stream);

/* The table of a2sf_rotary: row p holds magnitude * cos(p f_i), then magnitude * sin(p f_i), f_i = base^(-2 i /
 * rotary_dims) * (g + (1 - g) / factor), computed in 64 bits.
 * g, the share of a frequency that a longer context leaves as it is, is 0 for original_length = 0 (all positions are
 * divided by factor: linear scaling), else it grows from 0 to 1 where the turns that the pair makes over
 * original_length positions go from low to high. factor = 1: no scaling. */
a2sf_status a2sf_rotary_table(float* table, int32_t table_rows, int32_t rotary_dims, double base, double factor,
                              int32_t original_length, double low, double high, double magnitude, void* hip_stream);

/* One token of each row of logits.  The tokens of a row are ordered by logit, larger ones first, equal ones by index; the
 * filters keep, one after the other, the top_k first; of these the shortest prefix whose probabilities (softmax of
 * logit / temperature) reach top_p of their sum; of these the ones with at least min_p of the first one's probability.  The
 * first always stays.  Of what is left the token with the largest probability / noise is taken (the lower index where
 * equal): with exponential variates as noise, each with its probability.
 *   logits       [rows, n] dtype.  A NaN counts as -infinity and is never taken; where some are +infinity only those
 *                can be.  A row of -infinity: token -1, prob 0.
 *   noise        [rows, n] fp32, positive; NULL: the first token is taken.
 *   temperature  [rows] fp32, may be NULL (1); <= 0: the first token, whatever the filters.
 *   top_k        [rows] int32, may be NULL; <= 0 or >= n: all.
 *   top_p        [rows] fp32, may be NULL; >= 1: all.  Its sums are of whole numbers of 2^-41 of the first token's probability (for probabilities
 *                above 2^-10 of it: 2^-31), in 64 bits.
 *   min_p        [rows] fp32, may be NULL; <= 0: all.
 *   token        out [rows] int32.
 *   prob         out [rows] fp32, may be NULL: the token's probability among those that were left.
 * n <= A2SF_MAX_VOCABULARY. */
#define A2SF_MAX_VOCABULARY 4194304
a2sf_status a2sf_sample(const a2sf_rows* logits, const a2sf_rows* noise, int32_t rows, int32_t n, int32_t dtype,
                        const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                        int32_t* token, float* prob, void* hip_stream);

/* ---- Keys and values in pages -----------------------------------------------------------------------------------------
 * A cache that keeps every token (or, under a window, the newest and a few first ones) of sequences of different lengths that come and
 * go: the baseline without eviction, and the local one.  Keys and values lie in pages of page_size tokens; a table says which
 * page holds a sequence's tokens 0 .. page_size - 1, page_size .. 2 page_size - 1, and so on.  The conventions of the operators around
 * the attention hold.  At most 2^24 - 1 sequences and 2^28 - 1 tokens a call. */
typedef struct {
  void* k;                    /* page p, head h, token t of the page: d elements from p * stride[0] + h * stride[1] + t * stride[2] on */
  void* v;                    /* laid out as k */
  uint8_t* k_scales;          /* A2SF_E4M3: the scale of each token and head, a byte at p * scale_stride[0] + h * scale_stride[1] + t * */
  uint8_t* v_scales;          /*            scale_stride[2], as for a2sf_rows8.  Other types: NULL */
  int64_t stride[3];          /* elements; rows start at multiples of 16 bytes */
  int64_t scale_stride[3];    /* bytes */
  int32_t pages;
  int32_t page_size;          /* tokens, a power of two, at most 65536 */
  int32_t kv_heads;
  int32_t d;                  /* 64 or 128 */
  int32_t dtype;              /* that of the call's tensors, or A2SF_E4M3 (read as bf16 by bf16 calls of several tokens: scale bytes of 10 to 246) */
} a2sf_pages;

/* Which sequences a call is about, and which of its tokens are theirs. */
typedef struct {
  const int32_t* table;       /* [sequences, table_pages]: pages; an entry that no token of the call needs may be anything (-1) */
  const int32_t* len;         /* [sequences]: tokens of each sequence, the call's new ones among them */
  const int32_t* starts;      /* [sequences + 1]: sequence s has the call's tokens starts[s] .. starts[s + 1] - 1, its newest ones, in
                                 order.  NULL: token s is the newest of sequence s, and a sequence of length 0 is a place without one */
  int64_t table_stride;       /* entries from row to row */
  int32_t sequences;
  int32_t table_pages;
} a2sf_sequences;

typedef struct {
  void* data;                 /* [tokens, heads, d]; a head's elements are next to each other */
  int64_t stride[2];          /* elements from token to token, head to head */
} a2sf_heads;

/* A sequence is bad if its length is negative or more than table_pages * page_size, or if it has a negative number of new tokens or more
 * of them than tokens.  Starts do not fall and lie in 0 .. the call's tokens; where two of them fall, their sequence is bad, and rows of others may
 * be left alone.  Tokens of the call that no sequence has are left alone: nothing is written for them. */

/* New tokens: their keys and values go to their sequences' pages, k and q turned by their positions (a token's place in its sequence) on
 * the way, as a2sf_rotary turns them.
 *   q, q_out    [tokens, heads, d] dtype, both or neither; q_out may be q with the same strides.
 *   k, v        [tokens, cache->kv_heads, d] dtype.  What turning gives is rounded once, to the pages' type.
 *   dtype       A2SF_F32 or A2SF_BF16.
 *   table       [table_rows, rotary_dims] fp32 as a2sf_rotary takes it; NULL: nothing is turned.  A token whose position is no row of
 *               the table has NaN in the rotary_dims of q and k (pages of 8 bits: in all of k).
 * A token of a bad sequence, or one whose page is none of the cache's, leaves the cache alone and has NaN for its row of q_out.
 * starts NULL: a place without a sequence (length 0) leaves q_out as it is.  A page that two sequences share is not
 * written by both in one call. */
a2sf_status a2sf_paged_append(const a2sf_heads* q, const a2sf_heads* k, const a2sf_heads* v, int32_t tokens, int32_t heads,
                              int32_t dtype, const a2sf_sequences* sequences, const a2sf_pages* cache, const float* table,
                              int32_t table_rows, int32_t rotary_dims, int32_t pairs, const a2sf_heads* q_out,
                              void* hip_stream);

/* Attention of each sequence's newest tokens (already appended) over its pages: o_i = sum_j softmax_j(q_i . k_j / sqrt(d)) v_j over the
 * tokens j that token i sees: j <= i, and j > i - window or j < sinks (the window counts the token itself).
 *   q          [tokens, heads, d] dtype, heads a multiple of cache->kv_heads: query head h reads K/V head h / (heads / kv_heads).
 *   dtype      A2SF_F32 or A2SF_BF16.  Logits, maxima and sums are in 32 bits.  What a probability p is multiplied with v as: of fp32 calls 32
 *              bits; of bf16 calls without starts two bf16 numbers, within 2^-17 p; of bf16 calls with starts one, within 2^-8 p (so o is
 *              within 2^-8 sum p |v| before it is rounded to bf16), or with A2SF_BF16 | A2SF_WIDE_SUMS two (1.1 to 1.3 times the time).
 *   window     >= 1; A2SF_NO_WINDOW: every earlier token.
 *   sinks      >= 0: first tokens that stay visible.
 *   o          out [tokens, heads, d] dtype.  NaN for a bad sequence, and for a token that sees one whose page is none of the cache's;
 *              0 for a place without a sequence.  An infinity or NaN in a row of v reaches the tokens that see it alone, as one or the other.
 *   workspace  may be NULL; with a2sf_paged_workspace_bytes() bytes calls of few rows split their tokens over more of the chip, with less into
 *              fewer parts, and single tokens of up to 512 sequences, some of which may be much longer than others (by the size of the table), share
 *              it evenly.  The same sizes with the same workspace give the same bits.
 * What the table names for tokens that none of the call's sees does not matter, nor what lies there. */
#define A2SF_NO_WINDOW 0x7FFFFFFF
a2sf_status a2sf_paged_attention(const a2sf_heads* q, int32_t tokens, int32_t heads, int32_t dtype, const a2sf_sequences* sequences,
                                 const a2sf_pages* cache, int32_t window, int32_t sinks, const a2sf_heads* o, void* workspace,
                                 size_t workspace_bytes, void* hip_stream);
/* The most that a call of these sizes makes use of, whatever its window (0: nothing, or the sizes are wrong).
 *   table_tokens  table_pages * page_size. */
size_t a2sf_paged_workspace_bytes(int32_t tokens, int32_t heads, int32_t kv_heads, int32_t d, int32_t sequences, int64_t table_tokens);

/* What a row of logits says of given tokens, with y = logit - max, Z = sum exp(y): log p = y - log(Z), the entropy
 * log(Z) - sum(exp(y) y) / Z, and the tokens of the largest logits (equal ones: the lower index first).
 *   logits      [rows, n] dtype.  -infinity has probability 0.  A row with a NaN or +infinity, or of -infinity alone, has NaN for all
 *               its values; among its alternatives a NaN counts as -infinity.
 *   tokens      [rows, given] int32; NULL with given = 0.  A token outside 0 .. n - 1 has NaN.
 *   logp        out [rows, given] fp32.
 *   entropy     out [rows] fp32, may be NULL.
 *   top         out [rows, alternatives] fp32: their log p, falling; may be NULL.
 *   top_tokens  out [rows, alternatives] int32; may be NULL.
 * n <= A2SF_MAX_VOCABULARY, alternatives <= n and <= A2SF_MAX_ALTERNATIVES, 0 without top and top_tokens. */
#define A2SF_MAX_ALTERNATIVES 64
a2sf_status a2sf_log_probs(const a2sf_rows* logits, int32_t rows, int32_t n, int32_t dtype, const a2sf_rows* tokens, int32_t given,
                           const a2sf_rows* logp, float* entropy, const a2sf_rows* top, const a2sf_rows* top_tokens,
                           int32_t alternatives, void* hip_stream);

const char* a2sf_status_string(int32_t status);

#ifdef __cplusplus
}
#endif
#endif /* A2SF_H */
