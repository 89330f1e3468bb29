// Host-side launch functions of the kernel files, called by the C-ABI entry points.
// Every launcher only enqueues on `st`; shapes have been validated by the caller.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/a2sf.h"

namespace a2sf {

// select_compact.hip
void launch_select(const float* scores, const int32_t* pos, const int32_t* len, int G, int L,
                   int stride, int select, int recent, int32_t* keep_idx, int32_t* n_keep,
                   hipStream_t st);
// k2 / v2 [G, m2, d] set: the rows of the slots from off_heads[g] on are taken from there
// (a chunk whose rows were not copied into the cache); heads with a negative entry there are left alone
void launch_compact(const a2sf_cache& c, const int32_t* keep_idx, int keep_stride,
                    const int32_t* n_keep, hipStream_t st, const void* k2 = nullptr,
                    const void* v2 = nullptr, int m2 = 0, const int32_t* off_heads = nullptr,
                    bool mostly_done = false);  // hardly a head has rows to move
// Selection on the cache's scores and compaction in one kernel, for budgets it takes (selects_in_place).  k2 / v2 [G, m2, d]
// set: every head's last m2 tokens, still to be counted into its length, have their rows there; a head that has
// no room for them is left alone.  off_heads (may be null): heads with a negative entry are left alone.
bool selects_in_place(const a2sf_cache& c, int select, int recent, bool appends);
void launch_select_compact(const a2sf_cache& c, int select, int recent, hipStream_t st, const void* k2 = nullptr,
                           const void* v2 = nullptr, int m2 = 0, const int32_t* off_heads = nullptr);
// Selection on a prompt's scores [G, n] and gather of the surviving rows into the cache.
void launch_select_gather(const void* k, const void* v, const float* scores_full, int n, int select,
                          int recent, int32_t* keep_idx, int32_t* n_keep, const a2sf_cache& c,
                          hipStream_t st);

// decode.hip
struct DecodePlan {
  int nsplit;          // workgroups per head (1 = single fused kernel)
  int rows_per_split;  // multiple of 64
  int wave_slots;      // > 0: wave-per-head kernel holding 64*wave_slots slots in registers
  bool loop;           // wave-per-head path, fast mode: persistent workgroups, a wave works through several heads
  int wave_heads;      // ... that many (1 otherwise)
  bool small;          // one large workgroup per head, all rows in registers; does the stable eviction itself
  bool stream;         // single-kernel paths: load the cache rows with the non-temporal hint
  size_t ws_bytes;     // split-K scratch
};
DecodePlan plan_decode(int G, int capacity, int d);
bool decode_small(int G, int capacity, int d, int dtype, bool stable);  // whether DecodePlan::small applies
void launch_decode(const void* q, const void* k_new, const void* v_new, int t_pos,
                   const a2sf_cache& c, float alpha, const float* alpha_heads, int select,
                   int recent, bool evict_here, void* o, void* ws, const DecodePlan& plan,
                   hipStream_t st);

// Generation step of G K/V heads with `group` (2 .. 8) query heads each: q, o are
// [G, group, d]; group * capacity floats of LDS per workgroup.  ws (may be null) / ws_bytes:
// scratch memory for the token-split form that few K/V heads with long caches take.
void launch_decode_gqa(const void* q, const void* k_new, const void* v_new, int t_pos,
                       const a2sf_cache& c, int group, float alpha, int select, int recent,
                       bool evict_here, void* o, void* ws, size_t ws_bytes, hipStream_t st);

// chunk.hip: the chunk's K/V rows go behind each head's cached tokens (len grows by m, the old
// lengths are left in len_old, -1 where the chunk does not fit)
void launch_chunk_append(const void* k, const void* v, int m, int pos0, const a2sf_cache& c,
                         int32_t* len_old, bool copy_rows, hipStream_t st);

// similarity.hip: cosine between the policy's attention row (cache positions + the new token)
// and the Ideal row over the first L rows of k_all, per head.
void launch_ideal_similarity(const void* q, const void* k_all, int n_stride, int L,
                             const a2sf_cache& c, float* out, hipStream_t st);

void launch_similarity_mean(const float* cos, long long begin, long long end, float* out,
                            hipStream_t st);

// Geometry of one attention call: m query rows per head against keys that lie kv_stride rows
// apart from head to head; row i sees keys 0 .. off + i.  The prompt phase is the square case
// (off = 0, kv_stride = m); a chunk of a prompt runs against the head's cache, off = the tokens
// cached before the chunk (a head with off_heads[g] < 0, or without room for m more, is skipped).
// kv_group > 1: grouped-query heads.  The attention kernels then run over G * kv_group query
// heads, query head g reading the K/V rows of head g / kv_group; the column-score kernels run
// over the G K/V heads and sum the scores of each head's kv_group query heads.
struct AttnRect {
  int m;
  int kv_stride;
  const int32_t* off_heads;  // [G] device, or null: 0 for every head
  int kv_group = 1;
  // Second source of key / value rows (bf16 only): when set, a head's
  // keys 0 .. off-1 are rows of k / v and its keys off .. off+m-1 are the m rows [G, m, d] of
  // k2 / v2 -- a chunk whose rows have not been copied behind the cached ones.
  const void* k2 = nullptr;
  const void* v2 = nullptr;
  // Column scores with two sources: the positions pos0 + i of the keys off + i are written here, [G, kv_stride]
  int32_t* pos = nullptr;
  int pos0 = 0;
  // Calls without outputs: the log-sum-exp of the rows before first_row is not needed (the score
  // kernel that follows skips them), so their row blocks are not computed.
  int first_row = 0;
};
// prefill_f32.hip / prefill_bf16.hip
// lse2[g][i] = log2(sum_j exp(s_ij)) of the masked row i (s already scaled by 1/sqrt(d)).
void launch_prefill_f32(const float* q, const float* k, const float* v, int G, int n, int d,
                        float* o, float* lse2, hipStream_t st, int first_row = 0);
// First prompt row whose log-sum-exp the fp32 score kernel uses.
int f32_first_lse_row(int n, float alpha_max);
// alpha_heads (device [G]) may be null: then every head uses `alpha`; otherwise `alpha` is an
// upper bound of the per-head factors.
void launch_scores_f32(const float* q, const float* k, const float* lse2, int G, int n, int d,
                       float alpha, const float* alpha_heads, float* scores, hipStream_t st);
// The general (rectangular) forms, used for chunks of a prompt.  keys_per_head: upper bound of
// off + m over the heads (the grid is sized by it).  accumulate: the new column sums are added
// to decay * scores[] (the cached tokens' older scores) instead of replacing it.
void launch_attn_f32(const float* q, const float* k, const float* v, int G, const AttnRect& rc,
                     int d, float* o, float* lse2, hipStream_t st);
void launch_colscores_f32(const float* q, const float* k, const float* lse2, int G,
                          const AttnRect& rc, int keys_per_head, int d, float alpha,
                          const float* alpha_heads, float* scores, int s_stride, bool accumulate,
                          float decay, hipStream_t st);
void launch_attn_bf16(const void* q, const void* k, const void* v, int G, const AttnRect& rc, int d,
                      void* o, float* lse2, hipStream_t st);
void launch_colscores_bf16(const void* q, const void* k, const float* lse2, int G,
                           const AttnRect& rc, int keys_per_head, int d, float alpha, float* scores,
                           int s_stride, bool accumulate, float decay, hipStream_t st);
// Column scores, selection and moves in one kernel, where scores_select_fits (a prompt's score tolerance is not used): a prompt
// (square rc, into the empty cache; scores_full may be null) or, with rc.k2, a chunk (in place; `decay` as above).
bool scores_select_fits(int G, const AttnRect& rc, int keys_per_head, float alpha);
void launch_scores_select_bf16(const void* q, const void* k, const void* v, const float* lse2, const AttnRect& rc,
                               int keys_per_head, float alpha, const float* alpha_heads, float decay, float* scores_full,
                               int select, int recent, const a2sf_cache& c, hipStream_t st);
// first_row > 0 (only with o == null): rows before it need no log-sum-exp
void launch_prefill_bf16(const void* q, const void* k, const void* v, int G, int n, int d,
                         void* o, float* lse2, hipStream_t st, int first_row = 0);
// First prompt row whose log-sum-exp launch_scores_bf16 reads for these sizes (Section 3.3: the
// forgetting factor takes older rows' contributions to 0; exactly 0 in fp32 before that row).
int bf16_first_lse_row(int n, float alpha_max);
// tol > 0 (d = 128 only): rows whose whole remaining contribution is provably below tol * S_j
// are skipped (see RowWindow in prefill_bf16.hip); tol = 0 computes every row of nonzero weight.
void launch_scores_bf16(const void* q, const void* k, const float* lse2, int G, int n, int d,
                        float alpha, const float* alpha_heads, float tol, float* scores,
                        hipStream_t st);

// Rows i < first_row contribute exactly 0 to every fp32 score (their weight alpha^(n-1-i)
// is below the smallest fp32 subnormal while P <= 1), so the score kernels skip them.
// Also returns log2(alpha) as used in the exponent (0 for alpha == 0, whose only row is n-1).
int first_contributing_row(int n, float alpha, float* log2_alpha);

// ---- the operators around the attention ------------------------------------------------------------------------------------
// A launch's lanes are counted in 32 bits: false, and nothing launched, where a call would take more.
inline bool grid_fits(unsigned long long groups, unsigned lanes) { return groups * lanes <= 0xFFFFFFFFull; }
// rows.hip.  Strides in elements (8-bit rows and scales: bytes); absent tensors are null.
struct NormArgs {
  const void *x, *residual, *weight;
  void *total, *out;
  uint8_t *q, *scales;
  long long x_stride, residual_stride, total_stride, out_stride, q_stride, scale_stride;
  float eps;
  int rows, n;
};
bool launch_rms_norm(const NormArgs& a, int dtype, hipStream_t st);
struct QuantArgs {
  const void *x, *gate;
  void* out;
  uint8_t *q, *scales;
  long long x_stride, gate_stride, out_stride, q_stride, scale_stride;
  int rows, n, blocks_per_row;
};
bool launch_quantize(const QuantArgs& a, int dtype, hipStream_t st);
bool launch_quantize_weight(const QuantArgs& a, int dtype, hipStream_t st);

// matmul.hip: C[m, n] = A[m, k] B[n, k]^T
struct MatmulArgs {
  const uint8_t *a, *a_scales, *b, *b_scales;
  void* c;
  long long a_stride, a_scale_stride, b_stride, b_scale_stride, c_stride;
  int m, n, k;
};
size_t matmul_workspace(int m, int n, int k);
// wide_sums: a bf16 C too is summed in 32 bits
void launch_matmul(const MatmulArgs& a, int dtype, bool wide_sums, void* workspace, size_t workspace_bytes, hipStream_t st);

// rotary.hip
struct RotaryPart {
  const void* x;
  void* y;
  long long x_stride[3], y_stride[3];  // batch, position, head
  int heads, rotate, in_place;
  int lanes, tokens_per_block;  // set by the launcher
};
struct RotaryArgs {
  RotaryPart part[A2SF_MAX_ROTARY_PARTS];
  int parts, batch, length, d, rot, inverse;
  const int32_t* pos;
  long long pos_stride;
  const float* table;
  int table_rows;
  // set by the launcher
  int turning, items;
  uint32_t first_block[A2SF_MAX_ROTARY_PARTS];
};
bool launch_rotary(RotaryArgs a, int dtype, bool neighbours, hipStream_t st);
struct RotaryTableArgs {
  float* table;
  int rows, rot, original_length;
  double base, factor, low, high, magnitude;
};
void launch_rotary_table(const RotaryTableArgs& a, hipStream_t st);

// sample.hip
struct SampleArgs {
  const void* logits;
  const float* noise;
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* prob;
  long long stride, noise_stride;
  int rows, n;
};
bool launch_sample(const SampleArgs& a, int dtype, hipStream_t st);

// logprobs.hip
struct LogProbsArgs {
  const void* logits;
  const int32_t* tokens;
  float *logp, *entropy, *top;
  int32_t* top_tokens;
  long long stride, token_stride, logp_stride, top_stride, top_token_stride;
  int rows, n, given, alternatives;
};
bool launch_log_probs(const LogProbsArgs& a, int dtype, hipStream_t st);

// ---- keys and values in pages ----------------------------------------------------------------------------------------------
// The cache and the sequences of a call as the kernels take them: strides in bytes, page_size = 2^shift.
struct PagedCache {
  char *k, *v;
  uint8_t *k_scales, *v_scales;
  long long stride[3], scale_stride[3];
  const int32_t *table, *len, *starts;
  long long table_stride;
  int sequences, table_pages, pages, shift, kv_heads, d, dtype;
  int tokens;  // of the call
};
// paged_append.hip
struct AppendArgs {
  PagedCache c;
  const void *q, *k, *v;
  void* q_out;
  long long q_stride[2], k_stride[2], v_stride[2], q_out_stride[2];
  const float* table;
  int heads, table_rows, rot;
  int per_lane, groups;  // set by the launcher
};
bool launch_paged_append(AppendArgs a, int dtype, bool neighbours, hipStream_t st);
// paged_attention.hip
struct PagedArgs {
  PagedCache c;
  const void* q;
  void* o;
  long long q_stride[2], o_stride[2];
  int heads, group, window, sinks;
  bool wide;  // probabilities as two bf16 numbers in the tile form too
  float scale_log2e;
  // set by the launcher
  float *part, *part_ml;  // sums of parts of rows, their maxima and weights: [rows][splits] (a row is a (token, head)) or [even][2][part_rows]
  int splits, blocks, blocks_per;  // blocks of rows: of the call, of a sequence (one token each)
  int even, part_rows;             // workgroups that share the tokens evenly (one token each), or 0
};
size_t paged_workspace(int tokens, int heads, int kv_heads, int d, int sequences, long long table_tokens);
bool launch_paged_attention(PagedArgs a, int dtype, void* workspace, size_t workspace_bytes, hipStream_t st);

}  // namespace a2sf
