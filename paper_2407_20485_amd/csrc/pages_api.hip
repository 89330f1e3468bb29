// C-ABI entry points of keys and values in pages and of log probabilities: argument validation on the host, then one launch
// function each.
#include <math.h>
#include <stdint.h>

#include "a2sf_internal.h"

using namespace a2sf;

namespace {

inline bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
inline uintptr_t size_of(int32_t dtype) { return dtype == A2SF_F32 ? 4 : dtype == A2SF_BF16 ? 2 : 1; }

#define A2SF_TRY(call)                                   \
  do {                                                   \
    const a2sf_status status_ = (call);                  \
    if (status_ != A2SF_OK) return status_;              \
  } while (0)

a2sf_status check_heads(const a2sf_heads* x, int tokens, int heads, int d, int32_t dtype) {
  if (!x || !x->data || misaligned(x->data, size_of(dtype))) return A2SF_EINVAL;
  if (heads < 1 || heads > 0xFFFF) return A2SF_ESHAPE;
  if ((tokens > 1 && x->stride[0] < d) || (heads > 1 && x->stride[1] < d)) return A2SF_ESHAPE;
  return A2SF_OK;
}

a2sf_status check_pages(const a2sf_pages* c, int32_t dtype) {
  if (!c) return A2SF_EINVAL;
  if (dtype != A2SF_F32 && dtype != A2SF_BF16) return A2SF_EDTYPE;
  if (c->dtype != dtype && c->dtype != A2SF_E4M3) return A2SF_EDTYPE;
  if (!c->k || !c->v || misaligned(c->k, 16) || misaligned(c->v, 16)) return A2SF_EINVAL;
  if ((c->dtype == A2SF_E4M3) != (c->k_scales != nullptr) || (c->dtype == A2SF_E4M3) != (c->v_scales != nullptr)) return A2SF_EINVAL;
  if ((c->d != 64 && c->d != 128) || c->pages < 1 || c->kv_heads < 1 || c->kv_heads > 0xFFFF) return A2SF_ESHAPE;
  if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)) != 0) return A2SF_ESHAPE;
  const int32_t counts[3] = {c->pages, c->kv_heads, c->page_size};
  const int64_t unit = 16 / (int64_t)size_of(c->dtype);
  for (int i = 0; i < 3; ++i) {
    if (counts[i] == 1) continue;  // not looked at
    if (c->stride[i] < c->d || c->stride[i] % unit != 0 || c->stride[i] > (int64_t)1 << 44) return A2SF_ESHAPE;
    if (c->dtype == A2SF_E4M3 && (c->scale_stride[i] < 1 || c->scale_stride[i] > (int64_t)1 << 44)) return A2SF_ESHAPE;
  }
  return A2SF_OK;
}

a2sf_status check_sequences(const a2sf_sequences* s, int32_t tokens, const a2sf_pages* c) {
  if (!s || !s->table || !s->len || misaligned(s->table, 4) || misaligned(s->len, 4) || misaligned(s->starts, 4)) return A2SF_EINVAL;
  if (s->sequences < 1 || s->sequences > 0xFFFFFF || tokens < 1 || tokens > 0xFFFFFFF || s->table_pages < 1) return A2SF_ESHAPE;
  if (!s->starts && tokens != s->sequences) return A2SF_ESHAPE;
  if (s->sequences > 1 && s->table_stride < s->table_pages) return A2SF_ESHAPE;
  // positions have 32 bits
  if ((long long)s->table_pages * c->page_size > 0x7FFFFFFFLL - 256) return A2SF_ESHAPE;
  return A2SF_OK;
}

PagedCache paged(const a2sf_pages* c, const a2sf_sequences* s, int32_t tokens) {
  PagedCache p;
  const long long e = (long long)size_of(c->dtype);
  const int32_t counts[3] = {c->pages, c->kv_heads, c->page_size};
  p.k = (char*)c->k;
  p.v = (char*)c->v;
  p.k_scales = c->k_scales;
  p.v_scales = c->v_scales;
  for (int i = 0; i < 3; ++i) {
    p.stride[i] = counts[i] == 1 ? 0 : c->stride[i] * e;
    p.scale_stride[i] = counts[i] == 1 ? 0 : c->scale_stride[i];
  }
  p.table = s->table;
  p.len = s->len;
  p.starts = s->starts;
  p.table_stride = s->table_stride;
  p.sequences = s->sequences;
  p.table_pages = s->table_pages;
  p.pages = c->pages;
  p.shift = __builtin_ctz((unsigned)c->page_size);
  p.kv_heads = c->kv_heads;
  p.d = c->d;
  p.dtype = c->dtype;
  p.tokens = tokens;
  return p;
}

// (an error that an unrelated earlier call left on this thread is not this call's)
template <typename F>
a2sf_status launched(F launch) {
  (void)hipGetLastError();
  if (!launch()) return A2SF_ESHAPE;
  return hipGetLastError() == hipSuccess ? A2SF_OK : A2SF_EHIP;
}

// [rows, n] of 4-byte elements
a2sf_status check_rows4(const a2sf_rows* r, int rows, int n) {
  if (!r->data || misaligned(r->data, 4)) return A2SF_EINVAL;
  return rows > 1 && r->stride < n ? A2SF_ESHAPE : A2SF_OK;
}

}  // namespace

extern "C" {

a2sf_status a2sf_paged_append(const a2sf_heads* q, const a2sf_heads* k, const a2sf_heads* v, int32_t tokens, int32_t heads,
                              int32_t dtype, const a2sf_sequences* sequences, const a2sf_pages* cache, const float* table,
                              int32_t table_rows, int32_t rotary_dims, int32_t pairs, const a2sf_heads* q_out, void* hip_stream) {
  A2SF_TRY(check_pages(cache, dtype));
  A2SF_TRY(check_sequences(sequences, tokens, cache));
  const int d = cache->d;
  A2SF_TRY(check_heads(k, tokens, cache->kv_heads, d, dtype));
  A2SF_TRY(check_heads(v, tokens, cache->kv_heads, d, dtype));
  if ((q == nullptr) != (q_out == nullptr)) return A2SF_EINVAL;
  if (q) {
    A2SF_TRY(check_heads(q, tokens, heads, d, dtype));
    A2SF_TRY(check_heads(q_out, tokens, heads, d, dtype));
    if (q->data == q_out->data && ((tokens > 1 && q->stride[0] != q_out->stride[0]) || (heads > 1 && q->stride[1] != q_out->stride[1])))
      return A2SF_EINVAL;  // elements would be overwritten before they are read
  }
  if (table) {
    if (misaligned(table, 4) || (pairs != A2SF_ROTARY_HALVES && pairs != A2SF_ROTARY_NEIGHBOURS)) return A2SF_EINVAL;
    if (table_rows < 1 || rotary_dims < 2 || rotary_dims % 2 != 0 || rotary_dims > d) return A2SF_ESHAPE;
  }
  AppendArgs a = {};
  a.c = paged(cache, sequences, tokens);
  a.q = q ? q->data : nullptr;
  a.q_out = q ? q_out->data : nullptr;
  a.k = k->data;
  a.v = v->data;
  for (int i = 0; i < 2; ++i) {
    a.q_stride[i] = q ? q->stride[i] : 0;
    a.q_out_stride[i] = q ? q_out->stride[i] : 0;
    a.k_stride[i] = k->stride[i];
    a.v_stride[i] = v->stride[i];
  }
  a.heads = q ? heads : 0;
  a.table = table;
  a.table_rows = table ? table_rows : 0;
  a.rot = table ? rotary_dims : 0;
  return launched([&] { return launch_paged_append(a, dtype, table && pairs == A2SF_ROTARY_NEIGHBOURS, (hipStream_t)hip_stream); });
}

a2sf_status a2sf_paged_attention(const a2sf_heads* q, int32_t tokens, int32_t heads, int32_t dtype, const a2sf_sequences* sequences,
                                 const a2sf_pages* cache, int32_t window, int32_t sinks, const a2sf_heads* o, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  const bool wide = (dtype & A2SF_WIDE_SUMS) != 0;
  dtype &= ~A2SF_WIDE_SUMS;
  A2SF_TRY(check_pages(cache, dtype));
  A2SF_TRY(check_sequences(sequences, tokens, cache));
  A2SF_TRY(check_heads(q, tokens, heads, cache->d, dtype));
  A2SF_TRY(check_heads(o, tokens, heads, cache->d, dtype));
  if (heads % cache->kv_heads != 0) return A2SF_ESHAPE;
  if ((long long)tokens * heads > 0x7FFFFFFFLL) return A2SF_ESHAPE;
  if (window < 1 || sinks < 0 || q->data == o->data) return A2SF_EINVAL;
  if (misaligned(workspace, 16)) return A2SF_EWORKSPACE;
  PagedArgs a = {};
  a.c = paged(cache, sequences, tokens);
  a.q = q->data;
  a.o = o->data;
  for (int i = 0; i < 2; ++i) {
    a.q_stride[i] = q->stride[i];
    a.o_stride[i] = o->stride[i];
  }
  a.heads = heads;
  a.group = heads / cache->kv_heads;
  a.window = window;
  a.sinks = sinks;
  a.wide = wide;
  a.scale_log2e = 1.44269504088896340736f / sqrtf((float)cache->d);
  return launched([&] { return launch_paged_attention(a, dtype, workspace, workspace ? workspace_bytes : 0, (hipStream_t)hip_stream); });
}

size_t a2sf_paged_workspace_bytes(int32_t tokens, int32_t heads, int32_t kv_heads, int32_t d, int32_t sequences, int64_t table_tokens) {
  if (tokens < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads != 0 || (d != 64 && d != 128) || sequences < 1 || table_tokens < 1 ||
      (long long)tokens * heads > 0x7FFFFFFFLL)
    return 0;
  return paged_workspace(tokens, heads, kv_heads, d, sequences, table_tokens);
}

a2sf_status a2sf_log_probs(const a2sf_rows* logits, int32_t rows, int32_t n, int32_t dtype, const a2sf_rows* tokens, int32_t given,
                           const a2sf_rows* logp, float* entropy, const a2sf_rows* top, const a2sf_rows* top_tokens,
                           int32_t alternatives, void* hip_stream) {
  if (dtype != A2SF_F32 && dtype != A2SF_BF16) return A2SF_EDTYPE;
  if (rows < 1 || n < 1 || n > A2SF_MAX_VOCABULARY || given < 0 || alternatives < 0 || alternatives > A2SF_MAX_ALTERNATIVES ||
      alternatives > n)
    return A2SF_ESHAPE;
  if (!logits || !logits->data || misaligned(logits->data, size_of(dtype))) return A2SF_EINVAL;
  if (rows > 1 && logits->stride < n) return A2SF_ESHAPE;
  if ((given > 0) != (tokens != nullptr) || (given > 0) != (logp != nullptr)) return A2SF_EINVAL;
  if ((alternatives > 0) != (top || top_tokens)) return A2SF_EINVAL;
  if (!(given > 0 || entropy || alternatives > 0) || misaligned(entropy, 4)) return A2SF_EINVAL;
  if (given > 0) {
    A2SF_TRY(check_rows4(tokens, rows, given));
    A2SF_TRY(check_rows4(logp, rows, given));
  }
  if (top) A2SF_TRY(check_rows4(top, rows, alternatives));
  if (top_tokens) A2SF_TRY(check_rows4(top_tokens, rows, alternatives));
  LogProbsArgs a = {};
  a.logits = logits->data;
  a.stride = logits->stride;
  if (given > 0) {
    a.tokens = (const int32_t*)tokens->data;
    a.token_stride = tokens->stride;
    a.logp = (float*)logp->data;
    a.logp_stride = logp->stride;
  }
  if (top) {
    a.top = (float*)top->data;
    a.top_stride = top->stride;
  }
  if (top_tokens) {
    a.top_tokens = (int32_t*)top_tokens->data;
    a.top_token_stride = top_tokens->stride;
  }
  a.entropy = entropy;
  a.rows = rows;
  a.n = n;
  a.given = given;
  a.alternatives = alternatives;
  return launched([&] { return launch_log_probs(a, dtype, (hipStream_t)hip_stream); });
}

}  // extern "C"
