// C-ABI entry points of the operators around the attention: argument validation on the host, then one launch
// function each.
#include <math.h>
#include <stdint.h>

#include "a2sf_internal.h"

using namespace a2sf;

namespace {

inline bool misaligned(const void* p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }
inline int blocks(int n) { return n / 128 + (n % 128 != 0); }

a2sf_status check_sizes(int32_t rows, int32_t n, int32_t dtype) {
  if (dtype != A2SF_F32 && dtype != A2SF_BF16) return A2SF_EDTYPE;
  if (rows < 1 || n < 1) return A2SF_ESHAPE;
  if ((long long)rows * blocks(n) > 0x7FFFFFFFLL) return A2SF_ESHAPE;
  return A2SF_OK;
}
// Rows may be views that start inside a tensor: aligned to their elements.  `wanted`: may not be absent
inline uintptr_t size_of(int32_t dtype) { return dtype == A2SF_F32 ? 4 : 2; }
a2sf_status check_rows(const a2sf_rows* r, int rows, int n, int32_t dtype, bool wanted) {
  if (!r) return wanted ? A2SF_EINVAL : A2SF_OK;
  if (!r->data || misaligned(r->data, size_of(dtype))) return A2SF_EINVAL;
  if (rows > 1 && r->stride < n) return A2SF_ESHAPE;
  return A2SF_OK;
}
a2sf_status check_rows8(const a2sf_rows8* r, int rows, int scale_rows, int n, bool wanted) {
  if (!r) return wanted ? A2SF_EINVAL : A2SF_OK;
  if (!r->data || !r->scales || misaligned(r->data) || misaligned(r->scales, 4)) return A2SF_EINVAL;
  if (rows > 1 && (r->stride < n || r->stride % 16 != 0)) return A2SF_ESHAPE;
  if (scale_rows > 1 && (r->scale_stride < blocks(n) || r->scale_stride % 4 != 0)) return A2SF_ESHAPE;
  return A2SF_OK;
}
template <typename R>
auto data(const R* r) { return r ? r->data : nullptr; }
template <typename R>
long long stride(const R* r) { return r ? (long long)r->stride : 0; }

#define A2SF_TRY(call)                                   \
  do {                                                   \
    const a2sf_status status_ = (call);                  \
    if (status_ != A2SF_OK) return status_;              \
  } while (0)

// (an error that an unrelated earlier call left on this thread is not this call's)
template <typename F>
a2sf_status launched(F launch) {
  (void)hipGetLastError();
  if (!launch()) return A2SF_ESHAPE;
  return hipGetLastError() == hipSuccess ? A2SF_OK : A2SF_EHIP;
}

}  // namespace

extern "C" {

a2sf_status a2sf_rms_norm(const a2sf_rows* x, const a2sf_rows* residual, const void* weight, float eps, int32_t rows,
                          int32_t n, int32_t dtype, const a2sf_rows* total, const a2sf_rows* out,
                          const a2sf_rows8* out8, void* hip_stream) {
  A2SF_TRY(check_sizes(rows, n, dtype));
  if (n > A2SF_MAX_ROW) return A2SF_ESHAPE;
  A2SF_TRY(check_rows(x, rows, n, dtype, true));
  A2SF_TRY(check_rows(residual, rows, n, dtype, false));
  A2SF_TRY(check_rows(total, rows, n, dtype, false));
  A2SF_TRY(check_rows(out, rows, n, dtype, !out8));
  A2SF_TRY(check_rows8(out8, rows, rows, n, false));
  if (!weight || misaligned(weight, size_of(dtype)) || !(eps >= 0.f) || !isfinite(eps)) return A2SF_EINVAL;
  NormArgs a;
  a.x = x->data;
  a.residual = data(residual);
  a.weight = weight;
  a.total = data(total);
  a.out = data(out);
  a.q = (uint8_t*)data(out8);
  a.scales = out8 ? out8->scales : nullptr;
  a.x_stride = stride(x);
  a.residual_stride = stride(residual);
  a.total_stride = stride(total);
  a.out_stride = stride(out);
  a.q_stride = stride(out8);
  a.scale_stride = out8 ? out8->scale_stride : 0;
  a.eps = eps;
  a.rows = rows;
  a.n = n;
  return launched([&] { return launch_rms_norm(a, dtype, (hipStream_t)hip_stream); });
}

a2sf_status a2sf_quantize(const a2sf_rows* x, const a2sf_rows* gate, int32_t rows, int32_t n, int32_t dtype,
                          const a2sf_rows* out, const a2sf_rows8* out8, void* hip_stream) {
  A2SF_TRY(check_sizes(rows, n, dtype));
  A2SF_TRY(check_rows(x, rows, n, dtype, true));
  A2SF_TRY(check_rows(gate, rows, n, dtype, false));
  A2SF_TRY(check_rows(out, rows, n, dtype, !out8));
  A2SF_TRY(check_rows8(out8, rows, rows, n, false));
  QuantArgs a;
  a.x = x->data;
  a.gate = data(gate);
  a.out = data(out);
  a.q = (uint8_t*)data(out8);
  a.scales = out8 ? out8->scales : nullptr;
  a.x_stride = stride(x);
  a.gate_stride = stride(gate);
  a.out_stride = stride(out);
  a.q_stride = stride(out8);
  a.scale_stride = out8 ? out8->scale_stride : 0;
  a.rows = rows;
  a.n = n;
  a.blocks_per_row = blocks(n);
  return launched([&] { return launch_quantize(a, dtype, (hipStream_t)hip_stream); });
}

a2sf_status a2sf_quantize_weight(const a2sf_rows* w, int32_t n, int32_t k, int32_t dtype, const a2sf_rows8* out8,
                                 void* hip_stream) {
  A2SF_TRY(check_sizes(n, k, dtype));
  if (n > 0x7FFFFFFF - 128) return A2SF_ESHAPE;
  A2SF_TRY(check_rows(w, n, k, dtype, true));
  A2SF_TRY(check_rows8(out8, n, blocks(n), k, true));
  QuantArgs a;
  a.x = w->data;
  a.gate = nullptr;
  a.out = nullptr;
  a.q = (uint8_t*)out8->data;
  a.scales = out8->scales;
  a.x_stride = w->stride;
  a.gate_stride = a.out_stride = 0;
  a.q_stride = out8->stride;
  a.scale_stride = out8->scale_stride;
  a.rows = n;
  a.n = k;
  a.blocks_per_row = blocks(k);
  return launched([&] { return launch_quantize_weight(a, dtype, (hipStream_t)hip_stream); });
}

size_t a2sf_matmul_workspace_bytes(int32_t m, int32_t n, int32_t k) {
  return m < 1 || n < 1 || k < 1 || k > (1 << 20) ? 0 : matmul_workspace(m, n, k);
}

a2sf_status a2sf_matmul_scaled(const a2sf_rows8* a, const a2sf_rows8* b, int32_t m, int32_t n, int32_t k,
                               const a2sf_rows* c, int32_t c_dtype, void* workspace, size_t workspace_bytes,
                               void* hip_stream) {
  const bool wide_sums = (c_dtype & A2SF_WIDE_SUMS) != 0;
  c_dtype &= ~A2SF_WIDE_SUMS;
  A2SF_TRY(check_sizes(m, n, c_dtype));
  if (k < 1 || k > (1 << 20) || m > 0x7FFFFFFF - 256 || n > 0x7FFFFFFF - 256) return A2SF_ESHAPE;
  // tiles are counted in 32 bits, and a tile's 256 rows are addressed by 32-bit offsets
  if ((long long)blocks(m) * blocks(n) > 0x3FFFFFFFLL) return A2SF_ESHAPE;
  A2SF_TRY(check_rows8(a, m, m, k, true));
  A2SF_TRY(check_rows8(b, n, blocks(n), k, true));
  constexpr int64_t kFarthest = 1 << 23;
  if ((m > 1 && (a->stride > kFarthest || a->scale_stride > kFarthest)) || (n > 1 && b->stride > kFarthest) ||
      (n > 128 && b->scale_stride > kFarthest))
    return A2SF_ESHAPE;
  A2SF_TRY(check_rows(c, m, n, c_dtype, true));
  if (misaligned(workspace)) return A2SF_EWORKSPACE;
  MatmulArgs g;
  g.a = (const uint8_t*)a->data;
  g.a_scales = a->scales;
  g.b = (const uint8_t*)b->data;
  g.b_scales = b->scales;
  g.c = c->data;
  g.a_stride = m > 1 ? a->stride : 0;
  g.a_scale_stride = m > 1 ? a->scale_stride : 0;
  g.b_stride = n > 1 ? b->stride : 0;
  g.b_scale_stride = n > 128 ? b->scale_stride : 0;
  g.c_stride = c->stride;
  g.m = m;
  g.n = n;
  g.k = k;
  return launched([&] { return launch_matmul(g, c_dtype, wide_sums, workspace, workspace ? workspace_bytes : 0, (hipStream_t)hip_stream), true; });
}

a2sf_status a2sf_rotary(const a2sf_rotary_part* parts, int32_t n_parts, int32_t batch, int32_t length, int32_t d,
                        int32_t dtype, const int32_t* pos, int64_t pos_stride, const float* table, int32_t table_rows,
                        int32_t rotary_dims, int32_t pairs, int32_t inverse, void* hip_stream) {
  if (dtype != A2SF_F32 && dtype != A2SF_BF16) return A2SF_EDTYPE;
  if (!parts || n_parts < 1 || n_parts > A2SF_MAX_ROTARY_PARTS) return A2SF_EINVAL;
  if (pairs != A2SF_ROTARY_HALVES && pairs != A2SF_ROTARY_NEIGHBOURS) return A2SF_EINVAL;
  if (batch < 1 || length < 1 || d < 1 || d > 512 || table_rows < 1) return A2SF_ESHAPE;
  if (rotary_dims < 2 || rotary_dims % 2 != 0 || rotary_dims > d) return A2SF_ESHAPE;
  if ((long long)batch * length > 0x0FFFFFFFLL) return A2SF_ESHAPE;
  if (batch > 1 && pos_stride < length) return A2SF_ESHAPE;
  if (!pos || !table || misaligned(pos, 4) || misaligned(table, 4)) return A2SF_EINVAL;
  RotaryArgs a = {};
  for (int i = 0; i < n_parts; ++i) {
    const a2sf_rotary_part& p = parts[i];
    if (!p.x || !p.y || misaligned(p.x, size_of(dtype)) || misaligned(p.y, size_of(dtype))) return A2SF_EINVAL;
    if (p.heads < 1 || p.heads > 0xFFFFFF) return A2SF_ESHAPE;
    RotaryPart& to = a.part[i];
    to.x = p.x;
    to.y = p.y;
    to.heads = p.heads;
    to.in_place = p.x == p.y;
    to.rotate = p.rotate != 0;
    for (int j = 0; j < 3; ++j) {
      if (p.x_stride[j] < 0 || p.y_stride[j] < 0) return A2SF_ESHAPE;
      to.x_stride[j] = p.x_stride[j];
      to.y_stride[j] = p.y_stride[j];
      const int count = j == 0 ? batch : j == 1 ? length : p.heads;
      if (count > 1 && p.x_stride[j] != p.y_stride[j]) to.in_place = 0;
    }
    if (p.x == p.y && !to.in_place) return A2SF_EINVAL;  // elements would be overwritten before they are read
  }
  a.parts = n_parts;
  a.batch = batch;
  a.length = length;
  a.d = d;
  a.rot = rotary_dims;
  a.inverse = inverse != 0;
  a.pos = pos;
  a.pos_stride = pos_stride;
  a.table = table;
  a.table_rows = table_rows;
  return launched([&] { return launch_rotary(a, dtype, pairs == A2SF_ROTARY_NEIGHBOURS, (hipStream_t)hip_stream); });
}

a2sf_status a2sf_rotary_table(float* table, int32_t table_rows, int32_t rotary_dims, double base, double factor,
                              int32_t original_length, double low, double high, double magnitude, void* hip_stream) {
  if (!table || misaligned(table, 4)) return A2SF_EINVAL;
  if (table_rows < 1 || rotary_dims < 2 || rotary_dims % 2 != 0 || rotary_dims > 512) return A2SF_ESHAPE;
  if ((long long)table_rows * rotary_dims > 0xFFFFFFFFLL) return A2SF_ESHAPE;
  if (!(base > 0.0) || !(factor > 0.0) || !isfinite(base) || !isfinite(factor) || !isfinite(magnitude) ||
      original_length < 0 || !isfinite(low) || !isfinite(high) || low > high)
    return A2SF_EINVAL;
  const RotaryTableArgs a = {table, table_rows, rotary_dims, original_length, base, factor, low, high, magnitude};
  return launched([&] { return launch_rotary_table(a, (hipStream_t)hip_stream), true; });
}

a2sf_status a2sf_sample(const a2sf_rows* logits, const a2sf_rows* noise, int32_t rows, int32_t n, int32_t dtype,
                        const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                        int32_t* token, float* prob, void* hip_stream) {
  A2SF_TRY(check_sizes(rows, n, dtype));
  if (n > A2SF_MAX_VOCABULARY) return A2SF_ESHAPE;
  A2SF_TRY(check_rows(logits, rows, n, dtype, true));
  A2SF_TRY(check_rows(noise, rows, n, A2SF_F32, false));
  if (!token || misaligned(token, 4) || misaligned(prob, 4) || misaligned(temperature, 4) || misaligned(top_k, 4) ||
      misaligned(top_p, 4) || misaligned(min_p, 4))
    return A2SF_EINVAL;
  SampleArgs a;
  a.logits = logits->data;
  a.noise = (const float*)data(noise);
  a.temperature = temperature;
  a.top_p = top_p;
  a.min_p = min_p;
  a.top_k = top_k;
  a.token = token;
  a.prob = prob;
  a.stride = logits->stride;
  a.noise_stride = stride(noise);
  a.rows = rows;
  a.n = n;
  return launched([&] { return launch_sample(a, dtype, (hipStream_t)hip_stream); });
}

}  // extern "C"
