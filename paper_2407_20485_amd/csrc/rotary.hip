// Rotary positions: the pairs of a head's first `rot` elements turn by position * frequency, from a table of cosines and sines.
// The same pass takes the heads of a QKV product apart into the layouts of the attention calls.  Bound by memory: every element
// is read and written once, and the table's row of a token (rot floats) serves all its heads.
#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

template <typename T, int W> struct Chunk;  // W consecutive elements
template <typename T> struct Chunk<T, 8> {
  float f[8];
  __device__ __forceinline__ void load(const T* p) { load_unit(p, f); }
  __device__ __forceinline__ void store(T* p) const { store_unit(p, f); }
};
template <typename T> struct Chunk<T, 1> {
  float f[1];
  __device__ __forceinline__ void load(const T* p) { f[0] = load_one(p); }
  __device__ __forceinline__ void store(T* p) const { store_one(p, f[0]); }
};

// An item is what a lane reads before it writes: with halves W elements of the first half of the turned part and the W of the
// second that they pair with, with neighbours 2 W elements, behind the turned part 2 W elements as they are (W where an odd
// one is left).  A lane keeps its item's cosines and sines and goes through the heads.  Items read and write their own elements only,
// so a part may be turned in place.
// W = 8 where the item's parts are whole units of eight (any stride and alignment), W = 1 else.
template <typename T, int W, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  const int local = threadIdx.x;
  const long long token = (long long)blockIdx.x * a.tokens_per_block + local / a.lanes;
  const int lane = local % a.lanes;
  if (local >= a.tokens_per_block * a.lanes || token >= (long long)a.batch * a.length) return;
  const int item = lane % a.items, head_step = a.lanes / a.items;
  int head = lane / a.items;
  if (head >= head_step) return;  // lanes past the last whole head
  const int b = (int)(token / a.length), i = (int)(token - (long long)b * a.length);
  const int half = a.rot / 2;
  const int pairs = half / W;  // items that turn
  const bool turns = item < pairs;
  // first elements of the item's two parts
  int e0, e1;
  bool two = true;
  if (turns) {
    e0 = NEIGHBOURS ? 2 * item * W : item * W;
    e1 = NEIGHBOURS ? e0 + W : half + e0;
  } else {
    e0 = a.rot + 2 * (item - pairs) * W;
    e1 = e0 + W;
    two = e1 + W <= a.d;
  }
  float c[W], s[W];
  bool known = true;
  if (turns) {
    const int32_t p = a.pos[b * a.pos_stride + i];
    known = p >= 0 && p < a.table_rows;
    const float* row = a.table + (long long)(known ? p : 0) * a.rot + item * W;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      c[j] = row[j];
      s[j] = row[half + j];
      if (a.inverse) s[j] = -s[j];
    }
  }
  int part = 0;
  for (; head < a.heads; head += head_step) {
    while (head >= a.first_head[part + 1]) ++part;
    const int h = head - a.first_head[part];
    const RotaryPart& P = a.part[part];
    const T* x = (const T*)P.x + b * P.x_stride[0] + i * P.x_stride[1] + h * P.x_stride[2];
    T* y = (T*)P.y + b * P.y_stride[0] + i * P.y_stride[1] + h * P.y_stride[2];
    if (!(turns && P.rotate) && P.in_place) continue;
    Chunk<T, W> u, v;
    u.load(x + e0);
    if (two) v.load(x + e1);
    if (turns && P.rotate) {
      if (NEIGHBOURS && W > 1) {
        // pairs (0, 1) (2, 3) ... of the 2 W elements
        float z[2 * W];
#pragma unroll
        for (int j = 0; j < W; ++j) { z[j] = u.f[j]; z[W + j] = v.f[j]; }
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float p = z[2 * j], q = z[2 * j + 1];
          z[2 * j] = p * c[j] - q * s[j];
          z[2 * j + 1] = q * c[j] + p * s[j];
        }
#pragma unroll
        for (int j = 0; j < W; ++j) { u.f[j] = z[j]; v.f[j] = z[W + j]; }
      } else {
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float p = u.f[j], q = v.f[j];
          u.f[j] = p * c[j] - q * s[j];
          v.f[j] = q * c[j] + p * s[j];
        }
      }
      if (!known) {
#pragma unroll
        for (int j = 0; j < W; ++j) u.f[j] = v.f[j] = __uint_as_float(0x7FC00000u);
      }
    }
    u.store(y + e0);
    if (two) v.store(y + e1);
  }
}

// table[p] = cosines, then sines, of p * f_i, times `magnitude`.  64 bits: an angle of thousands of turns in 32 would
// be wrong in its third digit.
__global__ __launch_bounds__(256) void rotary_table_kernel(RotaryTableArgs a) {
  const int half = a.rot / 2;
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
  if (at >= (long long)a.rows * half) return;
  const int p = (int)(at / half), i = (int)(at - (long long)p * half);
  double f = pow(a.base, -2.0 * i / a.rot);
  if (a.factor != 1.0) {
    double keep = 0.0;  // the share of the frequency that is not scaled
    if (a.original_length > 0) {
      const double turns = a.original_length * f / 6.283185307179586476925286766559;
      keep = a.high > a.low ? (turns - a.low) / (a.high - a.low) : (turns >= a.low ? 1.0 : 0.0);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
    }
    f *= keep + (1.0 - keep) / a.factor;
  }
  double sn, cs;
  sincos(p * f, &sn, &cs);
  a.table[(long long)p * a.rot + i] = (float)(cs * a.magnitude);
  a.table[(long long)p * a.rot + half + i] = (float)(sn * a.magnitude);
}

template <typename T, int W>
void rotary(const RotaryArgs& a, uint32_t grid, bool neighbours, hipStream_t st) {
  if (neighbours) rotary_kernel<T, W, true><<<grid, 256, 0, st>>>(a);
  else rotary_kernel<T, W, false><<<grid, 256, 0, st>>>(a);
}

}  // namespace

void launch_rotary(RotaryArgs a, int dtype, bool neighbours, hipStream_t st) {
  const bool wide = a.rot % 16 == 0 && a.d % 16 == 0;
  const int W = wide ? 8 : 1;
  a.items = a.rot / 2 / W + (a.d - a.rot + 2 * W - 1) / (2 * W);
  // A token's heads over as many lanes as there are, up to a workgroup; several tokens per workgroup where they are fewer.
  const int want = a.heads * a.items;
  a.lanes = want < 256 ? want : 256 / a.items * a.items;
  a.tokens_per_block = 256 / a.lanes;
  const long long tokens = (long long)a.batch * a.length;
  const uint32_t grid = (uint32_t)((tokens + a.tokens_per_block - 1) / a.tokens_per_block);
  if (dtype == A2SF_F32) {
    if (wide) rotary<float, 8>(a, grid, neighbours, st);
    else rotary<float, 1>(a, grid, neighbours, st);
  } else {
    if (wide) rotary<bf16_t, 8>(a, grid, neighbours, st);
    else rotary<bf16_t, 1>(a, grid, neighbours, st);
  }
}

void launch_rotary_table(const RotaryTableArgs& a, hipStream_t st) {
  const long long count = (long long)a.rows * (a.rot / 2);
  rotary_table_kernel<<<(uint32_t)((count + 255) / 256), 256, 0, st>>>(a);
}

}  // namespace a2sf
