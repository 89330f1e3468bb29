// Rotary positions: the pairs of a head's first `rot` elements turn by position * frequency, from a table of cosines and sines.
// The same pass takes the heads of a QKV product apart into the layouts of the attention calls.  Bound by memory: every element
// is read and written once, and the table's row of a token (rot floats) serves all its heads.
#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

// Sixteen bytes of neighbouring elements, or fewer of them
template <typename T>
struct Chunk {
  static constexpr int kCount = 16 / (int)sizeof(T);
  float f[kCount];
  __device__ __forceinline__ void load(const T* p, int have) {
    if (have >= kCount) {
      const u32x4_t r = *(const u32x4_at2_t*)p;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(r[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[2 * i] = __uint_as_float(r[i] << 16);
          f[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kCount; ++i) f[i] = i < have ? load_one(p + i) : 0.f;
  }
  __device__ __forceinline__ void store(T* p, int have) const {
    if (have >= kCount) {
      u32x4_t r;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(f[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
      }
      *(u32x4_at2_t*)p = r;
      return;
    }
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      if (i < have) store_one(p + i, f[i]);
  }
};

// An item is what a lane reads before it writes: with halves 16 bytes of the first half of the turned part and the 16 of the
// second that they pair with, with neighbours 16 bytes, and 16 bytes behind the turned part as they are; so the lanes of a head
// read its elements in one row.  A workgroup takes some tokens of one part (its strides are then scalar), a lane one item of
// up to kHeads heads, with the item's cosines and sines: all of them are read before the first is written.  Items read and write
// their own elements only, so a part may be turned in place.  Any stride and alignment; WHOLE: no item is shorter than 16 bytes.
// 8 x 2048 tokens of 96 heads of 128 in bf16 (805 MB): halves 157 us = 5.1 TB/s, neighbours 151 = 5.3 (a copy of 1 GiB: 5.2).  With one item of all
// parts' heads in turn per lane, whose strides are then looked up lane by lane, 165 and 181.
// 16 tokens of 48 heads of 128: 3.3 us with a head to a lane, 4.6 with four.
// A turned part of 100 of 128, halves: 221 us, neighbours 175 (345 and 332 with the last item element by element, as it still is in place).
constexpr int kHeads = 4;

template <typename T, bool NEIGHBOURS, bool WHOLE>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  constexpr int W = Chunk<T>::kCount, kTable = NEIGHBOURS ? W / 2 : W;
  int part = 0;
#pragma unroll
  for (int k = 1; k < A2SF_MAX_ROTARY_PARTS; ++k) part += blockIdx.x >= a.first_block[k];
  const RotaryPart& P = a.part[part];
  const int local = threadIdx.x;
  const uint32_t token = (blockIdx.x - a.first_block[part]) * (uint32_t)P.tokens_per_block + (uint32_t)(local / P.lanes);  // (below 2^29)
  const int lane = local % P.lanes;
  if (local >= P.tokens_per_block * P.lanes || token >= (uint32_t)a.batch * (uint32_t)a.length) return;
  const int item = lane % a.items, head_step = P.lanes / a.items;
  const int b = (int)(token / (uint32_t)a.length), i = (int)(token - (uint32_t)b * (uint32_t)a.length);
  const int half = a.rot / 2;
  const bool turns = item < a.turning;
  if (!(turns && P.rotate) && P.in_place) return;
  // the item's elements: `have` from e0 on, with halves as many from e1 on
  int e0, e1 = 0, have;
  const int from = turns ? 0 : a.rot, upto = !turns ? a.d : NEIGHBOURS ? a.rot : half;
  e0 = from + (turns ? item : item - a.turning) * W;
  have = upto - e0;
  if (WHOLE) {
    have = W;
  } else if (have < W && upto - from >= W && !P.in_place) {
    // the last item moves back over elements of the one before it, which both then write the same (not in place, where it might read
    // what the other has written)
    e0 = upto - W;
    have = W;
  }
  if (turns && !NEIGHBOURS) e1 = half + e0;
  const bool two = !NEIGHBOURS && turns;
  const T* x = (const T*)P.x + b * P.x_stride[0] + i * P.x_stride[1];
  T* y = (T*)P.y + b * P.y_stride[0] + i * P.y_stride[1];
  float c[kTable], s[kTable];
  bool known = true;
  if (turns && P.rotate) {
    const int32_t p = a.pos[b * a.pos_stride + i];
    known = p >= 0 && p < a.table_rows;
    const int first = NEIGHBOURS ? e0 / 2 : e0;
    const float* row = a.table + (long long)(known ? p : 0) * a.rot + first;
#pragma unroll
    for (int j = 0; j < kTable; ++j) {
      const bool there = WHOLE || first + j < half;
      c[j] = there ? row[j] : 0.f;
      s[j] = there ? row[half + j] : 0.f;
    }
    if (a.inverse)
#pragma unroll
      for (int j = 0; j < kTable; ++j) s[j] = -s[j];
  }
  const int h0 = lane / a.items;
  for (int head = h0; head < P.heads; head += kHeads * head_step) {
    Chunk<T> u[kHeads], v[kHeads];
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
      const int h = head + k * head_step;
      if (h >= P.heads) break;
      const T* from = x + h * P.x_stride[2];
      u[k].load(from + e0, have);
      if (two) v[k].load(from + e1, have);
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
      const int h = head + k * head_step;
      if (h >= P.heads) break;
      if (turns && P.rotate) {
        if constexpr (NEIGHBOURS) {
#pragma unroll
          for (int j = 0; j < W / 2; ++j) {
            const float p = u[k].f[2 * j], q = u[k].f[2 * j + 1];
            u[k].f[2 * j] = p * c[j] - q * s[j];
            u[k].f[2 * j + 1] = q * c[j] + p * s[j];
          }
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) {
            const float p = u[k].f[j], q = v[k].f[j];
            u[k].f[j] = p * c[j] - q * s[j];
            v[k].f[j] = q * c[j] + p * s[j];
          }
        }
        if (!known) {
#pragma unroll
          for (int j = 0; j < W; ++j) u[k].f[j] = v[k].f[j] = __uint_as_float(0x7FC00000u);
        }
      }
      T* to = y + h * P.y_stride[2];
      u[k].store(to + e0, have);
      if (two) v[k].store(to + e1, have);
    }
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

template <typename T>
bool rotary(RotaryArgs a, bool neighbours, hipStream_t st) {
  constexpr int W = Chunk<T>::kCount;
  const int turned = neighbours ? a.rot : a.rot / 2;
  a.turning = (turned + W - 1) / W;
  a.items = a.turning + (a.d - a.rot + W - 1) / W;
  const bool whole = turned % W == 0 && (a.d - a.rot) % W == 0;
  const long long tokens = (long long)a.batch * a.length;
  const bool few = tokens <= 256;
  uint32_t grid = 0;
  for (int k = 0; k < A2SF_MAX_ROTARY_PARTS; ++k) {
    a.first_block[k] = k < a.parts ? grid : 0xFFFFFFFFu;
    if (k >= a.parts) continue;
    // as many lanes for a token as have kHeads heads each (one each if there are too few tokens to fill the chip anyway), fewer where a
    // workgroup has no more; several tokens per workgroup
    RotaryPart& P = a.part[k];
    const long long want = (long long)(few ? P.heads : (P.heads + kHeads - 1) / kHeads) * a.items;
    P.lanes = want < 256 ? (int)want : 256 / a.items * a.items;
    P.tokens_per_block = 256 / P.lanes;
    grid += (uint32_t)((tokens + P.tokens_per_block - 1) / P.tokens_per_block);
  }
  if (!grid_fits(grid, 256)) return false;
  if (neighbours) {
    if (whole) rotary_kernel<T, true, true><<<grid, 256, 0, st>>>(a);
    else rotary_kernel<T, true, false><<<grid, 256, 0, st>>>(a);
  } else {
    if (whole) rotary_kernel<T, false, true><<<grid, 256, 0, st>>>(a);
    else rotary_kernel<T, false, false><<<grid, 256, 0, st>>>(a);
  }
  return true;
}

}  // namespace

bool launch_rotary(RotaryArgs a, int dtype, bool neighbours, hipStream_t st) {
  return dtype == A2SF_F32 ? rotary<float>(a, neighbours, st) : rotary<bf16_t>(a, neighbours, st);
}

void launch_rotary_table(const RotaryTableArgs& a, hipStream_t st) {
  const long long count = (long long)a.rows * (a.rot / 2);
  rotary_table_kernel<<<(uint32_t)((count + 255) / 256), 256, 0, st>>>(a);
}

}  // namespace a2sf
