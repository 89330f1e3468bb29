// New keys and values into the pages of their sequences, keys and queries turned by their positions on the way: one pass over the
// rows of a QKV product, in the place of a rotation and a scatter.  Bound by memory: every element is read and written once.
#include "pages_dev.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

// Eight neighbouring elements of a head to a lane, so 16 (d = 128) or 8 lanes to a head, a few heads of one token each.  An element is
// turned with its partner, which with pairs of halves another lane holds as its own: where a whole head of 128 turns, it comes from there
// by a lane rotation, else it is read twice, the second time from the caches.  All lanes of a head are in one wave, which has read all it needs before it writes, so q may be turned in place.
constexpr int kMostHeads = 4;

template <typename T, bool EIGHT, int D, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
  constexpr int LANES = D / kUnit;
  const PagedCache& c = a.c;
  const uint32_t first_item = blockIdx.x * (256u / LANES) + (threadIdx.x & ~63u) / LANES;  // of the wave
  const uint32_t item = first_item + (threadIdx.x & 63) / LANES;
  const uint32_t token = item / (uint32_t)a.groups;
  const int group = (int)(item - token * (uint32_t)a.groups);
  const int e0 = (int)(threadIdx.x % LANES) * kUnit;
  const int total = a.heads + 2 * c.kv_heads;
  bool live = token < (uint32_t)c.tokens;
  int seq = live ? (int)token : 0;
  if (c.starts) {
    seq = max(0, sequence_of(c, (int)min(__builtin_amdgcn_readfirstlane(first_item / (uint32_t)a.groups), (uint32_t)c.tokens - 1)));
    while (live && seq + 1 < c.sequences && c.starts[seq + 1] <= (int)token) ++seq;
    live = live && c.starts[seq] <= (int)token && (int)token < c.starts[seq + 1];
  }
  const NewTokens t = new_tokens(c, seq);
  live = live && (t.past >= 0 || t.bad);
  const int pos = t.bad ? 0 : max(0, t.past + (int)token - t.first);
  bool lost = t.bad;  // there is no place for this token
  int page = 0;
  if (live && !t.bad) page = page_of(c, c.table + seq * c.table_stride, pos, lost);
  const int place = pos & ((1 << c.shift) - 1);

  // the cosines and sines of this lane's elements; partner: how far away the other element of a pair is
  const int half = a.rot / 2;
  const bool turns = e0 < a.rot;
  const bool known = pos < a.table_rows;
  float co[kUnit], si[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) { co[j] = 1.f; si[j] = 0.f; }
  // (a lane's partners are eight neighbours too, and so are its cosines, or four with pairs of neighbours)
  const bool whole = (NEIGHBOURS ? a.rot : half) % kUnit == 0;
  if (live && turns) {
    const float* row = a.table + (long long)(known ? pos : 0) * a.rot;
    if (whole) {
      float c8[kUnit], s8[kUnit];
      const int first = NEIGHBOURS ? e0 / 2 : e0 < half ? e0 : e0 - half;
      if (NEIGHBOURS) {
        const u32x4_t cv = *(const u32x4_at4_t*)(row + first), sv = *(const u32x4_at4_t*)(row + half + first);
#pragma unroll
        for (int j = 0; j < kUnit; ++j) {
          c8[j] = __uint_as_float(cv[j / 2]);
          s8[j] = j % 2 ? __uint_as_float(sv[j / 2]) : -__uint_as_float(sv[j / 2]);
        }
      } else {
        load_unit(row + first, c8);
        load_unit(row + half + first, s8);
        if (e0 < half)
#pragma unroll
          for (int j = 0; j < kUnit; ++j) s8[j] = -s8[j];
      }
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        co[j] = known ? c8[j] : __uint_as_float(0x7FC00000u);
        si[j] = s8[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const int e = e0 + j;
        if (e >= a.rot) break;
        const int pair = NEIGHBOURS ? e / 2 : e < half ? e : e - half;
        const bool second = NEIGHBOURS ? (e & 1) != 0 : e >= half;
        co[j] = known ? row[pair] : __uint_as_float(0x7FC00000u);
        si[j] = second ? row[half + pair] : -row[half + pair];
      }
    }
  }
  const bool swaps = !NEIGHBOURS && D == 128 && a.rot == D;  // the partners are in the lane eight further on in a row of 16
  float f[kMostHeads][kUnit];
#pragma unroll
  for (int i = 0; i < kMostHeads; ++i) {
    const int h = group * a.per_lane + i;
    if (!live || i >= a.per_lane || h >= total) continue;
    const int kind = h < a.heads ? 0 : h < a.heads + c.kv_heads ? 1 : 2;
    const T* x = kind == 0   ? (const T*)a.q + (long long)token * a.q_stride[0] + h * a.q_stride[1]
                 : kind == 1 ? (const T*)a.k + (long long)token * a.k_stride[0] + (h - a.heads) * a.k_stride[1]
                             : (const T*)a.v + (long long)token * a.v_stride[0] + (h - a.heads - c.kv_heads) * a.v_stride[1];
    load_unit(x + e0, f[i]);
    if (kind == 2 || !turns || swaps) continue;
    float other[kUnit];
    if (NEIGHBOURS) {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) other[j] = f[i][j ^ 1];
    } else if (whole) {
      load_unit(x + (e0 < half ? e0 + half : e0 - half), other);
    } else {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const int e = e0 + j;
        other[j] = e < a.rot ? load_one(x + (e < half ? e + half : e - half)) : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < kUnit; ++j)
      if (e0 + j < a.rot) f[i][j] = f[i][j] * co[j] + other[j] * si[j];
  }
  if (swaps) {
#pragma unroll
    for (int i = 0; i < kMostHeads; ++i) {
      const int h = group * a.per_lane + i;
      if (i >= a.per_lane) break;
      const bool turned = h < a.heads + c.kv_heads;
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const float other = dpp_move<0x128>(f[i][j]);  // (the lanes of a head are all here or none)
        f[i][j] = turned ? f[i][j] * co[j] + other * si[j] : f[i][j];
      }
    }
  }
  wait_vm<0>();  // (all of the wave's reads)
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < kMostHeads; ++i) {
    const int h = group * a.per_lane + i;
    const bool there = live && i < a.per_lane && h < total;
    const int kind = h < a.heads ? 0 : h < a.heads + c.kv_heads ? 1 : 2;
    const int kv = kind == 1 ? h - a.heads : h - a.heads - c.kv_heads;
    if (there && kind == 0) {
      if (lost)
#pragma unroll
        for (int j = 0; j < kUnit; ++j) f[i][j] = __uint_as_float(0x7FC00000u);
      store_unit((T*)a.q_out + (long long)token * a.q_out_stride[0] + h * a.q_out_stride[1] + e0, f[i]);
    }
    const bool kept = there && kind > 0 && !lost;
    const long long at = page * c.stride[0] + kv * c.stride[1] + place * c.stride[2];
    char* const rows = kind == 1 ? c.k : c.v;
    if constexpr (EIGHT) {
      uint32_t top = kept ? unit_top(f[i]) : 0u;  // (every lane of the wave takes part)
      top = max(top, dpp_move_u32<0xB1>(top));
      top = max(top, dpp_move_u32<0x4E>(top));
      top = max(top, dpp_move_u32<0x141>(top));
      if (LANES == 16) top = max(top, dpp_move_u32<0x140>(top));
      if (kept) {
        const uint32_t byte = scale_byte(top);
        *(uint2*)(rows + at + e0) = to_eight_bits(f[i], byte);
        if (e0 == 0)
          (kind == 1 ? c.k_scales : c.v_scales)[page * c.scale_stride[0] + kv * c.scale_stride[1] + place * c.scale_stride[2]] = (uint8_t)byte;
      }
    } else if (kept) {
      store_unit((T*)(rows + at) + e0, f[i]);
    }
  }
}

template <typename T, bool EIGHT, int D>
bool append(AppendArgs a, bool neighbours, hipStream_t st) {
  const int total = a.heads + 2 * a.c.kv_heads;
  // (us in the kernel with one head to a lane / four, 48 heads of 128: 16 tokens 3.3 / 4.1, 256 4.0 / 4.6, 341 4.4 / 4.7, 512 5.6 / 5.3, 1024 8.8 / 6.9)
  a.per_lane = (long long)a.c.tokens * total <= 16384 ? 1 : kMostHeads;
  a.groups = (total + a.per_lane - 1) / a.per_lane;
  const unsigned long long items = (unsigned long long)a.c.tokens * a.groups, grid = (items + 256 / (D / kUnit) - 1) / (256 / (D / kUnit));
  if (!grid_fits(grid, 256)) return false;
  if (neighbours) paged_append_kernel<T, EIGHT, D, true><<<(uint32_t)grid, 256, 0, st>>>(a);
  else paged_append_kernel<T, EIGHT, D, false><<<(uint32_t)grid, 256, 0, st>>>(a);
  return true;
}

template <typename T>
bool append(const AppendArgs& a, bool neighbours, hipStream_t st) {
  const bool eight = a.c.dtype == A2SF_E4M3;
  if (a.c.d == 128) return eight ? append<T, true, 128>(a, neighbours, st) : append<T, false, 128>(a, neighbours, st);
  return eight ? append<T, true, 64>(a, neighbours, st) : append<T, false, 64>(a, neighbours, st);
}

}  // namespace

bool launch_paged_append(AppendArgs a, int dtype, bool neighbours, hipStream_t st) {
  return dtype == A2SF_F32 ? append<float>(a, neighbours, st) : append<bf16_t>(a, neighbours, st);
}

}  // namespace a2sf
