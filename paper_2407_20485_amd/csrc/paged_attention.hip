// Attention over keys and values in pages.
//
//  paged_rows   up to 16 query rows (the heads that share a K/V head, of one token or of neighbouring ones) against a range of their
//               tokens, straight from memory into registers: the form for single tokens, whose every byte of the cache is
//               used once.  The range may be a share of what the rows see;
//  paged_tiles  (paged_tiles.hip) 128 query rows against tiles of 64 tokens through LDS: bf16 prompts and chunks;
//  paged_join   adds up the shares of either.
#include <float.h>

#include <algorithm>

#include "paged_tiles.h"
#include "pages_dev.h"
#include "rows_dev.h"

namespace a2sf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f32x4_t mfma16(const uint4& a, const uint4& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mfma16(float a, float b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// ---- even shares ---------------------------------------------------------------------------------------------------------------------
// The tokens that the sequences' rows see, in units, all pieces (a sequence's rows under one K/V head) one after the other, dealt out to the
// workgroups evenly (4 sequences of 16000 .. 65536 tokens 133 us, 170 with each sequence cut into as many shares): a workgroup takes `per`
// units in a row, whatever pieces they are of.  What it has of a piece that is not whole goes to one of two places of its own: the second if
// the piece goes on behind it, else the first.
__device__ __forceinline__ int units_of(const PagedArgs& a, int seq, int unit) {  // of a piece of the sequence
  const NewTokens t = new_tokens(a.c, seq);
  if (t.bad || t.past < 0) return 1;  // (there is something to write)
  return (visible(t.past, t.past, a.window, a.sinks).count + unit - 1) / unit;
}
struct EvenShares {
  int total, per;
};
__device__ __forceinline__ EvenShares even_shares(const PagedArgs& a, int unit) {
  const int lane = threadIdx.x & 63, pieces = a.blocks_per * a.c.kv_heads;
  int sum = 0;
  for (int s = lane; s < a.c.sequences; s += 64) sum += units_of(a, s, unit) * pieces;
  const int total = wave_sum_i(sum);
  return {total, (total + a.even - 1) / a.even};
}
// Where workgroup `group` begins: the sequence, its piece and the unit of that, and the units that the workgroup has (0: none)
struct EvenPlace {
  int seq, piece, unit, left;
};
__device__ __forceinline__ EvenPlace even_place(const PagedArgs& a, int unit, int group) {
  const int lane = threadIdx.x & 63, pieces = a.blocks_per * a.c.kv_heads;
  const bool few = a.c.sequences <= 64;  // all in the lanes at once
  EvenShares all;
  if (!few) all = even_shares(a, unit);
  int before = 0;
  for (int s = 0;; s += 64) {
    const int units = s + lane < a.c.sequences ? units_of(a, s + lane, unit) : 0;
    int upto = units * pieces;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
      const int other = __shfl_up(upto, step);
      if (lane >= step) upto += other;
    }
    if (few) {
      all.total = __builtin_amdgcn_readlane(upto, 63);
      all.per = (all.total + a.even - 1) / a.even;
    }
    const int at = group * all.per;
    if (at >= all.total) return {0, 0, 0, 0};
    const unsigned long long behind = __ballot(before + upto > at);
    if (behind) {
      const int l = __builtin_ctzll(behind);
      const int start = __builtin_amdgcn_readlane(before + upto - units * pieces, l), each = __builtin_amdgcn_readlane(units, l);
      const int piece = (at - start) / each;
      return {s + l, piece, at - start - piece * each, min(all.per, all.total - at)};
    }
    before += __builtin_amdgcn_readlane(upto, 63);
    if (s + 64 >= a.c.sequences) return {0, 0, 0, 0};  // (only if lengths change under the call)
  }
}

// ---- up to 16 rows, straight from memory ------------------------------------------------------------------------------------------
// S^T = K Q^T with the tokens as rows of the result: lane (g, q) = (l / 16, l % 16) gets the logits of query row q with tokens 4g .. 4g + 3
// of 16, which is how the second product, O^T = V^T P^T, takes its P^T -- if its k runs over the tokens in that order, which is free to
// choose: lane (g, x) of V^T then has tokens 4g .. of each 16, and of those the D / 16 values from dimension x * D / 16 on, whole 16 rows
// of V being read by 16 lanes side by side; a pair of tokens' values of one dimension is one byte permutation.
// So neither P nor V goes through LDS.  Q and K take their dimensions in the order in which K's 16 bytes per lane come.
// bf16: P goes into the product as two bf16 numbers, its value and what that leaves out (2^-17 of it stays out): the matrix pipe has room.
// Bound by memory: 4 x up to 65536 tokens of 8 K/V heads 118 us = 6.1 TB/s, 200 x 1004 of 40 heads 657 = 6.3; 48 x up to 8192 in 8 bits 98 = 5.4,
// in fp32 8 x up to 32768 265 = 5.7.  A wave has one tile's K and V
// in registers and asks for the next K when it has used this one's (two tiles at a time take 256 registers and spill: 200 x 1004
// 745 us without streaming loads and 951 with them).
constexpr int kRows = 16;
constexpr int kRowWaves = 4;

template <typename T, bool EIGHT, int D>
struct RowForm {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int BYTES = EIGHT ? 1 : (int)sizeof(T);
  static constexpr int H = F32 ? 1 : 2;                   // 16 tokens each
  static constexpr int TOKENS = 16 * H;                   // of a tile
  static constexpr int UNIT = kRowWaves * TOKENS;         // shares are multiples of this
  static constexpr int NK = D * BYTES / 64;               // 16-byte loads of a row of K per lane
  static constexpr int VD = D / 16;                       // dimensions of V per lane
  static constexpr int VW = VD * BYTES / 4;               // ... in dwords
  static constexpr int E = 4 * H;                         // tokens of V per lane
};

// SEVERAL: a block may hold the rows of several tokens, which do not all see the same
template <typename T, bool EIGHT, int D, bool SEVERAL>
__global__ __launch_bounds__(64 * kRowWaves, D == 64 ? 3 : 2) void paged_rows_kernel(PagedArgs a) {
  typedef RowForm<T, EIGHT, D> F;
  constexpr int H = F::H, NK = F::NK, VD = F::VD, VW = F::VW, E = F::E, TT = F::TOKENS;
  __shared__ float o_of[kRowWaves][kRows][D + 4];
  __shared__ float m_of[kRowWaves][kRows], l_of[kRowWaves][kRows];
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, x16 = lane & 15;
  const int out_q = threadIdx.x >> 4, out_d = (threadIdx.x & 15) * VD;  // the row that this thread writes, 16 threads to a row

  // Rows first_row .. of a sequence under one K/V head against its tokens v0 .. v1 - 1 (as they are numbered in `see`); part: where the
  // result goes, < 0: it is all there is, and goes to o.
  const auto attend = [&](int seq, const NewTokens& t, int kv, int first_row, const Visible& see, int v0, int v1, int part) {
    // this lane's query row
    const long long row = (long long)first_row + x16;
    const int i_row = (int)min(row / a.group, (long long)t.count - 1), head = kv * a.group + (int)(row % a.group);
    const int token_row = t.first + (int)(row / a.group);
    const bool there = row < (long long)t.count * a.group && token_row >= 0 && token_row < c.tokens;
    const int pos = t.past + i_row;
    // the row that this thread writes
    const long long out_row = (long long)first_row + out_q;
    const int out_token = t.first + (int)(out_row / a.group), out_head = kv * a.group + (int)(out_row % a.group);
    const bool out_there = out_row < (long long)t.count * a.group && out_token >= 0 && out_token < c.tokens;
    T* const out = (T*)a.o + (out_there ? out_token * a.o_stride[0] + out_head * a.o_stride[1] : 0) + out_d;
    if (t.bad || t.past < 0) {
      if (out_there && part < 0) {
        float f[VD];
#pragma unroll
        for (int i = 0; i < VD; ++i) f[i] = t.bad ? kNan : 0.f;
        store_n<VD>(out, f);
      }
      return;
    }
    // Q: dimensions in the order of K's loads
    uint4 qb[F::F32 ? 1 : D / 32];
    float qf[F::F32 ? D / 4 : 1];
    {
      const T* q = (const T*)a.q + (there ? token_row * a.q_stride[0] + head * a.q_stride[1] : 0);
      if constexpr (!F::F32) {
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          const int dim = EIGHT ? j / 2 * 64 + g * 16 + j % 2 * 8 : j * 32 + g * 8;
          qb[j] = make_uint4(0, 0, 0, 0);
          if (there) {
            const u32x4_t v = *(const u32x4_at2_t*)(q + dim);
            qb[j] = make_uint4(v[0], v[1], v[2], v[3]);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < D / 4; ++j) {
          const int dim = EIGHT ? j / 16 * 64 + g * 16 + j % 16 : j / 4 * 16 + g * 4 + j % 4;
          qf[j] = there ? q[dim] : 0.f;
        }
      }
    }

    const int32_t* const table = c.table + seq * c.table_stride;
    const char* const kbase = c.k + kv * c.stride[1];
    const char* const vbase = c.v + kv * c.stride[1];
    const int mask = (1 << c.shift) - 1;
    // the page of token number v0 + .. of a tile, one token to a lane (H = 1: twice)
    const auto lookup = [&](int base) -> int {
      const int i = min(base + lane % TT, v1 - 1);
      return table[see.token(i) >> c.shift];
    };
    // a tile's K and V; the scales of its tokens (k's byte, then v's) and the tokens whose page is none of the cache's (the same in all lanes)
    uint4 kr[H][NK];
    uint32_t vr[E][VW], both = 0, both_next = 0;
    unsigned long long lost = 0, lost_next = 0;
    const auto sound = [&](int pages) { return (uint32_t)pages < (uint32_t)c.pages ? pages : 0; };
    const auto at = [&](int base, int pages, int i) -> long long {  // element i of the tile -> its row
      const int token = see.token(min(base + i, v1 - 1));
      return (long long)__shfl(pages, i) * c.stride[0] + (long long)(token & mask) * c.stride[2];
    };
    // Sixteen tokens are in one page if it has so many, and then scalar instructions form their address (48 sequences of up to 8191 tokens in 8
    // bits 100 us, 108 with an address per row; d = 64 in bf16 99 and 109); smaller pages, and rows very far from each other, take one per row.
    const bool grouped = c.shift >= 4 && c.stride[2] < (1ll << 27);
    const uint32_t koff = x16 * (uint32_t)c.stride[2] + g * 16;
    uint32_t voff[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) voff[e] = (g * 4 + e) * (uint32_t)c.stride[2] + x16 * (VD * F::BYTES);
    const auto group_at = [&](int base, int pages, int h) -> long long {
      const int token = see.token(min(base + h * 16, (v1 - 1) & ~15));
      return (long long)__builtin_amdgcn_readlane(pages, h * 16) * c.stride[0] + (long long)(token & mask) * c.stride[2];
    };
    const auto load_k = [&](int h, const char* p) {
#pragma unroll
      for (int j = 0; j < NK; ++j) kr[h][j] = load16_as<!SEVERAL>(p + j * 64);
    };
    const auto load_v = [&](int e, const char* p) {
      if constexpr (VW == 1) {
        vr[e][0] = __builtin_nontemporal_load((const uint32_t*)p);
      } else if constexpr (VW == 2) {
        const u32x2_t v = __builtin_nontemporal_load((const u32x2_t*)p);
        vr[e][0] = v[0];
        vr[e][1] = v[1];
      } else {
#pragma unroll
        for (int j = 0; j < VW; j += 4) {
          const uint4 v = load16_as<!SEVERAL>(p + 4 * j);
          vr[e][j] = v.x;
          vr[e][j + 1] = v.y;
          vr[e][j + 2] = v.z;
          vr[e][j + 3] = v.w;
        }
      }
    };
    const auto fetch_k = [&](int base, int pages) {
      lost_next = __ballot((uint32_t)pages >= (uint32_t)c.pages);
      pages = sound(pages);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        if (grouped) load_k(h, kbase + group_at(base, pages, h) + koff);
        else load_k(h, kbase + at(base, pages, h * 16 + x16) + g * 16);
      }
      if constexpr (EIGHT) {
        const int token = see.token(min(base + lane % TT, v1 - 1));
        const long long p = (long long)pages * c.scale_stride[0] + kv * c.scale_stride[1] + (long long)(token & mask) * c.scale_stride[2];
        both_next = c.k_scales[p] | (uint32_t)c.v_scales[p] << 8;
      }
    };
    const auto fetch_v = [&](int base, int pages) {
      pages = sound(pages);
      if (grouped) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
          const char* p = vbase + group_at(base, pages, h);
#pragma unroll
          for (int e = 0; e < 4; ++e) load_v(4 * h + e, p + voff[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) load_v(e, vbase + at(base, pages, e / 4 * 16 + g * 4 + e % 4) + x16 * (VD * F::BYTES));
      }
    };

    float m = -FLT_MAX, l = 0.f;
    f32x4_t o[VD];
#pragma unroll
    for (int i = 0; i < VD; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // A tile with tokens that some rows see and others do not: a probability of 0 keeps no infinity or NaN of V out of a row.  Such values
    // are taken out, and the rows that see one of them get NaN for its dimension: those for which a product of marks is above 0.
    const auto separate = [&](uint32_t hidden, auto& vf) {
      const auto odd32 = [](float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; };
      uint32_t odd = 0;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < VD; ++i) odd |= (__float_as_uint(vf[e][i]) & 0x7F800000u) + 0x00800000u;
      if (!__any(odd >> 31)) return;
#pragma unroll
      for (int i = 0; i < VD; ++i) {
        f32x4_t marks = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) {
          marks = mfma16(odd32(vf[e][i]) ? 1.f : 0.f, hidden >> e & 1 ? 0.f : 1.f, marks);
          if (odd32(vf[e][i])) vf[e][i] = 0.f;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (marks[r] > 0.f) o[i][r] = kNan;
      }
    };

    const auto compute = [&](int base, int next, int pages) {
      f32x4_t s[H];
#pragma unroll
      for (int h = 0; h < H; ++h) {
        s[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NK; ++j) {
          const uint4 k = kr[h][j];
          const uint32_t w[4] = {k.x, k.y, k.z, k.w};
          if constexpr (!F::F32 && !EIGHT) {
            s[h] = mfma16(k, qb[j], s[h]);
          } else if constexpr (!F::F32) {
            uint32_t b[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              b[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[i], 1.0f, false));
              b[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[i], 1.0f, true));
            }
            s[h] = mfma16(make_uint4(b[0], b[1], b[2], b[3]), qb[2 * j], s[h]);
            s[h] = mfma16(make_uint4(b[4], b[5], b[6], b[7]), qb[2 * j + 1], s[h]);
          } else if constexpr (!EIGHT) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[h] = mfma16(__uint_as_float(w[i]), qf[4 * j + i], s[h]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
              s[h] = mfma16(lo[0], qf[16 * j + 4 * i], s[h]);
              s[h] = mfma16(lo[1], qf[16 * j + 4 * i + 1], s[h]);
              s[h] = mfma16(hi[0], qf[16 * j + 4 * i + 2], s[h]);
              s[h] = mfma16(hi[1], qf[16 * j + 4 * i + 3], s[h]);
            }
          }
        }
      }
      fetch_k(next, pages);  // (behind the last tile: its last token again)
      uint32_t scales[EIGHT ? E : 1];
      if constexpr (EIGHT) {
#pragma unroll
        for (int e = 0; e < E; ++e) scales[e] = (uint32_t)__shfl((int)both, e / 4 * 16 + g * 4 + e % 4);
      }
      float y[E], top = -FLT_MAX;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float k = a.scale_log2e;
        if constexpr (EIGHT) k *= scale_value(scales[e] & 255u);
        y[e] = s[e / 4][e % 4] * k;
      }
      if (lost) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (lost >> (e / 4 * 16 + g * 4 + e % 4) & 1) {
            y[e] = kNan;
#pragma unroll
            for (int j = 0; j < VW; ++j) vr[e][j] = 0;
          }
      }
      if (base + TT > v1 || (!SEVERAL && base < see.edge)) {  // numbers behind the end, and some that no row sees
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int i = base + e / 4 * 16 + g * 4 + e % 4, token = see.token(i);
          if (i >= v1 || (!SEVERAL && pos - token >= a.window && token >= a.sinks)) {
            y[e] = -INFINITY;
#pragma unroll
            for (int j = 0; j < VW; ++j) vr[e][j] = 0;
          }
        }
      }
      float vf[F::F32 ? E : 1][VD];  // V as fp32
      if constexpr (F::F32) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int j = 0; j < VW; ++j) {
            if constexpr (EIGHT) {
              const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)vr[e][j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)vr[e][j], true);
              vf[e][4 * j] = lo[0];
              vf[e][4 * j + 1] = lo[1];
              vf[e][4 * j + 2] = hi[0];
              vf[e][4 * j + 3] = hi[1];
            } else {
              vf[e][j] = __uint_as_float(vr[e][j]);
            }
          }
      }
      if constexpr (SEVERAL) {
        static_assert(F::F32, "several tokens of bf16 take the tile form");
        uint32_t hidden = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int token = see.token(base + e / 4 * 16 + g * 4 + e % 4);
          if (token > pos || (pos - token >= a.window && token >= a.sinks)) {
            y[e] = -INFINITY;
            hidden |= 1u << e;
          }
        }
        if (__any(hidden)) separate(hidden, vf);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, y[e]);
      // the running maximum moves when a logit is 2^8 above it: until then the sums have room
      if (__any(top > m + 8.f)) {
        const float m_new = fmaxf(m, across_rows(top, OpMax(), true, true)), shrink = fast_exp2(m - m_new);
        l *= shrink;
#pragma unroll
        for (int i = 0; i < VD; ++i) o[i] *= shrink;
        m = m_new;
      }
      float p[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        p[e] = fast_exp2(y[e] - m);
        l += p[e];
        if constexpr (EIGHT) p[e] = p[e] == 0.f ? 0.f : p[e] * scale_value(scales[e] >> 8);
      }
      if constexpr (!F::F32) {
#pragma unroll
        for (int e0 = 0; e0 < E; e0 += 8) {  // 32 tokens
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p0 = p[e0 + 2 * i], p1 = p[e0 + 2 * i + 1];
            hi[i] = pack_bf16(p0, p1);
            lo[i] = pack_bf16(p0 - __uint_as_float(hi[i] << 16), p1 - __uint_as_float(hi[i] & 0xFFFF0000u));
          }
          uint32_t vb[8][VD / 2];  // bf16, two dimensions to a register
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int j = 0; j < VW; ++j) {
              const uint32_t w = vr[e0 + e][j];
              if constexpr (EIGHT) {
                vb[e][2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false));
                vb[e][2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true));
              } else {
                vb[e][j] = w;
              }
            }
#pragma unroll
          for (int i = 0; i < VD; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
              w[j] = __builtin_amdgcn_perm(vb[2 * j + 1][i / 2], vb[2 * j][i / 2], i % 2 ? 0x07060302u : 0x05040100u);
            const uint4 v = make_uint4(w[0], w[1], w[2], w[3]);
            o[i] = mfma16(v, make_uint4(hi[0], hi[1], hi[2], hi[3]), o[i]);
            o[i] = mfma16(v, make_uint4(lo[0], lo[1], lo[2], lo[3]), o[i]);
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
          for (int i = 0; i < VD; ++i) o[i] = mfma16(vf[e][i], p[e], o[i]);
        }
      }
    };

    // tile after tile: the next one's K is asked for when this one's has been used, V likewise, its pages a tile before
    int base = v0 + wave * TT;
    if (base < v1) {
      int pages = lookup(base);
      fetch_k(base, pages);
      fetch_v(base, pages);
      pages = lookup(base + F::UNIT);
      for (;;) {
        both = both_next;
        lost = lost_next;
        const int next = base + F::UNIT;
        compute(base, next, pages);
        if (next >= v1) break;
        fetch_v(next, pages);
        pages = lookup(next + F::UNIT);
        base = next;
      }
    }
    l = across_rows(l, OpAdd(), true, true);
    if (g == 0) {
      m_of[wave][x16] = m;
      l_of[wave][x16] = l;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < VD; ++i) o_of[wave][x16][(4 * g + r) * VD + i] = o[i][r];
    __syncthreads();
    if (out_there) {
      float m_all = m_of[0][out_q];
#pragma unroll
      for (int w = 1; w < kRowWaves; ++w) m_all = fmaxf(m_all, m_of[w][out_q]);
      float l_all = 0.f, f[VD];
#pragma unroll
      for (int i = 0; i < VD; ++i) f[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) {
        const float k = fast_exp2(m_of[w][out_q] - m_all);
        l_all += k * l_of[w][out_q];
#pragma unroll
        for (int i = 0; i < VD; ++i) f[i] += k * o_of[w][out_q][out_d + i];
      }
      if (part < 0) {
        const float inv = 1.f / l_all;
#pragma unroll
        for (int i = 0; i < VD; ++i) f[i] *= inv;
        store_n<VD>(out, f);
      } else {
        const long long at = SEVERAL ? ((long long)out_token * a.heads + out_head) * a.splits + part : (long long)part * a.part_rows + out_q;
#pragma unroll
        for (int i = 0; i < VD; ++i) a.part[at * D + out_d + i] = f[i];
        if (out_d == 0) {
          a.part_ml[2 * at] = m_all;
          a.part_ml[2 * at + 1] = l_all;
        }
      }
    }
  };

  if constexpr (SEVERAL) {
    const int split = blockIdx.x % a.splits;
    const int kv = blockIdx.x / a.splits % c.kv_heads;
    const RowBlock rb = row_block(c, a.group, kRows, blockIdx.x / a.splits / c.kv_heads);
    if (!rb.any) return;
    const int seq = __builtin_amdgcn_readfirstlane(rb.seq), first_row = __builtin_amdgcn_readfirstlane(rb.first_row);
    const NewTokens t = new_tokens(c, seq);
    Share share = {Visible(), 0, 1};
    if (!t.bad) share = share_of(a, t, first_row, kRows, F::UNIT);
    const int v0 = split * share.size;  // (of a bad sequence paged_join writes the rows, if there are shares)
    if (split < share.parts) attend(seq, t, kv, first_row, share.see, v0, min(share.see.count, v0 + share.size), a.splits > 1 ? split : -1);
  } else {
    const int pieces = a.blocks_per * c.kv_heads;
    int seq = blockIdx.x / pieces, piece = blockIdx.x - seq * pieces;  // a piece to each workgroup
    int u0 = 0, left = 0x7FFFFFFF;                                    // the unit to begin with, units to do
    if (a.even) {
      const EvenPlace p = even_place(a, F::UNIT, blockIdx.x);
      if (p.left == 0) return;
      seq = p.seq;
      piece = p.piece;
      u0 = p.unit;
      left = p.left;
    }
    for (;;) {
      const NewTokens t = new_tokens(c, seq);
      Visible see = {0, 0, 0, 0};
      if (!t.bad && t.past >= 0) see = visible(t.past, t.past, a.window, a.sinks);
      const int units = max(1, (see.count + F::UNIT - 1) / F::UNIT);
      if (u0 >= units) return;  // (only if lengths change under the call)
      const int u1 = units - u0 < left ? units : u0 + left;
      const int part = u0 == 0 && u1 == units ? -1 : 2 * (int)blockIdx.x + (u1 < units);
      attend(seq, t, piece % c.kv_heads, piece / c.kv_heads * kRows, see, u0 * F::UNIT, min(see.count, u1 * F::UNIT), part);
      left -= u1 - u0;
      if (!a.even || left <= 0) return;
      __syncthreads();  // the sums of this piece have been read
      u0 = 0;
      if (++piece == pieces) {
        piece = 0;
        if (++seq >= c.sequences) return;  // (the same)
      }
    }
  }
}

// ---- the shares of a row, added up -------------------------------------------------------------------------------------------------
// WAVES waves take a row, 64 shares at a time: a share's maximum and sum to a lane, then the shares' vectors, 16 bytes to a lane and several
// shares side by side, four of them on their way.  (33 shares of 32 rows: 4.7 us, 12 with a wave that takes one after the other.)
constexpr int kMostSplits = 64;
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a, int unit) {  // unit: that of paged_rows' shares; 0: paged_tiles made them
  constexpr int LANES = D / 4, NG = 64 * WAVES / LANES;  // lanes of a vector, shares side by side
  __shared__ float sums[WAVES == 1 ? 1 : NG][WAVES == 1 ? 1 : D + 4];
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63, in_row = threadIdx.x % (64 * WAVES), x = in_row % LANES, side = in_row / LANES;
  const long long row = (long long)blockIdx.x * (4 / WAVES) + threadIdx.x / (64 * WAVES);
  if (row >= (long long)c.tokens * a.heads) return;
  const int token = __builtin_amdgcn_readfirstlane((int)(row / a.heads)), head = __builtin_amdgcn_readfirstlane((int)(row % a.heads));
  const int seq = c.starts ? sequence_of(c, token) : token;
  if (seq < 0) return;
  const NewTokens t = new_tokens(c, seq);
  if (c.starts && (token < c.starts[seq] || token >= c.starts[seq + 1])) return;  // no sequence has it
  // the row's parts lie `step` places apart from `first` on, but for the last, if `last` is not negative
  long long first = row * a.splits, last = -1;
  int parts = 0, step = 1;
  if (a.even) {
    const EvenShares all = even_shares(a, unit);
    const int g = head % a.group, units = units_of(a, seq, unit);
    int start = 0;
    for (int s = lane; s < seq; s += 64) start += units_of(a, s, unit) * a.blocks_per * c.kv_heads;
    start = wave_sum_i(start) + (g / kRows * c.kv_heads + head / a.group) * units;
    const int w0 = start / all.per, w1 = (start + units - 1) / all.per;
    if (w0 == w1) return;  // one workgroup had it all
    parts = w1 - w0 + 1;
    first = (2ll * w0 + 1) * a.part_rows + g % kRows;
    last = 2ll * w1 * a.part_rows + g % kRows;
    step = 2 * a.part_rows;
  } else if (!t.bad) {
    const int r = (token - t.first) * a.group + head % a.group;
    parts = unit ? share_of(a, t, r / kRows * kRows, kRows, unit).parts : tile_plan(a, t, r / kTileRows * kTileRows).parts;
  }
  const auto place = [&](int p) { return p == parts - 1 && last >= 0 ? last : first + (long long)p * step; };
  f32x4_t f = {0.f, 0.f, 0.f, 0.f};
  float m = -FLT_MAX, l = 0.f;
  for (int p0 = 0; p0 < parts; p0 += 64) {
    const int here = min(64, parts - p0);
    const f32x2_t ml = *(const f32x2_t*)(a.part_ml + 2 * place(p0 + min(lane, here - 1)));
    f32x4_t v[4];
    const auto ask = [&](int p) {  // (before the weights are known)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *(const f32x4_t*)(a.part + place(p0 + min(p + i * NG, here - 1)) * D + 4 * x);
    };
    ask(side);
    const float mine = lane < here ? ml[0] : -FLT_MAX;
    const float m_new = fmaxf(m, wave_max(mine)), shrink = fast_exp2(m - m_new), k = lane < here ? fast_exp2(mine - m_new) : 0.f;
    m = m_new;
    l = l * shrink + wave_sum(lane < here ? k * ml[1] : 0.f);
    f *= shrink;
    for (int p = 0; p < here; p += 4 * NG) {  // (the whole wave: a weight comes from the lane that has it)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int q = p + side + i * NG;
        const float w = __shfl(k, q & 63);
        if (q < here) f += w * v[i];
      }
      if (p + 4 * NG < here) ask(p + 4 * NG + side);
    }
  }
  if constexpr (WAVES == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = across_rows(f[i], OpAdd(), LANES == 16, true);
  } else {
    *(f32x4_t*)&sums[side][4 * x] = f;
    __syncthreads();
    if (side > 0) return;
    f = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NG; ++i) f += *(const f32x4_t*)&sums[i][4 * x];
  }
  if (side > 0) return;
  const float inv = t.bad ? kNan : 1.f / l;
  T* const out = (T*)a.o + token * a.o_stride[0] + head * a.o_stride[1] + 4 * x;
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = f[i] * inv;
  store_n<4>(out, r);
}

// Blocks of `rows` rows, or a few more than there are
int row_blocks(int tokens, int group, int sequences, bool one_each, int rows) {
  return one_each ? sequences * ((group + rows - 1) / rows) : (int)((long long)tokens * group / rows) + sequences;
}
// Several tokens of a sequence: shares of at least `unit` tokens for `groups` workgroups whose rows see at most `most`.  Two workgroups to a compute
// unit are on the chip at once, and as many are wanted (us with 256 / 512 / 1024 / 2048 of them, 32 heads on 8: 512 tokens behind 8192 113 / 92 / 108 / 108,
// over pages of 8 bits 145 / 101 / 119 / 119, 64 behind 8192 33 / 31 / 41 / 39; in fp32 64 behind 4096 94 / 82 / 94 / 118, 256 behind 2000 133 / 133 / 151 / 170).
constexpr int kWantedGroups = 512;
int splits_for(long long groups, long long most, long long unit) {
  const long long want = (kWantedGroups + groups - 1) / groups, units = most / unit;
  return (int)std::max(1ll, std::min({want, units, (long long)kMostSplits}));
}
// The tile form: a share costs each row of the call some writing and reading, so the more rows, the more tokens it has to have (us with shares of
// 128 / 512 / 1024 / 2048 tokens or more, and whole rows, 32 heads on 8: 16 tokens behind 4096 in 4 sequences, 2048 rows, 29 / 31 / 33 / 43, 93; 256 behind 4096, 8192
// rows, 40 / 40 / 44 / 47, 96; 512 alone, 16384 rows, 26 / 18 / 18 / 18, 18, behind 4096 60 / 60 / 60 / 66, 102; 4 x 256 behind 512, 32768 rows, 46 / 46 / 24 / 24, 24, behind
// 1024 54 / 54 / 54 / 35, 35).
constexpr int kRowsPerToken = 16;
long long tokens_of_share(long long rows) { return std::max((long long)kFewestTiles * kTileTokens, rows / kRowsPerToken); }
size_t part_bytes(long long rows, int splits, int d) { return splits > 1 ? (size_t)rows * splits * (d + 2) * 4 : 0; }
// One token of each: workgroups that share the tokens evenly, or 0 where a piece goes to each workgroup: if no piece has more than a unit, or if
// there are two pieces and more for each workgroup on the chip and none can be so long that it runs on alone, or the lengths are too many to be
// scanned by all.  us, a piece to each / even shares, 128 and 256 sequences on 8 K/V heads of d = 128 in tables for 8192 tokens (8 and 4 for a
// piece): one of 8192 beside others of 300 tokens 132 / 47 and 143 / 81, all of 300 32 / 37 and 60 / 71, of 75 to 300 up to 1000 66 / 75 and 122 / 139; in tables for
// 65536: one such beside 500 937 / 94 and 954 / 144.  1024 sequences of 300 on one head 32 / 53.
constexpr int kEvenGroups(int d) { return d == 64 ? 768 : 512; }  // as many as are on the chip at once
constexpr int kLongPiece = 4;          // tokens for each piece of the call
constexpr int kScannedLengths = 512;
constexpr long long kMostUnits = 0x3FFFFFFF;  // (counted in 32 bits)
int even_groups(long long pieces, long long most, int unit, int d, int sequences) {
  const long long units = (most + unit - 1) / unit;
  if (units < 2 || pieces * units > kMostUnits) return 0;
  if (pieces >= 2 * kEvenGroups(d) && (most < kLongPiece * pieces || sequences > kScannedLengths)) return 0;
  return (int)std::min((long long)kEvenGroups(d), pieces * units);
}
size_t even_bytes(int groups, int group, int d) { return (size_t)groups * 2 * std::min(group, kRows) * (d + 2) * 4; }

template <typename T, bool EIGHT, int D>
bool attend(PagedArgs a, void* workspace, size_t bytes, hipStream_t st) {
  typedef RowForm<T, EIGHT, D> F;
  const long long rows = (long long)a.c.tokens * a.heads;
  const bool tiles = a.c.starts && !F::F32;
  a.blocks = row_blocks(a.c.tokens, a.group, a.c.sequences, !a.c.starts, tiles ? kTileRows : kRows);
  a.blocks_per = (a.group + kRows - 1) / kRows;
  a.part_rows = std::min(a.group, kRows);
  const long long groups = (long long)a.blocks * a.c.kv_heads;
  const long long most = std::min((long long)a.c.table_pages << a.c.shift, (long long)a.window + a.sinks + (tiles ? kTileRows : a.c.starts ? kRows : 0));
  a.splits = 1;
  a.even = 0;
  a.part = (float*)workspace;
  unsigned long long grid = (unsigned long long)groups;
  if (!a.c.starts) {
    const int wanted = even_groups(groups, most, F::UNIT, D, a.c.sequences);
    a.even = (int)std::min((unsigned long long)wanted, (unsigned long long)(bytes / even_bytes(1, a.group, D)));
    if (a.even <= std::min(groups, (long long)wanted) / 2) a.even = 0;  // too little room to be of use
    if (a.even) grid = a.even;
    a.part_ml = a.part + 2ll * a.even * a.part_rows * D;
  } else {
    a.splits = splits_for(groups, most, tiles ? tokens_of_share(rows) : F::UNIT);
    while (a.splits > 1 && part_bytes(rows, a.splits, D) > bytes) --a.splits;
    a.part_ml = a.part + rows * a.splits * D;
    grid *= a.splits;
  }
  // four waves to a row (one token of 8000, 32 rows, 15.0 us, 17.9 with one; a chunk of 16, 512 rows, 19.9 and 20.8; 64 tokens of 8000, 2048 rows, 216 and 212)
  const bool few = rows <= 512;
  const unsigned long long join = few ? (unsigned long long)rows : (unsigned long long)(rows + 3) / 4;
  if (!grid_fits(grid, 64 * kRowWaves) || !grid_fits(join, 256)) return false;
  if (tiles) launch_paged_tiles(a, (uint32_t)grid, st);
  else if (!a.c.starts) paged_rows_kernel<T, EIGHT, D, false><<<(uint32_t)grid, 64 * kRowWaves, 0, st>>>(a);
  else if constexpr (F::F32) paged_rows_kernel<T, EIGHT, D, true><<<(uint32_t)grid, 64 * kRowWaves, 0, st>>>(a);
  if (a.splits > 1 || a.even) {
    const int unit = tiles ? 0 : F::UNIT;
    if (few) paged_join_kernel<T, D, 4><<<(uint32_t)join, 256, 0, st>>>(a, unit);
    else paged_join_kernel<T, D, 1><<<(uint32_t)join, 256, 0, st>>>(a, unit);
  }
  return true;
}

template <typename T>
bool attend(const PagedArgs& a, void* workspace, size_t bytes, hipStream_t st) {
  const bool eight = a.c.dtype == A2SF_E4M3;
  if (a.c.d == 128) return eight ? attend<T, true, 128>(a, workspace, bytes, st) : attend<T, false, 128>(a, workspace, bytes, st);
  return eight ? attend<T, true, 64>(a, workspace, bytes, st) : attend<T, false, 64>(a, workspace, bytes, st);
}

}  // namespace

size_t paged_workspace(int tokens, int heads, int kv_heads, int d, int sequences, long long table_tokens) {
  const long long rows = (long long)tokens * heads;
  const auto bytes = [&](int block, long long unit) {
    const long long groups = (long long)row_blocks(tokens, heads / kv_heads, sequences, false, block) * kv_heads;
    return part_bytes(rows, splits_for(groups, table_tokens, unit), d);
  };
  // (of the forms for single tokens that of fp32 has the smaller shares)
  size_t most = std::max(bytes(kRows, 16 * kRowWaves), bytes(kTileRows, tokens_of_share(rows)));
  if (tokens == sequences) {
    const long long pieces = (long long)row_blocks(tokens, heads / kv_heads, sequences, true, kRows) * kv_heads;
    const int unit = 16 * kRowWaves;
    const long long counted = std::min(table_tokens, kMostUnits / pieces * unit);  // (a call under a window may have few enough)
    most = std::max(most, even_bytes(even_groups(pieces, counted, unit, d, sequences), heads / kv_heads, d));
  }
  return most;
}

bool launch_paged_attention(PagedArgs a, int dtype, void* workspace, size_t bytes, hipStream_t st) {
  return dtype == A2SF_F32 ? attend<float>(a, workspace, bytes, st) : attend<bf16_t>(a, workspace, bytes, st);
}

}  // namespace a2sf
