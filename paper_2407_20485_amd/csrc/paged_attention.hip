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
// ---- up to 16 rows, straight from memory ------------------------------------------------------------------------------------------
// S^T = K Q^T with the tokens as rows of the result: lane (g, q) = (l / 16, l % 16) gets the logits of query row q with tokens 4g .. 4g + 3
// of 16, which is how the second product, O^T = V^T P^T, takes its P^T -- if its k runs over the tokens in that order, which is free to
// choose: lane (g, x) of V^T then has tokens 4g .. of each 16, and of those the D / 16 values from dimension x * D / 16 on, whole 16 rows
// of V being read by 16 lanes side by side; a pair of tokens' values of one dimension is one byte permutation.
// So neither P nor V goes through LDS.  Q and K take their dimensions in the order in which K's 16 bytes per lane come.
// bf16: P goes into the product as two bf16 numbers, its value and what that leaves out (2^-17 of it stays out): the matrix pipe has room.
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
__global__ __launch_bounds__(64 * kRowWaves, 2) void paged_rows_kernel(PagedArgs a) {
  typedef RowForm<T, EIGHT, D> F;
  constexpr int H = F::H, NK = F::NK, VD = F::VD, VW = F::VW, E = F::E, TT = F::TOKENS;
  __shared__ float o_of[kRowWaves][kRows][D + 4];
  __shared__ float m_of[kRowWaves][kRows], l_of[kRowWaves][kRows];
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, x16 = lane & 15;
  const int split = blockIdx.x % a.splits;
  const int kv = blockIdx.x / a.splits % c.kv_heads;
  const RowBlock rb = row_block(c, a.group, kRows, blockIdx.x / a.splits / c.kv_heads);
  if (!rb.any) return;
  const int seq = __builtin_amdgcn_readfirstlane(rb.seq), first_row = __builtin_amdgcn_readfirstlane(rb.first_row);
  const NewTokens t = new_tokens(c, seq);
  // this lane's query row
  const long long row = (long long)first_row + x16;
  const int i_row = (int)min(row / a.group, (long long)t.count - 1), head = kv * a.group + (int)(row % a.group);
  const int token_row = t.first + (int)(row / a.group);
  const bool there = row < (long long)t.count * a.group && token_row >= 0 && token_row < c.tokens;
  // the row that this thread writes: 16 threads to a row
  const long long out_row = (long long)first_row + (threadIdx.x >> 4);
  const int out_token = t.first + (int)(out_row / a.group), out_head = kv * a.group + (int)(out_row % a.group);
  const bool out_there = out_row < (long long)t.count * a.group && out_token >= 0 && out_token < c.tokens;
  T* const out = (T*)a.o + (out_there ? out_token * a.o_stride[0] + out_head * a.o_stride[1] : 0) + (threadIdx.x & 15) * VD;
  if (t.bad || t.past < 0) {  // (with shares paged_join writes these rows)
    if (a.splits == 1 && out_there) {
      float f[VD];
#pragma unroll
      for (int i = 0; i < VD; ++i) f[i] = t.bad ? kNan : 0.f;
      store_n<VD>(out, f);
    }
    return;
  }
  const Share share = share_of(a, t, first_row, kRows, F::UNIT);
  if (split >= share.parts) return;
  const Visible see = share.see;
  const int v0 = split * share.size, v1 = min(see.count, v0 + share.size);
  const int pos = t.past + i_row;

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

  struct Tile {
    uint4 k[H][NK];
    uint32_t v[E][VW];
    uint32_t scales[EIGHT ? E : 1];  // k's byte, then v's
    bool bad[E];
  };
  const int32_t* const table = c.table + seq * c.table_stride;
  const char* const kbase = c.k + kv * c.stride[1];
  const char* const vbase = c.v + kv * c.stride[1];
  const int mask = (1 << c.shift) - 1;
  // the page of token number v0 + .. of a tile, one token to a lane (H = 1: twice)
  const auto lookup = [&](int base) -> int {
    const int i = min(base + lane % TT, v1 - 1);
    return table[see.token(i) >> c.shift];
  };
  const auto fetch = [&](int base, int pages, Tile& T_) {
    // an element's place among the tile's tokens -> its row
    const auto at = [&](int i, bool& bad) -> long long {
      const int page = __shfl(pages, i);
      bad = (uint32_t)page >= (uint32_t)c.pages;
      const int token = see.token(min(base + i, v1 - 1));
      return (long long)(bad ? 0 : page) * c.stride[0] + (long long)(token & mask) * c.stride[2];
    };
    bool ignored;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const char* p = kbase + at(h * 16 + x16, ignored) + g * 16;
#pragma unroll
      for (int j = 0; j < NK; ++j) T_.k[h][j] = load16(p + j * 64);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const char* p = vbase + at(e / 4 * 16 + g * 4 + e % 4, T_.bad[e]) + x16 * (VD * F::BYTES);
      if constexpr (VW == 1) {
        T_.v[e][0] = *(const uint32_t*)p;
      } else if constexpr (VW == 2) {
        const uint2 v = *(const uint2*)p;
        T_.v[e][0] = v.x;
        T_.v[e][1] = v.y;
      } else {
#pragma unroll
        for (int j = 0; j < VW; j += 4) {
          const uint4 v = load16(p + 4 * j);
          T_.v[e][j] = v.x;
          T_.v[e][j + 1] = v.y;
          T_.v[e][j + 2] = v.z;
          T_.v[e][j + 3] = v.w;
        }
      }
    }
    if constexpr (EIGHT) {
      const int i = lane % TT, page = pages;
      const int token = see.token(min(base + i, v1 - 1));
      const long long p = (long long)((uint32_t)page < (uint32_t)c.pages ? page : 0) * c.scale_stride[0] + kv * c.scale_stride[1] +
                          (long long)(token & mask) * c.scale_stride[2];
      const int both = c.k_scales[p] | c.v_scales[p] << 8;
#pragma unroll
      for (int e = 0; e < E; ++e) T_.scales[e] = (uint32_t)__shfl(both, e / 4 * 16 + g * 4 + e % 4);
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

  const auto compute = [&](int base, Tile& T_) {
    f32x4_t s[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      s[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        const uint4 k = T_.k[h][j];
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
    // V as bf16, two dimensions to a register, or as fp32
    uint32_t vb[F::F32 ? 1 : E][VD / 2];
    float vf[F::F32 ? E : 1][VD];
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        const uint32_t w = T_.v[e][j];
        if constexpr (F::F32 && EIGHT) {
          const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
          vf[e][4 * j] = lo[0];
          vf[e][4 * j + 1] = lo[1];
          vf[e][4 * j + 2] = hi[0];
          vf[e][4 * j + 3] = hi[1];
        } else if constexpr (F::F32) {
          vf[e][j] = __uint_as_float(w);
        } else if constexpr (EIGHT) {
          vb[e][2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false));
          vb[e][2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true));
        } else {
          vb[e][j] = w;
        }
      }
    }
    const auto clear = [&](int e) {
#pragma unroll
      for (int j = 0; j < (F::F32 ? VD : VD / 2); ++j) {
        if constexpr (F::F32) vf[e][j] = 0.f;
        else vb[e][j] = 0;
      }
    };
    float y[E], top = -FLT_MAX;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float k = a.scale_log2e;
      if constexpr (EIGHT) k *= scale_value(T_.scales[e] & 255u);
      y[e] = s[e / 4][e % 4] * k;
      if (T_.bad[e]) {
        y[e] = kNan;
        clear(e);
      }
    }
    if (base + TT > v1) {  // the last tile: what is behind the end counts nothing
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (base + e / 4 * 16 + g * 4 + e % 4 >= v1) {
          y[e] = -INFINITY;
          clear(e);
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
      if constexpr (EIGHT) p[e] = p[e] == 0.f ? 0.f : p[e] * scale_value(T_.scales[e] >> 8);
    }
    if constexpr (!F::F32) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
        lo[i] = pack_bf16(p[2 * i] - __uint_as_float(hi[i] << 16), p[2 * i + 1] - __uint_as_float(hi[i] & 0xFFFF0000u));
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
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int i = 0; i < VD; ++i) o[i] = mfma16(vf[e][i], p[e], o[i]);
      }
    }
  };

  // tile after tile, the next one's rows on their way and the pages of the one after that
  int base = v0 + wave * TT;
  if (base < v1) {
    Tile A, B;
    int pages = lookup(base);
    fetch(base, pages, A);
    pages = lookup(base + F::UNIT);
    for (;;) {
      int next = base + F::UNIT;
      if (next < v1) {
        fetch(next, pages, B);
        pages = lookup(next + F::UNIT);
      }
      compute(base, A);
      if (next >= v1) break;
      base = next;
      next = base + F::UNIT;
      if (next < v1) {
        fetch(next, pages, A);
        pages = lookup(next + F::UNIT);
      }
      compute(base, B);
      if (next >= v1) break;
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
  if (!out_there) return;
  const int q = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * VD;
  float m_all = m_of[0][q];
#pragma unroll
  for (int w = 1; w < kRowWaves; ++w) m_all = fmaxf(m_all, m_of[w][q]);
  float l_all = 0.f, f[VD];
#pragma unroll
  for (int i = 0; i < VD; ++i) f[i] = 0.f;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    const float k = fast_exp2(m_of[w][q] - m_all);
    l_all += k * l_of[w][q];
#pragma unroll
    for (int i = 0; i < VD; ++i) f[i] += k * o_of[w][q][d0 + i];
  }
  if (a.splits == 1) {
    const float inv = 1.f / l_all;
#pragma unroll
    for (int i = 0; i < VD; ++i) f[i] *= inv;
    store_n<VD>(out, f);
  } else {
    const long long at = ((long long)out_token * a.heads + out_head) * a.splits + split;
#pragma unroll
    for (int i = 0; i < VD; ++i) a.part[at * D + d0 + i] = f[i];
    if (d0 == 0) {
      a.part_ml[2 * at] = m_all;
      a.part_ml[2 * at + 1] = l_all;
    }
  }
}

// ---- the shares of a row, added up -------------------------------------------------------------------------------------------------
// A wave takes a row: a share's maximum and sum to a lane, then the shares' vectors one after the other.
constexpr int kMostSplits = 64;
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a, int unit) {  // unit: that of paged_rows' shares; 0: paged_tiles made them
  constexpr int N = D / 64;
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 63;
  const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= (long long)c.tokens * a.heads) return;
  const int token = __builtin_amdgcn_readfirstlane((int)(at / a.heads)), head = __builtin_amdgcn_readfirstlane((int)(at % a.heads));
  const int seq = c.starts ? sequence_of(c, token) : token;
  if (seq < 0) return;
  const NewTokens t = new_tokens(c, seq);
  if (c.starts && (token < c.starts[seq] || token >= c.starts[seq + 1])) return;  // no sequence has it
  T* const out = (T*)a.o + token * a.o_stride[0] + head * a.o_stride[1] + lane * N;
  float f[N];
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = t.bad ? kNan : 0.f;
  if (!t.bad && t.past >= 0) {
    const int row = (token - t.first) * a.group + head % a.group;
    const int parts = unit ? share_of(a, t, row / kRows * kRows, kRows, unit).parts : tile_plan(a, t, row / kTileRows * kTileRows).parts;
    const float* part = a.part + at * a.splits * D + lane * N;
    float m = -FLT_MAX, l = 0.f;
    if (lane < parts) {
      m = a.part_ml[2 * (at * a.splits + lane)];
      l = a.part_ml[2 * (at * a.splits + lane) + 1];
    }
    const float k = fast_exp2(m - wave_max(m));
    const float inv = 1.f / wave_sum(k * l);
#pragma unroll 8
    for (int p = 0; p < parts; ++p) {
      const float w = wave_broadcast(k, p);
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] += w * part[(long long)p * D + i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] *= inv;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) store_one(out + i, f[i]);
}

// Blocks of `rows` rows, or a few more than there are
int row_blocks(int tokens, int group, int sequences, bool one_each, int rows) {
  return one_each ? sequences * ((group + rows - 1) / rows) : (int)((long long)tokens * group / rows) + sequences;
}
// Shares for `groups` workgroups whose rows see at most `most` tokens
constexpr int kWantedGroups = 2048, kWantedTileGroups = 1024;
int splits_for(long long groups, long long most, int unit, int wanted) {
  const long long want = (wanted + groups - 1) / groups, units = (most + unit - 1) / unit;
  return (int)std::max(1ll, std::min({want, units, (long long)kMostSplits}));
}
constexpr int kFewestTiles = 4;  // of a share
size_t part_bytes(long long rows, int splits, int d) { return splits > 1 ? (size_t)rows * splits * (d + 2) * 4 : 0; }

template <typename T, bool EIGHT, int D>
bool attend(PagedArgs a, void* workspace, size_t bytes, hipStream_t st) {
  typedef RowForm<T, EIGHT, D> F;
  const long long rows = (long long)a.c.tokens * a.heads;
  const bool tiles = a.c.starts && !F::F32;
  a.blocks = row_blocks(a.c.tokens, a.group, a.c.sequences, !a.c.starts, tiles ? kTileRows : kRows);
  const long long groups = (long long)a.blocks * a.c.kv_heads;
  const long long most = std::min((long long)a.c.table_pages << a.c.shift, (long long)a.window + a.sinks + (tiles ? kTileRows : a.c.starts ? kRows : 0));
  a.splits = tiles ? splits_for(groups, most, kFewestTiles * kTileTokens, kWantedTileGroups) : splits_for(groups, most, F::UNIT, kWantedGroups);
  while (a.splits > 1 && part_bytes(rows, a.splits, D) > bytes) --a.splits;
  a.part = (float*)workspace;
  a.part_ml = a.part + rows * a.splits * D;
  const unsigned long long grid = (unsigned long long)groups * a.splits, join = (unsigned long long)(rows + 3) / 4;
  if (!grid_fits(grid, 64 * kRowWaves) || !grid_fits(join, 256)) return false;
  if (tiles) launch_paged_tiles(a, (uint32_t)grid, st);
  else if (!a.c.starts) paged_rows_kernel<T, EIGHT, D, false><<<(uint32_t)grid, 64 * kRowWaves, 0, st>>>(a);
  else if constexpr (F::F32) paged_rows_kernel<T, EIGHT, D, true><<<(uint32_t)grid, 64 * kRowWaves, 0, st>>>(a);
  if (a.splits > 1) paged_join_kernel<T, D><<<(uint32_t)join, 256, 0, st>>>(a, tiles ? 0 : F::UNIT);
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
  const auto bytes = [&](bool one_each, int block, int unit, int wanted) {
    const long long groups = (long long)row_blocks(tokens, heads / kv_heads, sequences, one_each, block) * kv_heads;
    return part_bytes(rows, splits_for(groups, table_tokens, unit, wanted), d);
  };
  // (of the forms for single tokens that of fp32 has the smaller shares)
  size_t most = std::max(bytes(false, kRows, 16 * kRowWaves, kWantedGroups), bytes(false, kTileRows, kFewestTiles * kTileTokens, kWantedTileGroups));
  if (tokens == sequences) most = std::max(most, bytes(true, kRows, 16 * kRowWaves, kWantedGroups));
  return most;
}

bool launch_paged_attention(PagedArgs a, int dtype, void* workspace, size_t bytes, hipStream_t st) {
  return dtype == A2SF_F32 ? attend<float>(a, workspace, bytes, st) : attend<bf16_t>(a, workspace, bytes, st);
}

}  // namespace a2sf
