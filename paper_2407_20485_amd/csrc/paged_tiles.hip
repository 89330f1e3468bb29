// Attention of prompts and chunks over keys and values in pages, bf16: a block of 128 query rows against tiles of 64 tokens that come
// through LDS, on the conventions of the prompt kernels (tiles_dev.h, prefill_bf16.hip): S^T = K Q^T and O^T = V^T P^T on the 32 x 32
// matrix instruction, a lane holding one query row and 16 of 32 tokens, an online softmax whose maximum moves only when it has to.
//
// A block's rows are the heads of a K/V head's group, token by token, so a tile of K and V serves all heads of the group at once.
// Probabilities go into the second product as bf16 numbers, each within 2^-8 of itself, or with WIDE as two, its value and what that
// leaves out (2^-17 of it stays out); their sum is of the unrounded ones.  The caller chooses: the second number is a half more matrix
// instructions and three vector instructions a pair (4 prompts of up to 2048 tokens, 32 heads: 111 us without, 136 with it; 16384 tokens under a window of 2048
// 591 and 757, without a window 2145 and 2827; 8192 tokens over pages of 8 bits 643 and 781, of d = 64 345 and 448; a chunk of 512 with 15 single
// tokens 83 and 97).
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "paged_tiles.h"
#include "pages_dev.h"
#include "rows_dev.h"
#include "tiles_dev.h"

namespace a2sf {
namespace {

typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
__device__ __forceinline__ void lds_write16(lds_char* p, const uint4& v) { *reinterpret_cast<lds_u32x4*>(p) = u32x4_t{v.x, v.y, v.z, v.w}; }

// Infinities and NaN among packed bf16 numbers
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; }  // sets the upper bit of their halves
__device__ __forceinline__ uint32_t odd_marks(uint32_t w) {  // 1 for such a number, else 0
  return ((w & 0x7F80u) == 0x7F80u ? 0x3F80u : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0x3F800000u : 0u);
}
__device__ __forceinline__ uint32_t without_odd(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u);
}

// D: head dimension; EIGHT: pages of 8 bits, whose rows are unpacked to bf16 (with their scales) on their way into LDS.
template <int D, bool EIGHT, bool WIDE>
__global__ __launch_bounds__(kThreads, 2) void paged_tiles_kernel(PagedArgs a) {
  constexpr int KK = D / 16, DB = D / 32, ROW = D * 2, kTB = kTile * ROW;
  constexpr int RPL = 512 / D, NL = kTile / (4 * RPL);     // rows of a direct load, loads of a wave
  constexpr int NE = kTile * D / 16 / kThreads;            // EIGHT: 16-byte pieces of a tile per thread
  __shared__ __attribute__((aligned(1024))) char smem[4 * kTB];  // two stages of K, two of V
  const PagedCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  lds_char* const lds = (lds_char*)smem;
  lds_char* const vst = lds + 2 * kTB;

  // K/V heads fastest, so that with a multiple of eight of them a head's blocks are on one die; blocks whose rows see most first
  const int kv = blockIdx.x % c.kv_heads;
  const int split = blockIdx.x / c.kv_heads % a.splits;
  const int rank = (int)(blockIdx.x / c.kv_heads / a.splits);
  const RowBlock rb = c.sequences <= 64 ? ranked_block(a, rank) : row_block(c, a.group, kTileRows, a.blocks - 1 - rank);
  if (!rb.any) return;
  const int seq = __builtin_amdgcn_readfirstlane(rb.seq), first_row = __builtin_amdgcn_readfirstlane(rb.first_row);
  const NewTokens t = new_tokens(c, seq);
  const int rows = (int)min((long long)t.count * a.group - first_row, (long long)kTileRows);  // of this block
  // where a row of the block stands in the call
  const auto place = [&](int r, int& token, int& head) -> bool {
    const int row = first_row + r;
    token = t.first + row / a.group;
    head = kv * a.group + row % a.group;
    return r < rows && token >= 0 && token < c.tokens;
  };
  if (t.bad) {
    if (a.splits == 1)
      for (int e = tid; e < rows * D; e += kThreads) {
        int token, head;
        if (place(e / D, token, head)) store_one((bf16_t*)a.o + token * a.o_stride[0] + head * a.o_stride[1] + e % D, kNan);
      }
    return;
  }
  const TilePlan plan = tile_plan(a, t, first_row);
  if (split >= plan.parts) return;
  const int p0 = t.past + first_row / a.group, p1 = t.past + (first_row + rows - 1) / a.group;
  // this wave's rows see positions up to those of its first and last row
  const int wrow = wave * 32;
  const bool any_rows = wrow < rows;
  const int w0 = t.past + (first_row + min(wrow, rows - 1)) / a.group, w1 = t.past + (first_row + min(wrow + 31, rows - 1)) / a.group;
  const int pos = t.past + (first_row + min(wrow + l32, rows - 1)) / a.group;  // of this lane's row

  // Q fragments (B operand): lane (query l32, half h) holds Q[query][16kk + 8h .. +7]
  uint4 qf[KK];
  {
    int token, head;
    const bool there = place(wrow + l32, token, head);
    const bf16_t* q = (const bf16_t*)a.q + (there ? token * a.q_stride[0] + head * a.q_stride[1] : 0);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const u32x4_t v = there ? *(const u32x4_at2_t*)(q + kk * 16 + h * 8) : u32x4_t{0, 0, 0, 0};
      qf[kk] = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
  // per-lane LDS byte offsets inside a K / V tile
  int koff[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) koff[kk] = l32 * ROW + (((2 * kk + h) ^ k_swizzle<D>(l32)) << 4);
  int voff[DB];
  {
    const int i = lane & 15, r = i >> 2, qd = i & 3, gq = (lane >> 4) & 1;
    const int cl = 2 * gq + (qd >> 1), vs = v_swizzle<D>(4 * h + r);  // key = 8*x + 4h + r
#pragma unroll
    for (int db = 0; db < DB; ++db) voff[db] = (4 * h + r) * ROW + ((((4 * db + cl) ^ vs)) << 4) + (qd & 1) * 8;
  }

  // ---- tiles and their rows
  const int32_t* const table = c.table + seq * c.table_stride;
  const char* const kbase = c.k + kv * c.stride[1];
  const char* const vbase = c.v + kv * c.stride[1];
  const int mask_in_page = (1 << c.shift) - 1;
  const int t_first = split * plan.per, t_end = min(plan.tiles, t_first + plan.per);
  const auto base_of = [&](int i) { return i < plan.sink_tiles ? i * kTile : plan.from + (i - plan.sink_tiles) * kTile; };
  const auto last_of = [&](int i) { return i < plan.sink_tiles ? plan.sinks - 1 : p1; };  // newest token of the tile that a row sees
  // the page of token base + lane; behind the last token that one's
  const auto lookup = [&](int i) -> int {
    i = min(i, plan.tiles - 1);
    return table[min(base_of(i) + lane, last_of(i)) >> c.shift];
  };
  // Rows go in groups of eight that start at multiples of eight tokens, so with pages of eight or more a group is in one page and its
  // address is formed by scalar instructions (a direct load takes four or eight rows); smaller pages, and rows very far from each
  // other, take an address per lane.
  const bool grouped = c.shift >= 3 && c.stride[2] < (1ll << 28);
  const int lrow = wave * RPL + lane / (D / 8);            // + 4 * RPL * u
  const int kchunk = (lane % (D / 8)) ^ k_swizzle<D>(lrow), vchunk = (lane % (D / 8)) ^ v_swizzle<D>(lrow);
  const uint32_t in_group = (uint32_t)(lane / (D / 8)) * (uint32_t)(grouped ? c.stride[2] : 0);
  const auto fetch = [&](int i, int pages, lds_char* kt, lds_char* vt) {  // bf16
    const int base = base_of(i);
    const int sound = (uint32_t)pages < (uint32_t)c.pages ? pages : 0;
    if (grouped) {
#pragma unroll
      for (int u = 0; u < NL; ++u) {
        const uint32_t to = (u * 4 + wave) * 1024;
        const int r = (u * 4 + wave) * RPL;
        const long long at = (long long)__builtin_amdgcn_readlane(sound, r) * c.stride[0] + (long long)((base + r) & mask_in_page) * c.stride[2];
        dma16(kbase + at, in_group + kchunk * 16, (uint32_t)(size_t)kt + to);
        dma16(vbase + at, in_group + vchunk * 16, (uint32_t)(size_t)vt + to);
      }
    } else {
#pragma unroll 1
      for (int u = 0; u < NL; ++u) {
        const uint32_t to = (u * 4 + wave) * 1024;
        const int r = u * 4 * RPL + lrow;
        const long long at = (long long)__shfl(sound, r) * c.stride[0] + (long long)((base + r) & mask_in_page) * c.stride[2];
        dma16_at(kbase + at + kchunk * 16, (uint32_t)(size_t)kt + to);
        dma16_at(vbase + at + vchunk * 16, (uint32_t)(size_t)vt + to);
      }
    }
  };
  uint4 kraw[EIGHT ? NE : 1], vraw[EIGHT ? NE : 1];
  uint32_t both[EIGHT ? NE : 1];
  const auto request = [&](int i, int pages) {  // 8 bits
    const int base = base_of(i);
    int thread = tid;
    asm volatile("" : "+v"(thread));  // (what is formed of it is not kept over the loop: 8192 tokens 755 us, 679 so)
    const int sound = (uint32_t)pages < (uint32_t)c.pages ? pages : 0;
#pragma unroll
    for (int u = 0; u < NE; ++u) {
      const int r = (u * kThreads + thread) / (D / 16), col = thread % (D / 16);
      const long long page = __shfl(sound, r), in_page = (base + r) & mask_in_page;
      const long long at = page * c.stride[0] + in_page * c.stride[2] + col * 16;
      const long long s = page * c.scale_stride[0] + kv * c.scale_stride[1] + in_page * c.scale_stride[2];
      kraw[u] = load16(kbase + at);
      vraw[u] = load16(vbase + at);
      both[u] = c.k_scales[s] | (uint32_t)c.v_scales[s] << 16;
    }
  };
  const auto deliver = [&](lds_char* kt, lds_char* vt) {
    int thread = tid;
    asm volatile("" : "+v"(thread));  // (the same)
#pragma unroll
    for (int u = 0; u < NE; ++u) {
      const int r = (u * kThreads + thread) / (D / 16), col = thread % (D / 16);
      // (a power of two: values in bf16 are exact, from its subnormal numbers to where its range ends)
      const auto unpack = [&](const uint4& x, uint32_t byte, uint4& lo, uint4& hi) {
        const float scale = scale_value(byte);
        const auto two = [&](uint32_t w, auto half) {
          return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, decltype(half)::value));
        };
        constexpr std::false_type lower{};
        constexpr std::true_type upper{};
        lo = make_uint4(two(x.x, lower), two(x.x, upper), two(x.y, lower), two(x.y, upper));
        hi = make_uint4(two(x.z, lower), two(x.z, upper), two(x.w, lower), two(x.w, upper));
      };
      uint4 lo, hi;
      unpack(kraw[u], both[u] & 255u, lo, hi);
      lds_write16(kt + r * ROW + (((2 * col) ^ k_swizzle<D>(r)) << 4), lo);
      lds_write16(kt + r * ROW + (((2 * col + 1) ^ k_swizzle<D>(r)) << 4), hi);
      unpack(vraw[u], both[u] >> 16, lo, hi);
      lds_write16(vt + r * ROW + (((2 * col) ^ v_swizzle<D>(r)) << 4), lo);
      lds_write16(vt + r * ROW + (((2 * col + 1) ^ v_swizzle<D>(r)) << 4), hi);
    }
  };

  float m = -FLT_MAX, lsum = 0.f;
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;

  const auto logits = [&](const lds_char* kt, f32x16 (&s)[2]) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
    constexpr int NF = 2 * KK;  // fragment i = (kk, kb): the two key blocks alternate, so that no
    uint4 fr[NF];               // matrix op waits for the one before it
#pragma unroll
    for (int i = 0; i < kPrefetch; ++i) fr[i] = lds_read16(kt + (i & 1) * 32 * ROW + koff[i >> 1]);
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      if (i + kPrefetch < NF) fr[i + kPrefetch] = lds_read16(kt + ((i + kPrefetch) & 1) * 32 * ROW + koff[(i + kPrefetch) >> 1]);
      s[i & 1] = mfma_bf16(fr[i], qf[i >> 1], s[i & 1]);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, kPrefetch, 0);
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i + kPrefetch < NF) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
  };
  constexpr int kNumbers = WIDE ? 2 : 1;  // of a probability
  const auto add_values = [&](const lds_char* vt, const uint32_t (&pf)[kNumbers][16]) {  // O += V^T P
    constexpr int NF = DB * 4;  // fragment i = (kb, tt, db), db fastest
    uint2 lo[NF], hi[NF];
    const auto vread = [&](int i, uint2& x, uint2& y) {
      const lds_char* p = vt + ((i / DB) * 16) * ROW + voff[i % DB];
      x = lds_read_tr16(p);
      y = lds_read_tr16(p + 8 * ROW);
    };
#pragma unroll
    for (int i = 0; i < kPrefetch; ++i) vread(i, lo[i], hi[i]);
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      if (i + kPrefetch < NF) vread(i + kPrefetch, lo[i + kPrefetch], hi[i + kPrefetch]);
      const int w = 4 * (i / DB);
#pragma unroll
      for (int p = 0; p < kNumbers; ++p)
        oacc[i % DB] = mfma_bf16(make_uint4(lo[i].x, lo[i].y, hi[i].x, hi[i].y), make_uint4(pf[p][w], pf[p][w + 1], pf[p][w + 2], pf[p][w + 3]),
                                 oacc[i % DB]);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * kPrefetch, 0);
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, kNumbers, 0);
      if (i + kPrefetch < NF) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
  };
  // A tile with tokens that some rows see and others do not: a probability of 0 keeps no infinity or NaN of V out of a row.  Such values are
  // taken out of the tile, and the rows that see one of them get NaN for its dimension: those for which a product of marks is above 0.
  // The whole workgroup comes here.
  const auto separate = [&](bool need, auto hidden, lds_char* vt) {
    lds_char* const mine = vt + tid * (kTB / kThreads);
    uint32_t odd = 0;
#pragma unroll
    for (int j = 0; j < kTB / kThreads / 16; ++j) {
      const uint4 x = lds_read16(mine + j * 16);
      odd |= odd_bits(x.x) | odd_bits(x.y) | odd_bits(x.z) | odd_bits(x.w);
    }
    if (!__syncthreads_or(odd & 0x80008000u)) return;
    if (need) {
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        f32x16 marks;
#pragma unroll
        for (int i = 0; i < 16; ++i) marks[i] = 0.f;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {  // 16 tokens each
          const lds_char* p = vt + kt * 16 * ROW + voff[db];
          const uint2 x = lds_read_tr16(p), y = lds_read_tr16(p + 8 * ROW);
          uint32_t seen[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            seen[j] = (hidden(kt / 2, 8 * (kt % 2) + 2 * j) ? 0u : 0x3F80u) | (hidden(kt / 2, 8 * (kt % 2) + 2 * j + 1) ? 0u : 0x3F800000u);
          marks = mfma_bf16(make_uint4(odd_marks(x.x), odd_marks(x.y), odd_marks(y.x), odd_marks(y.y)),
                            make_uint4(seen[0], seen[1], seen[2], seen[3]), marks);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (marks[i] > 0.f) oacc[db][i] = kNan;
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kTB / kThreads / 16; ++j) {
      const uint4 x = lds_read16(mine + j * 16);
      lds_write16(mine + j * 16, make_uint4(without_odd(x.x), without_odd(x.y), without_odd(x.z), without_odd(x.w)));
    }
    __syncthreads();
  };

  const auto tile_step = [&](int i, unsigned long long bad, const lds_char* kt, lds_char* vt) {
    const int base = base_of(i);
    const bool sink_tile = i < plan.sink_tiles;
    const bool need = any_rows && (sink_tile || (base <= w1 && (w0 - (base + kTile - 1) < a.window || base < a.sinks)));
    const bool uneven = sink_tile ? base + kTile > plan.sinks : base + kTile - 1 > p0 || p1 - base >= a.window;
    const int limit = sink_tile ? plan.sinks - 1 : pos;
    // whether this lane's row does not see element e of key block kb (no branches: the comparisons of all 32 stand side by side)
    const auto hidden = [&](int kb, int e) -> bool {
      const int token = base + kb * 32 + 8 * (e >> 2) + 4 * h + (e & 3);
      return (token > limit) | ((pos - token >= a.window) & (token >= a.sinks));
    };
    f32x16 s[2];
    if (need) {
      logits(kt, s);
      if (bad) {  // a page that is none of the cache's
        const uint32_t of_lane[2] = {(uint32_t)bad >> (4 * h), (uint32_t)(bad >> 32) >> (4 * h)};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            s[kb][e] = of_lane[kb] & (1u << (8 * (e >> 2) + (e & 3))) ? kNan : s[kb][e];
      }
      if (uneven) {
        if (sink_tile || p1 - base < a.window) {  // no row's window ends here
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              s[kb][e] = base + kb * 32 + 8 * (e >> 2) + 4 * h + (e & 3) > limit ? -INFINITY : s[kb][e];
        } else {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kb][e] = hidden(kb, e) ? -INFINITY : s[kb][e];
        }
      }
    }
    if (uneven) separate(need, hidden, vt);
    if (!need) return;
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
    mx = across_rows(mx, OpMax(), false, true) * a.scale_log2e;
    if (__any(mx > m + 8.f)) {
      const float m_new = fmaxf(m, mx), shrink = fast_exp2(m - m_new);
      lsum *= shrink;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[db][e] *= shrink;
      m = m_new;
    }
    uint32_t pf[kNumbers][16];
    float rs = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float e0 = fast_exp2(fmaf(s[j >> 3][(2 * j) & 15], a.scale_log2e, -m));
      const float e1 = fast_exp2(fmaf(s[j >> 3][(2 * j + 1) & 15], a.scale_log2e, -m));
      rs += e0;
      rs += e1;
      const uint32_t both = pack_bf16(e0, e1);
      pf[0][j] = both;
      if constexpr (WIDE) pf[1][j] = pack_bf16(e0 - __uint_as_float(both << 16), e1 - __uint_as_float(both & 0xFFFF0000u));
    }
    lsum += rs;
    add_values(vt, pf);
  };

  int pages = lookup(t_first);
  unsigned long long bad = __ballot((uint32_t)pages >= (uint32_t)c.pages), bad_next = 0;
  if constexpr (EIGHT) {
    request(t_first, pages);
    deliver(lds, vst);
  } else {
    fetch(t_first, pages, lds, vst);
  }
  pages = lookup(t_first + 1);
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(qf[kk].x));  // waited for here, not in the loop
  wait_vm_barrier<0>();
  for (int t0 = t_first; t0 < t_end; t0 += 2) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {  // stage b: LDS offsets are immediates
      const int i = t0 + b;
      if (i >= t_end) break;
      // the stages of the tile before are free: every wave passed the barrier that ended its step
      if (i + 1 < t_end) {
        bad_next = __ballot((uint32_t)pages >= (uint32_t)c.pages);
        if constexpr (EIGHT) request(i + 1, pages);
        else fetch(i + 1, pages, lds + (1 - b) * kTB, vst + (1 - b) * kTB);
        pages = lookup(i + 2);
      }
      tile_step(i, bad, lds + b * kTB, vst + b * kTB);
      if constexpr (EIGHT)
        if (i + 1 < t_end) deliver(lds + (1 - b) * kTB, vst + (1 - b) * kTB);
      bad = bad_next;
      wait_vm_barrier<0>();  // the next tile for every wave of the workgroup
    }
  }

  const float l = across_rows(lsum, OpAdd(), false, true);
  if (a.splits > 1) {
    int token, head;
    if (place(wrow + l32, token, head)) {
      const long long at = ((long long)token * a.heads + head) * a.splits + split;
      float* const part = a.part + at * D;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4)
          *(f32x4_t*)(part + 32 * db + 8 * i4 + 4 * h) =
              f32x4_t{oacc[db][4 * i4], oacc[db][4 * i4 + 1], oacc[db][4 * i4 + 2], oacc[db][4 * i4 + 3]};
      if (h == 0) {
        a.part_ml[2 * at] = m;
        a.part_ml[2 * at + 1] = l;
      }
    }
    return;
  }
  // The accumulator layout gives a lane four neighbouring dimensions of one row at a time: each wave turns its 32 x D block round through a
  // strip of LDS of its own (free after the loop's last barrier) and stores whole rows.
  lds_char* const strip = lds + wave * 32 * ROW;
  const float inv = 1.0f / l;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      uint2 w;
      w.x = pack_bf16(oacc[db][4 * i4 + 0] * inv, oacc[db][4 * i4 + 1] * inv);
      w.y = pack_bf16(oacc[db][4 * i4 + 2] * inv, oacc[db][4 * i4 + 3] * inv);
      // row l32, elements 32db + 8*i4 + 4h .. +3  ->  chunk 4db + i4, half h
      lds_write8(strip + l32 * ROW + (((4 * db + i4) ^ k_swizzle<D>(l32)) << 4) + 8 * h, w);
    }
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int u = 0; u < 32 / RPL; ++u) {
    const int r = RPL * u + lane / (D / 8), ch = lane % (D / 8);
    const uint4 x = lds_read16(strip + r * ROW + ((ch ^ k_swizzle<D>(r)) << 4));
    int token, head;
    if (place(wrow + r, token, head))
      *(u32x4_at2_t*)((bf16_t*)a.o + token * a.o_stride[0] + head * a.o_stride[1] + ch * 8) = u32x4_t{x.x, x.y, x.z, x.w};
  }
}

}  // namespace

template <bool WIDE>
void tiles(const PagedArgs& a, uint32_t grid, hipStream_t st) {
  const bool eight = a.c.dtype == A2SF_E4M3;
  if (a.c.d == 128) {
    if (eight) paged_tiles_kernel<128, true, WIDE><<<grid, kThreads, 0, st>>>(a);
    else paged_tiles_kernel<128, false, WIDE><<<grid, kThreads, 0, st>>>(a);
  } else {
    if (eight) paged_tiles_kernel<64, true, WIDE><<<grid, kThreads, 0, st>>>(a);
    else paged_tiles_kernel<64, false, WIDE><<<grid, kThreads, 0, st>>>(a);
  }
}

void launch_paged_tiles(const PagedArgs& a, uint32_t grid, hipStream_t st) {
  if (a.wide) tiles<true>(a, grid, st);
  else tiles<false>(a, grid, st);
}

}  // namespace a2sf
