// Which sequence a token of a call belongs to, what it sees, and where a page's rows lie.  Lengths, starts and tables live on the
// device: whatever they hold, no address leaves the buffers that the caller has described.
#pragma once
#include "a2sf_dev.h"
#include "a2sf_internal.h"
#include "rows_dev.h"

namespace a2sf {

// The new tokens of a sequence: `count` from token `first` of the call on, at positions past, past + 1 ..
struct NewTokens {
  int first, count, past;
  bool bad;
};
__device__ __forceinline__ NewTokens new_tokens(const PagedCache& c, int seq) {
  NewTokens t;
  const int len = c.len[seq];
  if (c.starts) {
    t.first = c.starts[seq];
    const long long count = (long long)c.starts[seq + 1] - t.first;
    t.count = (int)max(0ll, min(count, (long long)c.tokens));
    t.bad = count < 0 || count > len || t.first < 0 || t.first + count > c.tokens;
  } else {
    t.first = seq;
    t.count = 1;
    t.bad = false;
  }
  t.past = len - t.count;
  t.bad |= len < 0 || (long long)len > (long long)c.table_pages << c.shift;
  return t;
}

// The sequence whose tokens hold token t of the call, if any has it (the caller checks): the number of sequences that start
// at or before t, less one.  t is the same for the whole wave, all of whose lanes come here.
__device__ __forceinline__ int sequence_of(const PagedCache& c, int t) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int s = 0; s < c.sequences; s += 64) before += __popcll(__ballot(s + lane < c.sequences && c.starts[s + lane] <= t));
  return before - 1;
}

// Tokens that positions p0 .. p1 of a sequence see between them: the first `sinks` and those from a position on.  They are numbered one
// after the other, sixteen that start at a multiple of sixteen together, so that such a group is in one page if pages have so many; the
// few that nobody sees are in the numbers below `edge`.
struct Visible {
  int sinks, from, count, edge;  // sinks, from: multiples of sixteen
  __device__ __forceinline__ int token(int i) const { return i < sinks ? i : i - sinks + from; }
};
__device__ __forceinline__ int first_in_window(int p0, int window) { return p0 < window ? 0 : p0 - window + 1; }
__device__ __forceinline__ Visible visible(int p0, int p1, int window, int sinks) {
  Visible v;
  const int from = first_in_window(p0, window);
  v.from = from & ~15;
  v.sinks = (min(sinks, from) + 15) & ~15;
  v.edge = from > 0 ? v.sinks + 16 : 0;
  if (v.sinks >= v.from) {  // nothing between them
    v.from = v.sinks = 0;
    v.edge = from;
  }
  v.count = v.sinks + p1 - v.from + 1;
  return v;
}

// The page that holds a token; page 0 with `bad` set where the table names none of the cache's
__device__ __forceinline__ int page_of(const PagedCache& c, const int32_t* row, int token, bool& bad) {
  const int page = row[token >> c.shift];
  bad = (uint32_t)page >= (uint32_t)c.pages;
  return bad ? 0 : page;
}

// The value that a scale's byte stands for (255 stands for no number, as its values' bytes do too)
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

constexpr float kNan = __builtin_nanf("");

// N neighbouring elements at an element's alignment
typedef uint32_t u32_at2_t __attribute__((aligned(2)));
template <int N>
__device__ __forceinline__ void store_n(bf16_t* p, const float* f) {
  if constexpr (N == 8) {
    store_unit(p, f);
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) ((u32_at2_t*)p)[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
  }
}
template <int N>
__device__ __forceinline__ void store_n(float* p, const float* f) {
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = f[i];
}

// Rows of a sequence's new tokens under one K/V head are counted token by token, the heads of a token next to each other; a block
// has ROWS of them.
struct RowBlock {
  int seq, first_row;  // of the sequence's
  bool any;            // there is such a block
};
// Block b of a call with starts: blocks of one sequence after the other.  The whole wave comes here with the same b.
__device__ __forceinline__ RowBlock row_block(const PagedCache& c, int group, int rows, int b) {
  RowBlock r = {0, 0, false};
  const int lane = threadIdx.x & 63;
  long long before = 0;
  for (int s = 0; s < c.sequences; s += 64) {
    long long n = 0;
    if (s + lane < c.sequences) {
      const long long count = (long long)c.starts[s + lane + 1] - c.starts[s + lane];
      n = (max(0ll, min(count, (long long)c.tokens)) * group + rows - 1) / rows;
    }
    long long upto = n;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
      const long long other = __shfl_up(upto, step);
      if (lane >= step) upto += other;
    }
    const unsigned long long behind = __ballot(before + upto > b);
    if (behind) {
      const int at = __builtin_ctzll(behind);
      r.seq = s + at;
      const long long prior = before + __shfl(upto - n, at);
      r.first_row = (int)(b - prior) * rows;
      r.any = true;
      return r;
    }
    before += __shfl(upto, 63);
  }
  return r;
}
// What the rows of a block see between them, and how it is shared out
struct Share {
  Visible see;
  int size, parts;  // tokens of a share, shares that have any
};
__device__ __forceinline__ Share share_of(const PagedArgs& a, const NewTokens& t, int first_row, int rows, int unit) {
  Share s;
  const int last_row = (int)min((long long)first_row + rows, (long long)t.count * a.group) - 1;
  s.see = visible(t.past + first_row / a.group, t.past + last_row / a.group, a.window, a.sinks);
  const int units = (s.see.count + unit - 1) / unit;
  s.size = (units + a.splits - 1) / a.splits * unit;
  s.parts = (s.see.count + s.size - 1) / s.size;
  return s;
}

}  // namespace a2sf
