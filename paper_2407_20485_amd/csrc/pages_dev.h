// Which sequence a token of a call belongs to, what it sees, and where a page's rows lie.  Lengths, starts and tables live on the
// device: whatever they hold, no address leaves the buffers that the caller has described.
#pragma once
#include "a2sf_dev.h"
#include "a2sf_internal.h"

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

// Tokens that positions p0 .. p1 of a sequence see between them: 0 .. sinks - 1 and from .. p1.  They are numbered one after the other.
struct Visible {
  int sinks, from, count;
  __device__ __forceinline__ int token(int i) const { return i < sinks ? i : i - sinks + from; }
};
__device__ __forceinline__ Visible visible(int p0, int p1, int window, int sinks) {
  Visible v;
  v.from = p0 < window ? 0 : p0 - window + 1;
  v.sinks = min(sinks, v.from);
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

}  // namespace a2sf
