// How the tile form of attention over pages shares out its work (paged_tiles.hip; paged_join of paged_attention.hip follows it).
#pragma once
#include "pages_dev.h"

namespace a2sf {

constexpr int kTileRows = 128;   // query rows of a workgroup
constexpr int kTileTokens = 64;
// Tiles of a share, unless the block has fewer (us with 1 / 2 / 4 / 8 of them, 32 heads on 8: 512 tokens in a table for 65536 34 / 29 / 28 / 31,
// 64 behind 1000 25 / 21 / 22 / 27, four of those 29 / 23 / 24 / 27, 16 x 4 behind 500 22 / 21 / 25 / 28, 512 behind 8192 105 with any)
constexpr int kFewestTiles = 2;

// The tiles of a block of rows: those of the first `sinks` tokens, if they lie apart, then those from token `from` (a multiple of eight, so
// that eight rows are in one page) to the block's newest token.
struct TilePlan {
  int sinks, sink_tiles, from, tiles;
  int per, parts;  // tiles of a share, shares that have any
};
__device__ __forceinline__ TilePlan tile_plan(const PagedArgs& a, const NewTokens& t, int first_row) {
  const int last_row = (int)min((long long)first_row + kTileRows, (long long)t.count * a.group) - 1;
  const int p0 = t.past + first_row / a.group, p1 = t.past + last_row / a.group;
  TilePlan p;
  const int from = first_in_window(p0, a.window);
  p.sinks = min(a.sinks, from);
  p.from = from & ~7;
  p.sink_tiles = (p.sinks + kTileTokens - 1) / kTileTokens;
  if (p.sinks >= p.from) p.from = p.sink_tiles = 0;
  p.tiles = p.sink_tiles + (p1 - p.from) / kTileTokens + 1;
  const int shares = max(1, min(a.splits, p.tiles / kFewestTiles));  // (the table may have room for many more tiles than there are)
  p.per = (p.tiles + shares - 1) / shares;
  p.parts = (p.tiles + p.per - 1) / p.per;
  return p;
}

// The block of a rank: the sequences by their lengths, longer ones first, and in a sequence the blocks from its end, whose rows see most (up
// to 64 sequences, one to a lane; the whole wave comes here).  What is begun last is then short, and blocks that
// run together share their tiles in the caches.
__device__ __forceinline__ RowBlock ranked_block(const PagedArgs& a, int rank) {
  const int lane = threadIdx.x & 63;
  int blocks = 0, len = -1;
  if (lane < a.c.sequences) {
    const NewTokens t = new_tokens(a.c, lane);
    blocks = (int)(((long long)t.count * a.group + kTileRows - 1) / kTileRows);
    len = t.bad ? 0 : t.past + t.count;
  }
  int before = 0;
  for (int s = 0; s < a.c.sequences; ++s) {
    const int other = __builtin_amdgcn_readlane(len, s);
    if (other > len || (other == len && s < lane)) before += __builtin_amdgcn_readlane(blocks, s);
  }
  const unsigned long long here = __ballot(before <= rank && rank < before + blocks);
  if (!here) return {0, 0, false};
  const int seq = __builtin_ctzll(here);
  return {seq, (__builtin_amdgcn_readlane(blocks, seq) - 1 - (rank - __builtin_amdgcn_readlane(before, seq))) * kTileRows, true};
}

void launch_paged_tiles(const PagedArgs& a, uint32_t grid, hipStream_t st);

}  // namespace a2sf
