// What the two ways of np_attn_decode_shared have in common: which groups of rows share how many tokens, and where parts of a row's result meet.  Small
// groups go through np_attn_decode.cu, beside their rows' own tokens; of large ones np_attn_shared.cu does the shared tokens, and leaves them for
// np_attn_rest.cu, which does the rows' own and the join.
#pragma once

#include <stdint.h>

#include "np_attn.h"

namespace npa {

constexpr int kSharedTile = 128;       // tokens of a tile of the first kernel
constexpr int kSharedBlocks = 320;     // its blocks, at most
constexpr int kSharedGroups = 512;     // groups that it keeps in mind, at most
constexpr int kRestBlocks = 640;       // blocks of the second kernel, at most, where it splits rows

// Of a row: where on the line of work its shared tokens' tiles begin, of key-value head 0, and how far it is to the next head's; its first query head's
// place among the rows of a block's part; the tokens that it shares.
struct __align__(32) RowPlan {
  int64_t first_w, step;
  int32_t place, shared;
};
// How the line is dealt out to `blocks` blocks: the first `more` take each + 1 tiles of it, the others each.
struct __align__(32) LinePlan {
  int64_t each, more;
  int32_t blocks;
};

// Where the parts of a (row, query head) meet, and counts of what has arrived, which are zero between calls.  Of one size for all calls, so that
// what one call leaves in a workspace is never another's count.
struct __align__(32) Record {
  float o[2][128];            // sums of the shared tokens and of the row's own
  float ml[2][2];             // their maxima (base two) and sums
  unsigned int count;         // at a key-value head's first query head: parts of the row
  unsigned int pair_count;    // at the first query head of a block of them: pieces of the row's own tokens
  unsigned int group_count;   // in a group's first row, by the number of the block of columns: joined pieces of the shared tokens
  unsigned int unused;
};

struct SharedArgs {
  const int32_t* cu;       // [n_groups + 1]
  const int32_t* tokens;   // [n_groups] that a group shares
  int n_groups;
  int columns;             // (row, query head) pairs of a group and key-value head, about
  Record* records;         // [n][n_heads]
  // large groups: rows of the call in a block of rows, and in each tile of 128 query rows
  int members, tile_members;
  LinePlan* line;
  RowPlan* plan;           // [n]
  float* part_ml;          // [2 * blocks][rows of a block][2]   of blocks that have not done all of a block of rows' tiles (the others: records)
  float* part_o;           // [2 * blocks][rows of a block][HD]
  int part_rows;
  // and of the rows' own tokens: what a block has of a split (row, key-value head, heads)
  float* rest_ml;          // [blocks][8][2]
  float* rest_o;           // [blocks][8][HD]
};

// What is known of a group: the tokens that it shares, its rows [lo, hi) of the call, and the sequence whose pages are read for them.
struct GroupInfo {
  int tokens;
  int16_t lo, hi;
  int seq;
};
__device__ __forceinline__ GroupInfo group_at(const SharedArgs& s, int n, int g) {
  const int lo = min(max(s.cu[g], 0), n), hi = max(lo, min(s.cu[g + 1], n));
  return GroupInfo{s.tokens[g], (int16_t)lo, (int16_t)hi, -1};
}
// By a whole warp: the group's sequence is that of its first row that has one; it shares nothing if there is none, or (NP_KV_S_LENGTH) if its rows do
// not all have that many tokens or they do not fill pages.  Of row i: seqs[i] (-1: none) and lens[i], as the tables say.
__device__ __forceinline__ void check_group(GroupInfo& x, const int16_t* seqs, const int* lens, int max_pages, int shift, int32_t* status) {
  const int lane = threadIdx.x & 31;
  if (x.tokens == 0) return;
  bool good = x.tokens > 0 && (x.tokens & ((1 << shift) - 1)) == 0 && (x.tokens >> shift) <= max_pages;
  for (int i0 = x.lo; i0 < x.hi; i0 += 32) {
    const int i = i0 + lane, seq = i < x.hi ? seqs[i] : -1;
    if (seq >= 0) good &= lens[i] >= x.tokens;
    const uint32_t all = __ballot_sync(0xffffffffu, seq >= 0);
    if (x.seq < 0 && all) x.seq = __shfl_sync(0xffffffffu, seq, __ffs(all) - 1);
  }
  good = __all_sync(0xffffffffu, good);
  if (!good && x.seq >= 0 && lane == 0) atomicOr(status, NP_KV_S_LENGTH);
  if (!good || x.seq < 0) x.tokens = 0;
}

__device__ __forceinline__ int64_t divide_up(int64_t a, int b) { return (a + b - 1) / b; }

}  // namespace npa
