// What the kernels of np_attn_decode_shared have in common: which groups of rows share how many tokens, and where the kernel of the shared tokens
// (np_attn_shared.cu) leaves its results for that of the rows' own (np_attn_decode.cu), which does both where groups are small.
#pragma once

#include <stdint.h>

#include "np_attn.h"

namespace npa {

constexpr int kSharedTile = 128;       // tokens of a tile of the first kernel
constexpr int kSharedBlocks = 320;     // its blocks, at most
constexpr int kSharedSlotRows = 256;   // rows of a block's partial result, at most

// Of a group: where its tiles begin on the line of work, its first row, and its blocks of rows.
struct __align__(16) GroupPlan {
  int64_t first_w;
  int32_t row0, row_blocks;
};
// How the line is dealt out: the first `more` blocks take each + 1 tiles of it, the others each.
struct __align__(16) LinePlan {
  int64_t each, more;
};

// Where the parts of a (row, query head) meet, and counts of what has arrived, which are zero between calls.  Of one size for all calls, so that
// what one call leaves in a workspace is never another's count.
struct __align__(32) Record {
  float o[2][128];            // sums of the shared tokens and of the row's own
  float ml[2][2];             // their maxima (base two) and sums
  unsigned int count;         // at a key-value head's first query head: parts of the row
  unsigned int pair_count;    // at the first query head of a block of them: joined pieces of the row's own tokens
  unsigned int group_count;   // in a group's first row, by the number of the block of columns: joined pieces of the shared tokens
  unsigned int unused;
};

struct SharedArgs {
  const int32_t* cu;       // [n_groups + 1]
  const int32_t* tokens;   // [n_groups] that a group shares
  int n_groups;
  bool together;           // one kernel for both
  int columns;             // together: (row, query head) pairs of a group and key-value head, about
  Record* records;         // [n][n_heads]
  // the two kernels apart: rows of the call in a block of rows, and in each tile of 128 query rows
  int members, tile_members;
  LinePlan* line;
  GroupPlan* plan;         // [n_groups]
  float* part_ml;          // [2 * blocks][rows of a block][2]   of blocks that have not done all of a block of rows' tiles (the others: records)
  float* part_o;           // [2 * blocks][rows of a block][HD]
  int part_rows;
};

// Rows [lo, hi) of a group.
__device__ __forceinline__ void group_rows(const SharedArgs& s, int n, int g, int* lo, int* hi) {
  *lo = min(max(s.cu[g], 0), n);
  *hi = max(*lo, min(s.cu[g + 1], n));
}

// By a whole warp: the tokens that group g shares; 0 where it has no row with a sequence, or (NP_KV_S_LENGTH) where its rows do not all have
// that many or they do not fill pages.  *seq: the sequence of its first row that has one.
__device__ __forceinline__ int group_tokens(const SharedArgs& s, int g, int lo, int hi, const int32_t* seqs, const int32_t* lens, int max_seqs, int max_pages,
                                            int shift, int32_t* status, int* seq) {
  const int lane = threadIdx.x & 31, tokens = s.tokens[g];
  *seq = -1;
  if (tokens == 0 || lo == hi) return 0;
  bool good = tokens > 0 && (tokens & ((1 << shift) - 1)) == 0 && (tokens >> shift) <= max_pages;
  for (int i0 = lo; i0 < hi; i0 += 32) {
    const int i = i0 + lane, q = i < hi ? (seqs ? seqs[i] : i) : -1;
    const bool has = q >= 0 && q < max_seqs;
    if (has) good &= lens[q] >= tokens;
    const uint32_t all = __ballot_sync(0xffffffffu, has);
    if (*seq < 0 && all) *seq = __shfl_sync(0xffffffffu, q, __ffs(all) - 1);
  }
  good = __all_sync(0xffffffffu, good);
  if (*seq < 0) return 0;
  if (!good) {
    if (lane == 0) atomicOr(status, NP_KV_S_LENGTH);
    return 0;
  }
  return tokens;
}

__device__ __forceinline__ int64_t divide_up(int64_t a, int b) { return (a + b - 1) / b; }

}  // namespace npa
