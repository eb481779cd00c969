// What the two kernels of np_attn_decode_shared have in common: which groups of rows share how many tokens, and where the first kernel
// (np_attn_shared.cu: the shared tokens, for all rows of a group at once) leaves its results for the second (np_attn_decode.cu: each row's own tokens,
// and the join).
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

struct SharedArgs {
  const int32_t* cu;       // [n_groups + 1]
  const int32_t* tokens;   // [n_groups] that a group shares
  int n_groups;
  int members;             // rows of the call in a block of rows
  int tile_members;        // and in each tile of 128 query rows
  LinePlan* line;
  GroupPlan* plan;         // [n_groups]
  float* row_ml;           // [n][n_heads][2]   maximum (base two) and sum, of rows that one block has done alone
  float* row_o;            // [n][n_heads][HD]
  float* part_ml;          // [2 * blocks][rows of a block][2]   of the others
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
