// Attention of one new token for each row of groups that share their first tokens (np_attn_decode_shared), the shared tokens' part: for all
// (row, query head) pairs of a group and key-value head at once
//
//   m = max_j s_j,   l = sum_j 2^(s_j - m),   O = sum_j 2^(s_j - m) v_j,   s_j = scale * log2(e) * q . k_j     over the shared tokens j
//
// in fp32; the rows' own tokens and the join are the second kernel's (np_attn_rest.cu).
//
// The shared keys and values are read once for up to 256 such pairs, so with few of them the cache's bytes bound the kernel, and with many the
// two matrix products.  They are the products of np_attn_prompt without its mask: tiles of 128 pairs against 128 tokens on the
// 5th-generation tensor cores, scores and accumulators in tensor memory, a softmax warp's lane to a row.
//
// * A tile's rows are pairs (row of the call, query head), rows outermost; one tiled TMA copy brings them.  Keys and values come a page's rows at a
//   time, up to sixteen copies to a tile; a lane of the loading warp each.
// * All (group, key-value head, block of rows, tile of tokens) form one line, of which each block takes an equal stretch.  What a block has
//   of a block of rows goes to the workspace: straight to the rows' places where it has all of their tiles.  Where those are is worked out by the first
//   block alone, for the second kernel.
// * One tile to a block, two blocks to an SM: while one does its softmax, the other has the tensor cores and its copies are under way.
//   Two tiles share keys and values where groups have more rows than fill one.
// * Weights are the sum of two terms of the rows' type, as in np_attn_decode.cu, so that a row's result does not hang on how many others its group has:
//   against 64 bits the last case below is off by 1.66e-3 (bf16; the rounding of the result alone), with one term by 2.31e-3.  The second term lies where
//   the second half of the scores was and is half a product more: 69.0 us in place of 61.9.
// * Tokens come in sixteens that are there or not (pages outside the pool, the end of the last tile); those that are not get scores of -inf
//   and values of 0.
//
// Measured, both kernels (pages of 64 scattered over the pool): 64 rows, 64 heads of 128 over 8, that share 32768 tokens and have one of their own, 131 us,
// 0.53 PFLOP/s; that share 8192 and have up to 200, 68.4 us; 4 such rows that share 8192 tokens, 30.0 us.  Of the 68.4 us this kernel takes some 34: 6.5 until
// the first scores are there, 3.4 for each tile of 256 rows by 128 tokens (2.2 at the rate of a large product), 3 to store.
//
// Every wait is bounded; after a time-out all roles leave, the block meets and tensor memory is released.
#include <algorithm>
#include <cmath>

#include "np_attn.h"
#include "np_attn_groups.cuh"
#include "np_attn_tc.cuh"
#include "np_device.cuh"
#include "np_internal.h"
#include "np_pipe.cuh"

namespace npa {
namespace {

constexpr int kWaitPolls = 1 << 26;  // that a wait may take, a second or two

struct Args {
  const char* cache;  // of the layer
  const int32_t* table;
  const int32_t* lens;
  const int32_t* seqs;
  int32_t* status;
  SharedArgs shared;
  int n, n_heads, n_kv_heads, group;
  int shift, n_pages, max_seqs, max_pages;
  int64_t page_bytes;
  float scale2;  // scale * log2(e)
};

template <int HD, int kTiles>
struct Shape {
  static constexpr int kHalves = HD / 64;                        // 64 values = 128 bytes: one swizzle row
  static constexpr uint32_t kHalfBytes = kRows * 128;            // a tile's rows of one half
  static constexpr uint32_t kTileBytes = kHalves * kHalfBytes;
  static constexpr int kStages = 2 * kTiles * (128 / HD);        // K0 V0 K1 V1 ...
  static constexpr size_t kSmem = (kTiles + kStages) * (size_t)kTileBytes + 1024;
  static constexpr int kSoftmaxWarps = 4 * kTiles, kMmaWarp = kSoftmaxWarps, kLoadWarp = kMmaWarp + 1;
  static constexpr int kThreads = 32 * kSoftmaxWarps + 128;      // the last two warps have nothing to do
  static constexpr int kColumns = kTiles * 256;                  // of tensor memory: scores, then accumulators
};

// Tiles that a block takes, at least, of those of one block of rows: more blocks would each do less, but what every one leaves for the join is as
// large.  64 rows of 64 heads over 8 that share 512, 2048 or 4096 tokens: 33.9, 42.7 and 47.6 us with four (33.6, 45.7 and 49.6 with one, 33.9, 46.7
// and 51.1 with six); 4 rows that share 2048 or 8192: 25.9 and 30.1 (21.5 and 31.3; 31.8 and 35.2).
constexpr int kFewestTiles = 4;

// keys or values of a page's rows: (64 values, rows of a page's heads, halves of head_dim, keys and values, pages)
__device__ __forceinline__ void tma_load_page(void* dst, const CUtensorMap* map, int row, int half, int kv, int page, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(
                   npp::smem_addr(dst)),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(half), "r"(kv), "r"(page), "r"(npp::smem_addr(bar))
               : "memory");
}

// Tiles [t0, t1) of a block of rows.
struct Piece {
  int kvh, row0, rows, tokens, t0, t1;   // its first row of the call, how many there are
  bool whole;
  const int32_t* pages;
};
// The line of work, in shared memory.
struct Groups {
  int64_t end[kSharedGroups];  // tiles of the groups up to and including this one
  int tokens[kSharedGroups];
  int16_t lo[kSharedGroups], hi[kSharedGroups], seq[kSharedGroups];
};
struct Line {
  const Args& a;
  const Groups& groups;
  int64_t w, end;  // what is left of this block's stretch
  int g;
  // false: nothing is left
  __device__ __forceinline__ bool next(Piece& p) {
    if (w >= end) return false;
    while (groups.end[g] <= w) ++g;
    const int64_t first = g ? groups.end[g - 1] : 0;
    const int lo = groups.lo[g], hi = groups.hi[g];
    p.tokens = groups.tokens[g];
    const int tiles = (p.tokens + kRows - 1) / kRows, blocks = (hi - lo + a.shared.members - 1) / a.shared.members;
    const int64_t item = (w - first) / tiles;
    p.t0 = (int)(w - first - item * tiles);
    p.t1 = (int)min((int64_t)tiles, p.t0 + (end - w));
    w += p.t1 - p.t0;
    p.whole = p.t0 == 0 && p.t1 == tiles;
    p.kvh = (int)(item / blocks);
    p.row0 = lo + (int)(item - (int64_t)p.kvh * blocks) * a.shared.members;
    p.rows = min(a.shared.members, hi - p.row0);
    p.pages = a.table + (size_t)groups.seq[g] * a.max_pages;
    return true;
  }
};

// The page of a lane's sixteen tokens of tile j (lanes 0 to 7); -1: none.
__device__ __forceinline__ int page_of(const Args& a, const Piece& p, int j, int lane) {
  const int64_t tok = (int64_t)j * kRows + lane * 16;
  return lane < 8 && j < p.t1 && tok < p.tokens ? p.pages[tok >> a.shift] : -1;
}

// Rows whose O is not finite though their sum is, by their warp: what the values make infinite or NaN is so (weights are above 0).  mine: a
// lane's row's O.
template <bool kBf16, int HD>
__device__ __noinline__ void mend_rows(const Args& a, const Piece& p, uint32_t rows, float* mine, int lane) {
  constexpr int N = HD / 32;
  int odd[N];  // 1 a NaN, 2 inf, 4 -inf
#pragma unroll
  for (int i = 0; i < N; ++i) odd[i] = 0;
  const int64_t head_bytes = (int64_t)(HD * 2) << a.shift;
  const char* v = a.cache + (a.n_kv_heads + p.kvh) * head_bytes + lane * 2;
  const int64_t last = min((int64_t)p.t1 * kRows, (int64_t)p.tokens);
  for (int64_t j = (int64_t)p.t0 * kRows; j < last; ++j) {
    const int pg = p.pages[j >> a.shift];
    if ((unsigned)pg >= (unsigned)a.n_pages) continue;
    const char* row = v + pg * a.page_bytes + (j & ((1 << a.shift) - 1)) * (HD * 2);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float x = widen<kBf16>(*reinterpret_cast<const uint16_t*>(row + i * 64));
      if (not_finite(x)) odd[i] |= x == INFINITY ? 2 : x == -INFINITY ? 4 : 1;
    }
  }
  __syncwarp();  // the rows are stored
  for (; rows; rows &= rows - 1) {
    float* o = reinterpret_cast<float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), __ffs(rows) - 1)) + lane;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (odd[i]) __stcg(o + i * 32, odd[i] == 2 ? INFINITY : odd[i] == 4 ? -INFINITY : __uint_as_float(0x7fffffffu));
  }
}

template <bool kBf16, int HD, int kTiles>
__global__ void __launch_bounds__(Shape<HD, kTiles>::kThreads, 3 - kTiles)
k_attn_shared(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ Args a) {
  using S = Shape<HD, kTiles>;
  extern __shared__ __align__(1024) unsigned char tsm[];
  __shared__ Groups s_groups;
  __shared__ __align__(8) uint64_t full[S::kStages], empty[S::kStages], q_full, q_empty, s_full[kTiles], p_half[kTiles], p_full[kTiles], o_full[kTiles], o_empty[kTiles];
  __shared__ uint32_t s_tmem;
  __shared__ int s_ok;     // 0: a wait has run out
  __shared__ int s_items;  // (group, key-value head, block of rows) that share anything
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int n_groups = a.shared.n_groups;
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(tsm) + 1023) & ~(uintptr_t)1023);
  unsigned char* q_sm = base;
  unsigned char* ring = base + kTiles * S::kTileBytes;
  if (tid == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      npp::mbar_init(&full[s], 1);
      npp::mbar_init(&empty[s], 1);
    }
    npp::mbar_init(&q_full, 1);
    npp::mbar_init(&q_empty, 1);
    for (int i = 0; i < kTiles; ++i) {
      npp::mbar_init(&s_full[i], 1);
      npp::mbar_init(&p_half[i], 4);
      npp::mbar_init(&p_full[i], 4);
      npp::mbar_init(&o_full[i], 1);
      npp::mbar_init(&o_empty[i], 4);
    }
    npp::fence_barrier_init();
    s_ok = 1;
    s_items = 0;
  }
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();

  // ---- the line of work.  Rows' sequences and lengths lie where the queries will be.
  int* const lens = reinterpret_cast<int*>(q_sm);
  int16_t* const seqs = reinterpret_cast<int16_t*>(q_sm + NP_KV_MAX_SEQS * 4);
  for (int i = tid; i < a.n; i += S::kThreads) {
    const int seq = a.seqs ? a.seqs[i] : i;
    const bool known = seq >= 0 && seq < a.max_seqs;
    if (seq >= a.max_seqs && blockIdx.x == 0) atomicOr(a.status, NP_KV_S_SEQ);
    seqs[i] = (int16_t)(known ? seq : -1);
    lens[i] = known ? a.lens[seq] : 0;
  }
  for (int g = tid; g < n_groups; g += S::kThreads) {
    const GroupInfo x = group_at(a.shared, a.n, g);
    s_groups.tokens[g] = x.tokens;
    s_groups.lo[g] = x.lo;
    s_groups.hi[g] = x.hi;
  }
  __syncthreads();
  auto tiles_in = [](int tokens) { return (tokens + kRows - 1) / kRows; };
  for (int g = wid; g < n_groups; g += S::kThreads / 32) {
    GroupInfo x = {s_groups.tokens[g], s_groups.lo[g], s_groups.hi[g], -1};
    check_group(x, seqs, lens, a.max_pages, a.shift, a.status);
    __syncwarp();
    if (lane == 0) {
      const int items = (x.hi - x.lo + a.shared.members - 1) / a.shared.members * a.n_kv_heads;
      s_groups.end[g] = (int64_t)tiles_in(x.tokens) * items;
      if (x.tokens) atomicAdd(&s_items, items);
      s_groups.tokens[g] = x.tokens;
      s_groups.seq[g] = (int16_t)x.seq;
    }
  }
  __syncthreads();
  if (wid == 0) {
    int64_t run = 0;
    for (int g0 = 0; g0 < n_groups; g0 += 32) {
      int64_t inc = g0 + lane < n_groups ? s_groups.end[g0 + lane] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      if (g0 + lane < n_groups) s_groups.end[g0 + lane] = run + inc;
      run += __shfl_sync(0xffffffffu, inc, 31);
    }
  }
  __syncthreads();
  const int64_t W = s_groups.end[n_groups - 1];
  const int G = (int)min((int64_t)gridDim.x, max(divide_up(W, kFewestTiles), (int64_t)s_items));
  const int64_t each = G ? W / G : 0, more = W - each * G;
  if (blockIdx.x == 0) {  // for the join
    if (tid == 0) *a.shared.line = LinePlan{each, more, G};
    for (int i = tid; i < a.n; i += S::kThreads) a.shared.plan[i] = RowPlan{0, 0, 0, 0};
    __syncthreads();
    for (int g = wid; g < n_groups; g += S::kThreads / 32) {
      const int lo = s_groups.lo[g], tokens = s_groups.tokens[g], tiles = tiles_in(tokens);
      const int blocks = (s_groups.hi[g] - lo + a.shared.members - 1) / a.shared.members;
      if (tokens == 0) continue;
      for (int i = lo + lane; i < s_groups.hi[g]; i += 32) {
        const int block = (i - lo) / a.shared.members, in_block = i - lo - block * a.shared.members, tile = in_block / a.shared.tile_members;
        if (seqs[i] >= 0)
          a.shared.plan[i] = RowPlan{(g ? s_groups.end[g - 1] : 0) + (int64_t)block * tiles, (int64_t)blocks * tiles,
                                     tile * kRows + (in_block - tile * a.shared.tile_members) * a.group, tokens};
      }
    }
  }
  if ((int)blockIdx.x >= G) return;
  Line line = {a, s_groups, blockIdx.x * each + min((int64_t)blockIdx.x, more), 0, 0};
  line.end = line.w + each + (blockIdx.x < more ? 1 : 0);
  npp::fence_proxy_async();  // copies will write over what the block has read
  if (wid == S::kLoadWarp && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_kv) : "memory");
  }
  if (wid == S::kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(npp::smem_addr(&s_tmem)), "r"(S::kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  // true: the phase is complete; false: this or another wait of the block has run out
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    int polls = 0;
#pragma unroll 1
    while (!npp::mbar_try_wait(bar, parity)) {
      if (*static_cast<volatile int*>(&s_ok) == 0) return false;
      if (++polls >= kWaitPolls) {
        *static_cast<volatile int*>(&s_ok) = 0;
        atomicOr(a.status, NP_KV_S_TIMEOUT);
      }
    }
    return true;
  };
  // the same by whole warps: all lanes go on, or none does
  auto wait_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
  // rows of a tile: none in the second where they all fit the first
  auto tiles_of = [&](const Piece& p) { return kTiles == 2 && p.rows > a.shared.tile_members ? 2 : 1; };
  // which sixteens of a tile's tokens are there
  auto seen_of = [&](int page) { return __ballot_sync(0xffffffffu, (unsigned)page < (unsigned)a.n_pages) & 0xffu; };

  if (wid >= S::kMmaWarp) {
   fewer_registers<kTiles>();
   if (wid == S::kLoadWarp) {
    // ------------------------------ loads ------------------------------
    int stage = 0;
    uint32_t use = 0, n = 0;
    Piece p;
    bool ok = true;
    const int box = min(1 << a.shift, kRows), lead = box / 16 - 1;  // tokens of a copy; lanes of one, less one
    for (; ok && line.next(p); ++n) {
      ok = wait_all(&q_empty, (n & 1u) ^ 1u);
      if (!ok) break;
      const int tiles = tiles_of(p);
      if (lane == 0) {
        npp::mbar_expect_tx(&q_full, (uint32_t)tiles * S::kHalves * 128 * a.group * a.shared.tile_members);
        for (int i = 0; i < tiles; ++i)
          for (int h = 0; h < S::kHalves; ++h)
            tma_load_3d(q_sm + i * S::kTileBytes + h * S::kHalfBytes, &map_q, h * 64, p.kvh * a.group, p.row0 + i * a.shared.tile_members, &q_full);
      }
      __syncwarp();
      int page = page_of(a, p, p.t0, lane);
      for (int j = p.t0; j < p.t1 && ok; ++j) {
        const uint32_t seen = seen_of(page);
        const bool wanted = lane < 8 && j * (int64_t)kRows + lane * 16 < p.tokens;
        if (wanted && !(seen >> lane & 1u)) atomicOr(a.status, NP_KV_S_PAGE);
        const int now = page;
        page = page_of(a, p, j + 1, lane);
        const bool mine = (lane & lead) == 0 && (seen >> lane & 1u) && lane < 8;
        for (int kv = 0; kv < 2; ++kv) {
          ok = wait_all(&empty[stage], (use & 1u) ^ 1u);
          if (!ok) break;
          if (lane == 0) npp::mbar_expect_tx(&full[stage], (uint32_t)__popc(seen) * 16 * 128 * S::kHalves);
          __syncwarp();
          if (mine)
            for (int h = 0; h < S::kHalves; ++h)
              tma_load_page(ring + stage * S::kTileBytes + h * S::kHalfBytes + lane * 16 * 128, &map_kv,
                            (p.kvh << a.shift) + (int)(((int64_t)j * kRows + lane * 16) & ((1 << a.shift) - 1)), h, kv, now, &full[stage]);
          __syncwarp();
          if (++stage == S::kStages) {
            stage = 0;
            ++use;
          }
        }
      }
    }
    if (lane == 0 && *static_cast<volatile int*>(&s_ok) == 0) {  // after a time-out nobody else waits for the copies
      uint32_t patience = npp::kSpinLimit;
      npp::drain_ring(full, S::kStages, stage, use & 1u, patience);
      npp::wait_landed(&q_full, n & 1u, patience);
      if (n > 0) npp::wait_landed(&q_full, (n & 1u) ^ 1u, patience);
    }
   } else if (wid == S::kMmaWarp) {
    // ------------------------------ products ------------------------------
    // The whole warp goes through the loop and one lane issues, as in np_attn_prompt.cu.
    const uint32_t fmt = kBf16 ? 1u : 0u;
    const uint32_t common = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(kRows >> 4) << 24);
    const uint32_t id_s = common | ((uint32_t)(kRows >> 3) << 17), id_o = common | (1u << 16) | ((uint32_t)(HD >> 3) << 17);
    const uint64_t q_desc = smem_desc(npp::smem_addr(q_sm), 16), k_desc = smem_desc(npp::smem_addr(ring), 16),
                   v_desc = smem_desc(npp::smem_addr(ring), S::kHalfBytes);
    auto scores = [&](int i, uint32_t st) {
      const uint64_t qd = q_desc + (uint32_t)i * (S::kTileBytes >> 4), kd = k_desc + st * (S::kTileBytes >> 4);
#pragma unroll
      for (int k = 0; k < HD / 16; ++k) {
        const uint32_t off = ((k >> 2) * S::kHalfBytes + (k & 3) * 32) >> 4;
        mma_ss(tmem + i * kRows, qd + off, kd + off, id_s, k > 0);
      }
      commit(&s_full[i]);
    };
    // both terms of sixteen tokens' weights times their values
    auto weighted = [&](uint32_t d_o, uint32_t d_s, uint64_t vd, int k, uint32_t acc) {
      mma_ts(d_o, d_s + k * 8, vd + k * 128, id_o, acc);
      mma_ts(d_o, d_s + kRows / 2 + k * 8, vd + k * 128, id_o, 1u);
    };
    uint32_t ld = 0, p_cnt[kTiles] = {}, o_cnt[kTiles] = {};  // loads, softmax steps and results so far
    auto wait_load = [&](uint32_t l) { return wait_all(&full[l % S::kStages], (l / S::kStages) & 1u); };
    Piece p;
    bool ok = true;
    for (uint32_t n = 0; ok && line.next(p); ++n) {
      const int tiles = tiles_of(p), steps = p.t1 - p.t0;
      int page = page_of(a, p, p.t0, lane);
      ok = wait_all(&q_full, n & 1u) && wait_load(ld);
      if (!ok) break;
      fence_after();
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          if (i < tiles) scores(i, ld % S::kStages);
        commit(&empty[ld % S::kStages]);
        if (steps == 1) commit(&q_empty);
      }
      __syncwarp();
      for (int j = 0; j < steps && ok; ++j) {
        const uint32_t lv = ld + 2 * j + 1, lk = lv + 1, sv = lv % S::kStages, sk = lk % S::kStages;
        const bool more = j + 1 < steps;
        const uint32_t seen = seen_of(page);
        page = page_of(a, p, p.t0 + j + 1, lane);
        ok = wait_load(lv) && (!more || wait_load(lk));
        if (ok && seen != 0xffu) {  // values that are not there: zero, whatever lies in their place
#pragma unroll
          for (int h = 0; h < S::kHalves; ++h)
            for (uint32_t e = lane * 16; e < S::kHalfBytes; e += 32 * 16)
              if (!(seen >> (e >> 11) & 1u)) *reinterpret_cast<uint4*>(ring + sv * S::kTileBytes + h * S::kHalfBytes + e) = make_uint4(0, 0, 0, 0);
          npp::fence_proxy_async();
          __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          if (i >= tiles || !ok) continue;
          if (j == 0) ok = wait_all(&o_empty[i], (o_cnt[i]++ & 1u) ^ 1u);  // the rows before have been read out of the accumulators
          const uint32_t par = p_cnt[i]++ & 1u, d_s = tmem + i * kRows, d_o = tmem + kTiles * kRows + i * HD;
          const uint64_t vd = v_desc + sv * (S::kTileBytes >> 4);
          ok = ok && wait_all(&p_half[i], par);
          if (!ok) continue;
          fence_after();
          if (elect_one()) {  // the first 64 tokens
#pragma unroll
            for (int k = 0; k < kRows / 32; ++k) weighted(d_o, d_s, vd, k, (j | k) > 0);
          }
          __syncwarp();
          ok = wait_all(&p_full[i], par);
          if (!ok) continue;
          fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = kRows / 32; k < kRows / 16; ++k) weighted(d_o, d_s, vd, k, 1u);
            if (more) scores(i, sk);
            else commit(&o_full[i]);
          }
          __syncwarp();
        }
        if (ok && elect_one()) {
          commit(&empty[sv]);
          if (more) commit(&empty[sk]);
          if (j + 2 == steps) commit(&q_empty);
        }
        __syncwarp();
      }
      ld += 2 * steps;
    }
   }
  } else {
    more_registers<kTiles>();
    // ------------------------------ softmax of a tile, and what is left of it ------------------------------
    const int i = wid >> 2, row = (wid & 3) * 32 + lane;
    const int in_tile = row / a.group, in_group = row - in_tile * a.group;
    const uint32_t lanes = tmem + ((uint32_t)((wid & 3) * 32) << 16), ts = lanes + i * kRows, to = lanes + kTiles * kRows + i * HD;
    uint32_t s_cnt = 0, o_cnt = 0;
    auto arrive = [&](uint64_t* bar) {
      wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) npp::mbar_arrive(bar);
    };
    Piece p;
    bool ok = true;
    while (ok && line.next(p)) {
      if (i >= tiles_of(p)) continue;
      const int member = i * a.shared.tile_members + in_tile;
      const bool valid = in_tile < a.shared.tile_members && member < p.rows;  // the other rows hold anything, and have no say
      float m = -INFINITY, l = 0.f;
      int page = page_of(a, p, p.t0, lane);
      for (int j = p.t0; j < p.t1; ++j) {
        const uint32_t seen = seen_of(page);
        page = page_of(a, p, j + 1, lane);
        ok = wait_all(&s_full[i], s_cnt++ & 1u);
        if (!ok) break;
        fence_after();
        uint32_t s[kRows];
#pragma unroll
        for (int c = 0; c < kRows; c += 32) tm_ld32(ts + c, s, c);
        wait_ld(s);
        if (seen != 0xffu) {
#pragma unroll
          for (int c = 0; c < kRows; ++c)
            if (!(seen >> (c >> 4) & 1u)) s[c] = __float_as_uint(-INFINITY);
        }
        // the first half's exponentials beside the maximum, on the assumption that it has not grown much (np_attn_prompt.cu)
        float part = 0.f, now, sc = a.scale2;
        bool fast = false;
        if (j > p.t0) {
          part = softmax_half<kBf16, 0, true>(s, a.scale2, m, ts);
          now = row_max(s) * a.scale2;
          fast = __all_sync(0xffffffffu, !valid || (now <= m + kGrow && fabsf(m) <= kLarge && now < INFINITY));
        } else {
          now = row_max(s) * a.scale2;
        }
        float use = m;
        if (!fast) {
          // a NaN makes the maximum NaN, and with it the row; an infinite score does, too (inf - inf)
          now = max3(m, now, now == INFINITY ? __uint_as_float(0x7fffffffu) : -INFINITY);
          if (j == p.t0) {
            m = now;
          } else if (__any_sync(0xffffffffu, valid && !(now <= m + kGrow))) {
            const float f = exp2_fast(m - (now == -INFINITY ? 0.f : now));
            m = now;
            l *= f;
#pragma unroll 1
            for (int c = 0; c < HD; c += 16) {
              uint32_t o[16];
              tm_ld16(to + c, o);
              wait_ld(o);
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
              tm_st16(to + c, o);
            }
          }
          use = m == -INFINITY ? 0.f : m;
          if (__any_sync(0xffffffffu, valid && fabsf(use) > kLarge)) {
#pragma unroll
            for (int c = 0; c < kRows; ++c) s[c] = __float_as_uint(__uint_as_float(s[c]) * sc);
            sc = 1.f;
          }
          part = softmax_half<kBf16, 0, true>(s, sc, use, ts);
        }
        arrive(&p_half[i]);
        l += part + softmax_half<kBf16, kRows / 2, true>(s, sc, use, ts);
        arrive(&p_full[i]);
      }
      if (ok) ok = wait_all(&o_full[i], o_cnt++ & 1u);
      if (!ok) break;
      // ---- the partial result
      fence_after();
      Record* const record = a.shared.records + ((int64_t)(p.row0 + member) * a.n_heads + p.kvh * a.group + in_group);
      const int64_t at = (int64_t)(2 * blockIdx.x + (p.t0 == 0)) * a.shared.part_rows + i * kRows + row;
      float* const part_o = p.whole ? record->o[0] : a.shared.part_o + at * HD;
      float* const part_ml = p.whole ? record->ml[0] : a.shared.part_ml + at * 2;
      uint32_t big = 0;
#pragma unroll 1
      for (int c = 0; c < HD; c += 32) {
        uint32_t o[32];
        tm_ld32(to + c, o, 0);
        wait_ld(o);
        if (c + 32 == HD) {  // the accumulators may be written again
          fence_before();
          __syncwarp();
          if (lane == 0) npp::mbar_arrive(&o_empty[i]);
        }
        if (!valid) continue;
#pragma unroll
        for (int x = 0; x < 32; ++x) {
          if (l == 0.f) o[x] = 0;  // nothing but scores of -inf
          big = max(big, o[x] & 0x7fffffffu);
        }
#pragma unroll
        for (int x = 0; x < 32; x += 8) {
          uint32_t v[8];
#pragma unroll
          for (int y = 0; y < 8; ++y) v[y] = o[x + y];
          store32(part_o + c + x, v);
        }
      }
      if (valid) *reinterpret_cast<float2*>(part_ml) = make_float2(m, l);
      const uint32_t odd = __ballot_sync(0xffffffffu, valid && big >= 0x7f800000u && !not_finite(l));
      if (odd) mend_rows<kBf16, HD>(a, p, odd, part_o, lane);
    }
  }
  fence_before();
  __syncthreads();
  if (wid == S::kMmaWarp) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kColumns) : "memory");
  }
}

// A layer of the cache as (64 values, rows of a page's heads, halves of head_dim, keys and values, pages); a box is one half of up to 128
// rows of a page.
bool make_map(CUtensorMap* map, const Args& a, int hd) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t row = (cuuint64_t)hd * 2, rows = (cuuint64_t)a.n_kv_heads << a.shift;
  const cuuint64_t dims[5] = {64, rows, (cuuint64_t)hd / 64, 2, (cuuint64_t)a.n_pages};
  const cuuint64_t strides[4] = {row, 128, rows * row, 2 * rows * row};
  const cuuint32_t box[5] = {64, (cuuint32_t)std::min(1 << a.shift, kRows), 1, 1, 1}, estr[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 5, const_cast<char*>(a.cache), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool kBf16, int HD, int kTiles>
cudaError_t launch(const CUtensorMap& q, const CUtensorMap& kv, const Args& a, int sms, cudaStream_t s) {
  using S = Shape<HD, kTiles>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = npi::allow_shared(reinterpret_cast<const void*>(k_attn_shared<kBf16, HD, kTiles>), &done);
  if (e != cudaSuccess) return e;
  const unsigned blocks = (unsigned)std::min((3 - kTiles) * sms, kSharedBlocks / kTiles);
  return launch_early(k_attn_shared<kBf16, HD, kTiles>, dim3(blocks), S::kThreads, S::kSmem, s, q, kv, a);
}
template <bool kBf16>
cudaError_t launch(const CUtensorMap& q, const CUtensorMap& kv, const Args& a, int hd, int tiles, int sms, cudaStream_t s) {
  if (hd == 128) return tiles == 2 ? launch<kBf16, 128, 2>(q, kv, a, sms, s) : launch<kBf16, 128, 1>(q, kv, a, sms, s);
  return tiles == 2 ? launch<kBf16, 64, 2>(q, kv, a, sms, s) : launch<kBf16, 64, 1>(q, kv, a, sms, s);
}

// [partial results and counts of np_attn_decode.cu][how the line is dealt out][plans][np_attn_rest.cu's parts][maxima and sums of blocks' parts][their
// O][records]: all but the last are at the same place for every call.  They begin at the first multiple of kSpaceAlign in what the caller gives, which is
// 16-byte aligned: results are stored 32 bytes at a time, and records are 32-byte aligned for the compiler.
constexpr uint64_t kSpaceAlign = 32;
static_assert(alignof(Record) <= kSpaceAlign && alignof(RowPlan) <= kSpaceAlign && alignof(LinePlan) <= kSpaceAlign && sizeof(Record) % 32 == 0, "");
struct Space {
  uint64_t line, plan, rest_ml, rest_o, part_ml, part_o, records, bytes;  // bytes: with what lies before the beginning, at most
  Space(int n_heads, int n) {
    uint64_t at = 0;
    auto take = [&at](uint64_t bytes) {
      const uint64_t from = (at + 255) & ~(uint64_t)255;
      at = from + bytes;
      return from;
    };
    take(decode_parts_bytes());
    line = take(sizeof(LinePlan));
    plan = take((uint64_t)NP_KV_MAX_SEQS * sizeof(RowPlan));
    rest_ml = take((uint64_t)kRestBlocks * 8 * 8);
    rest_o = take((uint64_t)kRestBlocks * 8 * 128 * 4);
    part_ml = take((uint64_t)2 * kSharedBlocks * kRows * 8);
    part_o = take((uint64_t)2 * kSharedBlocks * kRows * 128 * 4);
    records = take((uint64_t)n * n_heads * sizeof(Record));
    bytes = at + kSpaceAlign - 16;
  }
  static char* begin(void* workspace) {
    return reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + kSpaceAlign - 1) & ~(uintptr_t)(kSpaceAlign - 1));
  }
};

// Columns, (row, query head) pairs of a group and key-value head, on average, that one kernel does beside the rows' own tokens; more take the tensor
// cores' way.  Both sides, us: 8 rows of 32 heads over 32 that share 8192 tokens, 8 columns, 41.2 in one kernel, 53.6 in two; 16 columns, sharing 1024,
// 27.5 and 29.6; 2 rows of 64 heads over 8, 16 columns, sharing 8192, 29.6 and 29.1, with 600 of their own 30.7 and 39.4; 24 columns 35.5 and
// 29.8; 24 rows of 32 heads, 24 columns, 80 and 57, with 600 of their own 90 and 113.
constexpr int kFewColumns = 16;

const char* shared_heads_error(const np_kv_desc* d, int n_heads, int n) {
  if (const char* m = decode_heads_error(d, n_heads, n)) return m;
  return n_heads / d->n_kv_heads > NP_ATTN_MAX_GROUP ? "more than NP_ATTN_MAX_GROUP query heads to a key-value head" : nullptr;
}

}  // namespace
}  // namespace npa

using namespace npa;

extern "C" {

int np_attn_shared_workspace_bytes(const np_kv_desc* d, int32_t n_heads, int32_t n, uint64_t* out) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  if (const char* m = shared_heads_error(d, n_heads, n)) return fail(NP_E_INVAL, m);
  if (!out) return fail(NP_E_INVAL, "NULL argument");
  *out = Space(n_heads, n).bytes;
  return NP_OK;
}

int np_attn_decode_shared(const np_kv_desc* d, const void* cache, int32_t layer, const np_kv_tables* t, const np_rows* q, int32_t n_heads,
                          const int32_t* seqs, int32_t n, const int32_t* cu, const int32_t* shared, int32_t n_groups, float scale, const np_rows* out,
                          float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  if (const char* m = shared_heads_error(d, n_heads, n)) return fail(NP_E_INVAL, m);
  if (!seqs && n > d->max_seqs) return fail(NP_E_INVAL, "n is above max_seqs");
  if (n_groups < 0 || n_groups > NP_KV_MAX_SEQS) return fail(NP_E_INVAL, "n_groups outside [0, NP_KV_MAX_SEQS]");
  if (n == 0) return NP_OK;
  float scale2;
  if (const char* m = decode_error(d, cache, layer, t, q, n_heads, n, scale, out, workspace, &scale2)) return fail(NP_E_INVAL, m);
  if (n_groups > 0 && (!cu || !shared)) return fail(NP_E_INVAL, "NULL argument");
  const Space space(n_heads, n);
  if (workspace_bytes < space.bytes) return fail(NP_E_INVAL, "workspace is smaller than np_attn_shared_workspace_bytes says");
  int sms;
  if (!device_sms(&sms)) return fail(NP_E_CUDA, "no CUDA device");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (held_in_8(d)) n_groups = 0;
  char* const ws = Space::begin(workspace);
  const int group = n_heads / d->n_kv_heads, columns = n_groups ? (int)std::min<int64_t>(1 << 20, ((int64_t)n * group + n_groups - 1) / n_groups) : 0;
  Args a = {};
  a.shared.cu = cu;
  a.shared.tokens = shared;
  a.shared.n_groups = n_groups;
  a.shared.records = reinterpret_cast<Record*>(ws + space.records);
  a.shared.columns = columns;
  // queries that rows or heads have in common: a tensor map has no strides of 0
  const bool in_common = (n > 1 && q->token_stride == 0) || (n_heads > 1 && q->head_stride == 0);
  if (columns <= kFewColumns || n_groups > kSharedGroups || in_common)
    return decode(d, cache, layer, t, q, n_heads, seqs, n, scale2, out, lse, ws, &a.shared, sms, s);
  a.page_bytes = page_bytes(d);
  a.cache = static_cast<const char*>(cache) + (int64_t)layer * d->n_pages * a.page_bytes;
  a.table = t->page_table;
  a.lens = t->lens;
  a.seqs = seqs;
  a.status = t->status;
  a.n = n;
  a.n_heads = n_heads;
  a.n_kv_heads = d->n_kv_heads;
  a.group = group;
  a.shift = log2_of(d->page_tokens);
  a.n_pages = d->n_pages;
  a.max_seqs = d->max_seqs;
  a.max_pages = d->max_pages;
  a.scale2 = scale2;
  // two tiles of rows where an average group fills more than one
  const int tile_members = kRows / group, tiles = (int64_t)n > (int64_t)n_groups * tile_members ? 2 : 1;
  a.shared.tile_members = tile_members;
  a.shared.members = tiles * tile_members;
  a.shared.line = reinterpret_cast<LinePlan*>(ws + space.line);
  a.shared.plan = reinterpret_cast<RowPlan*>(ws + space.plan);
  a.shared.part_ml = reinterpret_cast<float*>(ws + space.part_ml);
  a.shared.part_o = reinterpret_cast<float*>(ws + space.part_o);
  a.shared.part_rows = tiles * kRows;
  a.shared.rest_ml = reinterpret_cast<float*>(ws + space.rest_ml);
  a.shared.rest_o = reinterpret_cast<float*>(ws + space.rest_o);
  CUtensorMap mq, mkv;
  if (!make_rows_map(&mq, *q, d->head_dim, n_heads, n, a.group, tile_members) || !make_map(&mkv, a, d->head_dim))
    return fail(NP_E_INVAL, "rows or a cache that a tensor map does not describe");
  const cudaError_t e = row_type(d) == NP_T_BF16 ? launch<true>(mq, mkv, a, d->head_dim, tiles, sms, s) : launch<false>(mq, mkv, a, d->head_dim, tiles, sms, s);
  if (e != cudaSuccess) return fail_cuda(e);
  return decode_rest(d, a.cache, t, q, n_heads, seqs, n, scale2, out, lse, a.shared, sms, s);
}

}  // extern "C"
