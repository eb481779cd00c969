// Attention of one new token per sequence over the paged cache (np_attn_decode).
//
//   out[i][h] = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale * q[i][h] . k_j - m),   m the row's maximum
//
// Every key and value is used once per query head of its group, so the cache's bytes bound the kernel: 2 * head_dim * 2
// bytes per token and key-value head against 4 * head_dim operations per query head.  What has to be done is to keep
// enough loads in flight and to split the tokens evenly.
//
// * A warp takes sixteen tokens at a time, all heads of a group (up to eight, or up to sixteen) at once, on the tensor cores'
//   mma.sync form, fp32 sums.
// * Up to eight heads: S^T = K Q^T and O^T = V^T P^T, tokens and head_dim on the wide side, so that a group of one wastes matrix
//   operations (there are plenty) and no bytes.  Keys and values go from global memory straight into the registers that the
//   products read, 16 bytes per lane, no shared memory: S sums over head_dim, so any order of head_dim does as long as q has
//   the same, and lane t of a quad takes pieces t, t + 4, ... of a row; O's rows are head_dim in an order that only the store
//   has to undo, and two tokens' values are interleaved with byte permutes.  The keys of the next sixteen tokens are asked for
//   when S is there, the values when O is, so a warp always has 4 KB in flight (head_dim 128).
// * Up to sixteen heads: S = Q K^T and O = P V, the queries in registers, two exchanges for a row's maximum in place of three, and P is where
//   the second product wants it.  The accumulators leave no registers for keys and values on their way: a warp has a ring of its own in shared
//   memory, two chunks of sixteen tokens, each filled by one tiled TMA copy of keys and values.  (The same ring for eight heads, two
//   blocks to an SM instead of three: 3 % less time for long work, 9 % more for one sequence of 4095.)
// * The running maximum and sum are per warp (base 2, fp32); the accumulators are rescaled only when a maximum grows.  P is
//   the sum of two terms of the cache's type, so it is good to 16 bits and more where one term has 8 or 11.
// * All (sequence, group, tile of 64 tokens) triples form one line; each block takes an equal stretch of it.  A group's start counts
//   as two tiles: that is about what it costs (queries, page numbers, the join of the warps), and a block with many short
//   sequences would be the last otherwise.  A block that has a group's tokens to itself stores the result; otherwise blocks leave
//   (m, l, O) in the workspace and the last to arrive joins them in the order of the tokens, so that results do not depend on
//   who was last.
// * The first keys and values of a block's next piece are asked for before the warps' results of the last are joined.
// * An infinity in V meets two terms of P, of which the second may be 0 or below it, and factors that underflow: the sums make a NaN of
//   it.  So where a piece's result is no finite number though its sum is one, the block looks through the piece's V (mend) and stores
//   what the tokens make of it; joins take infinities as they are.
//
// A cache of 8 bits (e4m3 values, a power of two for each token, head and keys or values) goes the way of up to eight heads, or of two times eight: values
// become fp16, which holds all of them, as they are read, and the products are of fp16 whatever the rows' type, with the queries times a power of two of
// their own (the largest magnitude 2^14), so that nothing is lost.  A key's power of two is a factor of its score.  A value's is one of its
// weight, which keeps the weights in fp16's range only if the maximum has it too:
//
//   m = max_j (s_j + v_j),   o = sum_j 2^(s_j + v_j - m) e4m3_j,   l = sum_j 2^(s_j - m),   out = o / l       v_j the exponents of V
//
// with two terms of fp16 for a weight, as above.  There are half the bytes, and each has to be widened before a product takes it.  Long sequences stream at
// 5.2 TB/s behind a start and joins of 14 us; with nothing but the loads the long one below would still take 56 of its 66.6 us.  (Keys and values
// through shared memory with asynchronous copies, deeper prefetch, more blocks: no gain.)
//
// Measured (pages of 64 scattered over the pool, caches larger than the L2 in turn): sixteen sequences of 0 to 4095 tokens, 32 heads
// of 128, 57.3 us, 5.8 TB/s, 89 % of the copy rate; 64 of 1000 in fp16 159 us, 100 %; one of 131071 tokens, 64 heads over 8, 91.9 us,
// 89 %; one of 100 tokens 4.7 us.  In 8 bits the sixteen, the long one
// and the short one take 44.7, 67.1 and 5.1 us, 59 % and 63 % of the copy rate.  What is not the stream is the launch, three loads that depend on one another (length, page
// number, keys) and the joins.  Groups of more than eight heads are bound by the steps
// between a warp's loads: sixteen heads of 128 to a key-value head, 64 sequences of 2000 tokens, 53.8 us, 74 % (69 % with keys and values
// in registers, 55 % with 16-byte asynchronous copies in place of TMA, 70 % with the chunks beyond asked into the L2 ahead, 74 % with
// keys and values as two copies).
#include <algorithm>

#include "np_attn.h"
#include "np_attn_groups.cuh"
#include "np_attn_mma.cuh"
#include "np_device.cuh"
#include "np_internal.h"
#include "np_pipe.cuh"

namespace npa {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kTile = kWarps * 16;    // tokens of a tile
// Units of a block at least, where there are so few that blocks stay idle.  4 x 900 tokens, 16 heads over one: 13.1 us; with 1 15.6, 4 14.9,
// 8 19.1.  One of 4095 tokens, 32 heads: 21.0 with 1, 2 and 4, 26.1 with 8.
constexpr int kMinTiles = 2;
// What a group's start counts, in tiles.  The sixteen sequences above: 57.7 us; with 0 78.4, 1 57.6, 4 59.4.  The long one 93.0, 96.1, 94.3,
// 91.7; 128 of 1 to 1600 tokens, 64 heads over 8, 71.2, 81.2, 72.9, 73.4; one of 100 tokens 4.7, 7.1, 8.4, 4.9.
constexpr int kStart = 2;
// Partial results that are joined at a time.  The long sequence: 93.0 us; with 4 94.9, 16 99.4 (registers).
constexpr int kJoin = 8;
constexpr int kMaxBlocks = 640;       // blocks of a launch (the workspace holds two partial results of each)

struct DecodeArgs {
  const char* cache;         // of the layer
  const int32_t* table;
  const int32_t* lens;
  const int32_t* seqs;
  int32_t* status;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_token, q_head, o_token, o_head;  // elements
  float* lse;
  unsigned int* count;       // [2 * kMaxBlocks] partial results that have arrived, at the place of their first; zero between calls
  unsigned int* pair_count;  // [n * pairs], pair_step apart: the same of joined ones
  int pair_step;
  float* part_ml;            // [2 * kMaxBlocks][HB][2]
  float* part_o;             // [2 * kMaxBlocks][HB][HD]
  float scale2;              // scale * log2(e)
  int n, n_heads, n_kv_heads, group, blocks_of_heads;  // heads of a group: blocks_of_heads pieces of HB
  int shift, n_pages, max_seqs, max_pages;
  int64_t page_bytes;
  SharedArgs shared;  // kTogether: what groups of rows share
};

// How keys and values get to the products: in the rows' type, up to eight or sixteen heads of a group at once; in 8 bits, the same.
enum Form { kEight, kSixteen, kHeldEight, kHeldSixteen };

// Four 8 x 8 tiles of 16-bit values; lane 8 i + j has the address of row j of tile i.
__device__ __forceinline__ void load_tiles(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_tiles_transposed(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// Four e4m3 values as fp16, which holds all of them: bytes 0 and 1, bytes 2 and 3.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
// Two of the queries' values in fp32.
template <class T>
__device__ __forceinline__ float2 widen2(uint32_t w) {
  if constexpr (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
// keys and values of sixteen tokens: (64 values, rows of a page's heads, halves of head_dim, keys and values, pages)
__device__ __forceinline__ void tma_load_chunk(uint32_t dst, const CUtensorMap* map, int row, int page, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %2, %4}], [%5];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(page), "r"(npp::smem_addr(bar))
               : "memory");
}

// 16 or 8 bytes that are used once
__device__ __forceinline__ void load_words(const char* p, uint32_t (&w)[4]) {
  const uint4 v = npd::ldg_stream(p);
  w[0] = v.x;
  w[1] = v.y;
  w[2] = v.z;
  w[3] = v.w;
}
__device__ __forceinline__ void load_words(const char* p, uint32_t (&w)[2]) {
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
}

// Tokens of row i of the call; 0 where there are none to read.
__device__ __forceinline__ int row_len(const DecodeArgs& a, int i, int* seq_out) {
  const int seq = a.seqs ? a.seqs[i] : i;
  *seq_out = seq;
  if (seq < 0) return 0;
  if (seq >= a.max_seqs) {
    atomicOr(a.status, NP_KV_S_SEQ);
    return 0;
  }
  const int len = a.lens[seq];
  if (len < 0 || ((int64_t)len + (1 << a.shift) - 1) >> a.shift > a.max_pages) {
    atomicOr(a.status, NP_KV_S_LENGTH);
    return 0;
  }
  return len;
}

// Four values of joined partial results that are not finite: factors that are 0 make a NaN of an infinity, so they are what the partial results
// that are not finite add up to by themselves.  part: the four values of the first, `next` to those of the next, n of them; the first
// `extra` further where it is in its block's second place.
__device__ __noinline__ float4 keep_infinite(float4 acc, const float* part, int64_t extra, int64_t next, int n) {
  float4 kept = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [](float& sum, float x) {
    if (not_finite(x)) sum += x;
  };
  for (int y = 0; y < n; ++y) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(part + y * next + (y ? 0 : extra)));
    add(kept.x, v.x);
    add(kept.y, v.y);
    add(kept.z, v.z);
    add(kept.w, v.w);
  }
  if (not_finite(kept.x)) acc.x = kept.x;
  if (not_finite(kept.y)) acc.y = kept.y;
  if (not_finite(kept.z)) acc.z = kept.z;
  if (not_finite(kept.w)) acc.w = kept.w;
  return acc;
}

// Blocks that share an SM.  More of them keep more loads in flight, until the registers no longer hold a warp's keys, values and
// accumulators.  us with one more and with this many (sixteen heads: with keys and values in registers): 128 values, eight heads, four blocks 113 (the
// long sequence) and 186 (64 of 1000), three 101 and 164; sixteen heads, 64 of 2000, three 73.8, two 62.4.  64 values, eight heads, 64 heads, 16
// sequences of 2000, five 91.2, four 86.8 (three 93.9); sixteen heads, one of 131071, four 43.3, three 40.2 (two 45.0).
// In 8 bits: 128 values, eight heads, the long sequence, four 66.4, three 66.7, two 81.2; 64 values, 16 of 2000, 64 heads, five 93.4, four 72.2,
// three 76.2; sixteen heads, 64 of 2000, three 54.6 and two 56.6 (one 88.9), with 64 values 35.1 and 38.3 (58.7); 55.3 and 35.6 since
// sums go by the square of a factor's root.
constexpr int blocks_per_sm(int hd, int form) {
  return form == kHeldEight ? (hd == 64 ? 4 : 3) : form == kHeldSixteen ? 3 : hd == 64 ? (form == kEight ? 4 : 3) : (form == kEight ? 3 : 2);
}

// In 8 bits sums are of 2^(s - m): s - m is between -120 and 60 for the token that m is of, so a sum may be up to 2^60 to a maximum and still be all that
// there is to one that is 2^180 as large.  Warps add up to 2^-149, what they have is 2^30 times as large from then on, and a sum goes from one maximum
// to another by the square of a factor that is a normal number down to 2^-252.  (By the factor itself, sums of values that are 2^126 apart were lost.)
constexpr float kHeldUp = 0x1p30f;
// a b + c, whose result may be below 2^-126
__device__ __forceinline__ float fma_full(float a, float b, float c) {
  float d;
  asm("fma.rn.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// a sum in 8 bits to one whose maximum is 2^-e as large, added to c
__device__ __forceinline__ float move_held(float sum, float e, float c) {
  const float root = exp2_fast(0.5f * e);
  return fma_full(fma_full(sum, root, 0.f), root, c);
}

// What a block knows of groups, in dynamic shared memory: for each row its tokens, how many of them it shares, its group and sequence; and the units of
// groups and rows.
struct GroupRoom {
  int64_t* end;
  int *len, *first;
  GroupInfo* info;
  int16_t *group, *seq;
  uint32_t bytes;
  __host__ __device__ GroupRoom(unsigned char* base, int n, int n_groups) {
    uint32_t at = 0;
    auto take = [&](uint32_t size) {
      unsigned char* p = base + at;
      at += (size + 15) & ~15u;
      return p;
    };
    end = reinterpret_cast<int64_t*>(take((n + n_groups) * 8));
    len = reinterpret_cast<int*>(take(n * 4));
    first = reinterpret_cast<int*>(take(n * 4));
    info = reinterpret_cast<GroupInfo*>(take(n_groups * sizeof(GroupInfo)));
    group = reinterpret_cast<int16_t*>(take(n * 2));
    seq = reinterpret_cast<int16_t*>(take(n * 2));
    bytes = at;
  }
};

constexpr int kSlots = 2;  // sixteen heads: chunks of a warp on their way

// What a warp's lanes tell each other of waits that were given up.
struct WarpWaits {
  volatile int* word;
  int32_t* status;
  __device__ __forceinline__ bool lost() { return *word != 0; }
  __device__ __forceinline__ void lose() {
    *word = 1;
    atomicOr(status, NP_KV_S_TIMEOUT);
  }
};

// kTogether: groups' shared tokens are items of work beside the rows, whose own begin behind them; the last part of a row to arrive is joined to the
// others.
template <class T, int HD, int kForm, bool kTogether>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(HD, kForm))
k_attn_decode(const __grid_constant__ CUtensorMap map, const __grid_constant__ DecodeArgs a) {
  constexpr bool kWide = kForm == kSixteen, kHeld = kForm == kHeldEight || kForm == kHeldSixteen;
  constexpr int HB = kForm == kSixteen || kForm == kHeldSixteen ? 16 : 8;  // heads of a block, at most
  constexpr int NT = HB / 8, NH = kHeld ? 2 * NT : 2;  // in 8 bits: eights of heads; heads of a lane's scores
  // Sixteens of tokens of a chunk.  In 8 bits a sixteen's rows of 64 values are 1 KB, too few for a trip to memory.  16 sequences of 2000, 64 heads of 64:
  // 72.2 us with two, 89.7 with one; one of 131071, 64 heads over 8, 41.7 and 49.8.  Of 128 values two are no better: 65.0 and 66.7, but 16 ragged
  // sequences of 2000, 32 heads, 31.7 and 29.1.
  constexpr int SC = kHeld && HD == 64 ? 2 : 1;
  constexpr int kTileTokens = kTile * SC, kUnitsBefore = kStart / SC;  // tokens of a tile, what a group's start counts
  constexpr int KV = kHeld ? HD / 64 : HD / 32;        // 16-byte pieces of a key row per lane
  constexpr int VW = HD / 32;                          // in 8 bits: words of a value row per lane
  constexpr int VC = HD / 64;        // 16-byte pieces of a value row per lane
  constexpr int QV = HB * HD / 8 / kThreads > 0 ? HB * HD / 8 / kThreads : 1;  // 16-byte pieces of the queries per thread
  // Sixteen heads: sixteen-value steps along head_dim; bytes of a chunk's keys, and of its keys and values
  constexpr int KS = HD / 16;
  constexpr uint32_t kHalf = 16 * HD * 2, kSlot = 2 * kHalf;
  // Bytes from query to query, values from head to head of a warp's result, in shared memory: reads and stores meet all banks
  constexpr int QR = HD * 2 + (kWide ? 16 : 64), SO = HD + (kWide ? 8 : 0);
  __shared__ int64_t s_ends[kTogether ? 1 : NP_KV_MAX_SEQS];
  __shared__ __align__(16) float s_o[kWarps][HB][SO];
  __shared__ __align__(8) uint64_t s_full[kWarps][kSlots];  // a warp's ring is its own
  extern __shared__ __align__(1024) unsigned char s_dyn[];
  __shared__ __align__(16) unsigned char s_q[kHeld ? 16 : HB * QR];
  // In 8 bits: the queries in fp16, sixteen bytes to a lane as the products read them, and what a head's scores are to be multiplied with
  __shared__ __align__(16) unsigned char s_qh[kHeld ? HB * HD * 2 : 16];
  __shared__ __align__(8) float s_up[HB];
  __shared__ float s_ml[kWarps][HB][2];
  __shared__ int64_t s_wsum[kWarps];
  __shared__ int s_last;
  __shared__ volatile int s_lost[kWarps];  // a wait of the warp was given up
  __shared__ int s_done[kTogether ? HB : 1];
  const int n_groups = kTogether ? a.shared.n_groups : 0, items = n_groups + a.n;  // items: groups, then rows
  const GroupRoom room(s_dyn, kTogether ? a.n : 0, n_groups);
  int64_t* const s_end = kTogether ? room.end : s_ends;  // units of the items up to and including this one
  if (kWide && (threadIdx.x & 31) == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory");
    for (int i = 0; i < kSlots; ++i) npp::mbar_init(&s_full[threadIdx.x >> 5][i], 1);
    s_lost[threadIdx.x >> 5] = 0;
    npp::fence_barrier_init();
  }
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
  const int pairs = a.n_kv_heads * a.blocks_of_heads;   // (key-value head, block of its query heads)

  if constexpr (kTogether) {
    for (int i = tid; i < a.n; i += kThreads) {
      int seq;
      const int len = row_len(a, i, &seq);
      const bool known = seq >= 0 && seq < a.max_seqs;
      room.len[i] = len;
      room.seq[i] = (int16_t)(known ? seq : -1);
      room.first[i] = len > 0 || !known ? len : a.lens[seq];  // as the tables say
    }
    for (int x = tid; x < a.shared.n_groups; x += kThreads) room.info[x] = group_at(a.shared, a.n, x);
    __syncthreads();
    for (int x = wid; x < a.shared.n_groups; x += kWarps) {
      GroupInfo of = room.info[x];
      check_group(of, room.seq, room.first, a.max_pages, a.shift, a.status);
      __syncwarp();
      if (lane == 0) room.info[x] = of;
    }
    __syncthreads();
    for (int i = tid; i < a.n; i += kThreads) room.first[i] = 0;
    __syncthreads();
    for (int x = wid; x < a.shared.n_groups; x += kWarps) {
      const GroupInfo of = room.info[x];
      for (int i = of.lo + lane; i < of.hi; i += 32) {
        room.first[i] = room.len[i] > 0 ? of.tokens : 0;
        room.group[i] = (int16_t)x;
      }
    }
    __syncthreads();
  }
  // tokens of row i of the call that are its own
  auto own_len = [&](int i, int* seq) {
    if (!kTogether) return row_len(a, i, seq);
    *seq = room.seq[i];
    return room.len[i] - room.first[i];
  };
  // blocks of columns, (row, query head) pairs of one key-value head, of a group
  auto column_blocks = [&](const GroupInfo& x) { return ((x.hi - x.lo) * a.group + HB - 1) / HB; };
  // units of an item; kTogether: of all its pairs
  auto units_of = [&](int i) {
    int seq;
    int len;
    int64_t of = 1;
    if (kTogether && i < n_groups) {
      const GroupInfo x = room.info[i];
      len = x.tokens;
      of = (int64_t)a.n_kv_heads * column_blocks(x);
    } else {
      len = own_len(i - n_groups, &seq);
      if (kTogether) of = pairs;
    }
    return len > 0 ? (((int64_t)len + kTileTokens - 1) / kTileTokens + kUnitsBefore) * of : 0;
  };

  // ---- units (tiles, and a group's start) of every row, summed up; rows without tokens are answered here
  int64_t run = 0;
  if (items <= 32) {  // every warp by itself: all write the same
    int64_t inc = lane < items ? units_of(lane) : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane < items) s_end[lane] = inc;
    run = __shfl_sync(0xffffffffu, inc, 31);
    __syncwarp();
  } else {
    for (int base = 0; base < items; base += kThreads) {
      const int i = base + tid;
      int64_t inc = i < items ? units_of(i) : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      if (lane == 31) s_wsum[wid] = inc;
      __syncthreads();
      for (int w = 0; w < wid; ++w) inc += s_wsum[w];
      if (i < items) s_end[i] = run + inc;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) run += s_wsum[w];
      __syncthreads();
    }
  }
  // Four values of a head's result; its log of the sum with the first.  Of that log's two products one is rounded by itself, and which one is spelled out,
  // so that results are the same in every build: the sum's, of a piece by itself; the maximum's, of joined ones.
  auto result = [&](int i, int h, int d, float4 acc, float top, float sum, auto joined) {
    const float use = top == -INFINITY ? 0.f : top;
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    uint2 r;
    if constexpr (kHeld) acc = make_float4(acc.x * kHeldUp, acc.y * kHeldUp, acc.z * kHeldUp, acc.w * kHeldUp);
    r.x = (uint32_t)Half2<T>::round(none ? 0.f : acc.x * inv) | (uint32_t)Half2<T>::round(none ? 0.f : acc.y * inv) << 16;
    r.y = (uint32_t)Half2<T>::round(none ? 0.f : acc.z * inv) | (uint32_t)Half2<T>::round(none ? 0.f : acc.w * inv) << 16;
    *reinterpret_cast<uint2*>(a.out + i * a.o_token + (int64_t)h * a.o_head + d) = r;
    if (a.lse && d == 0) {
      float m = use;
      if (kHeld) {  // the maximum has an exponent v of V's in it, which the sum takes back: a whole number, added at the scale of |v| and the scores (half a step)
        int up;
        sum = frexpf(sum, &up);
        m += (float)(up - 30);
      }
      a.lse[(size_t)i * a.n_heads + h] = none ? -INFINITY : decltype(joined)::value ? __fmaf_rn(__log2f(sum), kLn2, __fmul_rn(m, kLn2)) : __fmaf_rn(m, kLn2, logf(sum));
    }
  };
  // where the parts of (row i, head h) meet
  auto record = [&](int64_t i, int h) { return a.shared.records + (i * a.n_heads + h); };
  for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
    if (s_end[n_groups + i] != (n_groups + i ? s_end[n_groups + i - 1] : 0)) continue;
    if (kTogether && room.first[i] > 0) continue;  // all of its tokens are shared
    for (int e = tid; e < a.n_heads * (HD / 8); e += kThreads) {
      const int h = e / (HD / 8), d = e % (HD / 8) * 8;
      *reinterpret_cast<uint4*>(a.out + i * a.o_token + h * a.o_head + d) = make_uint4(0, 0, 0, 0);
      if (a.lse && d == 0) a.lse[(size_t)i * a.n_heads + h] = -INFINITY;
    }
  }
  // the line's W units over G blocks: the first `more` blocks take each + 1 of them, the others each
  const int per = kTogether ? 1 : pairs;
  const int64_t W = run * per;
  const int G = (int)min((int64_t)gridDim.x, (W + kMinTiles - 1) / kMinTiles);
  if ((int)blockIdx.x >= G) return;
  const int64_t each = divide(W, G), more = W - each * G;
  auto block_of = [&](int64_t w) { return (int)(w < more * (each + 1) ? divide(w, each + 1) : more + divide(w - more * (each + 1), each)); };
  int64_t w0 = blockIdx.x * each + min((int64_t)blockIdx.x, more);
  const int64_t w1 = w0 + each + (blockIdx.x < more ? 1 : 0);
  int row = 0;
  {
    int lo = 0, hi = items - 1;  // the first item whose units end after w0
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_end[mid] * per > w0) hi = mid;
      else lo = mid + 1;
    }
    row = lo;
  }

  constexpr int kRowBytes = kHeld ? HD : HD * 2;
  const int64_t head_bytes = (int64_t)kRowBytes << a.shift, page_bytes = a.page_bytes;
  const int64_t exponents = 2 * a.n_kv_heads * head_bytes;  // in 8 bits: of a page, from its start
  struct Piece {  // tiles [ta, tb) of one (row, pair), or of a group and a block of its columns: from h0 on, of key-value head kvh
    int row, pair, kvh, h0, heads, len, tiles, ta, tb;
    bool of_group;
    int64_t first_w;  // of its pair, on the line
    const int32_t* pages;
    int first_row;    // of its key-value head in a page
    const char* kbase;
    const char* vbase;
    const char* ebase;
  };
  // the next piece with tokens from w0 on; false: none is left
  auto next_piece = [&](Piece& p) {
    while (w0 < w1) {
      while (s_end[row] * per <= w0) ++row;
      p.of_group = kTogether && row < n_groups;
      const GroupInfo of = p.of_group ? room.info[row] : GroupInfo{};
      const int64_t before = row ? s_end[row - 1] : 0, r0 = w0 - before * per;
      const int64_t units = !kTogether ? s_end[row] - before : divide(s_end[row] - before, p.of_group ? a.n_kv_heads * column_blocks(of) : pairs);
      const int pair = (int)divide(r0, units);
      const int64_t ra = r0 - pair * units, rb = min(units, ra + (w1 - w0));
      p.first_w = w0 - ra;
      w0 += rb - ra;
      p.ta = (int)max((int64_t)0, ra - kUnitsBefore);
      p.tb = (int)max((int64_t)0, rb - kUnitsBefore);
      if (p.ta == p.tb) continue;  // the start alone: whoever has the first tile begins
      p.row = row - n_groups;
      p.pair = pair;
      p.tiles = (int)(units - kUnitsBefore);
      int seq, kvh;
      if (p.of_group) {
        const int blocks = column_blocks(of);
        kvh = pair / blocks;
        p.row = of.lo;
        p.len = of.tokens;
        p.h0 = (pair - kvh * blocks) * HB;
        p.heads = min(HB, (of.hi - of.lo) * a.group - p.h0);
        p.pages = a.table + (size_t)of.seq * a.max_pages;
      } else {
        p.len = own_len(p.row, &seq);
        kvh = pair / a.blocks_of_heads;
        const int hb = pair - kvh * a.blocks_of_heads;
        p.h0 = kvh * a.group + hb * HB;
        p.heads = min(HB, a.group - hb * HB);
        p.pages = a.table + (size_t)seq * a.max_pages + (kTogether ? room.first[p.row] >> a.shift : 0);
      }
      p.kvh = kvh;
      p.first_row = kvh << a.shift;
      p.kbase = a.cache + kvh * head_bytes;
      p.vbase = p.kbase + a.n_kv_heads * head_bytes;
      p.ebase = a.cache + exponents + ((int64_t)kvh << a.shift);
      return true;
    }
    return false;
  };

  uint4 qf[QV], kf[kHeld ? 1 : 2][KV], vf[kHeld ? 1 : 4][VC];
  // In 8 bits: keys of tokens g and g + 8 of each sixteen, values of 2t, 2t + 1, 2t + 8 and 2t + 9, exponents of keys and (from bit 8 on) values of
  // token `lane`; how many tokens of each sixteen there are, where they are, and their pages, of this chunk and the next
  uint4 kh[kHeld ? SC : 1][2][KV];
  uint32_t vh[kHeld ? SC : 1][4][VW], ex = 0, ex_next = 0;
  int have_h[SC], next_have_h[SC], page_h[SC];
  uint32_t end_h = 0;       // tokens up to the end of the piece
  bool next_whole = false;  // all tokens of the next chunk are there
  int64_t next_at_h[SC];
  Piece p = {};
  int chunk_end, c, have, have_next, pg_next;  // chunks of 16 tokens
  int64_t at, at_next;
  int waiting[kSlots];                 // tokens of the chunks in this warp's ring
  npp::WarpRing<kSlots> uses;
  WarpWaits waits = {&s_lost[wid], a.status};
  const uint32_t ring = ((npp::smem_addr(s_dyn) + (kTogether ? room.bytes : 0u) + 1023) & ~1023u) + wid * kSlots * kSlot;
  // what a lane reads with load_tiles: rows (tokens) 0-7 and 8-15 of two neighbouring 16-byte columns, 128-byte swizzle
  const uint32_t lane_row = ((lane & 7) + (lane >> 4) * 8) * 128, lane_col = ((lane >> 3 & 1) ^ (lane & 7)) << 4;
  auto tiles_at = [&](uint32_t base, int step) { return base + lane_row + (step >> 2) * 2048 + (((step & 3) << 5) ^ lane_col); };
  // where the chunk's page starts, and how many of its tokens there are (0: nothing to read)
  auto chunk_of = [&](int chunk, int pg, int& n, int64_t& off) {
    n = 0;
    off = 0;
    if (chunk >= chunk_end) return;
    if ((unsigned)pg >= (unsigned)a.n_pages) {
      atomicOr(a.status, NP_KV_S_PAGE);
      return;
    }
    n = (int)min((int64_t)16, p.len - (int64_t)chunk * 16);
    off = pg * page_bytes + (int64_t)((chunk * 16) & ((1 << a.shift) - 1)) * (HD * 2);
  };
  auto page_of = [&](int chunk) { return chunk < chunk_end ? p.pages[(int)(((int64_t)chunk * 16) >> a.shift)] : 0; };
  // in 8 bits: the pages of a chunk's sixteens (0 where there are no tokens)
  auto pages_of_held = [&](int chunk) {
#pragma unroll
    for (int x = 0; x < SC; ++x) {
      const uint32_t tok = ((uint32_t)chunk * SC + x) * 16;
      page_h[x] = tok < end_h ? p.pages[tok >> a.shift] : 0;
    }
  };
  // asks for the exponents of the chunk with the pages page_h, and works out where the rest of it is
  auto ask_held = [&](int chunk) {
    next_whole = true;
    const char* e = nullptr;
    bool mine = false;
#pragma unroll
    for (int x = 0; x < SC; ++x) {
      const uint32_t tok = ((uint32_t)chunk * SC + x) * 16, place = tok & ((1u << a.shift) - 1);
      next_have_h[x] = tok < end_h ? (int)min(16u, end_h - tok) : 0;
      if ((unsigned)page_h[x] >= (unsigned)a.n_pages) {
        atomicOr(a.status, NP_KV_S_PAGE);
        next_have_h[x] = page_h[x] = 0;
      }
      next_whole &= next_have_h[x] == 16;
      const int64_t page = page_h[x] * page_bytes;
      next_at_h[x] = page + place * HD;
      if (SC == 1 || lane >> 4 == x) {
        e = p.ebase + page + (place + (lane & 15));
        mine = lane < 16 * SC && (lane & 15) < next_have_h[x];
      }
    }
    ex_next = 0;
    if (mine) ex_next = (uint8_t)__ldg(e) | (uint32_t)(uint8_t)__ldg(e + ((int64_t)a.n_kv_heads << a.shift)) << 8;
  };
  auto load_k_held = [&] {
#pragma unroll
    for (int x = 0; x < SC; ++x) {
      const char* k = p.kbase + next_at_h[x] + (g * HD + t * 16);
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int j = 0; j < KV; ++j) {
          if (next_whole) {
            kh[x][r][j] = npd::ldg_stream(k + r * 8 * HD + j * 64);
          } else {
            kh[x][r][j] = make_uint4(0, 0, 0, 0);
            if (g + 8 * r < next_have_h[x]) kh[x][r][j] = npd::ldg_stream(k + r * 8 * HD + j * 64);
          }
        }
    }
  };
  auto load_v_held = [&] {
#pragma unroll
    for (int x = 0; x < SC; ++x) {
      const char* v = p.vbase + next_at_h[x] + (2 * t * HD + g * (HD / 8));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int tok = (r & 1) + (r >> 1) * 8;
        if (next_whole) {
          load_words(v + tok * HD, vh[x][r]);
        } else {
#pragma unroll
          for (int w = 0; w < VW; ++w) vh[x][r][w] = 0;
          if (2 * t + tok < next_have_h[x]) load_words(v + tok * HD, vh[x][r]);
        }
      }
      have_h[x] = next_have_h[x];
    }
    ex = ex_next;
  };
  auto load_k = [&](int n, int64_t off) {
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < KV; ++j) {
        kf[r][j] = make_uint4(0, 0, 0, 0);
        if (g + 8 * r < n) kf[r][j] = npd::ldg_stream(p.kbase + off + (g + 8 * r) * (HD * 2) + (t + 4 * j) * 16);
      }
  };
  auto load_v = [&](int n, int64_t off) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int tok = 2 * t + (r & 1) + (r >> 1) * 8;
#pragma unroll
      for (int x = 0; x < VC; ++x) {
        vf[r][x] = make_uint4(0, 0, 0, 0);
        if (tok < n) vf[r][x] = npd::ldg_stream(p.vbase + off + tok * (HD * 2) + (g + 8 * x) * 16);
      }
    }
  };
  // asks for a chunk for the ring; how many of its tokens there are (0: nothing to read)
  auto ask = [&](int chunk, int pg) {
    if (chunk >= chunk_end) return 0;
    if ((unsigned)pg >= (unsigned)a.n_pages) {
      atomicOr(a.status, NP_KV_S_PAGE);
      return 0;
    }
    if (lane == 0 && uses.may_ask()) {
      const uint32_t slot = uses.slot(uses.asked++);
      npp::mbar_expect_tx(&s_full[wid][slot], kSlot);
      tma_load_chunk(ring + slot * kSlot, &map, p.first_row + (int)(((int64_t)chunk * 16) & ((1 << a.shift) - 1)), pg, &s_full[wid][slot]);
    }
    return (int)min((int64_t)16, p.len - (int64_t)chunk * 16);
  };
  // asks for the queries and the first keys and values of a piece
  auto begin = [&] {
    chunk_end = (int)min(((int64_t)p.len + 16 * SC - 1) / (16 * SC), (int64_t)p.tb * kWarps);
    c = p.ta * kWarps + wid;
    int pg[kSlots + 1] = {};
    if constexpr (kHeld) {
      end_h = (uint32_t)min((int64_t)p.len, (int64_t)p.tb * kTileTokens);
      pages_of_held(c);
    } else {
#pragma unroll
      for (int i = 0; i < (kWide ? kSlots : 1) + 1; ++i) pg[i] = page_of(c + i * kWarps);
    }
#pragma unroll
    for (int j = 0; j < QV; ++j) {
      const int x = j * kThreads + tid, h = x / (HD / 8), d = x % (HD / 8) * 8;
      qf[j] = make_uint4(0, 0, 0, 0);
      if (h < p.heads) {
        int64_t i = p.row, head = p.h0 + h;
        if (kTogether && p.of_group) {  // columns go through the rows' heads
          const int at = p.h0 + h, member = at / a.group;
          i += member;
          head = p.kvh * a.group + at - member * a.group;
        }
        qf[j] = *reinterpret_cast<const uint4*>(a.q + i * a.q_token + head * a.q_head + d);
      }
    }
    if constexpr (kWide) {
      __syncwarp();  // all lanes have read what the ring held
#pragma unroll
      for (int i = 0; i < kSlots; ++i) waiting[i] = ask(c + i * kWarps, pg[i]);
      pg_next = pg[kSlots];
    } else if constexpr (kHeld) {
      ask_held(c);
      load_k_held();
      load_v_held();
      pages_of_held(c + kWarps);
    } else {
      chunk_of(c, pg[0], have, at);
      load_k(have, at);
      load_v(have, at);
      pg_next = pg[1];
    }
  };
  auto add = [](float4& acc, float f, const float4& v) {
    acc.x += f * v.x;
    acc.y += f * v.y;
    acc.z += f * v.z;
    acc.w += f * v.w;
  };
  auto odd_four = [](const float4& v) { return not_finite(v.x) || not_finite(v.y) || not_finite(v.z) || not_finite(v.w); };
  // the queries that begin() asked for go where all warps read them; a barrier follows
  auto keep_queries = [&] {
#pragma unroll
    for (int j = 0; j < QV; ++j) {
      const int x = j * kThreads + tid, h = x / (HD / 8), d = x % (HD / 8);
      if constexpr (kHeld) {  // in fp16, times a power of two that brings the largest finite one of a head to 2^14
        float2 f[4];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[i] = widen2<T>(word(qf[j], i));
          const uint32_t b0 = __float_as_uint(f[i].x) & 0x7fffffffu, b1 = __float_as_uint(f[i].y) & 0x7fffffffu;
          top = max(top, max(b0 < 0x7f800000u ? b0 : 0u, b1 < 0x7f800000u ? b1 : 0u));
        }
#pragma unroll
        for (int y = 1; y < HD / 8; y <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, y));
        // biased exponent of the power of two to divide by, 1 to 240; of small scales so large that the product of the two is a normal number (queries are
        // then smaller than they could be, and off by 2^-25, which moves a score by 2^-15 at most, with 128 of the largest keys)
        const int e = max(max((int)(top >> 23), 15) - 14, 128 - (int)(__float_as_uint(a.scale2) >> 23));
        const float by = __uint_as_float((uint32_t)(254 - e) << 23), back = __uint_as_float((uint32_t)e << 23);
        if (h < HB) {
          __half2 r[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = __floats2half2_rn(fma_full(f[i].x, by, 0.f), fma_full(f[i].y, by, 0.f));
          // the halves of sixteen values d / 2, at lane 4 * (h % 8) + d / 2 % 4
          *reinterpret_cast<uint4*>(s_qh + (h >> 3) * (HD * 16) + (((d >> 3) * 2 + (d & 1)) * 32 + (h & 7) * 4 + (d >> 1 & 3)) * 16) = *reinterpret_cast<const uint4*>(r);
          if (d == 0) s_up[h] = fminf(a.scale2 * back, FLT_MAX);
        }
        continue;
      }
      if (h < HB) *reinterpret_cast<uint4*>(s_q + h * QR + d * 16) = qf[j];
    }
  };
  bool any = next_piece(p);
  if (any) {
    begin();
    keep_queries();
  }
  __syncthreads();
  while (any) {
    float m[NH], l[NH], o[kWide ? 2 * KS : kHeld ? NT * (HD / 16) : VC * 4][4];
#pragma unroll
    for (int i = 0; i < NH; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
    }
#pragma unroll
    for (auto& x : o) x[0] = x[1] = x[2] = x[3] = 0.f;
    uint32_t qr[kWide ? KS : 1][4];  // sixteen heads: the queries of heads g and g + 8, values 16 j + 2t, + 1 and those eight further
    if constexpr (kWide) {
#pragma unroll
      for (int j = 0; j < KS; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) qr[j][i] = *reinterpret_cast<const uint32_t*>(s_q + (g + (i & 1) * 8) * QR + j * 32 + t * 4 + (i >> 1) * 16);
    }
    // the maxima of the two heads grow to `top`, what has been added up is rescaled (by(i, factor) for the accumulators of head i), `use` is
    // what to take off
    auto raise = [&](const auto& top, auto& use, auto by) {
      float now[NH];
      bool grew = false;
#pragma unroll
      for (int i = 0; i < NH; ++i) {
        now[i] = fmaxf(m[i], top[i]);
        use[i] = now[i] == -INFINITY ? 0.f : now[i];  // -inf so far: nothing has been added up yet
        grew |= now[i] > m[i];
      }
      if (!__any_sync(0xffffffffu, grew)) return;
#pragma unroll
      for (int i = 0; i < NH; ++i) {
        const float f = exp2_fast(m[i] - use[i]);
        l[i] = kHeld ? move_held(l[i], m[i] - use[i], 0.f) : l[i] * f;
        m[i] = now[i];
        by(i, f);
      }
    };
    if constexpr (kHeld) {
      float up[NH];
#pragma unroll
      for (int i = 0; i < NH; ++i) up[i] = s_up[(i >> 1) * 8 + 2 * t + (i & 1)];
      for (; c < chunk_end; c += kWarps) {
        ask_held(c + kWarps);
        pages_of_held(c + 2 * kWarps);
        // ---- S^T = K Q^T, without their powers of two
        float s[SC][NT][4];
#pragma unroll
        for (int y = 0; y < SC; ++y)
#pragma unroll
          for (int x = 0; x < NT; ++x) s[y][x][0] = s[y][x][1] = s[y][x][2] = s[y][x][3] = 0.f;
#pragma unroll
        for (int j = 0; j < KV; ++j)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint4 q[NT];
#pragma unroll
            for (int x = 0; x < NT; ++x) q[x] = *reinterpret_cast<const uint4*>(s_qh + x * (HD * 16) + ((j * 2 + half) * 32 + lane) * 16);
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
              for (int y = 0; y < SC; ++y) {
                uint32_t a0, a1, a2, a3;
                widen4(word(kh[y][0][j], 2 * half + w), a0, a2);
                widen4(word(kh[y][1][j], 2 * half + w), a1, a3);
#pragma unroll
                for (int x = 0; x < NT; ++x) Half2<__half>::mma(s[y][x], a0, a1, a2, a3, w ? q[x].z : q[x].x, w ? q[x].w : q[x].y);
              }
          }
        load_k_held();
        // ---- softmax: s[y][x][0], s[y][x][1] are token g of a sixteen, s[y][x][2], s[y][x][3] token g + 8; heads 8x + 2t and 8x + 2t + 1.  A
        // token's values are times 2^lv: their weight is 2^(s + lv - m), m the largest s + lv, and the sum is of 2^(s - m).
        float lv[SC][2], top[NH], use[NH];
#pragma unroll
        for (int i = 0; i < NH; ++i) top[i] = -INFINITY;
#pragma unroll
        for (int y = 0; y < SC; ++y)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const uint32_t e = __shfl_sync(0xffffffffu, ex, 16 * y + g + 8 * r);
            const float power = __uint_as_float((e & 0xffu) << 23);
            const bool there = g + 8 * r < have_h[y];
            lv[y][r] = (float)(int)(e >> 8) - 127.f;
#pragma unroll
            for (int x = 0; x < NT; ++x)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float z = s[y][x][2 * r + i] * (up[2 * x + i] * power);  // either factor may be too large for the score by itself
                s[y][x][2 * r + i] = there ? z : -INFINITY;
                top[2 * x + i] = fmaxf(top[2 * x + i], s[y][x][2 * r + i] + lv[y][r]);
              }
          }
#pragma unroll
        for (int i = 0; i < NH; ++i)
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], x));
        raise(top, use, [&](int i, float f) {
#pragma unroll
          for (int v = 0; v < HD / 16; ++v) {
            o[(i >> 1) * (HD / 16) + v][i & 1] *= f;
            o[(i >> 1) * (HD / 16) + v][(i & 1) + 2] *= f;
          }
        });
#pragma unroll
        for (int y = 0; y < SC; ++y) {
          uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
          for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              float w[2];
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float e = s[y][x][2 * r + i] - use[2 * x + i];
                const float root = exp2_fast(0.5f * e);  // e + 30 would be rounded at 30's scale
                l[2 * x + i] = fma_full(root, root, l[2 * x + i]);
                w[i] = exp2_fast(e + lv[y][r]);
              }
              uint32_t hi, lo;
              Half2<__half>::split(w[0], w[1], hi, lo);
              ph[x][r] = transpose8x8(hi);
              pl[x][r] = transpose8x8(lo);
            }
          // ---- O^T += V^T W^T
#pragma unroll
          for (int w = 0; w < VW; ++w)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t order = half ? 0x7362 : 0x5140;
              uint32_t a0, a1, a2, a3;
              widen4(__byte_perm(vh[y][0][w], vh[y][1][w], order), a0, a1);
              widen4(__byte_perm(vh[y][2][w], vh[y][3][w], order), a2, a3);
#pragma unroll
              for (int x = 0; x < NT; ++x) {
                Half2<__half>::mma(o[x * (HD / 16) + 2 * w + half], a0, a1, a2, a3, ph[x][0], ph[x][1]);
                Half2<__half>::mma(o[x * (HD / 16) + 2 * w + half], a0, a1, a2, a3, pl[x][0], pl[x][1]);
              }
            }
        }
        load_v_held();
      }
    } else if constexpr (!kWide) {
      for (; c < chunk_end; c += kWarps) {
        chunk_of(c + kWarps, pg_next, have_next, at_next);
        pg_next = page_of(c + 2 * kWarps);
        uint32_t ph[2], pl[2];
        // ---- S^T = K Q^T
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KV; ++j) {
          const uint4 q = *reinterpret_cast<const uint4*>(s_q + g * QR + (t + 4 * j) * 16);
          Half2<T>::mma(s, kf[0][j].x, kf[1][j].x, kf[0][j].y, kf[1][j].y, q.x, q.y);
          Half2<T>::mma(s, kf[0][j].z, kf[1][j].z, kf[0][j].w, kf[1][j].w, q.z, q.w);
        }
        load_k(have_next, at_next);
        // ---- softmax: s[0], s[1] are token g, s[2], s[3] token g + 8; heads 2t and 2t + 1
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = g + 8 * (i >> 1) < have ? s[i] * a.scale2 : -INFINITY;
        float top[2], use[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          top[i] = fmaxf(s[i], s[i + 2]);
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], x));
        }
        raise(top, use, [&](int i, float f) {
#pragma unroll
          for (auto& x : o) {
            x[i] *= f;
            x[i + 2] *= f;
          }
        });
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = exp2_fast(s[i] - use[i & 1]);
        l[0] += p[0] + p[2];
        l[1] += p[1] + p[3];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t hi, lo;
          Half2<T>::split(p[2 * i], p[2 * i + 1], hi, lo);
          ph[i] = transpose8x8(hi);
          pl[i] = transpose8x8(lo);
        }
        // ---- O^T += V^T P^T
#pragma unroll
        for (int v = 0; v < VC; ++v)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t x0 = word(vf[0][v], w), x1 = word(vf[1][v], w), x2 = word(vf[2][v], w), x3 = word(vf[3][v], w);
            const uint32_t a0 = __byte_perm(x0, x1, 0x5410), a1 = __byte_perm(x0, x1, 0x7632);
            const uint32_t a2 = __byte_perm(x2, x3, 0x5410), a3 = __byte_perm(x2, x3, 0x7632);
            Half2<T>::mma(o[v * 4 + w], a0, a1, a2, a3, ph[0], ph[1]);
            Half2<T>::mma(o[v * 4 + w], a0, a1, a2, a3, pl[0], pl[1]);
          }
        load_v(have_next, at_next);
        have = have_next;
        at = at_next;
      }
    } else {
      for (; c < chunk_end; c += kWarps) {
        const int now = waiting[0], pg = pg_next;
        pg_next = page_of(c + (kSlots + 1) * kWarps);
        if (now > 0) {
          const uint32_t k_at = ring + uses.slot(uses.used) * kSlot, v_at = k_at + kHalf;
          uint32_t polls = 0;
#pragma unroll 1
          while (!npp::mbar_try_wait(&s_full[wid][uses.slot(uses.used)], uses.parity(uses.used)))
            if (npp::warp_ring_wait_step<npp::kSpinLimit>(polls, waits)) {
              uses.lost = true;
              break;
            }
          ++uses.used;
          if (now < 16) {  // tokens that are not there: zero, whatever their places hold
            for (int e = lane; e < (16 - now) * (HD / 8); e += 32) {
              const int r = now + e / (HD / 8), d = e % (HD / 8);
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v_at + (d >> 3) * 2048 + r * 128 + (((d ^ r) & 7) << 4)), "r"(0) : "memory");
            }
            npp::fence_proxy_async();
            __syncwarp();
          }
          uint32_t ph[4], pl[4];
          // ---- S = Q K^T, eight tokens at a time
          float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            uint32_t x[4];
            load_tiles(tiles_at(k_at, j), x);
            Half2<T>::mma(s[0], qr[j][0], qr[j][1], qr[j][2], qr[j][3], x[0], x[1]);
            Half2<T>::mma(s[1], qr[j][0], qr[j][1], qr[j][2], qr[j][3], x[2], x[3]);
          }
          // ---- softmax: s[r][0], s[r][1] are head g, s[r][2], s[r][3] head g + 8; tokens 8r + 2t and 8r + 2t + 1
          float top[2], use[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
              for (int x = 0; x < 2; ++x) s[r][2 * i + x] = 8 * r + 2 * t + x < now ? s[r][2 * i + x] * a.scale2 : -INFINITY;
            top[i] = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
#pragma unroll
            for (int x = 1; x < 4; x <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], x));
          }
          raise(top, use, [&](int i, float f) {
#pragma unroll
            for (auto& x : o) {
              x[2 * i] *= f;
              x[2 * i + 1] *= f;
            }
          });
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const float p0 = exp2_fast(s[r][2 * i] - use[i]), p1 = exp2_fast(s[r][2 * i + 1] - use[i]);
              l[i] += p0 + p1;
              Half2<T>::split(p0, p1, ph[2 * r + i], pl[2 * r + i]);
            }
          // ---- O += P V
#pragma unroll
          for (int j = 0; j < KS; ++j) {
            uint32_t x[4];
            load_tiles_transposed(tiles_at(v_at, j), x);
            Half2<T>::mma(o[2 * j], ph[0], ph[1], ph[2], ph[3], x[0], x[2]);
            Half2<T>::mma(o[2 * j + 1], ph[0], ph[1], ph[2], ph[3], x[1], x[3]);
            Half2<T>::mma(o[2 * j], pl[0], pl[1], pl[2], pl[3], x[0], x[2]);
            Half2<T>::mma(o[2 * j + 1], pl[0], pl[1], pl[2], pl[3], x[1], x[3]);
          }
          __syncwarp();
        }
#pragma unroll
        for (int i = 0; i + 1 < kSlots; ++i) waiting[i] = waiting[i + 1];
        waiting[kSlots - 1] = ask(c + kSlots * kWarps, pg);
      }
    }

    // ---- on to the next piece; this one's results meet in shared memory meanwhile
    const Piece e = p;
    any = next_piece(p);
    if (any) begin();
#pragma unroll
    for (int i = 0; i < NH; ++i) {
      const int h = kWide ? g + 8 * i : kHeld ? (i >> 1) * 8 + 2 * t + (i & 1) : 2 * t + i;
      if (kHeld) l[i] = fma_full(l[i], kHeldUp, 0.f);
#pragma unroll
      for (int x = kWide ? 1 : 4; x < (kWide ? 4 : 32); x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
      if (h < e.heads) {
        if ((kWide ? t : g) == 0) {
          s_ml[wid][h][0] = m[i];
          s_ml[wid][h][1] = l[i];
        }
        if constexpr (kHeld) {
#pragma unroll
          for (int k = 0; k < HD / 16; ++k)
            *reinterpret_cast<float2*>(&s_o[wid][h][g * (HD / 8) + 2 * k]) =
                make_float2(o[(i >> 1) * (HD / 16) + k][i & 1], o[(i >> 1) * (HD / 16) + k][(i & 1) + 2]);
        } else if constexpr (!kWide) {
#pragma unroll
          for (int k = 0; k < VC * 4; ++k)
            *reinterpret_cast<float2*>(&s_o[wid][h][(g + 8 * (k >> 2)) * 8 + 2 * (k & 3)]) = make_float2(o[k][i], o[k][i + 2]);
        } else {
#pragma unroll
          for (int k = 0; k < 2 * KS; ++k) *reinterpret_cast<float2*>(&s_o[wid][h][8 * k + 2 * t]) = make_float2(o[k][2 * i], o[k][2 * i + 1]);
        }
      }
    }
    __syncthreads();
    if (any) keep_queries();
    const bool whole = e.ta == 0 && e.tb == e.tiles;
    const bool meets = kTogether && (e.of_group || room.first[e.row] > 0);  // its result is a part
    auto record_of = [&](int h) {
      if (!e.of_group) return record(e.row, e.h0 + h);
      const int at = e.h0 + h, member = at / a.group;
      return record(e.row + member, e.kvh * a.group + at - member * a.group);
    };
    auto emit = [&](int h, int d, float4 acc, float top, float sum, auto joined) {
      if (kTogether && meets) {
        Record* r = record_of(h);
        const int part = e.of_group ? 0 : 1;
        __stcg(reinterpret_cast<float4*>(&r->o[part][d]), sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : acc);
        if (d == 0) __stcg(reinterpret_cast<float2*>(r->ml[part]), make_float2(top, sum));
        return;
      }
      result(e.row, e.h0 + h, d, acc, top, sum, joined);
    };
    const int slot = 2 * blockIdx.x + (e.ta == 0 ? 1 : 0);
    uint32_t odd = 0, turn = 1;  // bit k: the values of turn k below are not finite, and the sum does not say why
    for (int x = tid; x < e.heads * (HD / 4); x += kThreads, turn <<= 1) {
      const int h = x / (HD / 4), d = x % (HD / 4) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_ml[w][h][0]);
      const float use = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_fast(s_ml[w][h][0] - use);
        const float4 v = *reinterpret_cast<const float4*>(&s_o[w][h][d]);
        if (kHeld) sum = move_held(s_ml[w][h][1], s_ml[w][h][0] - use, sum);
        else sum += f * s_ml[w][h][1];
        add(acc, f, v);
      }
      if (odd_four(acc) && !not_finite(sum) && !(whole && sum == 0.f)) odd |= turn;
      if (whole) {
        emit(h, d, acc, top, sum, std::false_type{});
      } else {
        __stcg(reinterpret_cast<float4*>(&a.part_o[((size_t)slot * HB + h) * HD + d]), acc);
        if (d == 0) __stcg(reinterpret_cast<float2*>(&a.part_ml[(slot * HB + h) * 2]), make_float2(top, sum));
      }
    }
    if (kHeld) {
      __syncthreads();  // e4m3 has no infinities, and a NaN stays one by itself
    } else if (__syncthreads_or(odd)) {  // s_o and s_ml are free from here on, the next piece's queries are where all warps read them
      int* const seen = reinterpret_cast<int*>(&s_o[0][0][0]);
      int seq, len, from = 0;
      if (kTogether && e.of_group) {
        const GroupInfo of = room.info[room.group[e.row]];
        seq = of.seq;
        len = of.tokens;
      } else {
        len = own_len(e.row, &seq);
        if (kTogether) from = room.first[e.row];
      }
      look_through<T, HD>(Layer{a.cache, a.n_kv_heads, a.shift, a.n_pages}, a.table + (size_t)seq * a.max_pages + (from >> a.shift),
                          kTogether ? e.kvh : e.pair / a.blocks_of_heads, (int64_t)e.ta * kTile,
                          min((int64_t)len, (int64_t)e.tb * kTile), seen);
      for (int x = tid; odd && x < e.heads * (HD / 4); x += kThreads, odd >>= 1) {
        if (!(odd & 1u)) continue;
        const int h = x / (HD / 4), d = x % (HD / 4) * 4;
        for (int i = d; i < d + 4; ++i) {
          const float now = made_of(seen[i]);
          if (now == 0.f) continue;
          if (!whole) __stcg(&a.part_o[((size_t)slot * HB + h) * HD + i], now);
          else if (kTogether && meets) __stcg(&record_of(h)->o[e.of_group ? 0 : 1][i], now);
          else a.out[e.row * a.o_token + (int64_t)(e.h0 + h) * a.o_head + i] = (uint16_t)(infinity_bits<T>() | (now > 0.f ? 0u : now < 0.f ? 0x8000u : 0x7fffu));
        }
      }
      __syncthreads();
    }
    bool finished = whole;  // by this block
    if (!whole) {
      // ---- the last block to arrive joins up to kJoin neighbouring pieces; the last of those that did joins what they got
      const int c0 = block_of(e.first_w + kUnitsBefore), c1 = block_of(e.first_w + kUnitsBefore + e.tiles - 1), pieces = c1 - c0 + 1;
      auto slot_of = [&](int b) { return (2 * b + (b == c0)) * HB; };
      // true in the block that is the last of n to arrive at a count, which is zero again then
      auto last_of = [&](unsigned int* count, int n) {
        __threadfence();
        __syncthreads();
        if (tid == 0) {
          s_last = atomicAdd(count, 1u) + 1u == (unsigned)n;
          if (s_last) *count = 0u;
        }
        __syncthreads();
        if (s_last) __threadfence();
        return s_last != 0;
      };
      // the partial results of n blocks, `step` apart, from b on: to the result, or to b's place
      auto join = [&](int b, int n, int step, bool final) {
        for (int x0 = wid * 32; x0 < e.heads * (HD / 4); x0 += kThreads) {  // whole warps
          const int x = x0 + lane, h = x / (HD / 4), d = x % (HD / 4) * 4;
          const bool there = h < e.heads;
          float top = -INFINITY, sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int y0 = 0; y0 < n; y0 += kJoin) {
            float2 ml[kJoin];
            float4 v[kJoin];
#pragma unroll
            for (int y = 0; y < kJoin; ++y) {
              ml[y] = make_float2(-INFINITY, 0.f);
              v[y] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (there && y0 + y < n) {
                const int sl = slot_of(b + (y0 + y) * step) + h;
                ml[y] = __ldcg(reinterpret_cast<const float2*>(&a.part_ml[sl * 2]));
                v[y] = __ldcg(reinterpret_cast<const float4*>(&a.part_o[(size_t)sl * HD + d]));
              }
            }
            float now = top;
#pragma unroll
            for (int y = 0; y < kJoin; ++y) now = fmaxf(now, ml[y].x);
            const float use = now == -INFINITY ? 0.f : now, f0 = exp2_fast(top - use);
            sum = kHeld ? move_held(sum, top - use, 0.f) : sum * f0;
            top = now;
            acc = make_float4(acc.x * f0, acc.y * f0, acc.z * f0, acc.w * f0);
#pragma unroll
            for (int y = 0; y < kJoin; ++y) {
              const float f = exp2_fast(ml[y].x - use);
              if (kHeld) sum = move_held(ml[y].y, ml[y].x - use, sum);
              else sum += f * ml[y].y;
              add(acc, f, v[y]);
            }
          }
          if (there && odd_four(acc))
            acc = keep_infinite(acc, a.part_o + (size_t)(2 * b * HB + h) * HD + d, b == c0 ? HB * HD : 0, (int64_t)2 * step * HB * HD, n);
          __syncwarp();  // b's place is read by the HD / 4 lanes of a head, all of this warp: they are done
          if (!there) continue;
          if (final) {
            emit(h, d, acc, top, sum, std::true_type{});
          } else {
            const int sl = slot_of(b) + h;
            __stcg(reinterpret_cast<float4*>(&a.part_o[(size_t)sl * HD + d]), acc);
            if (d == 0) __stcg(reinterpret_cast<float2*>(&a.part_ml[sl * 2]), make_float2(top, sum));
          }
        }
      };
      const int mine = ((int)blockIdx.x - c0) / kJoin, groups = (pieces + kJoin - 1) / kJoin, b0 = c0 + mine * kJoin;
      if (last_of(&a.count[2 * b0 + (b0 == c0)], min(kJoin, pieces - mine * kJoin))) {
        join(b0, min(kJoin, pieces - mine * kJoin), 1, groups == 1);
        finished = groups == 1;
        unsigned int* count = a.pair_count + ((size_t)e.row * pairs + e.pair) * a.pair_step;
        if (kTogether) count = e.of_group ? &record(e.row, e.pair)->group_count : &record(e.row, e.h0)->pair_count;
        if (groups > 1 && last_of(count, groups)) {
          join(c0, groups, kJoin, true);
          finished = true;
        }
      }
    }
    if constexpr (kTogether) {
      if (finished && meets) {
        // ---- a part of one row, or of a group's up to HB rows: the last part of a row and key-value head to arrive joins them
        const int m0 = e.of_group ? e.h0 / a.group : 0, rows = e.of_group ? (e.h0 + e.heads - 1) / a.group - m0 + 1 : 1;
        auto has_own = [&](int i) { return s_end[n_groups + i] != s_end[n_groups + i - 1]; };
        __threadfence();
        __syncthreads();
        if (tid < rows) {
          const int i = e.row + m0 + tid;
          bool last = false;
          if (room.first[i] > 0 && (!e.of_group || room.group[i] == room.group[e.row])) {
            const int member = i - room.info[room.group[i]].lo;
            const int parts = ((member + 1) * a.group - 1) / HB - member * a.group / HB + 1 + (has_own(i) ? a.blocks_of_heads : 0);
            unsigned int* count = &record(i, e.kvh * a.group)->count;
            last = atomicAdd(count, 1u) + 1u == (unsigned)parts;
            if (last) *count = 0u;
          }
          s_done[tid] = last;
        }
        __syncthreads();
        __threadfence();
        for (int x = tid; x < rows * a.group * (HD / 4); x += kThreads) {
          const int at = x / (HD / 4), d = x % (HD / 4) * 4, r = at / a.group, i = e.row + m0 + r, h = e.kvh * a.group + at - r * a.group;
          if (!s_done[r]) continue;
          const Record* from = record(i, h);
          const bool own = has_own(i);
          const float2 m0 = __ldcg(reinterpret_cast<const float2*>(from->ml[0])), m1 = own ? __ldcg(reinterpret_cast<const float2*>(from->ml[1])) : make_float2(-INFINITY, 0.f);
          const float4 v0 = __ldcg(reinterpret_cast<const float4*>(&from->o[0][d]));
          const float4 v1 = own ? __ldcg(reinterpret_cast<const float4*>(&from->o[1][d])) : make_float4(0.f, 0.f, 0.f, 0.f);
          const float top = fmaxf(m0.x, m1.x), use = top == -INFINITY ? 0.f : top, f0 = exp2_fast(m0.x - use), f1 = exp2_fast(m1.x - use);
          const float sum = f0 * m0.y + f1 * m1.y;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          add(acc, f0, v0);
          add(acc, f1, v1);
          if (odd_four(acc) && !not_finite(sum)) {  // a factor that is 0 makes a NaN of an infinity
            auto kept = [](float now, float u, float w) {
              const float both = (not_finite(u) ? u : 0.f) + (not_finite(w) ? w : 0.f);
              return not_finite(both) ? both : now;
            };
            acc = make_float4(kept(acc.x, v0.x, v1.x), kept(acc.y, v0.y, v1.y), kept(acc.z, v0.z, v1.z), kept(acc.w, v0.w, v1.w));
          }
          result(i, h, d, acc, top, sum, std::true_type{});
        }
        __syncthreads();
      }
    }
  }
  if (kWide && lane == 0 && uses.lost) {  // a block leaves when its copies have landed
    uint32_t patience = npp::kSpinLimit;
    npp::drain_ring(s_full[wid], kSlots, uses.slot(uses.asked), uses.parity(uses.asked), patience);
  }
}

// Heads of a block.  Sixteen read keys and values once for up to sixteen heads, eight have more warps: 64 sequences of 2000 tokens, 64
// heads over 4, 54 us with sixteen and 81 with eight, which read everything twice.
int heads_per_block(int group) { return group <= 8 ? 8 : 16; }

// A layer of the cache as (64 values, rows of a page's heads, halves of head_dim, keys and values, pages); a box is a chunk.
bool make_map(CUtensorMap* map, const DecodeArgs& a, int hd) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t row = (cuuint64_t)hd * 2, rows = (cuuint64_t)a.n_kv_heads << a.shift;
  const cuuint64_t dims[5] = {64, rows, (cuuint64_t)hd / 64, 2, (cuuint64_t)a.n_pages};
  const cuuint64_t strides[4] = {row, 128, rows * row, 2 * rows * row};
  const cuuint32_t box[5] = {64, 16, (cuuint32_t)hd / 64, 2, 1}, estr[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 5, const_cast<char*>(a.cache), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int HD, int kForm, bool kTogether>
cudaError_t launch(const CUtensorMap& map, const DecodeArgs& a, int sms, cudaStream_t s) {
  size_t room = kTogether ? GroupRoom(nullptr, a.n, a.shared.n_groups).bytes : 0;
  if (kForm == kSixteen) room += (size_t)kWarps * kSlots * 16 * HD * 4 + 1024;
  if (kForm == kSixteen || kTogether) {
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = npi::allow_shared(reinterpret_cast<const void*>(k_attn_decode<T, HD, kForm, kTogether>), &done);
    if (e != cudaSuccess) return e;
  }
  const dim3 grid(std::min(kMaxBlocks, blocks_per_sm(HD, kForm) * sms));
  return launch_early(k_attn_decode<T, HD, kForm, kTogether>, grid, kThreads, room, s, map, a);
}
template <class T, int HD>
cudaError_t launch(const CUtensorMap& map, const DecodeArgs& a, int hb, bool held, bool together, int sms, cudaStream_t s) {
  if (held) return hb == 8 ? launch<T, HD, kHeldEight, false>(map, a, sms, s) : launch<T, HD, kHeldSixteen, false>(map, a, sms, s);
  if (together) return hb == 8 ? launch<T, HD, kEight, true>(map, a, sms, s) : launch<T, HD, kSixteen, true>(map, a, sms, s);
  return hb == 8 ? launch<T, HD, kEight, false>(map, a, sms, s) : launch<T, HD, kSixteen, false>(map, a, sms, s);
}

// [(m, l) of the partial results][their O][counts]: the counts start at the same place for every description and n, and the
// rest needs no particular contents, so one workspace serves calls of different sizes in turn.
constexpr uint64_t kSpaceO = (uint64_t)2 * kMaxBlocks * 16 * 8, kSpaceCounts = kSpaceO + (uint64_t)2 * kMaxBlocks * 16 * 128 * 4;
constexpr uint64_t kSpacePairs = kSpaceCounts + (uint64_t)2 * kMaxBlocks * 4;
uint64_t space_bytes(int n_kv_heads, int group, int n) {
  const int hb = heads_per_block(group);
  return kSpacePairs + (uint64_t)n * n_kv_heads * ((group + hb - 1) / hb) * 4;
}

const char* heads_error(const np_kv_desc* d, int n_heads, int n) {
  if (n_heads < 1 || n_heads > (1 << 17) || n_heads % d->n_kv_heads) return "n_heads must be a positive multiple of n_kv_heads, at most 131072";
  if (n < 0 || n > NP_KV_MAX_SEQS) return "n outside [0, NP_KV_MAX_SEQS]";
  return nullptr;
}

}  // namespace

uint64_t decode_parts_bytes() { return kSpacePairs; }

int decode(const np_kv_desc* d, const void* cache, int32_t layer, const np_kv_tables* t, const np_rows* q, int32_t n_heads, const int32_t* seqs, int32_t n,
           float scale2, const np_rows* out, float* lse, void* workspace, const SharedArgs* shared, int sms, cudaStream_t s) {
  DecodeArgs a = {};
  a.page_bytes = page_bytes(d);
  a.cache = static_cast<const char*>(cache) + (int64_t)layer * d->n_pages * a.page_bytes;
  a.table = t->page_table;
  a.lens = t->lens;
  a.seqs = seqs;
  a.status = t->status;
  a.q = static_cast<const uint16_t*>(q->data);
  a.out = static_cast<uint16_t*>(out->data);
  a.q_token = q->token_stride;
  a.q_head = q->head_stride;
  a.o_token = out->token_stride;
  a.o_head = out->head_stride;
  a.lse = lse;
  a.n = n;
  a.n_heads = n_heads;
  a.n_kv_heads = d->n_kv_heads;
  a.group = n_heads / d->n_kv_heads;
  const int hb = heads_per_block(shared && shared->n_groups > 0 ? std::max(a.group, shared->columns) : a.group);
  a.blocks_of_heads = (a.group + hb - 1) / hb;
  a.scale2 = scale2;
  a.shift = log2_of(d->page_tokens);
  a.n_pages = d->n_pages;
  a.max_seqs = d->max_seqs;
  a.max_pages = d->max_pages;
  if (shared) a.shared = *shared;
  char* ws = static_cast<char*>(workspace);
  a.part_ml = reinterpret_cast<float*>(ws);
  a.part_o = reinterpret_cast<float*>(ws + kSpaceO);
  a.count = reinterpret_cast<unsigned int*>(ws + kSpaceCounts);
  a.pair_count = reinterpret_cast<unsigned int*>(ws + kSpacePairs);
  a.pair_step = 1;
  if (shared && shared->n_groups == 0) {  // nothing is shared, but the workspace is of that kind
    a.pair_count = &shared->records->pair_count;
    a.pair_step = sizeof(Record) / 4;
  }
  const bool held = held_in_8(d);
  const bool together = shared && shared->n_groups > 0;
  CUtensorMap map = {};
  if (hb == 16 && !held && !make_map(&map, a, d->head_dim)) return fail(NP_E_INVAL, "a cache that a tensor map does not describe");
  cudaError_t e;
  if (row_type(d) == NP_T_BF16) e = d->head_dim == 128 ? launch<__nv_bfloat16, 128>(map, a, hb, held, together, sms, s) : launch<__nv_bfloat16, 64>(map, a, hb, held, together, sms, s);
  else e = d->head_dim == 128 ? launch<__half, 128>(map, a, hb, held, together, sms, s) : launch<__half, 64>(map, a, hb, held, together, sms, s);
  return e == cudaSuccess ? NP_OK : fail_cuda(e);
}

const char* decode_error(const np_kv_desc* d, const void* cache, int32_t layer, const np_kv_tables* t, const np_rows* q, int32_t n_heads, int32_t n,
                         float scale, const np_rows* out, const void* workspace, float* scale2) {
  if (!cache || !workspace || !t || !t->page_table || !t->lens || !t->status) return "NULL argument";
  if ((uintptr_t)cache % 16 || (uintptr_t)workspace % 16) return "cache and workspace must be 16-byte aligned";
  if (layer < 0 || layer >= d->n_layers) return "layer outside the cache";
  if (!scale_base2(scale, scale2)) return kScaleError;
  if (const char* m = rows_error(q)) return m;
  if (const char* m = rows_error(out)) return m;
  if ((n > 1 && out->token_stride == 0) || (n_heads > 1 && out->head_stride == 0)) return "rows of the result need strides above 0";
  return nullptr;
}

const char* decode_heads_error(const np_kv_desc* d, int n_heads, int n) { return heads_error(d, n_heads, n); }

}  // namespace npa

using namespace npa;

extern "C" {

int np_attn_workspace_bytes(const np_kv_desc* d, int32_t n_heads, int32_t n, uint64_t* out) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  if (const char* m = heads_error(d, n_heads, n)) return fail(NP_E_INVAL, m);
  if (!out) return fail(NP_E_INVAL, "NULL argument");
  *out = space_bytes(d->n_kv_heads, n_heads / d->n_kv_heads, n);
  return NP_OK;
}

int np_attn_decode(const np_kv_desc* d, const void* cache, int32_t layer, const np_kv_tables* t, const np_rows* q, int32_t n_heads,
                   const int32_t* seqs, int32_t n, float scale, const np_rows* out, float* lse, void* workspace,
                   uint64_t workspace_bytes, void* stream) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  if (const char* m = heads_error(d, n_heads, n)) return fail(NP_E_INVAL, m);
  if (!seqs && n > d->max_seqs) return fail(NP_E_INVAL, "n is above max_seqs");
  if (n == 0) return NP_OK;
  float scale2;
  if (const char* m = decode_error(d, cache, layer, t, q, n_heads, n, scale, out, workspace, &scale2)) return fail(NP_E_INVAL, m);
  if (workspace_bytes < space_bytes(d->n_kv_heads, n_heads / d->n_kv_heads, n)) return fail(NP_E_INVAL, "workspace is smaller than np_attn_workspace_bytes says");
  int sms;
  if (!device_sms(&sms)) return fail(NP_E_CUDA, "no CUDA device");
  return decode(d, cache, layer, t, q, n_heads, seqs, n, scale2, out, lse, workspace, nullptr, sms, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
