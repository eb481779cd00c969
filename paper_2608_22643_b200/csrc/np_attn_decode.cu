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
// Measured (pages of 64 scattered over the pool, caches larger than the L2 in turn): sixteen sequences of 0 to 4095 tokens, 32 heads
// of 128, 57.3 us, 5.8 TB/s, 89 % of the copy rate; 64 of 1000 in fp16 159 us, 100 %; one of 131071 tokens, 64 heads over 8, 91.9 us,
// 89 %; one of 100 tokens 4.7 us.  What is not the stream is the launch, three loads that depend on one another (length, page
// number, keys) and the joins.  Groups of more than eight heads are bound by the steps
// between a warp's loads: sixteen heads of 128 to a key-value head, 64 sequences of 2000 tokens, 53.8 us, 74 % (69 % with keys and values
// in registers, 55 % with 16-byte asynchronous copies in place of TMA, 70 % with the chunks beyond asked into the L2 ahead, 74 % with
// keys and values as two copies).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "np_attn.h"
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
  unsigned int* pair_count;  // [n * pairs] the same of joined ones
  float* part_ml;            // [2 * kMaxBlocks][HB][2]
  float* part_o;             // [2 * kMaxBlocks][HB][HD]
  float scale2;              // scale * log2(e)
  int n, n_heads, n_kv_heads, group, blocks_of_heads;  // heads of a group: blocks_of_heads pieces of HB
  int shift, n_pages, max_seqs, max_pages;
};

template <class T>
struct Half2;
template <>
struct Half2<__nv_bfloat16> {
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
  // (x, y) rounded, and what the rounding left, rounded
  static __device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    const float2 f = __bfloat1622float2(h);
    const __nv_bfloat162 l = __floats2bfloat162_rn(x - f.x, y - f.y);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = *reinterpret_cast<const uint32_t*>(&l);
  }
  static __device__ __forceinline__ uint16_t round(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
};
template <>
struct Half2<__half> {
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
  static __device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo) {
    const __half2 h = __floats2half2_rn(x, y);
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(x - f.x, y - f.y);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = *reinterpret_cast<const uint32_t*>(&l);
  }
  static __device__ __forceinline__ uint16_t round(float x) { return __half_as_ushort(__float2half_rn(x)); }
};

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
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
// keys and values of sixteen tokens: (64 values, rows of a page's heads, halves of head_dim, keys and values, pages)
__device__ __forceinline__ void tma_load_chunk(uint32_t dst, const CUtensorMap* map, int row, int page, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %2, %4}], [%5];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(page), "r"(npp::smem_addr(bar))
               : "memory");
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// a / b, by 32 bits where they do
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
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

template <class T>
__device__ __forceinline__ constexpr uint32_t infinity_bits() {
  return std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
}
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// By a whole block: results of tiles [ta, tb) of (row, pair) that are not finite, where V has anything of that kind among them.  Weights are
// above 0, so an infinity stays one, and two of different signs or a NaN make a NaN; what the sums made of finite values stays.  V is looked
// through once for all heads, eight values to a thread.  `odd`: bit k if the thread is to look at the four values of its turn k over heads and
// head_dim; part_o: of the partial result, nullptr: out.  seen: HD ints of shared memory that are free.  One of 131071 tokens a NaN, 64
// heads over 8: 201 us a call in place of 93. (One block that looks through all of V behind the join: 10 ms.)
template <class T, int HD>
__device__ __noinline__ void mend(const DecodeArgs& a, uint32_t odd, int row, int pair, int ta, int tb, int h0, int heads, float* part_o, int* seen) {
  constexpr int kCols = HD / 8, kStep = kThreads / kCols, kAhead = 4;
  constexpr uint32_t kInf = infinity_bits<T>();
  const int tid = threadIdx.x;
  for (int d = tid; d < HD; d += kThreads) seen[d] = 0;
  __syncthreads();
  int seq;
  const int64_t len = min((int64_t)row_len(a, row, &seq), (int64_t)tb * kTile);
  const int col = tid % kCols;
  const int32_t* pages = a.table + (size_t)seq * a.max_pages;
  const int64_t head_bytes = (int64_t)(HD * 2) << a.shift;
  const char* v = a.cache + (a.n_kv_heads + pair / a.blocks_of_heads) * head_bytes + col * 16;
  uint32_t bits = 0;  // value x of the column: 1 << x a NaN, 256 << x inf, 65536 << x -inf
  for (int64_t j0 = (int64_t)ta * kTile + tid / kCols; j0 < len; j0 += kAhead * kStep) {
    int pg[kAhead];
    uint4 w[kAhead];
#pragma unroll
    for (int y = 0; y < kAhead; ++y) pg[y] = j0 + y * kStep < len ? pages[(j0 + y * kStep) >> a.shift] : -1;
#pragma unroll
    for (int y = 0; y < kAhead; ++y) {
      w[y] = make_uint4(0, 0, 0, 0);
      if ((unsigned)pg[y] < (unsigned)a.n_pages)
        w[y] = npd::ldg_stream(v + (int64_t)pg[y] * 2 * a.n_kv_heads * head_bytes + ((j0 + y * kStep) & ((1 << a.shift) - 1)) * (HD * 2));
    }
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const uint32_t b = word(w[y], x >> 1) >> (x & 1) * 16 & 0xffffu;
        if ((b & kInf) == kInf) bits |= (b & 0x7fffu) != kInf ? 1u << x : b == kInf ? 256u << x : 65536u << x;
      }
  }
  for (int x = 0; bits && x < 8; ++x)
    if (const int what = bits >> x & 0x10101) atomicOr(&seen[col * 8 + x], what);
  __syncthreads();
  for (int x = tid; odd && x < heads * (HD / 4); x += kThreads, odd >>= 1) {
    if (!(odd & 1u)) continue;
    const int h = x / (HD / 4), d = x % (HD / 4) * 4;
    uint16_t* out = a.out + row * a.o_token + (int64_t)(h0 + h) * a.o_head + d;
    float* part = part_o + h * HD + d;
    for (int i = 0; i < 4; ++i) {
      const int what = seen[d + i];
      if (!what) continue;
      const uint32_t now = what == 0x100 ? kInf : what == 0x10000 ? kInf | 0x8000u : 0x7fffu;
      if (part_o == nullptr) out[i] = (uint16_t)now;
      else __stcg(&part[i], what == 0x100 ? INFINITY : what == 0x10000 ? -INFINITY : __uint_as_float(0x7fffffffu));
    }
  }
  __syncthreads();
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
// accumulators.  us with one more and with this many (sixteen heads: with keys and values in registers): 128 values, eight heads, four blocks 113 (the long sequence) and 186 (64 of 1000),
// three 101 and 164; sixteen heads, 64 of 2000, three 73.8, two 62.4.  64 values, eight heads, 64 heads, 16 sequences of 2000, five
// 91.2, four 86.8 (three 93.9); sixteen heads, one of 131071, four 43.3, three 40.2 (two 45.0).
constexpr int blocks_per_sm(int hd, int heads) { return hd == 64 ? (heads == 8 ? 4 : 3) : (heads == 8 ? 3 : 2); }

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

template <class T, int HD, bool kWide>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(HD, kWide ? 16 : 8))
k_attn_decode(const __grid_constant__ CUtensorMap map, const __grid_constant__ DecodeArgs a) {
  constexpr int HB = kWide ? 16 : 8;  // heads of a block, at most
  constexpr int KV = HD / 32;        // 16-byte pieces of a key row per lane
  constexpr int VC = HD / 64;        // 16-byte pieces of a value row per lane
  constexpr int QV = HB * HD / 8 / kThreads > 0 ? HB * HD / 8 / kThreads : 1;  // 16-byte pieces of the queries per thread
  // Sixteen heads: sixteen-value steps along head_dim; bytes of a chunk's keys, and of its keys and values
  constexpr int KS = HD / 16;
  constexpr uint32_t kHalf = 16 * HD * 2, kSlot = 2 * kHalf;
  // Bytes from query to query, values from head to head of a warp's result, in shared memory: reads and stores meet all banks
  constexpr int QR = HD * 2 + (kWide ? 16 : 64), SO = HD + (kWide ? 8 : 0);
  __shared__ int64_t s_end[NP_KV_MAX_SEQS];             // tiles of the rows up to and including this one
  __shared__ __align__(16) float s_o[kWarps][HB][SO];
  __shared__ __align__(8) uint64_t s_full[kWarps][kSlots];  // a warp's ring is its own
  extern __shared__ __align__(1024) unsigned char s_dyn[];
  __shared__ __align__(16) unsigned char s_q[HB * QR];
  __shared__ float s_ml[kWarps][HB][2];
  __shared__ int64_t s_wsum[kWarps];
  __shared__ int s_last;
  __shared__ volatile int s_lost[kWarps];  // a wait of the warp was given up
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

  // ---- units (tiles, and a group's start) of every row, summed up; rows without tokens are answered here
  int64_t run = 0;
  if (a.n <= 32) {  // every warp by itself: all write the same
    int len = 0, seq = -1;
    if (lane < a.n) len = row_len(a, lane, &seq);
    int64_t inc = len > 0 ? ((int64_t)len + kTile - 1) / kTile + kStart : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane < a.n) s_end[lane] = inc;
    run = __shfl_sync(0xffffffffu, inc, 31);
    __syncwarp();
  } else {
    for (int base = 0; base < a.n; base += kThreads) {
      const int i = base + tid;
      int len = 0, seq = -1;
      if (i < a.n) len = row_len(a, i, &seq);
      int64_t inc = len > 0 ? ((int64_t)len + kTile - 1) / kTile + kStart : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
      }
      if (lane == 31) s_wsum[wid] = inc;
      __syncthreads();
      for (int w = 0; w < wid; ++w) inc += s_wsum[w];
      if (i < a.n) s_end[i] = run + inc;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) run += s_wsum[w];
      __syncthreads();
    }
  }
  for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
    if (s_end[i] != (i ? s_end[i - 1] : 0)) continue;
    for (int e = tid; e < a.n_heads * (HD / 8); e += kThreads) {
      const int h = e / (HD / 8), d = e % (HD / 8) * 8;
      *reinterpret_cast<uint4*>(a.out + i * a.o_token + h * a.o_head + d) = make_uint4(0, 0, 0, 0);
      if (a.lse && d == 0) a.lse[(size_t)i * a.n_heads + h] = -INFINITY;
    }
  }
  // the line's W units over G blocks: the first `more` blocks take each + 1 of them, the others each
  const int64_t W = run * pairs;
  const int G = (int)min((int64_t)gridDim.x, (W + kMinTiles - 1) / kMinTiles);
  if ((int)blockIdx.x >= G) return;
  const int64_t each = divide(W, G), more = W - each * G;
  auto block_of = [&](int64_t w) { return (int)(w < more * (each + 1) ? divide(w, each + 1) : more + divide(w - more * (each + 1), each)); };
  int64_t w0 = blockIdx.x * each + min((int64_t)blockIdx.x, more);
  const int64_t w1 = w0 + each + (blockIdx.x < more ? 1 : 0);
  int row = 0;
  {
    int lo = 0, hi = a.n - 1;  // the first row whose units end after w0
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_end[mid] * pairs > w0) hi = mid;
      else lo = mid + 1;
    }
    row = lo;
  }

  const int64_t head_bytes = (int64_t)(HD * 2) << a.shift, page_bytes = 2 * a.n_kv_heads * head_bytes;
  struct Piece {  // tiles [ta, tb) of one (row, pair)
    int row, pair, h0, heads, len, tiles, ta, tb;
    int64_t first_w;  // of its pair, on the line
    const int32_t* pages;
    int first_row;    // of its key-value head in a page
    const char* kbase;
    const char* vbase;
  };
  // the next piece with tokens from w0 on; false: none is left
  auto next_piece = [&](Piece& p) {
    while (w0 < w1) {
      while (s_end[row] * pairs <= w0) ++row;
      const int64_t before = row ? s_end[row - 1] : 0, units = s_end[row] - before, r0 = w0 - before * pairs;
      const int pair = (int)divide(r0, units);
      const int64_t ra = r0 - pair * units, rb = min(units, ra + (w1 - w0));
      p.first_w = w0 - ra;
      w0 += rb - ra;
      p.ta = (int)max((int64_t)0, ra - kStart);
      p.tb = (int)max((int64_t)0, rb - kStart);
      if (p.ta == p.tb) continue;  // the start alone: whoever has the first tile begins
      p.row = row;
      p.pair = pair;
      p.tiles = (int)(units - kStart);
      int seq;
      p.len = row_len(a, row, &seq);
      const int kvh = pair / a.blocks_of_heads, hb = pair - kvh * a.blocks_of_heads;
      p.h0 = kvh * a.group + hb * HB;
      p.heads = min(HB, a.group - hb * HB);
      p.pages = a.table + (size_t)seq * a.max_pages;
      p.first_row = kvh << a.shift;
      p.kbase = a.cache + kvh * head_bytes;
      p.vbase = p.kbase + a.n_kv_heads * head_bytes;
      return true;
    }
    return false;
  };

  uint4 qf[QV], kf[2][KV], vf[4][VC];
  Piece p = {};
  int chunk_end, c, have, have_next, pg_next;  // chunks of 16 tokens
  int64_t at, at_next;
  int waiting[kSlots];                 // tokens of the chunks in this warp's ring
  npp::WarpRing<kSlots> uses;
  WarpWaits waits = {&s_lost[wid], a.status};
  const uint32_t ring = ((npp::smem_addr(s_dyn) + 1023) & ~1023u) + wid * kSlots * kSlot;
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
    chunk_end = (int)min(((int64_t)p.len + 15) >> 4, (int64_t)p.tb * kWarps);
    c = p.ta * kWarps + wid;
    int pg[kSlots + 1];
#pragma unroll
    for (int i = 0; i < (kWide ? kSlots : 1) + 1; ++i) pg[i] = page_of(c + i * kWarps);
#pragma unroll
    for (int j = 0; j < QV; ++j) {
      const int x = j * kThreads + tid, h = x / (HD / 8), d = x % (HD / 8) * 8;
      qf[j] = make_uint4(0, 0, 0, 0);
      if (h < p.heads) qf[j] = *reinterpret_cast<const uint4*>(a.q + p.row * a.q_token + (int64_t)(p.h0 + h) * a.q_head + d);
    }
    if constexpr (kWide) {
      __syncwarp();  // all lanes have read what the ring held
#pragma unroll
      for (int i = 0; i < kSlots; ++i) waiting[i] = ask(c + i * kWarps, pg[i]);
      pg_next = pg[kSlots];
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
  // four values of a head's result; its log of the sum with the first
  auto result = [&](int i, int h, int d, const float4& acc, float use, float sum) {
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    uint2 r;
    r.x = (uint32_t)Half2<T>::round(none ? 0.f : acc.x * inv) | (uint32_t)Half2<T>::round(none ? 0.f : acc.y * inv) << 16;
    r.y = (uint32_t)Half2<T>::round(none ? 0.f : acc.z * inv) | (uint32_t)Half2<T>::round(none ? 0.f : acc.w * inv) << 16;
    *reinterpret_cast<uint2*>(a.out + i * a.o_token + (int64_t)h * a.o_head + d) = r;
    if (a.lse && d == 0) a.lse[(size_t)i * a.n_heads + h] = none ? -INFINITY : use * kLn2 + logf(sum);
  };
  // the queries that begin() asked for go where all warps read them; a barrier follows
  auto keep_queries = [&] {
#pragma unroll
    for (int j = 0; j < QV; ++j) {
      const int x = j * kThreads + tid, h = x / (HD / 8), d = x % (HD / 8);
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
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[kWide ? 2 * KS : VC * 4][4];
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
    auto raise = [&](const float (&top)[2], float (&use)[2], auto by) {
      float now[2];
      bool grew = false;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        now[i] = fmaxf(m[i], top[i]);
        use[i] = now[i] == -INFINITY ? 0.f : now[i];  // -inf so far: nothing has been added up yet
        grew |= now[i] > m[i];
      }
      if (!__any_sync(0xffffffffu, grew)) return;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float f = exp2_fast(m[i] - use[i]);
        m[i] = now[i];
        l[i] *= f;
        by(i, f);
      }
    };
    if constexpr (!kWide) {
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
    for (int i = 0; i < 2; ++i) {
      const int h = kWide ? g + 8 * i : 2 * t + i;
#pragma unroll
      for (int x = kWide ? 1 : 4; x < (kWide ? 4 : 32); x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
      if (h < e.heads) {
        if ((kWide ? t : g) == 0) {
          s_ml[wid][h][0] = m[i];
          s_ml[wid][h][1] = l[i];
        }
        if constexpr (!kWide) {
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
        sum += f * s_ml[w][h][1];
        add(acc, f, v);
      }
      if (odd_four(acc) && !not_finite(sum) && !(whole && sum == 0.f)) odd |= turn;
      if (whole) {
        result(e.row, e.h0 + h, d, acc, use, sum);
      } else {
        __stcg(reinterpret_cast<float4*>(&a.part_o[((size_t)slot * HB + h) * HD + d]), acc);
        if (d == 0) __stcg(reinterpret_cast<float2*>(&a.part_ml[(slot * HB + h) * 2]), make_float2(top, sum));
      }
    }
    if (__syncthreads_or(odd))  // s_o and s_ml are free from here on, the next piece's queries are where all warps read them
      mend<T, HD>(a, odd, e.row, e.pair, e.ta, e.tb, e.h0, e.heads, whole ? nullptr : a.part_o + (size_t)slot * HB * HD, reinterpret_cast<int*>(&s_o[0][0][0]));
    if (!whole) {
      // ---- the last block to arrive joins up to kJoin neighbouring pieces; the last of those that did joins what they got
      const int c0 = block_of(e.first_w + kStart), c1 = block_of(e.first_w + kStart + e.tiles - 1), pieces = c1 - c0 + 1;
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
            top = now;
            sum *= f0;
            acc = make_float4(acc.x * f0, acc.y * f0, acc.z * f0, acc.w * f0);
#pragma unroll
            for (int y = 0; y < kJoin; ++y) {
              const float f = exp2_fast(ml[y].x - use);
              sum += f * ml[y].y;
              add(acc, f, v[y]);
            }
          }
          if (there && odd_four(acc))
            acc = keep_infinite(acc, a.part_o + (size_t)(2 * b * HB + h) * HD + d, b == c0 ? HB * HD : 0, (int64_t)2 * step * HB * HD, n);
          __syncwarp();  // b's place is read by the HD / 4 lanes of a head, all of this warp: they are done
          if (!there) continue;
          if (final) {
            result(e.row, e.h0 + h, d, acc, top == -INFINITY ? 0.f : top, sum);
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
        if (groups > 1 && last_of(&a.pair_count[(size_t)e.row * pairs + e.pair], groups)) join(c0, groups, kJoin, true);
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

template <class T, int HD, bool kWide>
cudaError_t launch(const CUtensorMap& map, const DecodeArgs& a, int sms, cudaStream_t s) {
  size_t ring = 0;
  if (kWide) {
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = npi::allow_shared(reinterpret_cast<const void*>(k_attn_decode<T, HD, kWide>), &done);
    if (e != cudaSuccess) return e;
    ring = (size_t)kWarps * kSlots * 16 * HD * 4 + 1024;
  }
  const dim3 grid(std::min(kMaxBlocks, blocks_per_sm(HD, kWide ? 16 : 8) * sms));
  return launch_early(k_attn_decode<T, HD, kWide>, grid, kThreads, ring, s, map, a);
}
template <class T>
cudaError_t launch(const CUtensorMap& map, const DecodeArgs& a, int hd, int hb, int sms, cudaStream_t s) {
  if (hd == 128) return hb == 8 ? launch<T, 128, false>(map, a, sms, s) : launch<T, 128, true>(map, a, sms, s);
  return hb == 8 ? launch<T, 64, false>(map, a, sms, s) : launch<T, 64, true>(map, a, sms, s);
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
  if (!cache || !workspace || !t || !t->page_table || !t->lens || !t->status) return fail(NP_E_INVAL, "NULL argument");
  if ((uintptr_t)cache % 16 || (uintptr_t)workspace % 16) return fail(NP_E_INVAL, "cache and workspace must be 16-byte aligned");
  if (workspace_bytes < space_bytes(d->n_kv_heads, n_heads / d->n_kv_heads, n)) return fail(NP_E_INVAL, "workspace is smaller than np_attn_workspace_bytes says");
  if (layer < 0 || layer >= d->n_layers) return fail(NP_E_INVAL, "layer outside the cache");
  float scale2;
  if (!scale_base2(scale, &scale2)) return fail(NP_E_INVAL, kScaleError);
  if (const char* m = rows_error(q)) return fail(NP_E_INVAL, m);
  if (const char* m = rows_error(out)) return fail(NP_E_INVAL, m);
  if ((n > 1 && out->token_stride == 0) || (n_heads > 1 && out->head_stride == 0)) return fail(NP_E_INVAL, "rows of the result need strides above 0");
  int sms;
  if (!device_sms(&sms)) return fail(NP_E_CUDA, "no CUDA device");
  const int64_t page = (int64_t)2 * d->n_kv_heads * d->page_tokens * d->head_dim * 2;
  DecodeArgs a = {};
  a.cache = static_cast<const char*>(cache) + (int64_t)layer * d->n_pages * page;
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
  const int hb = heads_per_block(a.group);
  a.blocks_of_heads = (a.group + hb - 1) / hb;
  a.scale2 = scale2;
  a.shift = log2_of(d->page_tokens);
  a.n_pages = d->n_pages;
  a.max_seqs = d->max_seqs;
  a.max_pages = d->max_pages;
  char* ws = static_cast<char*>(workspace);
  a.part_ml = reinterpret_cast<float*>(ws);
  a.part_o = reinterpret_cast<float*>(ws + kSpaceO);
  a.count = reinterpret_cast<unsigned int*>(ws + kSpaceCounts);
  a.pair_count = reinterpret_cast<unsigned int*>(ws + kSpacePairs);
  CUtensorMap map = {};
  if (hb == 16 && !make_map(&map, a, d->head_dim)) return fail(NP_E_INVAL, "a cache that a tensor map does not describe");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = d->dtype == NP_T_BF16 ? launch<__nv_bfloat16>(map, a, d->head_dim, hb, sms, s) : launch<__half>(map, a, d->head_dim, hb, sms, s);
  return e == cudaSuccess ? NP_OK : fail_cuda(e);
}

}  // extern "C"
