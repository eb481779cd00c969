// Causal attention over packed prompts (np_attn_prompt).
//
//   o[i] = sum_{j <= i} p_ij v_j / sum_{j <= i} p_ij,   p_ij = exp(scale * q_i . k_j - m_i)     i, j rows of one prompt
//
// Two matrix products per block of rows and 128 keys, S = Q K^T and O += P V, run on the 5th-generation tensor cores with
// S, P and O in tensor memory; the softmax between them runs on the plain cores.  Per 128 x 128 scores at head_dim 128 the
// products take 1024 cycles of the tensor cores and the exponentials 1024 cycles of the special function units, so the two
// have to overlap completely:
//
// * A block holds two tiles of 128 query rows of the same key-value head.  While the plain cores do one tile's softmax, the
//   tensor cores do the other's products.  Roles: two groups of four warps (softmax and result of a tile, a row per lane),
//   one warp that issues the products, one that loads.
// * A tile's 128 rows are (token, query head) pairs of one group, tokens outermost: with eight heads to a group a tile is
//   sixteen tokens, keys and values are read once for all eight, and a short prompt fills its tiles.  Heads that do not
//   divide 128 leave the last rows of a tile unused.
// * Q, K and V come by tiled TMA (128-byte swizzle).  V is the product's B operand with head_dim contiguous, P its A operand in
//   tensor memory, where the softmax overwrites the scores it came from.
// * O is rescaled in tensor memory only when a row's maximum has grown by more than 2^8 since it was last taken; until then
//   probabilities are up to 2^8 instead of 1, which fp32 sums and 16-bit factors hold.  P is rounded to the rows' type (the
//   product takes nothing wider at this rate), the sum l is of the unrounded values.
// * Only tiles that reach past a row are masked.  Rows of the tail tile that belong to the next prompt (or to nobody) are zeroed
//   in V; within a prompt a later token's V meets P = 0 exactly, so only an infinity or a NaN there can reach an earlier row,
//   and a row whose result is not finite is computed again from plain loads over the tokens that it sees.
//
// Every wait is bounded (np_pipe.cuh); after a time-out all roles leave, the block meets and tensor memory is released.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "np_attn.h"
#include "np_device.cuh"
#include "np_internal.h"
#include "np_pipe.cuh"

namespace npa {
namespace {

constexpr int kRows = 128;              // query rows of a tile, keys of a tile
constexpr int kThreads = 320;
constexpr int kMmaWarp = 8, kLoadWarp = 9;
constexpr float kGrow = 8.f;            // log2 of the growth of a maximum that is let pass

struct PromptArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  const int32_t* cu;
  float* lse;
  int32_t* status;
  int n, n_tokens, n_heads, n_kv_heads, group, tile_tokens;
  float scale2;  // scale * log2(e)
};

__device__ __forceinline__ void tma_load_3d(void* dst_smem, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          npp::smem_addr(dst_smem)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(npp::smem_addr(bar))
      : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(npp::smem_addr(bar)) : "memory");
}
// 128-byte swizzle, groups of eight 128-byte rows 1024 bytes apart.  K-major: a row is 64 values along K (lead unused).
// Other way round: a row is 64 values along N for one k, `lead` bytes to the next 64 along N.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(0u)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(0u)
      : "memory");
}

#define NP_R32(r, o)                                                                                                                   \
  "=r"(r[o + 0]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7]),      \
      "=r"(r[o + 8]), "=r"(r[o + 9]), "=r"(r[o + 10]), "=r"(r[o + 11]), "=r"(r[o + 12]), "=r"(r[o + 13]), "=r"(r[o + 14]),             \
      "=r"(r[o + 15]), "=r"(r[o + 16]), "=r"(r[o + 17]), "=r"(r[o + 18]), "=r"(r[o + 19]), "=r"(r[o + 20]), "=r"(r[o + 21]),           \
      "=r"(r[o + 22]), "=r"(r[o + 23]), "=r"(r[o + 24]), "=r"(r[o + 25]), "=r"(r[o + 26]), "=r"(r[o + 27]), "=r"(r[o + 28]),           \
      "=r"(r[o + 29]), "=r"(r[o + 30]), "=r"(r[o + 31])
// 32 columns of this warp's 32 lanes: a lane gets its row's
template <int N>
__device__ __forceinline__ void tm_ld32(uint32_t taddr, uint32_t (&r)[N], int o) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : NP_R32(r, o)
      : "r"(taddr));
}
__device__ __forceinline__ void tm_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  if (kBf16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <bool kBf16>
__device__ __forceinline__ float widen(uint16_t x) {
  return kBf16 ? __uint_as_float((uint32_t)x << 16) : __half2float(__ushort_as_half(x));
}

// One row from plain loads, by a warp: the tokens it sees and no other.
template <bool kBf16, int HD>
__device__ __noinline__ void row_again(const PromptArgs& a, int start, int tok, int head, int kvh, int lane) {
  const uint16_t* q = a.q + (int64_t)(start + tok) * a.q_token + (int64_t)head * a.q_head;
  float top = -INFINITY, sum = 0.f, acc[HD / 32];
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) acc[i] = 0.f;
  for (int base = 0; base <= tok; base += 32) {
    const int j = base + lane;
    float s = -INFINITY;
    if (j <= tok) {
      const uint16_t* k = a.k + (int64_t)(start + j) * a.k_token + (int64_t)kvh * a.k_head;
      s = 0.f;
      for (int d = 0; d < HD; ++d) s = fmaf(widen<kBf16>(q[d]), widen<kBf16>(k[d]), s);
      s *= a.scale2;
    }
    float now = fmaxf(top, s);
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, x));
    const float use = now == -INFINITY ? 0.f : now, f = exp2_fast(top - use), p = j <= tok ? exp2_fast(s - use) : 0.f;
    top = now;
    sum = sum * f + p;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) acc[i] *= f;
    const int most = min(32, tok + 1 - base);
    for (int l = 0; l < most; ++l) {
      const float pl = __shfl_sync(0xffffffffu, p, l);
      const uint16_t* v = a.v + (int64_t)(start + base + l) * a.v_token + (int64_t)kvh * a.v_head;
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) acc[i] = fmaf(pl, widen<kBf16>(v[i * 32 + lane]), acc[i]);
    }
  }
  sum = npd::warp_sum(sum);
  uint16_t* out = a.out + (int64_t)(start + tok) * a.o_token + (int64_t)head * a.o_head;
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) out[i * 32 + lane] = (uint16_t)pack<kBf16>(sum == 0.f ? 0.f : acc[i] / sum, 0.f);
  if (a.lse && lane == 0)
    a.lse[(size_t)(start + tok) * a.n_heads + head] = sum == 0.f ? -INFINITY : (top == -INFINITY ? 0.f : top) * kLn2 + logf(sum);
}

template <int HD>
struct Shape {
  static constexpr int kHalves = HD / 64;                        // 64 values = 128 bytes: one swizzle row
  static constexpr uint32_t kHalfBytes = kRows * 128;            // a tile's rows of one half
  static constexpr uint32_t kTileBytes = kHalves * kHalfBytes;
  static constexpr int kStages = 4;                              // K0 V0 K1 V1 ...
  static constexpr size_t kSmem = (2 + kStages) * (size_t)kTileBytes + 1024;
};

template <bool kBf16, int HD>
__global__ void __launch_bounds__(kThreads, 1)
k_attn_prompt(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
              const __grid_constant__ PromptArgs a) {
  using S = Shape<HD>;
  extern __shared__ __align__(1024) unsigned char tsm[];
  __shared__ int s_end[NP_KV_MAX_SEQS];  // blocks of the prompts up to and including this one
  __shared__ int s_wsum[kThreads / 32];
  __shared__ __align__(8) uint64_t full[S::kStages], empty[S::kStages], q_full, s_full[2], p_full[2], o_full[2], v_fixed;
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_ok[2];
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int block_tokens = 2 * a.tile_tokens;

  // ---- which prompt, which tokens
  int run = 0;
  for (int base = 0; base < a.n; base += kThreads) {
    const int i = base + tid;
    int inc = 0;
    if (i < a.n) {
      const int lo = min(max(a.cu[i], 0), a.n_tokens), hi = min(max(a.cu[i + 1], 0), a.n_tokens);
      inc = hi > lo ? (hi - lo + block_tokens - 1) / block_tokens : 0;
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane == 31) s_wsum[wid] = inc;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < wid) inc += s_wsum[w];
      all += s_wsum[w];
    }
    if (i < a.n) s_end[i] = run + inc;
    run += all;
    __syncthreads();
  }
  // the blocks with the most keys first: a prompt's last tokens
  const int kvh = blockIdx.x % a.n_kv_heads, at = run - 1 - (int)(blockIdx.x / a.n_kv_heads);
  if (at < 0) return;
  int lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (s_end[mid] > at) hi = mid;
    else lo = mid + 1;
  }
  const int start = min(max(a.cu[lo], 0), a.n_tokens), len = min(max(a.cu[lo + 1], 0), a.n_tokens) - start;
  const int q0 = (at - (lo ? s_end[lo - 1] : 0)) * block_tokens;
  // tiles of keys that each tile of rows sees; the second tile may have no row
  int n_kv[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int first = q0 + i * a.tile_tokens, end = min(first + a.tile_tokens, len);
    n_kv[i] = end > first ? (end + kRows - 1) / kRows : 0;
  }
  const int n_tiles = max(n_kv[0], n_kv[1]);
  const bool tail = n_tiles * kRows > len;  // the last tile of keys reaches past the prompt

  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(tsm) + 1023) & ~(uintptr_t)1023);
  unsigned char* q_sm = base;
  unsigned char* ring = base + 2 * S::kTileBytes;

  if (tid == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      npp::mbar_init(&full[s], 1);
      npp::mbar_init(&empty[s], 1);
    }
    npp::mbar_init(&q_full, 1);
    npp::mbar_init(&v_fixed, 1);
    for (int i = 0; i < 2; ++i) {
      npp::mbar_init(&s_full[i], 1);
      npp::mbar_init(&p_full[i], 4);
      npp::mbar_init(&o_full[i], 1);
    }
    npp::fence_barrier_init();
    s_ok[0] = 1;
    s_ok[1] = 0;
  }
  if (wid == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(npp::smem_addr(&s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  auto wait = [&](uint64_t* bar, uint32_t parity) { return npp::wait_or_flag(bar, parity, s_ok, a.status); };

  if (wid == kLoadWarp) {
    // ------------------------------ loads ------------------------------
    int stage = 0;
    uint32_t use = 0;
    bool ok = true;
    if (lane == 0) {
      const int tiles = n_kv[1] > 0 ? 2 : 1;
      npp::mbar_expect_tx(&q_full, (uint32_t)tiles * S::kHalves * 128 * a.group * a.tile_tokens);
      for (int i = 0; i < tiles; ++i)
        for (int h = 0; h < S::kHalves; ++h)
          tma_load_3d(q_sm + i * S::kTileBytes + h * S::kHalfBytes, &map_q, h * 64, kvh * a.group, start + q0 + i * a.tile_tokens, &q_full);
      for (int j = 0; j < 2 * n_tiles; ++j) {
        ok = wait(&empty[stage], (use & 1u) ^ 1u);
        if (!ok) break;
        npp::mbar_expect_tx(&full[stage], S::kTileBytes);
        for (int h = 0; h < S::kHalves; ++h)
          tma_load_3d(ring + stage * S::kTileBytes + h * S::kHalfBytes, j & 1 ? &map_v : &map_k, h * 64, kvh, start + (j >> 1) * kRows, &full[stage]);
        if (++stage == S::kStages) {
          stage = 0;
          ++use;
        }
      }
    }
    ok = __shfl_sync(0xffffffffu, ok, 0);
    if (tail && ok) {
      // rows past the prompt in the last V tile: zero, whatever lies there
      const int s = (2 * n_tiles - 1) % S::kStages;
      if (wait(&full[s], (uint32_t)((2 * n_tiles - 1) / S::kStages) & 1u)) {
        const int from = len - (n_tiles - 1) * kRows, words = (kRows - from) * 8;  // 16-byte words of a half
        for (int e = lane; e < words * S::kHalves; e += 32) {
          const int h = e / words, w = e - h * words;
          *reinterpret_cast<uint4*>(ring + s * S::kTileBytes + h * S::kHalfBytes + from * 128 + w * 16) = make_uint4(0, 0, 0, 0);
        }
      }
      npp::fence_proxy_async();
      __syncwarp();
      if (lane == 0) npp::mbar_arrive(&v_fixed);
    }
    if (lane == 0 && !s_ok[0]) {  // after a time-out nobody else waits for the copies
      uint32_t patience = npp::kSpinLimit;
      npp::drain_ring(full, S::kStages, stage, use & 1u, patience);
      npp::wait_landed(&q_full, 0, patience);
    }
  } else if (wid == kMmaWarp) {
    // ------------------------------ products ------------------------------
    if (lane == 0) {
      const uint32_t fmt = kBf16 ? 1u : 0u;
      const uint32_t common = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(kRows >> 4) << 24);
      const uint32_t id_s = common | ((uint32_t)(kRows >> 3) << 17), id_o = common | (1u << 16) | ((uint32_t)(HD >> 3) << 17);
      const uint32_t q_addr = npp::smem_addr(q_sm), ring_addr = npp::smem_addr(ring);
      auto scores = [&](int i, int st) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint32_t off = (k >> 2) * S::kHalfBytes + (k & 3) * 32;
          mma_ss(tmem + i * kRows, smem_desc(q_addr + i * S::kTileBytes + off, 16), smem_desc(ring_addr + st * S::kTileBytes + off, 16), id_s, k > 0);
        }
        commit(&s_full[i]);
      };
      bool ok = wait(&q_full, 0) && wait(&full[0], 0);
      if (ok) {
        fence_after();
        for (int i = 0; i < 2; ++i)
          if (n_kv[i] > 0) scores(i, 0);
        commit(&empty[0]);
      }
      for (int j = 0; j < n_tiles && ok; ++j) {
        const int sv = (2 * j + 1) % S::kStages, sk = (2 * j + 2) % S::kStages;
        ok = wait(&full[sv], (uint32_t)((2 * j + 1) / S::kStages) & 1u);
        if (ok && j + 1 < n_tiles) ok = wait(&full[sk], (uint32_t)((2 * j + 2) / S::kStages) & 1u);
        if (ok && tail && j + 1 == n_tiles) ok = wait(&v_fixed, 0);
        for (int i = 0; i < 2 && ok; ++i) {
          if (j >= n_kv[i]) continue;
          ok = wait(&p_full[i], (uint32_t)j & 1u);
          if (!ok) break;
          fence_after();
#pragma unroll
          for (int k = 0; k < kRows / 16; ++k)
            mma_ts(tmem + 256 + i * HD, tmem + i * kRows + k * 8, smem_desc(ring_addr + sv * S::kTileBytes + k * 2048, S::kHalfBytes), id_o, (j | k) > 0);
          if (j + 1 < n_kv[i]) scores(i, sk);
          else commit(&o_full[i]);
        }
        if (ok) {
          commit(&empty[sv]);
          if (j + 1 < n_tiles) commit(&empty[sk]);
        }
      }
    }
  } else {
    // ------------------------------ softmax and result of a tile ------------------------------
    const int i = wid >> 2, row = (wid & 3) * 32 + lane;
    const int in_tile = row / a.group, head = kvh * a.group + row - in_tile * a.group;
    const int first = q0 + i * a.tile_tokens, tok = first + in_tile;
    const bool valid = in_tile < a.tile_tokens && tok < len;
    const uint32_t ts = tmem + ((uint32_t)((wid & 3) * 32) << 16) + i * kRows, to = tmem + ((uint32_t)((wid & 3) * 32) << 16) + 256 + i * HD;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int j = 0; j < n_kv[i]; ++j) {
      ok = wait(&s_full[i], (uint32_t)j & 1u);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      fence_after();
      uint32_t s[kRows];
#pragma unroll
      for (int c = 0; c < kRows; c += 32) tm_ld32(ts + c, s, c);
      wait_ld();
      if ((j + 1) * kRows - 1 > first) {  // the tile reaches past the first row
        const int see = tok - j * kRows;
#pragma unroll
        for (int c = 0; c < kRows; ++c)
          if (c > see) s[c] = __float_as_uint(-INFINITY);
      }
      float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int c = 0; c < kRows; c += 4) {
#pragma unroll
        for (int x = 0; x < 4; ++x) top[x] = fmaxf(top[x], __uint_as_float(s[c + x]));
      }
      const float now = fmaxf(m, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.scale2);
      if (j == 0) {
        m = now;
      } else if (__any_sync(0xffffffffu, now > m + kGrow)) {
        const float f = exp2_fast(m - (now == -INFINITY ? 0.f : now));
        m = now;
        l *= f;
#pragma unroll
        for (int c = 0; c < HD; c += 32) {
          uint32_t o[32];
          tm_ld32(to + c, o, 0);
          wait_ld();
          uint32_t w[16];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int x = 0; x < 16; ++x) w[x] = __float_as_uint(__uint_as_float(o[h * 16 + x]) * f);
            tm_st16(to + c + h * 16, w);
          }
        }
      }
      const float use = m == -INFINITY ? 0.f : m;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < kRows; c += 32) {
        uint32_t w[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const float p0 = exp2_fast(fmaf(__uint_as_float(s[c + 2 * x]), a.scale2, -use));
          const float p1 = exp2_fast(fmaf(__uint_as_float(s[c + 2 * x + 1]), a.scale2, -use));
          sum[(2 * x) & 3] += p0;
          sum[(2 * x + 1) & 3] += p1;
          w[x] = pack<kBf16>(p0, p1);
        }
        tm_st16(ts + c / 2, w);
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) npp::mbar_arrive(&p_full[i]);
    }
    if (ok && n_kv[i] > 0) ok = __all_sync(0xffffffffu, wait(&o_full[i], 0));
    if (ok && n_kv[i] > 0) {
      fence_after();
      const float inv = l == 0.f ? 0.f : 1.f / l;
      uint16_t* out = a.out + (int64_t)(start + tok) * a.o_token + (int64_t)head * a.o_head;
      uint32_t big = __float_as_uint(l) & 0x7fffffffu;
#pragma unroll
      for (int c = 0; c < HD; c += 32) {
        uint32_t o[32];
        tm_ld32(to + c, o, 0);
        wait_ld();
#pragma unroll
        for (int x = 0; x < 32; ++x) big = max(big, o[x] & 0x7fffffffu);
        if (valid) {
#pragma unroll
          for (int x = 0; x < 32; x += 8) {
            uint4 v;
            v.x = pack<kBf16>(__uint_as_float(o[x]) * inv, __uint_as_float(o[x + 1]) * inv);
            v.y = pack<kBf16>(__uint_as_float(o[x + 2]) * inv, __uint_as_float(o[x + 3]) * inv);
            v.z = pack<kBf16>(__uint_as_float(o[x + 4]) * inv, __uint_as_float(o[x + 5]) * inv);
            v.w = pack<kBf16>(__uint_as_float(o[x + 6]) * inv, __uint_as_float(o[x + 7]) * inv);
            *reinterpret_cast<uint4*>(out + c + x) = v;
          }
        }
      }
      if (valid && a.lse) a.lse[(size_t)(start + tok) * a.n_heads + head] = l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m) * kLn2 + logf(l);
      uint32_t again = __ballot_sync(0xffffffffu, valid && big >= 0x7f800000u);
      while (again) {
        const int src = __ffs(again) - 1;
        again &= again - 1;
        row_again<kBf16, HD>(a, start, __shfl_sync(0xffffffffu, tok, src), __shfl_sync(0xffffffffu, head, src), kvh, lane);
      }
    }
  }
  fence_before();
  __syncthreads();
  if (wid == kMmaWarp) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess
               ? reinterpret_cast<EncodeFn>(p)
               : nullptr;
  }();
  return fn;
}

// Rows of heads as (head_dim, heads, tokens); a box is 64 values of `box_heads` heads of `box_tokens` tokens.
bool make_map(CUtensorMap* map, const np_rows& r, int hd, int heads, int tokens, int box_heads, int box_tokens) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)hd, (cuuint64_t)heads, (cuuint64_t)tokens};
  // a stride along one element is never used, but has to be a valid one
  const cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)r.head_stride * 2 : (cuuint64_t)hd * 2, tokens > 1 ? (cuuint64_t)r.token_stride * 2 : (cuuint64_t)hd * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, r.data, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool kBf16, int HD>
cudaError_t launch(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const PromptArgs& a, unsigned blocks, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = npi::allow_shared(reinterpret_cast<const void*>(k_attn_prompt<kBf16, HD>), &done);
  return e != cudaSuccess ? e : launch_early(k_attn_prompt<kBf16, HD>, dim3(blocks), kThreads, Shape<HD>::kSmem, s, q, k, v, a);
}

}  // namespace
}  // namespace npa

using namespace npa;

extern "C" int np_attn_prompt(const np_attn_shape* d, const np_rows* q, const np_rows* k, const np_rows* v, const int32_t* cu, int32_t n,
                              int32_t n_tokens, float scale, const np_rows* out, float* lse, int32_t* status, void* stream) {
  if (!d) return fail(NP_E_INVAL, "NULL argument");
  if (d->dtype != NP_T_BF16 && d->dtype != NP_T_FP16) return fail(NP_E_INVAL, "dtype must be NP_T_BF16 or NP_T_FP16");
  if (d->head_dim != 64 && d->head_dim != 128) return fail(NP_E_INVAL, "head_dim must be 64 or 128");
  if (d->n_kv_heads < 1 || d->n_kv_heads > 1024 || d->n_heads < 1 || d->n_heads % d->n_kv_heads)
    return fail(NP_E_INVAL, "n_kv_heads must be in [1, 1024] and divide n_heads");
  for (int r : d->reserved)
    if (r) return fail(NP_E_INVAL, "reserved must be 0");
  const int group = d->n_heads / d->n_kv_heads;
  if (group > NP_ATTN_MAX_GROUP) return fail(NP_E_INVAL, "more than NP_ATTN_MAX_GROUP query heads to a key-value head");
  if (n < 1 || n > NP_KV_MAX_SEQS) return fail(NP_E_INVAL, "n outside [1, NP_KV_MAX_SEQS]");
  if (n_tokens < 0) return fail(NP_E_INVAL, "n_tokens must not be negative");
  if (!std::isfinite(scale) || scale <= 0.f) return fail(NP_E_INVAL, "scale must be positive and finite");
  if (n_tokens == 0) return NP_OK;
  if (!cu || !status) return fail(NP_E_INVAL, "NULL argument");
  for (const np_rows* r : {q, k, v, out})
    if (const char* m = rows_error(r)) return fail(NP_E_INVAL, m);
  for (const np_rows* r : {q, k, v, out}) {
    const bool query = r == q || r == out;
    if ((n_tokens > 1 && r->token_stride == 0) || ((query ? d->n_heads : d->n_kv_heads) > 1 && r->head_stride == 0))
      return fail(NP_E_INVAL, "rows of a prompt need strides above 0");
  }
  PromptArgs a = {};
  a.q = static_cast<const uint16_t*>(q->data);
  a.k = static_cast<const uint16_t*>(k->data);
  a.v = static_cast<const uint16_t*>(v->data);
  a.out = static_cast<uint16_t*>(out->data);
  a.q_token = q->token_stride;
  a.q_head = q->head_stride;
  a.k_token = k->token_stride;
  a.k_head = k->head_stride;
  a.v_token = v->token_stride;
  a.v_head = v->head_stride;
  a.o_token = out->token_stride;
  a.o_head = out->head_stride;
  a.cu = cu;
  a.lse = lse;
  a.status = status;
  a.n = n;
  a.n_tokens = n_tokens;
  a.n_heads = d->n_heads;
  a.n_kv_heads = d->n_kv_heads;
  a.group = group;
  a.tile_tokens = kRows / group;
  a.scale2 = scale * kLog2e;
  // a prompt of x tokens has ceil(x / block) blocks: together at most this many
  const int block_tokens = 2 * a.tile_tokens;
  const int64_t blocks = ((int64_t)n_tokens / block_tokens + std::min<int64_t>(n, n_tokens)) * d->n_kv_heads;
  if (blocks > 0x7fffffffLL) return fail(NP_E_INVAL, "too many tokens for one call");
  int sms;
  if (!device_sms(&sms)) return fail(NP_E_CUDA, "no CUDA device");
  CUtensorMap mq, mk, mv;
  if (!make_map(&mq, *q, d->head_dim, d->n_heads, n_tokens, group, a.tile_tokens) || !make_map(&mk, *k, d->head_dim, d->n_kv_heads, n_tokens, 1, kRows) ||
      !make_map(&mv, *v, d->head_dim, d->n_kv_heads, n_tokens, 1, kRows))
    return fail(NP_E_INVAL, "rows that a tensor map does not describe (strides of 2^40 bytes and more)");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (d->dtype == NP_T_BF16) e = d->head_dim == 128 ? launch<true, 128>(mq, mk, mv, a, (unsigned)blocks, s) : launch<true, 64>(mq, mk, mv, a, (unsigned)blocks, s);
  else e = d->head_dim == 128 ? launch<false, 128>(mq, mk, mv, a, (unsigned)blocks, s) : launch<false, 64>(mq, mk, mv, a, (unsigned)blocks, s);
  return e == cudaSuccess ? NP_OK : fail_cuda(e);
}
