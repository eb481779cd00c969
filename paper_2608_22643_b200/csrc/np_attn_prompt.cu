// Causal attention over packed prompts (np_attn_prompt).
//
//   o[i] = sum_{j <= i} p_ij v_j / sum_{j <= i} p_ij,   p_ij = exp(scale * q_i . k_j - m_i)     i, j rows of one prompt
//
// Two matrix products per block of rows and 128 keys, S = Q K^T and O += P V, run on the 5th-generation tensor cores with
// S, P and O in tensor memory; the softmax between them runs on the plain cores.  Per 128 x 128 scores at head_dim 128 the
// products take 1024 cycles of the tensor cores, their operands as many of shared memory's bandwidth, and the exponentials 1024
// cycles of the special function units, so all three have to overlap completely.  They do to 60 % (3260 cycles for two such tiles,
// both pipes busy 60 % of the time); what is left is hand-overs between the roles.  8192 tokens, 64 heads over 8: 900 us (1220
// TFLOP/s) as long as the clock holds, 960 to 1015 (1080 to 1150) in the long run, at the power limit.  With heads of 64 the exponentials
// stay what they are and the products halve: 8192 tokens, 64 heads, 764 us (720 TFLOP/s), exponential units busy 66 %.
//
// * A block holds two tiles of 128 query rows of the same key-value head (or an SM two blocks of one tile, for short prompts).
//   While the plain cores do one tile's softmax, the tensor cores do the other's products.  Roles: four warps to a tile (softmax and
//   result, a row per lane), one warp each that issues the products, loads, and lays out the block's next work.
// * Blocks stay and take one block of work after the other, the ones with the most keys first; loads and the first scores of the
//   next run while the result of the last is stored.
// * A tile's 128 rows are (token, query head) pairs of one group, tokens outermost: with eight heads to a group a tile is
//   sixteen tokens, keys and values are read once for all eight, and a short prompt fills its tiles.  Heads that do not
//   divide 128 leave the last rows of a tile unused.
// * Q, K and V come by tiled TMA (128-byte swizzle).  V is the product's B operand with head_dim contiguous, P its A operand in
//   tensor memory, where the softmax overwrites the scores it came from; the product over the first 64 keys starts while the
//   exponentials of the others are on their way.
// * O is rescaled in tensor memory only when a row's maximum has grown by more than 2^8 since it was last taken; until then
//   probabilities are up to 2^8 instead of 1, which fp32 sums and 16-bit factors hold.  P is rounded to the rows' type (the
//   product takes nothing wider at this rate), the sum l is of the unrounded values.
// * Only tiles that reach past a row are masked.  Rows of the last tile that belong to the next prompt (or to nobody) are zeroed in V;
//   within a prompt a later token's V meets P = 0 exactly, which only an infinity or a NaN survives: where a result is not finite,
//   mend_rows looks up whether the tokens that the row sees make it so.  (A warp that looks through these tiles' V beforehand is
//   simpler, and cost 2 to 10 %: its code, mostly.)
// * Short prompts wait for instructions: what is off the usual path (rescaling, the result) is kept in loops.  Unrolled, twelve
//   prompts of 0 to 1500 tokens, 32 heads, took 90 us instead of 80.  Measured and dropped: exponentials on the FMA units by a
//   polynomial (they are no less busy; heads of 128), two lanes to a row (the exchange costs what the halves save), scores read from tensor
//   memory 32 at a time, a warp of products for each tile (the tiles fall into step), the next block's first scores before the
//   other tile's last product.
//
// Every wait is bounded; after a time-out all roles leave, the block meets and tensor memory is released.
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
constexpr float kGrow = 8.f;            // log2 of the growth of a maximum that is let pass
// The largest score (times log2(e), either sign) that an exponent may be formed from by one fused step, s * scale2 - m.  m is a rounded product;
// what the rounding took off stays in the exponent, 1 at most up to here, and cancels between P and its sum.  Past it that passes the range
// of P (2^16 in fp16) and in the end of fp32, so the products are rounded first, as m is.
constexpr float kLarge = 16777216.f;
constexpr int kPlans = 2;               // blocks of work that are laid out ahead
// Polls that a wait may take, a second or two: a tile without rows waits for a whole block of work of the other.  Rows that are computed again
// take longer than that from a million tokens on, and the block's other roles wait for them; so a warp that does it raises the block's
// limit by 2^22 polls (100 ms) for every kBeat tokens (12 ms), to 2^30 (half a minute) at most.
constexpr int kWaitPolls = 1 << 26, kMostPolls = 1 << 30, kBeatPolls = 1 << 22, kBeat = 1 << 16;
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
  int out32;     // rows of out start on 32-byte boundaries
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
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
// one lane of a warp, the same every time
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
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
__device__ __forceinline__ void tm_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tm_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// The block's registers are dealt out anew: 192 or 200 for each thread of the softmax warps, which hold a row of scores, the rest for the
// four others.  Two tiles: 384 threads x 168 = 8 warps x 200 + 4 x 104; one tile: 256 x 128 = 4 x 192 + 4 x 64.
template <int kTiles>
__device__ __forceinline__ void more_registers() {
  if (kTiles == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
}
template <int kTiles>
__device__ __forceinline__ void fewer_registers() {
  if (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
}
// 32 bytes, 32-byte aligned: a whole sector
__device__ __forceinline__ void store32(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
               "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// The loads have arrived.  Their registers pass through: what uses them comes behind the wait.
template <int N>
__device__ __forceinline__ void wait_ld(uint32_t (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int o = 0; o < N; o += 16)
    asm volatile(""
                 : "+r"(r[o + 0]), "+r"(r[o + 1]), "+r"(r[o + 2]), "+r"(r[o + 3]), "+r"(r[o + 4]), "+r"(r[o + 5]), "+r"(r[o + 6]), "+r"(r[o + 7]),
                   "+r"(r[o + 8]), "+r"(r[o + 9]), "+r"(r[o + 10]), "+r"(r[o + 11]), "+r"(r[o + 12]), "+r"(r[o + 13]), "+r"(r[o + 14]),
                   "+r"(r[o + 15]));
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
typedef unsigned long long f32x2;  // two fp32 that one instruction works on
__device__ __forceinline__ f32x2 two(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void apart(f32x2 x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// the largest of three; a NaN among them is the result
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
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

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// A step of rows that are computed again: what waits for them may take longer.  A limit of 0 stays.
__device__ __forceinline__ void raise_limit(int* limit) {
  const int was = *static_cast<volatile int*>(limit);
  if (was > 0 && was < kMostPolls) atomicCAS(limit, was, was + kBeatPolls);
}

// Rows by plain loads, over the tokens that they see and no others; results replace what is not finite, where they are finite themselves.
// Four rows and eight tokens at a time: a lane has HD / 32 values of head_dim, then one of the 32 scores.
template <bool kBf16, int HD>
__device__ __noinline__ void rows_again(const PromptArgs& a, uint32_t rows, int start, int row_tok, int row_head, int kvh, int lane, int* limit) {
  constexpr int N = HD / 32, R = 4, T = 8;
  auto load = [](const uint16_t* p, float (&x)[N]) {
    uint32_t w[N / 2];
    if constexpr (N == 4) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x;
      w[1] = v.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = widen<kBf16>((uint16_t)(w[i / 2] >> (i & 1) * 16));
  };
  const uint16_t* k0 = a.k + (int64_t)start * a.k_token + (int64_t)kvh * a.k_head + lane * N;
  const uint16_t* v0 = a.v + (int64_t)start * a.v_token + (int64_t)kvh * a.v_head + lane * N;
  while (rows) {
    int tok[R], head[R], last = 0;
    float q[R][N], acc[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int src = rows ? __ffs(rows) - 1 : 0;
      tok[r] = __shfl_sync(0xffffffffu, row_tok, src);
      head[r] = __shfl_sync(0xffffffffu, row_head, src);
      if (!rows) tok[r] = -1;  // no row: sees nothing
      rows &= rows - 1;
      last = max(last, tok[r]);
      load(a.q + (int64_t)(start + max(tok[r], 0)) * a.q_token + (int64_t)head[r] * a.q_head + lane * N, q[r]);
#pragma unroll
      for (int i = 0; i < N; ++i) acc[r][i] = 0.f;
    }
    const int mine = lane < 8 ? tok[0] : lane < 16 ? tok[1] : lane < 24 ? tok[2] : tok[3];
    float top = -INFINITY, sum = 0.f;  // of row lane / 8; the sum of tokens lane % 8, + 8, ...
    for (int base = 0; base <= last; base += T) {
      if ((base & (kBeat - 1)) == 0 && lane == 0) raise_limit(limit);
      float s[R * T], v[T][N];
#pragma unroll
      for (int x = 0; x < T; ++x) {
        const int64_t j = min(base + x, last);
        float k[N];
        load(k0 + j * a.k_token, k);
        load(v0 + j * a.v_token, v[x]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          s[r * T + x] = q[r][0] * k[0];
#pragma unroll
          for (int i = 1; i < N; ++i) s[r * T + x] = fmaf(q[r][i], k[i], s[r * T + x]);
        }
      }
#pragma unroll
      for (int w = 16; w >= 1; w >>= 1)  // lane l gets the sum over all lanes of s[l]
#pragma unroll
        for (int i = 0; i < w; ++i) {
          const bool up = lane & w;
          s[i] = (up ? s[i + w] : s[i]) + __shfl_xor_sync(0xffffffffu, up ? s[i] : s[i + w], w);
        }
      const float score = base + (lane & 7) <= mine ? s[0] * a.scale2 : -INFINITY;
      float now = fmaxf(top, score);
#pragma unroll
      for (int x = 1; x < T; x <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, x));
      const float use = now == -INFINITY ? 0.f : now, f = exp2_fast(top - use), p = exp2_fast(score - use);
      top = now;
      sum = sum * f + p;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float fr = __shfl_sync(0xffffffffu, f, r * T);
#pragma unroll
        for (int i = 0; i < N; ++i) acc[r][i] *= fr;
#pragma unroll
        for (int x = 0; x < T; ++x) {
          const float pr = __shfl_sync(0xffffffffu, p, r * T + x);
          if (base + x > tok[r]) continue;
#pragma unroll
          for (int i = 0; i < N; ++i) acc[r][i] = fmaf(pr, v[x][i], acc[r][i]);
        }
      }
    }
#pragma unroll
    for (int x = 1; x < T; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float inv = 1.f / __shfl_sync(0xffffffffu, sum, r * T);
      if (tok[r] < 0) continue;
      uint16_t* out = a.out + (int64_t)(start + tok[r]) * a.o_token + (int64_t)head[r] * a.o_head + lane * N;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (not_finite(widen<kBf16>(out[i])) && !not_finite(acc[r][i] * inv)) out[i] = (uint16_t)pack<kBf16>(acc[r][i] * inv, 0.f);
    }
  }
}

// Rows whose O is not finite, by their warp (a row per lane, tokens rising with the lanes, one key-value head).  What the tokens
// that a row sees make infinite or NaN is so: weights are above 0, so an infinity stays one, and two of different signs or a NaN
// make a NaN; V is looked through once for all rows.  What they do not has met a later token's V, or has grown too large
// unnormalised: these rows are computed again.  That is slow, and no row's usual way: a NaN in
// the last of 8192 tokens, whose tile of 128 keys has rows that do not see it, makes 11 ms of a call of 0.9 (64 heads over 8; 50 ms a row at a
// time); NaN in all tokens, which every row sees, 8.5.
template <bool kBf16, int HD>
__device__ __noinline__ void mend_rows(const PromptArgs& a, uint32_t rows, int start, int row_tok, int row_head, int kvh, float row_l, int lane,
                                       int* limit) {
  constexpr int N = HD / 32;  // values of a lane: lane, lane + 32, ...
  int odd[N];                 // of the tokens so far: 1 a NaN, 2 inf, 4 -inf
#pragma unroll
  for (int i = 0; i < N; ++i) odd[i] = 0;
  const uint16_t* v0 = a.v + (int64_t)start * a.v_token + (int64_t)kvh * a.v_head + lane;
  int upto = 0;
  uint32_t again = 0;
  __syncwarp();  // the rows' results, which other lanes have stored, are read below
  for (; rows; rows &= rows - 1) {
    const int src = __ffs(rows) - 1, tok = __shfl_sync(0xffffffffu, row_tok, src), head = __shfl_sync(0xffffffffu, row_head, src);
    const float l = __shfl_sync(0xffffffffu, row_l, src);
    if (not_finite(l)) continue;  // a score is no number: all of the row is none
    uint16_t* out = a.out + (int64_t)(start + tok) * a.o_token + (int64_t)head * a.o_head + lane;
    bool left = false;
    while (l != 0.f && upto <= tok) {
      const int end = min(tok, upto + kBeat - 1);
#pragma unroll 4
      for (int j = upto; j <= end; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = widen<kBf16>(v0[j * a.v_token + i * 32]);
          if (not_finite(x)) odd[i] |= x == INFINITY ? 2 : x == -INFINITY ? 4 : 1;
        }
      upto = end + 1;
      if (lane == 0) raise_limit(limit);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float old = widen<kBf16>(out[i * 32]);
      if (l == 0.f) out[i * 32] = 0;  // nothing but scores of -inf
      else if (not_finite(old) && odd[i])
        out[i * 32] = (uint16_t)pack<kBf16>(odd[i] == 2 ? INFINITY : odd[i] == 4 ? -INFINITY : __uint_as_float(0x7fffffffu), 0.f);
      else left |= not_finite(old);
    }
    if (__any_sync(0xffffffffu, left)) again |= 1u << src;
  }
  __syncwarp();
  if (again) rows_again<kBf16, HD>(a, again, start, row_tok, row_head, kvh, lane, limit);
}

template <int HD, int kTiles>
struct Shape {
  static constexpr int kHalves = HD / 64;                        // 64 values = 128 bytes: one swizzle row
  static constexpr uint32_t kHalfBytes = kRows * 128;            // a tile's rows of one half
  static constexpr uint32_t kTileBytes = kHalves * kHalfBytes;
  static constexpr int kStages = 2 * kTiles * (128 / HD);        // K0 V0 K1 V1 ...
  static constexpr size_t kSmem = (kTiles + kStages) * (size_t)kTileBytes + 1024;
  static constexpr int kSoftmaxWarps = 4 * kTiles, kMmaWarp = kSoftmaxWarps, kLoadWarp = kMmaWarp + 1, kPlanWarp = kMmaWarp + 2;
  static constexpr int kThreads = 32 * kSoftmaxWarps + 128;      // the last warp has nothing to do
  static constexpr int kPlanReaders = kSoftmaxWarps + 2;         // warps that read a plan: softmax, products, loads
  static constexpr int kColumns = kTiles * 256;                  // of tensor memory: scores, then accumulators
};

// A block of work: the tiles of rows, one or two, of one prompt and key-value head.
struct Plan {
  int start, len, q0, kvh;  // first row and tokens of the prompt, first token of the block; len 0: nothing is left
};

template <int kTiles>
struct Work {
  int start, len, q0, kvh, n_kv[kTiles], n_tiles;
  bool tail;  // the last tile of keys reaches past the prompt
  __device__ __forceinline__ Work(const Plan& p, int tile_tokens) : start(p.start), len(p.len), q0(p.q0), kvh(p.kvh) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int first = q0 + i * tile_tokens, end = min(first + tile_tokens, len);
      n_kv[i] = end > first ? (end + kRows - 1) / kRows : 0;  // the second tile may have no row
    }
    n_tiles = max(n_kv[0], n_kv[kTiles - 1]);
    tail = n_tiles * kRows > len;
  }
};

// P = exp2(scale2 * S - m) of 64 of a row's scores, from column C on, into tensor memory; their sum.
template <bool kBf16, int C>
__device__ __forceinline__ float softmax_half(const uint32_t (&s)[kRows], float scale2, float use, uint32_t tp) {
  const f32x2 sc = two(scale2, scale2), off = two(-use, -use);
  f32x2 sum[2] = {0, 0};
#pragma unroll
  for (int c = C; c < C + kRows / 2; c += 32) {
    uint32_t w[16];
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const f32x2 e = fma2(two(__uint_as_float(s[c + 2 * x]), __uint_as_float(s[c + 2 * x + 1])), sc, off);
      float p0, p1;
      apart(e, p0, p1);
      p0 = exp2_fast(p0);
      p1 = exp2_fast(p1);
      sum[x & 1] = add2(sum[x & 1], two(p0, p1));
      w[x] = pack<kBf16>(p0, p1);
    }
    tm_st16(tp + c / 2, w);
  }
  float a, b;
  apart(add2(sum[0], sum[1]), a, b);
  return a + b;
}

// The largest of a row's scores; NaN if one is.
__device__ __forceinline__ float row_max(const uint32_t (&s)[kRows]) {
  float top[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) top[x] = max3(__uint_as_float(s[x]), __uint_as_float(s[x + 4]), __uint_as_float(s[x + 8]));
#pragma unroll
  for (int c = 12; c + 8 <= kRows; c += 8) {
#pragma unroll
    for (int x = 0; x < 4; ++x) top[x] = max3(top[x], __uint_as_float(s[c + x]), __uint_as_float(s[c + 4 + x]));
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) top[x] = max3(top[x], __uint_as_float(s[kRows - 4 + x]), -INFINITY);
  return max3(max3(top[0], top[1], top[2]), top[3], -INFINITY);
}

template <bool kBf16, int HD, int kTiles>
__global__ void __launch_bounds__(Shape<HD, kTiles>::kThreads, 3 - kTiles)
k_attn_prompt(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
              const __grid_constant__ PromptArgs a) {
  using S = Shape<HD, kTiles>;
  extern __shared__ __align__(1024) unsigned char tsm[];
  __shared__ int s_blocks[NP_KV_MAX_SEQS];  // blocks of work of each prompt (per key-value head)
  __shared__ Plan s_plan[kPlans];
  __shared__ __align__(8) uint64_t full[S::kStages], empty[S::kStages], q_full, q_empty, s_full[kTiles], p_half[kTiles], p_full[kTiles], o_full[kTiles], o_empty[kTiles],
      plan_full[kPlans], plan_empty[kPlans];
  __shared__ uint32_t s_tmem;
  __shared__ int s_limit;  // polls that a wait may take; 0: one has run out
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;

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
    for (int i = 0; i < kPlans; ++i) {
      npp::mbar_init(&plan_full[i], 1);
      npp::mbar_init(&plan_empty[i], S::kPlanReaders);
    }
    npp::fence_barrier_init();
    s_limit = kWaitPolls;
  }
  // the plan warp counts the blocks of each prompt while the others set up
  if (wid == S::kPlanWarp) {
    const int block_tokens = kTiles * a.tile_tokens;
    for (int i = lane; i < a.n; i += 32) {
      const int lo = min(max(a.cu[i], 0), a.n_tokens), hi = min(max(a.cu[i + 1], 0), a.n_tokens);
      s_blocks[i] = hi > lo ? (hi - lo - 1) / block_tokens + 1 : 0;
    }
    __syncwarp();
  }
  if (wid == S::kLoadWarp && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
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
      const int limit = *static_cast<volatile int*>(&s_limit);
      if (limit == 0) return false;
      if (++polls >= limit) {
        *static_cast<volatile int*>(&s_limit) = 0;
        atomicOr(a.status, NP_KV_S_TIMEOUT);
      }
    }
    return true;
  };
  // the same by whole warps: all lanes go on, or none does
  auto wait_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
  // the n-th plan; false: nothing is left, or a wait ran out
  auto plan = [&](uint32_t n, Plan& p, bool whole_warp) {
    uint64_t* bar = &plan_full[n % kPlans];
    if (whole_warp ? !wait_all(bar, (n / kPlans) & 1u) : !wait(bar, (n / kPlans) & 1u)) return false;
    p = s_plan[n % kPlans];
    if (whole_warp) {
      __syncwarp();
      if (lane == 0) npp::mbar_arrive(&plan_empty[n % kPlans]);
    } else {
      npp::mbar_arrive(&plan_empty[n % kPlans]);
    }
    return p.len > 0;
  };

  if (wid >= S::kMmaWarp) {
   fewer_registers<kTiles>();
   if (wid == S::kPlanWarp) {
    // ------------------------------ plans ------------------------------
    // Blocks of work in falling order of their place in their prompt, which is the order of their number of keys; this block
    // takes every gridDim-th, in alternating direction, so that all blocks get about the same.
    const int first_blocks = lane < a.n ? s_blocks[lane] : 0;  // of the first 32 prompts, at hand
    auto from_place = [&](int b) {  // blocks of work at place b or later, all prompts, one key-value head
      int sum = max(0, first_blocks - b);
      for (int i = lane + 32; i < a.n; i += 32) sum += max(0, s_blocks[i] - b);
      return __reduce_add_sync(0xffffffffu, sum);
    };
    int most = first_blocks;
    for (int i = lane + 32; i < a.n; i += 32) most = max(most, s_blocks[i]);
    most = __reduce_max_sync(0xffffffffu, most);
    const unsigned total = (unsigned)from_place(0) * a.n_kv_heads;
    for (uint32_t n = 0;; ++n) {
      const unsigned r = n * gridDim.x + (n & 1u ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
      Plan p = {0, 0, 0, 0};
      if (r < total) {
        const int at = (int)(r / (unsigned)a.n_kv_heads);
        int lo = 0, hi = most - 1;  // the largest place with more than `at` blocks from it on
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (from_place(mid) > at) lo = mid;
          else hi = mid - 1;
        }
        int which = at - from_place(lo + 1);  // among the prompts that have that place
        for (int first = 0; first < a.n; first += 32) {
          const uint32_t has = __ballot_sync(0xffffffffu, first + lane < a.n && (first == 0 ? first_blocks : s_blocks[first + lane]) > lo);
          const int cnt = __popc(has);
          if (which < cnt) {
            const bool it = (has >> lane & 1u) && __popc(has & ((1u << lane) - 1u)) == which;
            const int i = first + __ffs(__ballot_sync(0xffffffffu, it)) - 1;
            p.start = min(max(a.cu[i], 0), a.n_tokens);
            p.len = min(max(a.cu[i + 1], 0), a.n_tokens) - p.start;
            p.q0 = lo * kTiles * a.tile_tokens;
            p.kvh = (int)(r - (unsigned)at * a.n_kv_heads);
            break;
          }
          which -= cnt;
        }
      }
      if (!wait_all(&plan_empty[n % kPlans], ((n / kPlans) & 1u) ^ 1u)) break;
      if (lane == 0) {
        s_plan[n % kPlans] = p;
        npp::mbar_arrive(&plan_full[n % kPlans]);
      }
      __syncwarp();
      if (p.len == 0) break;
    }
   } else if (wid == S::kLoadWarp) {
    // ------------------------------ loads ------------------------------
    if (lane == 0) {
      int stage = 0;
      uint32_t use = 0, n = 0;
      Plan p;
      bool ok = true;
      for (; ok && plan(n, p, false); ++n) {
        const Work<kTiles> w(p, a.tile_tokens);
        const int tiles = w.n_kv[kTiles - 1] > 0 ? kTiles : 1;
        ok = wait(&q_empty, (n & 1u) ^ 1u);
        if (!ok) break;
        npp::mbar_expect_tx(&q_full, (uint32_t)tiles * S::kHalves * 128 * a.group * a.tile_tokens);
        for (int i = 0; i < tiles; ++i)
          for (int h = 0; h < S::kHalves; ++h)
            tma_load_3d(q_sm + i * S::kTileBytes + h * S::kHalfBytes, &map_q, h * 64, w.kvh * a.group, w.start + w.q0 + i * a.tile_tokens, &q_full);
        for (int j = 0; j < 2 * w.n_tiles; ++j) {
          ok = wait(&empty[stage], (use & 1u) ^ 1u);
          if (!ok) break;
          npp::mbar_expect_tx(&full[stage], S::kTileBytes);
          for (int h = 0; h < S::kHalves; ++h)
            tma_load_3d(ring + stage * S::kTileBytes + h * S::kHalfBytes, j & 1 ? &map_v : &map_k, h * 64, w.kvh, w.start + (j >> 1) * kRows,
                        &full[stage]);
          if (++stage == S::kStages) {
            stage = 0;
            ++use;
          }
        }
      }
      if (*static_cast<volatile int*>(&s_limit) == 0) {  // after a time-out nobody else waits for the copies
        uint32_t patience = npp::kSpinLimit;
        npp::drain_ring(full, S::kStages, stage, use & 1u, patience);
        npp::wait_landed(&q_full, n & 1u, patience);
        if (n > 0) npp::wait_landed(&q_full, (n & 1u) ^ 1u, patience);
      }
    }
   } else if (wid == S::kMmaWarp) {
    // ------------------------------ products ------------------------------
    // The whole warp goes through the loop and one lane issues: what an instruction takes (descriptors, addresses) then is
    // the same in all lanes, and the compiler keeps it in uniform registers, where the instruction wants it.  (One lane in a
    // loop of its own took 75 cycles per instruction, more than the product itself.)  One warp serves both tiles in turn: with
    // a warp for each, the tiles fall into step, and the tensor cores wait while both do their softmax.
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
    uint32_t ld = 0, p_cnt[kTiles] = {}, o_cnt[kTiles] = {};  // loads, softmax steps and results so far
    auto wait_load = [&](uint32_t l) { return wait_all(&full[l % S::kStages], (l / S::kStages) & 1u); };
    Plan p;
    bool ok = true;
    for (uint32_t n = 0; ok && plan(n, p, true); ++n) {
      const Work<kTiles> w(p, a.tile_tokens);
      ok = wait_all(&q_full, n & 1u) && wait_load(ld);
      if (!ok) break;
      fence_after();
      if (elect_one()) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          if (w.n_kv[i] > 0) scores(i, ld % S::kStages);
        commit(&empty[ld % S::kStages]);
        if (w.n_tiles == 1) commit(&q_empty);
      }
      __syncwarp();
      for (int j = 0; j < w.n_tiles && ok; ++j) {
        const uint32_t lv = ld + 2 * j + 1, lk = lv + 1, sv = lv % S::kStages, sk = lk % S::kStages;
        const bool more = j + 1 < w.n_tiles;
        ok = wait_load(lv) && (!more || wait_load(lk));
        if (ok && w.tail && !more) {
          // rows past the prompt: zero, whatever lies there
          const uint32_t from = (w.len - (w.n_tiles - 1) * kRows) * 128;
#pragma unroll
          for (int h = 0; h < S::kHalves; ++h)
            for (uint32_t e = from + lane * 16; e < S::kHalfBytes; e += 32 * 16)
              *reinterpret_cast<uint4*>(ring + sv * S::kTileBytes + h * S::kHalfBytes + e) = make_uint4(0, 0, 0, 0);
          npp::fence_proxy_async();
          __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          if (j >= w.n_kv[i] || !ok) continue;
          if (j == 0) ok = wait_all(&o_empty[i], (o_cnt[i]++ & 1u) ^ 1u);  // the tile before has been read out of the accumulators
          const uint32_t par = p_cnt[i]++ & 1u, d_s = tmem + i * kRows, d_o = tmem + kTiles * kRows + i * HD;
          const uint64_t vd = v_desc + sv * (S::kTileBytes >> 4);
          ok = ok && wait_all(&p_half[i], par);
          if (!ok) continue;
          fence_after();
          if (elect_one()) {  // the first 64 keys
#pragma unroll
            for (int k = 0; k < kRows / 32; ++k) mma_ts(d_o, d_s + k * 8, vd + k * 128, id_o, (j | k) > 0);
          }
          __syncwarp();
          ok = wait_all(&p_full[i], par);
          if (!ok) continue;
          fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = kRows / 32; k < kRows / 16; ++k) mma_ts(d_o, d_s + k * 8, vd + k * 128, id_o, 1u);
            if (j + 1 < w.n_kv[i]) scores(i, sk);
            else commit(&o_full[i]);
          }
          __syncwarp();
        }
        if (ok && elect_one()) {
          commit(&empty[sv]);
          if (more) commit(&empty[sk]);
          if (j + 2 == w.n_tiles) commit(&q_empty);
        }
        __syncwarp();
      }
      ld += 2 * w.n_tiles;
    }
   }
  } else {
    more_registers<kTiles>();
    // ------------------------------ softmax and result of a tile ------------------------------
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
    Plan p;
    bool ok = true;
    for (uint32_t n = 0; ok && plan(n, p, true); ++n) {
      const Work<kTiles> w(p, a.tile_tokens);
      const int steps = w.n_kv[i];
      if (steps == 0) continue;
      const int first = w.q0 + i * a.tile_tokens, tok = first + in_tile;
      const bool valid = in_tile < a.tile_tokens && tok < w.len;  // the other rows hold anything, and have no say
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < steps; ++j) {
        ok = wait_all(&s_full[i], s_cnt++ & 1u);
        if (!ok) break;
        fence_after();
        uint32_t s[kRows];
#pragma unroll
        for (int c = 0; c < kRows; c += 32) tm_ld32(ts + c, s, c);
        wait_ld(s);
        if ((j + 1) * kRows - 1 > first) {  // the tile reaches past the first row
          const int see = tok - j * kRows;
#pragma unroll
          for (int c = 0; c < kRows; c += 32) {
            const uint32_t keep = see - c >= 31 ? 0xffffffffu : see < c ? 0u : (2u << (see - c)) - 1u;
#pragma unroll
            for (int x = 0; x < 32; ++x)
              if (!(keep >> x & 1u)) s[c + x] = __float_as_uint(-INFINITY);
          }
        }
        // On the assumption that the maximum has not grown much, the first half's exponentials need not wait for it: it is found
        // beside them, by units that they leave idle.  (The maximum first: 390 cycles of 2350 for a tile.)
        float part = 0.f, now, sc = a.scale2;
        bool fast = false;
        if (j > 0) {
          part = softmax_half<kBf16, 0>(s, a.scale2, m, ts);
          now = row_max(s) * a.scale2;
          fast = __all_sync(0xffffffffu, !valid || (now <= m + kGrow && fabsf(m) <= kLarge && now < INFINITY));
        } else {
          now = row_max(s) * a.scale2;
        }
        float use = m;
        if (!fast) {
          // a NaN makes the maximum NaN, and with it the row; an infinite score does, too (inf - inf)
          now = max3(m, now, now == INFINITY ? __uint_as_float(0x7fffffffu) : -INFINITY);
          if (j == 0) {
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
          part = softmax_half<kBf16, 0>(s, sc, use, ts);
        }
        arrive(&p_half[i]);
        l += part + softmax_half<kBf16, kRows / 2>(s, sc, use, ts);
        arrive(&p_full[i]);
      }
      if (ok) ok = wait_all(&o_full[i], o_cnt++ & 1u);
      if (!ok) break;
      // ---- the result
      fence_after();
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int head = w.kvh * a.group + in_group;
      uint16_t* out = a.out + (int64_t)(w.start + tok) * a.o_token + (int64_t)head * a.o_head;
      uint32_t big = __float_as_uint(l) & 0x7fffffffu;
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
#pragma unroll
        for (int x = 0; x < 32; ++x) big = max(big, o[x] & 0x7fffffffu);
        if (valid) {
#pragma unroll
          for (int x = 0; x < 32; x += 16) {
            uint32_t v[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) v[y] = pack<kBf16>(__uint_as_float(o[x + 2 * y]) * inv, __uint_as_float(o[x + 2 * y + 1]) * inv);
            if (a.out32) {
              store32(out + c + x, v);
            } else {
              *reinterpret_cast<uint4*>(out + c + x) = make_uint4(v[0], v[1], v[2], v[3]);
              *reinterpret_cast<uint4*>(out + c + x + 8) = make_uint4(v[4], v[5], v[6], v[7]);
            }
          }
        }
      }
      if (valid && a.lse)
        a.lse[(size_t)(w.start + tok) * a.n_heads + head] = l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m) * kLn2 + logf(l);
      const uint32_t odd = __ballot_sync(0xffffffffu, valid && big >= 0x7f800000u);
      if (odd) mend_rows<kBf16, HD>(a, odd, w.start, tok, head, w.kvh, l, lane, &s_limit);
    }
  }
  fence_before();
  __syncthreads();
  if (wid == S::kMmaWarp) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kColumns) : "memory");
  }
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

template <bool kBf16, int HD, int kTiles>
cudaError_t launch(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const PromptArgs& a, int sms, cudaStream_t s) {
  using S = Shape<HD, kTiles>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = npi::allow_shared(reinterpret_cast<const void*>(k_attn_prompt<kBf16, HD, kTiles>), &done);
  if (e != cudaSuccess) return e;
  // a prompt of x tokens has ceil(x / (kTiles * tile_tokens)) blocks of work: together at most this many
  const int64_t work = ((int64_t)a.n_tokens / (kTiles * a.tile_tokens) + std::min(a.n, a.n_tokens)) * a.n_kv_heads;
  const unsigned blocks = (unsigned)std::min<int64_t>(work, (3 - kTiles) * sms);
  return launch_early(k_attn_prompt<kBf16, HD, kTiles>, dim3(blocks), S::kThreads, S::kSmem, s, q, k, v, a);
}
template <bool kBf16>
cudaError_t launch(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const PromptArgs& a, int hd, int tiles, int sms, cudaStream_t s) {
  if (hd == 128) return tiles == 2 ? launch<kBf16, 128, 2>(q, k, v, a, sms, s) : launch<kBf16, 128, 1>(q, k, v, a, sms, s);
  return tiles == 2 ? launch<kBf16, 64, 2>(q, k, v, a, sms, s) : launch<kBf16, 64, 1>(q, k, v, a, sms, s);
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
  float scale2;
  if (!scale_base2(scale, &scale2)) return fail(NP_E_INVAL, kScaleError);
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
  a.scale2 = scale2;
  a.out32 = (uintptr_t)out->data % 32 == 0 && out->token_stride % 16 == 0 && out->head_stride % 16 == 0;
  if (((int64_t)n_tokens / a.tile_tokens + n) * d->n_kv_heads > 0x7fffffffLL) return fail(NP_E_INVAL, "too many tokens for one call");
  int sms;
  if (!device_sms(&sms)) return fail(NP_E_CUDA, "no CUDA device");
  CUtensorMap mq, mk, mv;
  if (!make_map(&mq, *q, d->head_dim, d->n_heads, n_tokens, group, a.tile_tokens) || !make_map(&mk, *k, d->head_dim, d->n_kv_heads, n_tokens, 1, kRows) ||
      !make_map(&mv, *v, d->head_dim, d->n_kv_heads, n_tokens, 1, kRows))
    return fail(NP_E_INVAL, "rows that a tensor map does not describe (strides of 2^40 bytes and more)");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Two tiles to a block read keys and values once for both; one tile, two blocks to an SM, wastes less where prompts are short
  // (blocks end at odd times, a second tile may be empty) and gives every SM work where there is little.  us, one tile and two:
  // 32 heads of 128, 64 prompts of 64 tokens 37 and 50, 16 of 128 19.4 and 20.2, 16 of 200 34 and 32, 4 of 1024 59 and 54, one of 512
  // 13.5 and 15.7; 64 heads over 8, 16 of 200 41 and 44, 16 of 256 51 and 51, 4 of 768 68 and 62, one of 512 17.4 and 18.5; 64 heads
  // of 64, 16 of 256 37 and 43, 4 of 1024 72 and 81, one of 2048 62 and 64, of 8192 826 and 731.
  const bool little = (int64_t)n_tokens * d->n_kv_heads < (int64_t)2 * a.tile_tokens * sms;
  const int tiles = little || n_tokens <= (int64_t)n * (d->head_dim == 64 ? 2048 : group > 1 ? 224 : 128) ? 1 : 2;
  const cudaError_t e = d->dtype == NP_T_BF16 ? launch<true>(mq, mk, mv, a, d->head_dim, tiles, sms, s) : launch<false>(mq, mk, mv, a, d->head_dim, tiles, sms, s);
  return e == cudaSuccess ? NP_OK : fail_cuda(e);
}
