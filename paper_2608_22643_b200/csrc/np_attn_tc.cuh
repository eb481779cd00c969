// Shared by the attention kernels on the 5th-generation tensor cores (np_attn_prompt.cu, np_attn_shared.cu): tiles of 128 query rows and
// 128 keys, their products, and the softmax of a tile's rows.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "np_attn.h"
#include "np_pipe.cuh"

namespace npa {

constexpr int kRows = 128;              // query rows of a tile, keys of a tile
constexpr float kGrow = 8.f;            // log2 of the growth of a maximum that is let pass
// The largest score (times log2(e), either sign) that an exponent may be formed from by one fused step, s * scale2 - m.  m is a rounded product;
// what the rounding took off stays in the exponent, 1 at most up to here, and cancels between P and its sum.  Past it that passes the range
// of P (2^16 in fp16) and in the end of fp32, so the products are rounded first, as m is.
constexpr float kLarge = 16777216.f;

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

// (p0, p1) in the rows' type, and what that leaves of them, in it.  Together they are the value to 2^-16 in bf16, where the
// first is cut off (a byte permute), and to 2^-22 in fp16, or 2^-25.
template <bool kBf16>
__device__ __forceinline__ void split(float p0, float p1, uint32_t& hi, uint32_t& lo) {
  if (kBf16) {
    const uint32_t b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
    hi = __byte_perm(b0, b1, 0x7632);
    lo = pack<true>(p0 - __uint_as_float(b0 & 0xffff0000u), p1 - __uint_as_float(b1 & 0xffff0000u));
  } else {
    hi = pack<false>(p0, p1);
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    lo = pack<false>(p0 - h.x, p1 - h.y);
  }
}

// P = exp2(scale2 * S - m) of 64 of a row's scores, from column C on, into tensor memory; their sum.  kTwo: P in two terms, the second of all 128 behind
// the first of all 128, where S was.
template <bool kBf16, int C, bool kTwo = false>
__device__ __forceinline__ float softmax_half(const uint32_t (&s)[kRows], float scale2, float use, uint32_t tp) {
  const f32x2 sc = two(scale2, scale2), off = two(-use, -use);
  f32x2 sum[2] = {0, 0};
#pragma unroll
  for (int c = C; c < C + kRows / 2; c += 32) {
    uint32_t w[16], rest[kTwo ? 16 : 1];
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      const f32x2 e = fma2(two(__uint_as_float(s[c + 2 * x]), __uint_as_float(s[c + 2 * x + 1])), sc, off);
      float p0, p1;
      apart(e, p0, p1);
      p0 = exp2_fast(p0);
      p1 = exp2_fast(p1);
      sum[x & 1] = add2(sum[x & 1], two(p0, p1));
      if constexpr (kTwo) split<kBf16>(p0, p1, w[x], rest[x]);
      else w[x] = pack<kBf16>(p0, p1);
    }
    tm_st16(tp + c / 2, w);
    if constexpr (kTwo) tm_st16(tp + kRows / 2 + c / 2, rest);
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

// Rows of heads as (head_dim, heads, tokens); a box is 64 values of `box_heads` heads of `box_tokens` tokens.
inline bool make_rows_map(CUtensorMap* map, const np_rows& r, int hd, int heads, int tokens, int box_heads, int box_tokens) {
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

}  // namespace npa
