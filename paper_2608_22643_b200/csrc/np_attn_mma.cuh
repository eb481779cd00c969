// Shared by the attention kernels on mma.sync (np_attn_decode.cu, np_attn_rest.cu): products, exponentials, and what is done about infinities.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

#include "np_attn.h"
#include "np_device.cuh"

namespace npa {

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
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// a / b, by 32 bits where they do
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

template <class T>
__device__ __forceinline__ constexpr uint32_t infinity_bits() {
  return std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
}
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// By a block of 128 threads: what values that are not finite there are among V's of tokens [from, len) of the pages, for each of head_dim (bit 0 a NaN, 8
// inf, 16 -inf).  Weights are above 0, so an infinity stays one, and two of different signs or a NaN make a NaN; what the sums made of finite values
// stays.  V is looked through once for all heads, eight values to a thread.  seen: HD ints of shared memory that are free.  One of 131071 tokens a
// NaN, 64 heads over 8: 201 us a call in place of 93. (One block that looks through all of V behind the join: 10 ms.)
struct Layer {
  const char* cache;
  int n_kv_heads, shift, n_pages;
};
template <class T, int HD>
__device__ __noinline__ void look_through(const Layer& a, const int32_t* pages, int kvh, int64_t from, int64_t len, int* seen) {
  constexpr int kThreads = 128, kCols = HD / 8, kStep = kThreads / kCols, kAhead = 4;
  constexpr uint32_t kInf = infinity_bits<T>();
  const int tid = threadIdx.x;
  for (int d = tid; d < HD; d += kThreads) seen[d] = 0;
  __syncthreads();
  const int col = tid % kCols;
  const int64_t head_bytes = (int64_t)(HD * 2) << a.shift;
  const char* v = a.cache + (a.n_kv_heads + kvh) * head_bytes + col * 16;
  uint32_t bits = 0;  // value x of the column: 1 << x a NaN, 256 << x inf, 65536 << x -inf
  for (int64_t j0 = from + tid / kCols; j0 < len; j0 += kAhead * kStep) {
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
}
// What a result that such values go into is, as fp32; 0: as it was.
__device__ __forceinline__ float made_of(int seen) {
  return seen == 0 ? 0.f : seen == 0x100 ? INFINITY : seen == 0x10000 ? -INFINITY : __uint_as_float(0x7fffffffu);
}

}  // namespace npa
