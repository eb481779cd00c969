// Rows of heads on their way: norm and rotation of queries and keys (np_attn_rotate), the same into the cache's pages
// (np_kv_append_rotated), into and out of a cache of 8 bits (np_kv_append, np_kv_read).
//
//   y = x / sqrt(mean(x^2) + eps) * gain,   (a, b) -> (a cos t - b sin t, b cos t + a sin t),   t = position * freq[i]
//   e = the least of -60 .. 120 with max|x| <= 448 * 2^e,   x -> e4m3(x * 2^-e)
//
// Every value is read and written once, so the bytes bound all of this, if the instructions are few enough.  A row of head_dim values belongs
// to head_dim / 16 lanes; a lane has two rows on their way before it works on the first.  Its values are eight and the eight that they are
// pairs with, so nothing but the sum of squares and the largest magnitude goes from lane to lane.
//
// Cosines and sines belong to a token, not to a head: a block works them out once for its few tokens, while its loads are on their way.
// The angle is a product in fp64 that is brought to a fraction of a turn there (a position of 2^31 leaves 2^-24 of a turn), so fp32 does for the
// rest.
//
// Powers of two as scales make the 8 bits a matter of integers and one rounding: x * 2^-e is exact, so nothing of what is held depends on
// how it was computed.
//
// Measured (tokens of 64 heads of 128 over 8, each set of inputs in turn larger than the L2): 9 prompts of up to 2000 tokens with norms, 33.9 us, 61 % of the
// copy rate; 8192 tokens without norms into the cache 59.7 us, 87 %; 5 prompts into 8 bits and out again, two kernels, 18.6 us.  Issue slots are busy
// 60 to 70 % in the first two; a block's start (where its rows come from and go to, three loads that depend on one another; its angles) is the rest, and
// all that there is of the small calls: sixteen tokens 3.5 us, into 8 bits and out again 5.1, one token 2.4.  The first two took 46 and 92 us when
// pairs lay in two lanes and every lane worked out its rows' places, and 35.6 and 62.0 when each pair's angle began with a search for its token's
// sequence, and tokens were found by divisions.  (No better: blocks that stay, a warp for the
// loads, sixteen values to a lane.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "np_attn.h"
#include "np_device.cuh"
#include "np_internal.h"
#include "np_pipe.cuh"

namespace npa {
namespace {

constexpr int kThreads = 128, kFew = 32, kMany = 64;  // values of a lane on their way
template <int HD, int kEach, int kValues = kFew>
struct Rows {
  static constexpr int kLanes = HD / kEach;                  // of a row: a lane has that many of its values
  static constexpr int kTurn = kThreads / kLanes;            // rows of a block at a time
  static constexpr int kVecs = kValues / kEach;
  static constexpr int kBlock = kTurn * kVecs;
};

struct RowsArgs {
  const uint16_t* q;
  uint16_t* k;
  uint16_t* v;
  uint16_t* q_out;
  uint16_t* k_out;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, qo_token, qo_head, ko_token, ko_head;  // elements
  const int32_t* seqs;
  const int32_t* cu;
  const int32_t* start;
  int n, n_tokens, nq, nkv, rows;  // rows of a token: queries, keys, then values if there is a cache
  // x / rows = x * mul >> 32 + shift for x below 2^31: mul = floor(2^(32 + shift) / rows) + 1 with 2^shift < rows <= 2^(shift + 1), so that what mul is too
  // large by adds less than 1 / rows
  uint32_t mul;
  int mul_shift;
  __device__ __forceinline__ int token_of(uint32_t x) const { return (int)(__umulhi(x, mul) >> mul_shift); }
  // the cache
  char* cache;  // of the layer; nullptr: none
  const int32_t* table;
  const int32_t* lens;
  int32_t* status;
  int64_t page_bytes;
  int shift, n_pages, max_seqs, max_pages;
  // the rotation
  const double* freq;
  const float* q_gain;
  const float* k_gain;
  float eps, small;      // sums of squares below `small`, where squares are lost that an eps as small does not cover
  int half, neighbours;  // 16-byte pieces of half the values that turn
};

template <class T>
__device__ __forceinline__ float2 widen(uint32_t w);
template <>
__device__ __forceinline__ float2 widen<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 widen<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <class T>
__device__ __forceinline__ uint32_t pack(float x, float y);
template <>
__device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float x, float y) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack<__half>(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// No further from 0 than the type's largest number; NaN stays.
template <class T>
__device__ __forceinline__ float to_finite(float x) {
  const float most = std::is_same<T, __half>::value ? 65504.f : __uint_as_float(0x7f7f0000u);
  return x > most ? most : x < -most ? -most : x;
}

template <class T>
__device__ __forceinline__ void widen4(const uint2& v, float* x) {
  const float2 a = widen<T>(v.x), b = widen<T>(v.y);
  x[0] = a.x;
  x[1] = a.y;
  x[2] = b.x;
  x[3] = b.y;
}
__device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s) {
  const float u = a, w = b;
  a = u * c - w * s;
  b = w * c + u * s;
}

// Where a token is: its position (-1: the row is passed over), its page (-1: no place in the cache) and its place in that.
struct Place {
  int64_t pos;
  int page, at;
};
// cu of the call goes to shared memory, where a block's threads find their tokens' sequences without a trip to memory for each step.
__device__ __forceinline__ void keep_starts(const RowsArgs& a, int* cu) {
  if (a.cu)
    for (int i = threadIdx.x; i <= a.n; i += kThreads) cu[i] = a.cu[i];
}
// The sequence of token t, as a place in the call's lists; -1: none.  *off: the token's number in it.
__device__ __forceinline__ int sequence_of(const RowsArgs& a, const int* cu, int t, int* off) {
  *off = 0;
  if (!a.cu) return t < a.n ? t : -1;
  if (t < cu[0] || t >= cu[a.n]) return -1;
  int lo = 0, hi = a.n - 1;  // the last i with cu[i] <= t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  *off = t - cu[lo];
  return *off < 0 ? -1 : lo;
}
// The position of token t (-1: the row is passed over), and its sequence, if there is a cache.
__device__ __forceinline__ int64_t position_of(const RowsArgs& a, const int* cu, int t, int* seq) {
  int off;
  const int i = sequence_of(a, cu, t, &off);
  if (i < 0) return -1;
  const int st = a.start[i];
  *seq = !a.cache ? 0 : a.seqs ? a.seqs[i] : i;
  return st < 0 ? -1 : (int64_t)st + off;
}
__device__ __forceinline__ Place place_of(const RowsArgs& a, int64_t pos, int seq) {
  Place p = {pos, -1, 0};
  if (pos < 0 || !a.cache) return p;
  if (seq < 0 || seq >= a.max_seqs) {
    atomicOr(a.status, NP_KV_S_SEQ);
    return p;
  }
  const int64_t j = p.pos >> a.shift;
  const int len = a.lens[seq], pg = j < a.max_pages ? a.table[(size_t)seq * a.max_pages + j] : -1;  // on their way together
  if (p.pos >= len) return p;
  if ((unsigned)pg < (unsigned)a.n_pages) {
    p.page = pg;
    p.at = (int)(p.pos & ((1 << a.shift) - 1));
  } else {
    atomicOr(a.status, NP_KV_S_PAGE);
  }
  return p;
}

// The biased exponent of a row's power of two, from the bits of its largest finite magnitude: 448 = 1.75 * 2^8.
__device__ __forceinline__ int exponent_of(uint32_t top) {
  return min(max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 67), 247);
}
// Eight values times a power of two as e4m3; infinities become NaN.
__device__ __forceinline__ uint2 to_e4m3(const float (&x)[8], float power) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float z = x[2 * i + j];
      y[j] = (__float_as_uint(z) & 0x7fffffffu) == 0x7f800000u ? __uint_as_float(0x7fffffffu) : z * power;
    }
    w[i] = __nv_cvt_float2_to_fp8x2(make_float2(y[0], y[1]), __NV_SATFINITE, __NV_E4M3);
  }
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}

enum Kind { kQuery, kKey, kValue };

// kRotate: norm and rotation.  kHeld: keys and values go into pages of 8 bits.
template <class T, int HD, bool kRotate, bool kHeld, int kValues>
__global__ void __launch_bounds__(kThreads)
k_rows_in(const __grid_constant__ RowsArgs a) {
  using R = Rows<HD, 8, kValues>;
  constexpr int L = R::kLanes, kVecs = R::kVecs, kTokens = R::kBlock / 2 + 2;  // of a block at most: a token has two rows or more
  extern __shared__ int s_cu[];
  __shared__ const uint16_t* s_src[R::kBlock];
  __shared__ char* s_dst[R::kBlock];              // nullptr: the row is not written
  __shared__ char* s_exponent[kHeld ? R::kBlock : 1];
  __shared__ int64_t s_pos[kTokens];              // positions of the block's tokens, and their sequences
  __shared__ int s_seq[kTokens];
  __shared__ int s_row[R::kBlock];                // token of the block << 3 | whether it is normed << 2 | kind
  __shared__ __align__(16) float s_gain[kRotate ? 2 : 1][HD];
  __shared__ double s_freq[kRotate ? HD / 2 : 1];  // turns per position
  __shared__ __align__(16) float s_cos[kRotate ? kTokens : 1][HD / 2], s_sin[kRotate ? kTokens : 1][HD / 2];
  const int tid = threadIdx.x, piece = tid % L, slot = tid / L;
  const uint32_t total = (uint32_t)a.n_tokens * a.rows, first = blockIdx.x * R::kBlock;
  const int rows = (int)(min(total, first + R::kBlock) - first);
  const int t0 = a.token_of(first), tokens = a.token_of(first + rows - 1) - t0 + 1;
  // ---- where rows come from
  int t = 0, r = 0;
  if (tid < rows) {
    t = a.token_of(first + tid);
    r = (int)(first + tid - (uint32_t)t * a.rows);
    const int kind = r < a.nq ? kQuery : r < a.nq + a.nkv ? kKey : kValue;
    s_src[tid] = kind == kQuery ? a.q + t * a.q_token + r * a.q_head
                 : kind == kKey ? a.k + t * a.k_token + (r - a.nq) * a.k_head
                                : a.v + t * a.v_token + (r - a.nq - a.nkv) * a.v_head;
    const bool normed = kind == kQuery ? a.q_gain != nullptr : kind == kKey && a.k_gain != nullptr;
    s_row[tid] = (t - t0) << 3 | (normed ? 4 : 0) | kind;
  }
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  keep_starts(a, s_cu);
  if (kRotate && tid < a.half * 8) s_freq[tid] = a.freq[tid] * 0.15915494309189533577;  // 1 / (2 pi)
  if (kRotate && tid < HD / 2) {  // two gains of each kind
    const float2 one = make_float2(1.f, 1.f);
    *reinterpret_cast<float2*>(&s_gain[0][2 * tid]) = a.q_gain ? *reinterpret_cast<const float2*>(a.q_gain + 2 * tid) : one;
    *reinterpret_cast<float2*>(&s_gain[1][2 * tid]) = a.k_gain ? *reinterpret_cast<const float2*>(a.k_gain + 2 * tid) : one;
  }
  __syncthreads();
  // A lane's eight values: four from o0 and four from o1 on.  Of halves that turn, so that pairs meet in a lane.
  const bool turns = kRotate && piece < 2 * a.half, halves = turns && !a.neighbours;
  const int o0 = halves ? 4 * piece : 8 * piece, o1 = halves ? 8 * a.half + 4 * piece : 8 * piece + 4;
  uint2 raw[kVecs][2];
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    raw[j][0] = raw[j][1] = make_uint2(0, 0);
    const int i = j * R::kTurn + slot;
    if (i >= rows) continue;
    const uint16_t* src = s_src[i];
    if (kRotate) {
      raw[j][0] = *reinterpret_cast<const uint2*>(src + o0);
      raw[j][1] = *reinterpret_cast<const uint2*>(src + o1);
    } else {
      const uint4 v = *reinterpret_cast<const uint4*>(src + o0);
      raw[j][0] = make_uint2(v.x, v.y);
      raw[j][1] = make_uint2(v.z, v.w);
    }
  }
  // ---- where they go, and the angles of their tokens
  if (tid < tokens) s_pos[tid] = position_of(a, s_cu, t0 + tid, &s_seq[tid]);
  __syncthreads();
  if (tid < rows) {
    const Place p = place_of(a, s_pos[t - t0], s_seq[t - t0]);
    char* dst = nullptr;
    if (kRotate && r < a.nq) {
      if (p.pos >= 0) dst = reinterpret_cast<char*>(a.q_out + t * a.qo_token + r * a.qo_head);
    } else if (kRotate && !a.cache) {
      if (p.pos >= 0) dst = reinterpret_cast<char*>(a.k_out + t * a.ko_token + (r - a.nq) * a.ko_head);
    } else if (p.page >= 0) {
      const int64_t row = ((int64_t)(r - a.nq) << a.shift) + p.at;  // of the page
      char* page = a.cache + p.page * a.page_bytes;
      dst = page + row * (kHeld ? HD : HD * 2);
      if (kHeld) s_exponent[tid] = page + ((int64_t)2 * a.nkv << a.shift) * HD + row;
    }
    s_dst[tid] = dst;
  }
  if (kRotate && a.half) {
    const int pairs = a.half * 8, step = 32 - __clz(pairs - 1);  // a token's pairs, up to the next power of two
    for (int x = tid; x < tokens << step; x += kThreads) {
      const int u = x >> step, i = x - (u << step);
      if (i >= pairs) continue;
      double turn = (double)s_pos[u] * s_freq[i];
      turn -= rint(turn);
      float sin, cos;
      sincospif(2.f * (float)turn, &sin, &cos);
      s_cos[u][i] = cos;
      s_sin[u][i] = sin;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    const int i = j * R::kTurn + slot;
    const bool there = i < rows;
    const int row = there ? s_row[i] : kValue, kind = row & 3;
    char* dst = there ? s_dst[i] : nullptr;
    float x[8];
    if (kRotate && __any_sync(0xffffffffu, kind != kValue)) {
      widen4<T>(raw[j][0], x);
      widen4<T>(raw[j][1], x + 4);
      if (a.q_gain || a.k_gain) {
        auto sum_of_squares = [&] {
          float ss = x[0] * x[0];
#pragma unroll
          for (int z = 1; z < 8; ++z) ss = fmaf(x[z], x[z], ss);
#pragma unroll
          for (int o = 1; o < L; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          return ss;
        };
        float ss = sum_of_squares(), eps = a.eps;
        const bool normed = row & 4, past = normed && (ss == INFINITY || ss < a.small);
        if (__any_sync(0xffffffffu, past)) {  // squares past fp32's range, of values 2^-80 as large, or below its normal numbers, of values 2^60 as large
          if (past) {
            const float by = ss == INFINITY ? 0x1p-80f : 0x1p60f;
            eps = ss == INFINITY ? 0.f : eps * 0x1p120f;  // nothing beside large squares
#pragma unroll
            for (int z = 0; z < 8; ++z) x[z] *= by;
          }
          const float again = sum_of_squares();
          if (past) ss = again;
        }
        if (normed) {
          const float f = rsqrtf(ss * (1.f / HD) + eps);
          const float4 g0 = *reinterpret_cast<const float4*>(&s_gain[kind][o0]), g1 = *reinterpret_cast<const float4*>(&s_gain[kind][o1]);
          const float g[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
#pragma unroll
          for (int z = 0; z < 8; ++z) x[z] = x[z] * f * g[z];
        }
      }
      if (turns && kind != kValue) {
        const float4 c4 = *reinterpret_cast<const float4*>(&s_cos[row >> 3][4 * piece]), s4 = *reinterpret_cast<const float4*>(&s_sin[row >> 3][4 * piece]);
        const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
        if (halves) {
#pragma unroll
          for (int z = 0; z < 4; ++z) turn_pair(x[z], x[z + 4], c[z], s[z]);
        } else {
#pragma unroll
          for (int z = 0; z < 4; ++z) turn_pair(x[2 * z], x[2 * z + 1], c[z], s[z]);
        }
      }
      if (kind != kValue) {
        raw[j][0] = make_uint2(pack<T>(x[0], x[1]), pack<T>(x[2], x[3]));
        raw[j][1] = make_uint2(pack<T>(x[4], x[5]), pack<T>(x[6], x[7]));
      }
    }
    if (kHeld && __any_sync(0xffffffffu, kind != kQuery)) {
      widen4<T>(raw[j][0], x);
      widen4<T>(raw[j][1], x + 4);
      uint32_t top = 0;
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        const uint32_t b = __float_as_uint(x[z]) & 0x7fffffffu;
        top = max(top, b < 0x7f800000u ? b : 0u);
      }
#pragma unroll
      for (int o = 1; o < L; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (kind != kQuery && dst) {
        const int e = exponent_of(top);
        const uint2 w = to_e4m3(x, __uint_as_float((uint32_t)(254 - e) << 23));
        if (kRotate) {
          *reinterpret_cast<uint32_t*>(dst + o0) = w.x;
          *reinterpret_cast<uint32_t*>(dst + o1) = w.y;
        } else {
          *reinterpret_cast<uint2*>(dst + o0) = w;
        }
        if (piece == 0) *s_exponent[i] = (char)e;
      }
    }
    if ((!kHeld || kind == kQuery) && dst) {
      *reinterpret_cast<uint2*>(dst + 2 * o0) = raw[j][0];
      *reinterpret_cast<uint2*>(dst + 2 * o1) = raw[j][1];
    }
  }
}

template <class T, int HD, bool kHeld>
__global__ void __launch_bounds__(kThreads)
k_rows_out(const __grid_constant__ RowsArgs a) {
  using R = Rows<HD, 16>;
  constexpr int L = R::kLanes, kVecs = R::kVecs;
  extern __shared__ int s_cu[];
  __shared__ const char* s_src[R::kBlock];  // nullptr: not there
  __shared__ uint16_t* s_dst[R::kBlock];
  __shared__ const uint8_t* s_exponent[kHeld ? R::kBlock : 1];
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  keep_starts(a, s_cu);
  __syncthreads();
  const int tid = threadIdx.x, piece = tid % L, slot = tid / L;
  const uint32_t total = (uint32_t)a.n_tokens * a.rows, first = blockIdx.x * R::kBlock;
  const int rows = (int)(min(total, first + R::kBlock) - first);
  if (tid < rows) {
    const int t = a.token_of(first + tid), r = (int)(first + tid - (uint32_t)t * a.rows);
    int seq = 0;
    const int64_t pos = position_of(a, s_cu, t, &seq);
    const Place p = place_of(a, pos, seq);
    const char* page = a.cache + p.page * a.page_bytes;
    const int64_t at = ((int64_t)r << a.shift) + p.at;
    s_src[tid] = p.page < 0 ? nullptr : page + at * (kHeld ? HD : HD * 2);
    if (kHeld) s_exponent[tid] = reinterpret_cast<const uint8_t*>(page) + ((int64_t)2 * a.nkv << a.shift) * HD + at;
    s_dst[tid] = r < a.nkv ? a.k + t * a.k_token + r * a.k_head : a.v + t * a.v_token + (r - a.nkv) * a.v_head;
  }
  __syncthreads();
  uint4 raw[kVecs][kHeld ? 1 : 2];
  float power[kVecs];
  uint16_t* to[kVecs];
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    const int i = j * R::kTurn + slot;
    to[j] = nullptr;
    const char* src = i < rows ? s_src[i] : nullptr;
    if (!src) continue;
    to[j] = s_dst[i] + piece * 16;
    if constexpr (kHeld) {
      raw[j][0] = *reinterpret_cast<const uint4*>(src + piece * 16);
      power[j] = __uint_as_float((uint32_t)*s_exponent[i] << 23);
    } else {
      raw[j][0] = *reinterpret_cast<const uint4*>(src + piece * 32);
      raw[j][1] = *reinterpret_cast<const uint4*>(src + piece * 32 + 16);
    }
  }
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    if (!to[j]) continue;
    if constexpr (kHeld) {
      const uint32_t w[4] = {raw[j][0].x, raw[j][0].y, raw[j][0].z, raw[j][0].w};
      uint32_t o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (i & 1) * 16), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        o[i] = pack<T>(to_finite<T>(f.x * power[j]), to_finite<T>(f.y * power[j]));
      }
      *reinterpret_cast<uint4*>(to[j]) = make_uint4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<uint4*>(to[j] + 8) = make_uint4(o[4], o[5], o[6], o[7]);
    } else {
      *reinterpret_cast<uint4*>(to[j]) = raw[j][0];
      *reinterpret_cast<uint4*>(to[j] + 8) = raw[j][1];
    }
  }
}

// Values of a call from which a lane of a rotation has kMany of them on their way: fewer blocks work out the same angles, and more loads wait for each
// other's start.  64 heads of 128 over 8 into the cache, us with kMany and kFew: 64 tokens 3.95 and 3.16, 1024 (10 million) 13.0 and 11.9, 4096 (42 million)
// 33.2 and 33.5, 8192 59.7 and 61.8; 32 heads of 64, 4096 tokens (25 million) 25.9 and 25.7; normed queries and keys of 8000 tokens 64.7 and 65.7.
constexpr int64_t kManyFrom = 1 << 25;
template <class T>
cudaError_t launch_in(const RowsArgs& a, int hd, bool rotate, bool held, cudaStream_t s) {
  const int64_t rows = (int64_t)a.n_tokens * a.rows;
  const bool many = rotate && rows * hd >= kManyFrom;
  const int block = kThreads * 8 / hd * (many ? kMany : kFew) / 8;
  const dim3 grid((unsigned)((rows + block - 1) / block));
  auto go = [&](auto kernel) { return launch_early(kernel, grid, kThreads, a.cu ? (a.n + 1) * sizeof(int) : 0, s, a); };
  auto of_width = [&](auto width) {
    constexpr int HD = decltype(width)::value;
    if (!rotate) return go(k_rows_in<T, HD, false, true, kFew>);
    if (many) return held ? go(k_rows_in<T, HD, true, true, kMany>) : go(k_rows_in<T, HD, true, false, kMany>);
    return held ? go(k_rows_in<T, HD, true, true, kFew>) : go(k_rows_in<T, HD, true, false, kFew>);
  };
  return hd == 128 ? of_width(std::integral_constant<int, 128>{}) : of_width(std::integral_constant<int, 64>{});
}
template <class T>
cudaError_t launch_out(const RowsArgs& a, int hd, bool held, cudaStream_t s) {
  const int block = hd == 128 ? Rows<128, 16>::kBlock : Rows<64, 16>::kBlock;
  const dim3 grid((unsigned)(((int64_t)a.n_tokens * a.rows + block - 1) / block));
  auto go = [&](auto kernel) { return launch_early(kernel, grid, kThreads, a.cu ? (a.n + 1) * sizeof(int) : 0, s, a); };
  if (hd == 128) return held ? go(k_rows_out<T, 128, true>) : go(k_rows_out<T, 128, false>);
  return held ? go(k_rows_out<T, 64, true>) : go(k_rows_out<T, 64, false>);
}

// What is wrong with rows that are written.
const char* out_error(const np_rows* r, int n_tokens, int heads) {
  if (const char* m = rows_error(r)) return m;
  if ((n_tokens > 1 && r->token_stride == 0) || (heads > 1 && r->head_stride == 0)) return "rows of a result need strides above 0";
  return nullptr;
}

const char* rotation_error(const np_rotation* r, int head_dim) {
  if (!r) return "NULL rotation";
  if (r->rot_dim < 0 || r->rot_dim > head_dim || r->rot_dim % 16) return "rot_dim must be a multiple of 16 in [0, head_dim]";
  if (r->pairs != NP_ROT_HALVES && r->pairs != NP_ROT_NEIGHBOURS) return "pairs must be NP_ROT_HALVES or NP_ROT_NEIGHBOURS";
  if (r->rot_dim && (!r->freq || (uintptr_t)r->freq % 8)) return "freq must be there, and 8-byte aligned";
  if ((uintptr_t)r->q_gain % 16 || (uintptr_t)r->k_gain % 16) return "gains must be 16-byte aligned";
  if (!(r->eps >= FLT_MIN) || !std::isfinite(r->eps)) return "eps must be positive, not below the normal numbers, and finite";
  for (int x : r->reserved)
    if (x) return "reserved must be 0";
  return nullptr;
}

// Counts and places of tokens, the same for all calls.
const char* tokens_error(int32_t n_tokens, const int32_t* cu, int32_t n) {
  if (n < 0 || n_tokens < 0) return "n and n_tokens must not be negative";
  if (!cu && n_tokens != n) return "without cu there is one token for each sequence";
  if (cu && n > NP_KV_MAX_SEQS) return "n outside [0, NP_KV_MAX_SEQS]";
  return nullptr;
}

void put_rotation(RowsArgs& a, const np_rotation* r) {
  a.freq = r->freq;
  a.q_gain = r->q_gain;
  a.k_gain = r->k_gain;
  a.eps = r->eps;
  a.small = r->eps < 0x1p-80f ? 0x1p-80f : 0.f;
  a.half = r->rot_dim / 16;
  a.neighbours = r->pairs == NP_ROT_NEIGHBOURS;
}
void put_tokens(RowsArgs& a, int n_tokens, const int32_t* seqs, const int32_t* cu, const int32_t* start, int n) {
  a.seqs = seqs;
  a.cu = cu;
  a.start = start;
  a.n = n;
  a.n_tokens = n_tokens;
}
void put_rows(const np_rows* r, uint16_t** data, int64_t* token, int64_t* head) {
  *data = static_cast<uint16_t*>(r->data);
  *token = r->token_stride;
  *head = r->head_stride;
}
void put_cache(RowsArgs& a, const np_kv_desc* d, const void* cache, int layer, const np_kv_tables* t) {
  a.page_bytes = page_bytes(d);
  a.cache = static_cast<char*>(const_cast<void*>(cache)) + (int64_t)layer * d->n_pages * a.page_bytes;
  a.table = t->page_table;
  a.lens = t->lens;
  a.status = t->status;
  a.shift = log2_of(d->page_tokens);
  a.n_pages = d->n_pages;
  a.max_seqs = d->max_seqs;
  a.max_pages = d->max_pages;
  a.nkv = d->n_kv_heads;
}
constexpr const char* kTooMany = "too many rows for one call";
bool too_many(const RowsArgs& a) { return (int64_t)a.n_tokens * a.rows > 0x7fffffffLL - 2 * Rows<64, 16>::kBlock; }

// What every call over a cache checks; 1: there is nothing to do.
int enter(const np_kv_desc* d, const void* cache, int32_t layer, const np_kv_tables* t, const np_rows* k, const np_rows* v, int32_t n_tokens,
          const int32_t* cu, const int32_t* start, int32_t n) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  if (!t || !t->page_table || !t->lens || !t->status) return fail(NP_E_INVAL, "a table pointer is NULL");
  if (const char* m = tokens_error(n_tokens, cu, n)) return fail(NP_E_INVAL, m);
  if (n > d->max_seqs) return fail(NP_E_INVAL, "n outside [0, max_seqs]");
  if (n == 0 || n_tokens == 0) return 1;
  if (!cache || !start) return fail(NP_E_INVAL, "NULL argument");
  if ((uintptr_t)cache % 16) return fail(NP_E_INVAL, "cache must be 16-byte aligned");
  if (layer < 0 || layer >= d->n_layers) return fail(NP_E_INVAL, "layer outside the cache");
  if (const char* m = rows_error(k)) return fail(NP_E_INVAL, m);
  if (const char* m = rows_error(v)) return fail(NP_E_INVAL, m);
  return NP_OK;
}

int run(RowsArgs& a, int type, int hd, bool out, bool rotate, bool held, void* stream) {
  if (too_many(a)) return fail(NP_E_INVAL, kTooMany);
  while (1 << (a.mul_shift + 1) < a.rows) ++a.mul_shift;  // there are two rows or more, and fewer than 2^18
  a.mul = (uint32_t)((1ULL << (32 + a.mul_shift)) / a.rows + 1);
  int sms;
  if (!device_sms(&sms)) return fail(NP_E_CUDA, "no CUDA device");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (out) e = type == NP_T_BF16 ? launch_out<__nv_bfloat16>(a, hd, held, s) : launch_out<__half>(a, hd, held, s);
  else e = type == NP_T_BF16 ? launch_in<__nv_bfloat16>(a, hd, rotate, held, s) : launch_in<__half>(a, hd, rotate, held, s);
  return e == cudaSuccess ? NP_OK : fail_cuda(e);
}

}  // namespace

int append_held(const np_kv_desc* d, void* cache, int32_t layer, const np_kv_tables* t, const np_rows* k, const np_rows* v, int32_t n_tokens,
                const int32_t* seqs, const int32_t* cu, const int32_t* start, int32_t n, void* stream) {
  RowsArgs a = {};
  put_tokens(a, n_tokens, seqs, cu, start, n);
  put_cache(a, d, cache, layer, t);
  put_rows(k, &a.k, &a.k_token, &a.k_head);
  put_rows(v, &a.v, &a.v_token, &a.v_head);
  a.rows = 2 * a.nkv;
  return run(a, row_type(d), d->head_dim, false, false, true, stream);
}

}  // namespace npa

using namespace npa;

extern "C" {

int np_attn_rotate(const np_attn_shape* d, const np_rotation* r, const np_rows* q, const np_rows* k, const np_rows* q_out, const np_rows* k_out,
                   int32_t n_tokens, const int32_t* cu, const int32_t* start, int32_t n, void* stream) {
  if (!d) return fail(NP_E_INVAL, "NULL argument");
  if (d->dtype != NP_T_BF16 && d->dtype != NP_T_FP16) return fail(NP_E_INVAL, "dtype must be NP_T_BF16 or NP_T_FP16");
  if (d->head_dim != 64 && d->head_dim != 128) return fail(NP_E_INVAL, "head_dim must be 64 or 128");
  if (d->n_kv_heads < 1 || d->n_kv_heads > 1024 || d->n_heads < 1 || d->n_heads > (1 << 17))
    return fail(NP_E_INVAL, "n_kv_heads must be in [1, 1024], n_heads in [1, 131072]");
  for (int x : d->reserved)
    if (x) return fail(NP_E_INVAL, "reserved must be 0");
  if (const char* m = rotation_error(r, d->head_dim)) return fail(NP_E_INVAL, m);
  if (const char* m = tokens_error(n_tokens, cu, n)) return fail(NP_E_INVAL, m);
  if (n == 0 || n_tokens == 0) return NP_OK;
  if (!start) return fail(NP_E_INVAL, "NULL argument");
  if (const char* m = rows_error(q)) return fail(NP_E_INVAL, m);
  if (const char* m = rows_error(k)) return fail(NP_E_INVAL, m);
  if (const char* m = out_error(q_out, n_tokens, d->n_heads)) return fail(NP_E_INVAL, m);
  if (const char* m = out_error(k_out, n_tokens, d->n_kv_heads)) return fail(NP_E_INVAL, m);
  RowsArgs a = {};
  put_tokens(a, n_tokens, nullptr, cu, start, n);
  put_rotation(a, r);
  uint16_t* qd;
  put_rows(q, &qd, &a.q_token, &a.q_head);
  a.q = qd;
  put_rows(k, &a.k, &a.k_token, &a.k_head);
  put_rows(q_out, &a.q_out, &a.qo_token, &a.qo_head);
  put_rows(k_out, &a.k_out, &a.ko_token, &a.ko_head);
  a.nq = d->n_heads;
  a.nkv = d->n_kv_heads;
  a.rows = a.nq + a.nkv;
  return run(a, d->dtype, d->head_dim, false, true, false, stream);
}

int np_kv_append_rotated(const np_kv_desc* d, void* cache, int32_t layer, const np_kv_tables* t, const np_rotation* r, const np_rows* q,
                         int32_t n_heads, const np_rows* k, const np_rows* v, const np_rows* q_out, int32_t n_tokens, const int32_t* seqs,
                         const int32_t* cu, const int32_t* start, int32_t n, void* stream) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  if (const char* m = rotation_error(r, d->head_dim)) return fail(NP_E_INVAL, m);
  if (n_heads < 1 || n_heads > (1 << 17)) return fail(NP_E_INVAL, "n_heads outside [1, 131072]");
  if (int rc = enter(d, cache, layer, t, k, v, n_tokens, cu, start, n)) return rc == 1 ? NP_OK : rc;
  if (const char* m = rows_error(q)) return fail(NP_E_INVAL, m);
  if (const char* m = out_error(q_out, n_tokens, n_heads)) return fail(NP_E_INVAL, m);
  RowsArgs a = {};
  put_tokens(a, n_tokens, seqs, cu, start, n);
  put_rotation(a, r);
  put_cache(a, d, cache, layer, t);
  uint16_t* qd;
  put_rows(q, &qd, &a.q_token, &a.q_head);
  a.q = qd;
  put_rows(k, &a.k, &a.k_token, &a.k_head);
  put_rows(v, &a.v, &a.v_token, &a.v_head);
  put_rows(q_out, &a.q_out, &a.qo_token, &a.qo_head);
  a.nq = n_heads;
  a.rows = a.nq + 2 * a.nkv;
  return run(a, row_type(d), d->head_dim, false, true, held_in_8(d), stream);
}

int np_kv_read(const np_kv_desc* d, const void* cache, int32_t layer, const np_kv_tables* t, const np_rows* k, const np_rows* v, int32_t n_tokens,
               const int32_t* seqs, const int32_t* cu, const int32_t* start, int32_t n, void* stream) {
  if (int rc = enter(d, cache, layer, t, k, v, n_tokens, cu, start, n)) return rc == 1 ? NP_OK : rc;
  if (const char* m = out_error(k, n_tokens, d->n_kv_heads)) return fail(NP_E_INVAL, m);
  if (const char* m = out_error(v, n_tokens, d->n_kv_heads)) return fail(NP_E_INVAL, m);
  RowsArgs a = {};
  put_tokens(a, n_tokens, seqs, cu, start, n);
  put_cache(a, d, cache, layer, t);
  put_rows(k, &a.k, &a.k_token, &a.k_head);
  put_rows(v, &a.v, &a.v_token, &a.v_head);
  a.rows = 2 * a.nkv;
  return run(a, row_type(d), d->head_dim, true, false, held_in_8(d), stream);
}

}  // extern "C"
