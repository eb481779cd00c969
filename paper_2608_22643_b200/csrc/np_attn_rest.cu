// Attention of one new token for each row of groups that share their first tokens (np_attn_decode_shared), the second of two kernels: what a row has
// behind those, and the join with what np_attn_shared.cu has left of them.
//
// A block takes up to eight heads of a row and key-value head, four warps sixteen tokens each at a time, as in np_attn_decode.cu: S^T = K Q^T and
// O^T = V^T P^T on mma.sync, keys and values from global memory into the registers that the products read.  Rows' own tokens are often few, and then
// what counts is how short the way from the launch to the result is, so this is its own small kernel (np_attn_decode.cu's, with an even line of work
// and another kernel for the join, took 24 us in place of 20 for the 64 rows below).  Times of both kernels that are compared here are from before the first
// had its weights in two terms, which adds 3 to 8 us to either side:
// * It begins as soon as the first kernel's blocks leave room, works out by itself what its row shares, and waits only before the join.  (With the
//   first kernel telling what is where: 66.3 us for both in place of 61.)
// * Only where there are fewer blocks than the GPU holds are rows split; the last split to arrive joins them, in the order of the tokens.  Where a row
//   has too few tokens for that, all the blocks compute the same and each joins some of the heads: 4 rows that share 8192 tokens, 64 heads over 8,
//   46.2 us with one block to join eight heads, 32.2 so.
// * Where there are more blocks than the GPU holds and groups have one head or two, a warp to each of four key-value heads: one start for
//   four of them.  64 rows that share 8192 tokens and have 64 of their own, 32 heads: 69.7 us in place of 84.8; 24 rows 61.4 in place of 59.5, with
//   600 tokens 94 in place of 103.  (Several pairs one after the other to a block, the next one's keys asked for before the join: 94.6.)
//
// Measured alone: 64 rows of 1 to 200 tokens (4190 together), 64 heads over 8, nine parts of what they share: 20 us for 17 MB of the cache and 19 MB of
// parts, so it is latency that bounds it: four loads that depend on one another before the first keys, up to four steps of them, and two
// rounds of parts.
#include <algorithm>

#include "np_attn.h"
#include "np_attn_groups.cuh"
#include "np_attn_mma.cuh"
#include "np_device.cuh"
#include "np_internal.h"
#include "np_pipe.cuh"

namespace npa {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32, kHeads = 8;
constexpr int kSplitTokens = 128;  // tokens of a split, at least
constexpr int kAhead = 5;          // parts that a thread asks for at a time

struct RestArgs {
  Layer layer;
  const int32_t *seqs, *lens, *table;
  int32_t* status;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_token, q_head, o_token, o_head;  // elements
  float* lse;
  SharedArgs shared;
  float scale2;  // scale * log2(e)
  int n_heads, group, blocks_of_heads, splits, max_pages, max_seqs, n;
};
__device__ __forceinline__ int sequence(const RestArgs& a, int i) {
  const int seq = a.seqs ? a.seqs[i] : i;
  return seq < a.max_seqs ? max(seq, -1) : -1;
}
__device__ __forceinline__ int length(const RestArgs& a, int seq) {
  const int len = a.lens[seq];
  if (len >= 0 && ((int64_t)len + (1 << a.layer.shift) - 1) >> a.layer.shift <= a.max_pages) return len;
  atomicOr(a.status, NP_KV_S_LENGTH);
  return 0;
}

// Where the parts of a row's shared tokens are, for one head: of `count` blocks, or of the one that has done all of them; 0: none.
template <int HD>
struct SharedParts {
  const SharedArgs& s;
  const Record* whole;
  int first, count, place;
  __device__ __forceinline__ int64_t slot(int y) const { return (int64_t)(2 * (first + y) + (y == 0)) * s.part_rows + place; }
  __device__ __forceinline__ const float* ml(int y) const { return count == 1 ? whole->ml[0] : s.part_ml + slot(y) * 2; }
  __device__ __forceinline__ const float* o(int y) const { return count == 1 ? whole->o[0] : s.part_o + slot(y) * HD; }
};

struct Sum {
  float top, sum, acc[4];
};
__device__ __forceinline__ bool odd_four(const float (&x)[4]) { return not_finite(x[0]) || not_finite(x[1]) || not_finite(x[2]) || not_finite(x[3]); }
// `count` parts joined to x, kAhead at a time
template <class Ml, class O>
__device__ __forceinline__ void join(Sum& x, int count, Ml ml_of, O o_of) {
  for (int y0 = 0; y0 < count; y0 += kAhead) {
    float2 ml[kAhead];
    float4 v[kAhead];
#pragma unroll
    for (int y = 0; y < kAhead; ++y) {
      ml[y] = make_float2(-INFINITY, 0.f);
      v[y] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (y0 + y >= count) continue;
      ml[y] = __ldcg(reinterpret_cast<const float2*>(ml_of(y0 + y)));
      v[y] = __ldcg(reinterpret_cast<const float4*>(o_of(y0 + y)));
    }
    float now = x.top;
#pragma unroll
    for (int y = 0; y < kAhead; ++y) now = fmaxf(now, ml[y].x);
    const float use = now == -INFINITY ? 0.f : now, f0 = exp2_fast(x.top - use);
    x.top = now;
    x.sum *= f0;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.acc[i] *= f0;
#pragma unroll
    for (int y = 0; y < kAhead; ++y) {
      const float f = exp2_fast(ml[y].x - use);
      x.sum += f * ml[y].y;
      x.acc[0] += f * v[y].x;
      x.acc[1] += f * v[y].y;
      x.acc[2] += f * v[y].z;
      x.acc[3] += f * v[y].w;
    }
  }
}
// Factors that are 0 make a NaN of an infinity: what is not finite is what the parts that are not, and `own`, add up to.
template <class O>
__device__ __noinline__ void keep_not_finite(Sum& x, const float (&own)[4], int count, O o_of) {
  for (int i = 0; i < 4; ++i) {
    float kept = not_finite(own[i]) ? own[i] : 0.f;
    for (int y = 0; y < count; ++y) {
      const float v = __ldcg(o_of(y) + i);
      if (not_finite(v)) kept += v;
    }
    if (not_finite(kept)) x.acc[i] = kept;
  }
}

// kApart: a warp to each of four key-value heads of at most two heads, in place of four warps to one.
template <class T, int HD, bool kApart>
__global__ void __launch_bounds__(kThreads, HD == 64 ? 5 : 4)
k_attn_rest(const __grid_constant__ RestArgs a) {
  constexpr int KV = HD / 32;             // 16-byte pieces of a key row per lane
  constexpr int VC = HD / 64;             // 16-byte pieces of a value row per lane
  constexpr int QR = HD * 2 + 64;         // bytes from query to query: reads meet all banks
  constexpr int kFours = HD / 4;
  constexpr int kKvHeads = kApart ? kWarps : 1;     // of a block
  constexpr int kStep = kApart ? 1 : kWarps;        // sixteens of tokens from one of a warp's to its next
  __shared__ __align__(16) float s_o[kWarps][kHeads][HD];
  __shared__ __align__(16) unsigned char s_q[kHeads * QR];
  __shared__ float s_ml[kWarps][kHeads][2];
  __shared__ int s_seen[kKvHeads][HD];
  __shared__ Sum s_turns[kThreads];
  __shared__ int s_group, s_last;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
  const int pairs = kApart ? (a.layer.n_kv_heads + kKvHeads - 1) / kKvHeads : a.layer.n_kv_heads * a.blocks_of_heads;
  const int split = blockIdx.x % a.splits, of = blockIdx.x / a.splits, i = of / pairs, pair = of - i * pairs;
  const int kvh0 = kApart ? pair * kKvHeads : pair / a.blocks_of_heads, kv_heads = min(kKvHeads, a.layer.n_kv_heads - kvh0);
  const int hb = kApart ? 0 : pair - kvh0 * a.blocks_of_heads;
  const int h0 = kvh0 * a.group + hb * kHeads, heads = kApart ? kv_heads * a.group : min(kHeads, a.group - hb * kHeads);
  auto kv_of = [&](int h) { return kApart && a.group == 1 ? h : kApart ? h >> 1 : 0; };   // which of the block's a head's is
  const bool there = !kApart || wid < kv_heads;
  // The first kernel lets this one begin once what came before itself is done, so the tables and the caller's groups can be read; only what that
  // kernel writes has to be waited for.
  npp::pdl_launch_dependents();
  for (int x = tid; x < kHeads * (HD / 8); x += kThreads) {
    const int h = x / (HD / 8), d = x % (HD / 8) * 8;
    uint4 q = make_uint4(0, 0, 0, 0);
    if (h < heads) q = *reinterpret_cast<const uint4*>(a.q + i * a.q_token + (int64_t)(h0 + h) * a.q_head + d);
    *reinterpret_cast<uint4*>(s_q + h * QR + d * 2) = q;
  }
  // the row's sequence and tokens (0: no sequence, or more than its table holds), and those that it shares
  const int seq = sequence(a, i), len = seq < 0 ? 0 : length(a, seq);
  if (tid == 0) s_group = -1;
  __syncthreads();
  for (int x = tid; x < a.shared.n_groups; x += kThreads) {
    const GroupInfo group = group_at(a.shared, a.n, x);
    if (i >= group.lo && i < group.hi) atomicMax(&s_group, x);
  }
  __syncthreads();
  int held = 0;
  if (s_group >= 0) {  // as check_group() has it
    const GroupInfo group = group_at(a.shared, a.n, s_group);
    held = group.tokens;
    bool good = held > 0 && (held & ((1 << a.layer.shift) - 1)) == 0 && (held >> a.layer.shift) <= a.max_pages;
    for (int x = group.lo + tid; x < group.hi; x += kThreads) {
      const int of = sequence(a, x);
      good &= of < 0 || a.lens[of] >= held;
    }
    if (!__syncthreads_and(good)) held = 0;
  }
  const int own = max(len - held, 0);
  // this block's tokens of the row's own, sixteens of them: [c0, c1)
  const int sixteens = (int)(((int64_t)own + 15) >> 4);
  const int splits = min(a.splits, max(1, (sixteens + kSplitTokens / 16 - 1) / (kSplitTokens / 16))), each = (sixteens + splits - 1) / splits;
  // what needs no splits is computed by all of their blocks, and each has the result of some of the heads: [from_head, to_head)
  const int each_head = splits > 1 ? heads : (heads + a.splits - 1) / a.splits;
  const int from_head = splits > 1 ? 0 : split * each_head, to_head = min(heads, from_head + each_head);
  if (splits > 1 ? split >= splits : from_head >= heads) return;
  const int part = splits == 1 ? 0 : split, c0 = part * each, c1 = there ? min(sixteens, c0 + each) : c0, ce = min(sixteens, c0 + each);
  const int32_t* const pages = a.table + (size_t)max(seq, 0) * a.max_pages + (held >> a.layer.shift);
  const int64_t head_bytes = (int64_t)(HD * 2) << a.layer.shift, page_bytes = 2 * a.layer.n_kv_heads * head_bytes;
  const char* const keys = a.layer.cache + (kvh0 + (kApart && there ? wid : 0)) * head_bytes;
  const int64_t to_values = a.layer.n_kv_heads * head_bytes;

  uint4 kf[2][KV], vf[4][VC];
  // where chunk c with page pg is, and how many of its tokens there are (0: none)
  auto place = [&](int c, int pg, int& n) -> int64_t {
    n = c < c1 ? min(16, own - c * 16) : 0;
    if (n > 0 && (unsigned)pg >= (unsigned)a.layer.n_pages) {
      atomicOr(a.status, NP_KV_S_PAGE);
      n = 0;
    }
    return n > 0 ? pg * page_bytes + (int64_t)((c * 16) & ((1 << a.layer.shift) - 1)) * (HD * 2) : 0;
  };
  auto page_of = [&](int c) { return c < c1 ? pages[(c * 16) >> a.layer.shift] : 0; };
  auto load_k = [&](int64_t from, int n) {
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < KV; ++j) {
        kf[r][j] = make_uint4(0, 0, 0, 0);
        if (g + 8 * r < n) kf[r][j] = npd::ldg_stream(keys + from + (g + 8 * r) * (HD * 2) + (t + 4 * j) * 16);
      }
  };
  auto load_v = [&](int64_t from, int n) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int tok = 2 * t + (r & 1) + (r >> 1) * 8;
#pragma unroll
      for (int x = 0; x < VC; ++x) {
        vf[r][x] = make_uint4(0, 0, 0, 0);
        if (tok < n) vf[r][x] = npd::ldg_stream(keys + to_values + from + tok * (HD * 2) + (g + 8 * x) * 16);
      }
    }
  };
  const int begin = c0 + (kApart ? 0 : wid), second_page = page_of(begin + kStep);
  int first_have;
  const int64_t first_at = place(begin, page_of(begin), first_have);
  load_k(first_at, first_have);
  load_v(first_at, first_have);
  int have = first_have, page = second_page;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[VC * 4][4];
#pragma unroll
  for (auto& x : o) x[0] = x[1] = x[2] = x[3] = 0.f;
  __syncthreads();
  for (int c = begin; c < c1; c += kStep) {
    int next_have;
    const int64_t next_at = place(c + kStep, page, next_have);
    page = page_of(c + 2 * kStep);
    // ---- S^T = K Q^T
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < KV; ++j) {
      uint4 q = make_uint4(0, 0, 0, 0);
      if (!kApart || g < a.group) q = *reinterpret_cast<const uint4*>(s_q + (kApart ? wid * a.group + g : g) * QR + (t + 4 * j) * 16);
      Half2<T>::mma(s, kf[0][j].x, kf[1][j].x, kf[0][j].y, kf[1][j].y, q.x, q.y);
      Half2<T>::mma(s, kf[0][j].z, kf[1][j].z, kf[0][j].w, kf[1][j].w, q.z, q.w);
    }
    load_k(next_at, next_have);
    // ---- softmax: s[0], s[1] are token g, s[2], s[3] token g + 8; heads 2t and 2t + 1
    uint32_t ph[2], pl[2];
    float p[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) s[x] = g + 8 * (x >> 1) < have ? s[x] * a.scale2 : -INFINITY;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float top = fmaxf(s[x], s[x + 2]);
#pragma unroll
      for (int y = 4; y < 32; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, y));
      const float now = fmaxf(m[x], top), use = now == -INFINITY ? 0.f : now, f = exp2_fast(m[x] - use);
      m[x] = now;
      p[x] = exp2_fast(s[x] - use);
      p[x + 2] = exp2_fast(s[x + 2] - use);
      l[x] = l[x] * f + p[x] + p[x + 2];
#pragma unroll
      for (auto& y : o) {
        y[x] *= f;
        y[x + 2] *= f;
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint32_t hi, lo;
      Half2<T>::split(p[2 * x], p[2 * x + 1], hi, lo);
      ph[x] = transpose8x8(hi);
      pl[x] = transpose8x8(lo);
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
    load_v(next_at, next_have);
    have = next_have;
  }

  // ---- the warps' results meet
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int h = 2 * t + x;
#pragma unroll
    for (int y = 4; y < 32; y <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], y);
    if (g == 0) {
      s_ml[wid][h][0] = m[x];
      s_ml[wid][h][1] = l[x];
    }
#pragma unroll
    for (int k = 0; k < VC * 4; ++k) *reinterpret_cast<float2*>(&s_o[wid][h][(g + 8 * (k >> 2)) * 8 + 2 * (k & 3)]) = make_float2(o[k][x], o[k][x + 2]);
  }
  __syncthreads();
  auto of_warps = [&](int h, int d) {
    Sum x = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    if (kApart) {
      const int w = kv_of(h), in = h - w * a.group;
      const float4 v = *reinterpret_cast<const float4*>(&s_o[w][in][d]);
      x = Sum{s_ml[w][in][0], s_ml[w][in][1], {v.x, v.y, v.z, v.w}};
    } else {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) x.top = fmaxf(x.top, s_ml[w][h][0]);
      const float use = x.top == -INFINITY ? 0.f : x.top;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_fast(s_ml[w][h][0] - use);
        const float4 v = *reinterpret_cast<const float4*>(&s_o[w][h][d]);
        x.sum += f * s_ml[w][h][1];
        x.acc[0] += f * v.x;
        x.acc[1] += f * v.y;
        x.acc[2] += f * v.z;
        x.acc[3] += f * v.w;
      }
    }
    if (x.sum == 0.f) x.acc[0] = x.acc[1] = x.acc[2] = x.acc[3] = 0.f;  // nothing but scores of -inf
    return x;
  };
  bool odd = false;  // what the values make infinite or NaN has to be looked up
  for (int x = from_head * kFours + tid; x < to_head * kFours; x += kThreads) {
    const Sum mine = of_warps(x / kFours, x % kFours * 4);
    odd |= odd_four(mine.acc) && !not_finite(mine.sum);
  }
  const bool look = __syncthreads_or(odd);
  if (look)
    for (int x = 0; x < kv_heads; ++x) look_through<T, HD>(a.layer, pages, kvh0 + x, (int64_t)c0 * 16, min((int64_t)own, (int64_t)ce * 16), s_seen[x]);
  auto own_of = [&](int h, int d) {
    Sum x = of_warps(h, d);
    if (look && !not_finite(x.sum) && x.sum != 0.f)
      for (int y = 0; y < 4; ++y)
        if (not_finite(x.acc[y]) && s_seen[kv_of(h)][d + y]) x.acc[y] = made_of(s_seen[kv_of(h)][d + y]);
    return x;
  };
  float* const rest_o = a.shared.rest_o + (int64_t)(blockIdx.x - split) * kHeads * HD;  // of the row's first split
  float* const rest_ml = a.shared.rest_ml + (int64_t)(blockIdx.x - split) * kHeads * 2;
  if (splits > 1) {
    for (int x = tid; x < heads * kFours; x += kThreads) {
      const int h = x / kFours, d = x % kFours * 4;
      const Sum mine = own_of(h, d);
      __stcg(reinterpret_cast<float4*>(rest_o + (split * kHeads + h) * HD + d), make_float4(mine.acc[0], mine.acc[1], mine.acc[2], mine.acc[3]));
      if (d == 0) __stcg(reinterpret_cast<float2*>(rest_ml + (split * kHeads + h) * 2), make_float2(mine.top, mine.sum));
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      unsigned int* count = &a.shared.records[(int64_t)i * a.n_heads + h0].pair_count;
      s_last = atomicAdd(count, 1u) + 1u == (unsigned)splits;
      if (s_last) *count = 0u;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
  }

  // ---- and with what the row shares
  npp::pdl_wait_prior();
  const RowPlan plan = a.shared.plan[i];
  const LinePlan line = *a.shared.line;
  const int64_t longer = line.more * (line.each + 1);
  auto block_of = [&](int64_t x) {
    return (int)min((int64_t)line.blocks - 1, x < longer ? divide(x, line.each + 1) : line.more + divide(x - longer, line.each));
  };
  // where there are fewer results than threads, several threads take turns at a result's parts
  const int results = (to_head - from_head) * kFours, turns = max(1, kThreads / results), turn = turns > 1 ? tid / results : 0;
  for (int x = turns > 1 ? tid - turn * results : tid; x < results; x += kThreads) {
    const int h = from_head + x / kFours, d = x % kFours * 4;
    int first = 0, parts = 0;
    if (plan.shared && len > 0) {
      const int64_t w = plan.first_w + (kvh0 + kv_of(h)) * plan.step;
      first = block_of(w);
      parts = block_of(w + (plan.shared + kSharedTile - 1) / kSharedTile - 1) - first + 1;
    }
    const SharedParts<HD> of_group = {a.shared, a.shared.records + ((int64_t)i * a.n_heads + h0 + h), first, parts,
                                      plan.place + hb * kHeads + h - kv_of(h) * a.group};
    auto split_o = [&](int y) { return rest_o + (y * kHeads + h) * HD + d; };
    auto group_o = [&](int y) { return of_group.o(y) + d; };
    Sum all = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    if (turn == 0 && splits == 1) all = own_of(h, d);
    if (turn == 0 && splits > 1) {
      join(all, splits, [&](int y) { return rest_ml + (y * kHeads + h) * 2; }, split_o);
      if (odd_four(all.acc) && !not_finite(all.sum)) keep_not_finite(all, {0.f, 0.f, 0.f, 0.f}, splits, split_o);
    }
    const float own[4] = {all.acc[0], all.acc[1], all.acc[2], all.acc[3]};
    join(
        all, turn < turns ? (parts - turn + turns - 1) / turns : 0, [&](int y) { return of_group.ml(turn + y * turns); },
        [&](int y) { return group_o(turn + y * turns); });
    if (turns > 1) {
      s_turns[tid] = all;
      __syncthreads();
      if (turn > 0) return;
      float top = all.top;
      for (int y = 1; y < turns; ++y) top = fmaxf(top, s_turns[y * results + x].top);
      const float use = top == -INFINITY ? 0.f : top, f0 = exp2_fast(all.top - use);
      all.top = top;
      all.sum *= f0;
#pragma unroll
      for (int z = 0; z < 4; ++z) all.acc[z] *= f0;
      for (int y = 1; y < turns; ++y) {
        const Sum& other = s_turns[y * results + x];
        const float f = exp2_fast(other.top - use);
        all.sum += f * other.sum;
#pragma unroll
        for (int z = 0; z < 4; ++z) all.acc[z] += f * other.acc[z];
      }
    }
    if (parts && odd_four(all.acc) && !not_finite(all.sum)) keep_not_finite(all, own, parts, group_o);
    const bool none = all.sum == 0.f;
    const float inv = none ? 0.f : 1.f / all.sum;
    uint32_t r[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) r[y] = none ? 0u : Half2<T>::round(all.acc[y] * inv);
    *reinterpret_cast<uint2*>(a.out + i * a.o_token + (int64_t)(h0 + h) * a.o_head + d) = make_uint2(r[0] | r[1] << 16, r[2] | r[3] << 16);
    if (a.lse && d == 0) a.lse[(size_t)i * a.n_heads + h0 + h] = none ? -INFINITY : (all.top == -INFINITY ? 0.f : all.top) * kLn2 + logf(all.sum);
  }
}

}  // namespace

int decode_rest(const np_kv_desc* d, const char* cache, const np_kv_tables* t, const np_rows* q, int32_t n_heads, const int32_t* seqs, int32_t n, float scale2,
                const np_rows* out, float* lse, const SharedArgs& shared, int sms, cudaStream_t s) {
  RestArgs a = {};
  a.layer = Layer{cache, d->n_kv_heads, log2_of(d->page_tokens), d->n_pages};
  a.seqs = seqs;
  a.lens = t->lens;
  a.table = t->page_table;
  a.status = t->status;
  a.q = static_cast<const uint16_t*>(q->data);
  a.out = static_cast<uint16_t*>(out->data);
  a.q_token = q->token_stride;
  a.q_head = q->head_stride;
  a.o_token = out->token_stride;
  a.o_head = out->head_stride;
  a.lse = lse;
  a.shared = shared;
  a.scale2 = scale2;
  a.n_heads = n_heads;
  a.group = n_heads / d->n_kv_heads;
  a.blocks_of_heads = (a.group + kHeads - 1) / kHeads;
  a.max_pages = d->max_pages;
  a.max_seqs = d->max_seqs;
  a.n = n;
  const int room = 4 * sms;
  int64_t blocks = (int64_t)n * d->n_kv_heads * a.blocks_of_heads;
  const bool apart = a.group <= 2 && blocks > room;
  if (apart) blocks = (int64_t)n * ((d->n_kv_heads + kWarps - 1) / kWarps);
  a.splits = (int)std::max<int64_t>(1, std::min<int64_t>(64, std::min(kRestBlocks, room) / blocks));
  const dim3 grid((unsigned)(blocks * a.splits));
  auto go = [&](auto kernel) { return launch_early(kernel, grid, kThreads, 0, s, a); };
  auto of_width = [&](auto type) {
    using T = decltype(type);
    if (d->head_dim == 128) return apart ? go(k_attn_rest<T, 128, true>) : go(k_attn_rest<T, 128, false>);
    return apart ? go(k_attn_rest<T, 64, true>) : go(k_attn_rest<T, 64, false>);
  };
  const cudaError_t e = row_type(d) == NP_T_BF16 ? of_width(__nv_bfloat16{}) : of_width(__half{});
  return e == cudaSuccess ? NP_OK : fail_cuda(e);
}

}  // namespace npa
