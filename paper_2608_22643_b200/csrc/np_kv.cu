// The paged key-value cache: who owns which page (reserve, fork, free, compact) and the bytes that move (append, page
// copies).
//
// Measured: np_kv_append of 8192 tokens, 8 heads of 128, 11 us (67 MB read and written, 6.1 TB/s); page copies of a compaction, 880 MB,
// 139 us (6.3 TB/s, 97 % of the copy rate), of a fork, 268 MB in pages of 16 tokens, 38 us; np_kv_reserve 3.5 us, np_kv_free 1.5.
//
// The table work is integers in one block: a scan over the listed sequences says how many pages each needs, a scan over
// the reference counts lists the free pages (lowest number first), and both are exact, so what a call does depends on
// nothing but its inputs.  It is bound by the latency of its few dependent loads and by the launch (a call on a pool of a
// few thousand pages is a handful of barriers).  Freeing takes a block per sequence: nothing in it is ordered.
//
// The copies are bound by memory: 16 bytes per lane, four loads in flight per lane before the first store, pages cut into
// units of 16 KB that all blocks of the grid take in turn (a page is contiguous per layer only, so a unit is (layer, pair of
// pages, piece)).
#include <algorithm>
#include <atomic>
#include <cstdio>

#include "np_attn.h"
#include "np_device.cuh"
#include "np_internal.h"
#include "np_pipe.cuh"

namespace npa {

static thread_local char g_err[256] = "";
int fail(int code, const char* msg) {
  snprintf(g_err, sizeof g_err, "%s", msg);
  return code;
}
int fail_cuda(cudaError_t e) { return fail(NP_E_CUDA, cudaGetErrorString(e)); }

const char* desc_error(const np_kv_desc* d) {
  if (!d) return "NULL description";
  if (d->dtype != NP_T_BF16 && d->dtype != NP_T_FP16) return "dtype must be NP_T_BF16 or NP_T_FP16";
  if (d->n_layers < 1 || d->n_kv_heads < 1 || d->n_kv_heads > 1024) return "n_layers must be positive, n_kv_heads in [1, 1024]";
  if (d->head_dim != 64 && d->head_dim != 128) return "head_dim must be 64 or 128";
  const int p = d->page_tokens;
  if (p != 16 && p != 32 && p != 64 && p != 128 && p != 256) return "page_tokens must be 16, 32, 64, 128 or 256";
  if (d->n_pages < 1 || d->n_pages > NP_KV_MAX_PAGES) return "n_pages outside [1, NP_KV_MAX_PAGES]";
  if (d->max_seqs < 1 || d->max_seqs > NP_KV_MAX_SEQS) return "max_seqs outside [1, NP_KV_MAX_SEQS]";
  if (d->max_pages < 1 || d->max_pages > d->n_pages || (int64_t)d->max_pages * p > 0x7fffffffLL)
    return "max_pages outside [1, n_pages], or its tokens do not fit in 31 bits";
  for (int r : d->reserved)
    if (r) return "reserved must be 0";
  return nullptr;
}

const char* rows_error(const np_rows* r) {
  if (!r || !r->data) return "NULL rows";
  if ((uintptr_t)r->data % 16) return "rows must be 16-byte aligned";
  if (r->token_stride < 0 || r->head_stride < 0 || r->token_stride % 8 || r->head_stride % 8)
    return "strides of rows must be multiples of 8 elements and not negative";
  return nullptr;
}

bool tables_ok(const np_kv_tables* t) { return t && t->page_table && t->lens && t->refs && t->scratch && t->status; }

bool device_sms(int* sms) {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  if (dev < 64 && (*sms = known[dev].load(std::memory_order_relaxed)) > 0) return true;
  if (cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return false;
  if (dev < 64) known[dev].store(*sms, std::memory_order_relaxed);
  return true;
}

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPerThread = 8;                             // reference counts per thread and round of a scan
constexpr int kRound = kPlanThreads * kPerThread;
constexpr int kFewPages = 2048;                           // page numbers that need no trip through memory

// What the kernels need of a description, and where the pieces of the scratch are.
struct Pool {
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int32_t* scratch;
  int32_t* status;
  int shift, n_pages, max_seqs, max_pages;
  __host__ __device__ int list_len() const { return n_pages > NP_KV_MAX_SEQS ? n_pages : NP_KV_MAX_SEQS; }
  __host__ __device__ int32_t* pages() const { return scratch; }                       // [n_pages] free pages, or the map
  __host__ __device__ int32_t* pair_src() const { return scratch + n_pages; }          // [list_len]
  __host__ __device__ int32_t* pair_dst() const { return pair_src() + list_len(); }    // [list_len]
  __host__ __device__ int32_t* pair_count() const { return pair_dst() + list_len(); }  // [1]
};

uint64_t scratch_ints(const np_kv_desc* d) {
  const uint64_t list = d->n_pages > NP_KV_MAX_SEQS ? d->n_pages : NP_KV_MAX_SEQS;
  return d->n_pages + 2 * list + 16;
}

Pool pool_of(const np_kv_desc* d, const np_kv_tables* t) {
  return Pool{t->page_table, t->lens, t->refs, t->scratch, t->status, log2_of(d->page_tokens), d->n_pages, d->max_seqs, d->max_pages};
}

// Pages of a sequence's table row that its length uses; -1: the row does not hold that length.
__device__ __forceinline__ int pages_of(const Pool& p, int len) {
  if (len < 0) return -1;
  const int n = (int)(((int64_t)len + (1 << p.shift) - 1) >> p.shift);
  return n > p.max_pages ? -1 : n;
}

// The pages that a thread looks at in the round of a scan that begins at page `base`: bit j where take(refs[p], p), p its j-th.
template <class Take>
__device__ __forceinline__ uint32_t pages_taken(const int32_t* refs, int n, int base, Take take) {
  const int first = base + threadIdx.x * kPerThread;
  uint32_t mine = 0;
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int q = first + j;
    if (q < n && take(refs[q], q)) mine |= 1u << j;
  }
  return mine;
}

// Lists, in ascending order, the first `want` pages p of [0, n) for which take(refs[p], p); returns how many there are (at most
// `want`).  The whole block calls it.  round0: pages_taken for the first round.  red: 34 ints.
template <class Take>
__device__ int list_pages(const int32_t* refs, int n, int want, uint32_t round0, int32_t* out, int* red, Take take) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  int found = 0;
  for (int base = 0; base < n && found < want; base += kRound) {
    const int first = base + tid * kPerThread;
    uint32_t mine = base ? pages_taken(refs, n, base, take) : round0;
    const int cnt = __popc(mine);
    const int inc = npd::block_inclusive_scan_1024(cnt, red, lane, wid);
    int at = found + inc - cnt;
    const int total = red[32];
    while (mine && at < want) {
      const int j = __ffs(mine) - 1;
      mine &= mine - 1;
      out[at++] = first + j;
    }
    found += total;
    __syncthreads();
  }
  return min(found, want);
}

// Whether entry i of a list is the first of its value.
__device__ __forceinline__ bool first_of_its_value(const int* list, int i) {
  for (int j = 0; j < i; ++j)
    if (list[j] == list[i]) return false;
  return true;
}

// reserve (kFork false) and fork (true): who gets which pages.
template <bool kFork>
__global__ void __launch_bounds__(kPlanThreads, 1)
k_kv_take(Pool p, const int32_t* __restrict__ a, const int32_t* __restrict__ b, int n, int32_t* __restrict__ start_out) {
  __shared__ int s_seq[NP_KV_MAX_SEQS], s_src[kFork ? NP_KV_MAX_SEQS : 1], s_end[NP_KV_MAX_SEQS], s_old[NP_KV_MAX_SEQS];
  __shared__ int s_pages[kFewPages];
  __shared__ int red[34];
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  auto is_free = [](int r, int) { return r <= 0; };
  const uint32_t round0 = pages_taken(p.refs, p.n_pages, 0, is_free);  // on its way beside the sequences' lengths
  // reserve: a = sequences (NULL: 0..n-1), b = new tokens.  fork: a = sources, b = targets.
  int seq = -1, src = -1, add = 0;
  if (tid < n) {
    seq = kFork ? b[tid] : (a ? a[tid] : tid);
    if (kFork) src = a[tid];
    else add = b[tid];
    s_seq[tid] = seq;
  }
  __syncthreads();
  int bad = 0, need = 0, old = 0, len = 0, grown = 0;
  bool ok = false;
  if (tid < n) {
    const bool known = seq >= 0 && seq < p.max_seqs && (!kFork || (src >= 0 && src < p.max_seqs)) && first_of_its_value(s_seq, tid);
    if (!known) {
      bad = NP_KV_S_SEQ;
    } else if (kFork) {
      len = p.lens[src];
      old = pages_of(p, len);
      if (p.lens[seq] != 0) bad = NP_KV_S_SEQ;
      else if (old < 0) bad = NP_KV_S_LENGTH;
      else need = (len & ((1 << p.shift) - 1)) ? 1 : 0;
      grown = len;
      old -= need;  // full pages
    } else {
      len = p.lens[seq];
      old = pages_of(p, len);
      const int64_t to = (int64_t)len + add;
      const int now = to > 0x7fffffffLL ? -1 : pages_of(p, (int)to);
      if (add < 0 || old < 0 || now < 0) bad = NP_KV_S_LENGTH;
      else need = now - old;
      grown = (int)to;
    }
    ok = bad == 0;
    if (!ok) need = 0;
  }
  __syncthreads();
  // sums past the pool are too many, however many: up to 1024 sequences may ask for 2^22 pages each
  static_assert(NP_KV_MAX_PAGES < npd::kSumTop, "a sum that stops is more than a pool has");
  const int end = npd::block_inclusive_scan_to_top_1024(need, red, lane, wid);
  const int total = red[32];
  __syncthreads();
  int32_t* pages = total <= kFewPages ? s_pages : p.pages();
  const int have = total > 0 ? list_pages(p.refs, p.n_pages, min(total, p.n_pages), round0, pages, red, is_free) : 0;
  if (ok && need > 0 && end > have) {
    bad = NP_KV_S_FULL;
    ok = false;
  }
  __syncthreads();  // the list is in place; all lengths are read
  if (tid < n) {
    s_end[tid] = end;
    s_old[tid] = ok ? old : -1;
    if (kFork) s_src[tid] = src;
    if (ok) p.lens[seq] = grown;
    if (start_out) start_out[tid] = ok ? len : -1;
    if (bad) atomicOr(p.status, bad);
  }
  __syncthreads();
  // the new pages: item f of the scan belongs to the first sequence whose end is above f
  const int given = min(total, have);
  for (int f = tid; f < given; f += kPlanThreads) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (s_end[mid] > f) hi = mid;
      else lo = mid + 1;
    }
    if (s_old[lo] < 0) continue;
    const int before = lo ? s_end[lo - 1] : 0, pg = pages[f];
    p.table[(size_t)s_seq[lo] * p.max_pages + s_old[lo] + (f - before)] = pg;
    p.refs[pg] = 1;
  }
  if (kFork) {
    for (int i = tid; i < n; i += kPlanThreads) {
      int from = -1, to = -1;
      const int before = i ? s_end[i - 1] : 0;
      if (s_old[i] >= 0 && s_end[i] > before) {
        from = p.table[(size_t)s_src[i] * p.max_pages + s_old[i]];
        to = pages[before];
        if ((unsigned)from >= (unsigned)p.n_pages) atomicOr(p.status, NP_KV_S_PAGE);  // the target's page keeps what it held
      }
      p.pair_src()[i] = from;
      p.pair_dst()[i] = to;
    }
    // full pages are shared: a warp per sequence
    for (int i = wid; i < n; i += kPlanThreads / 32) {
      if (s_old[i] < 0) continue;
      const int32_t* from = p.table + (size_t)s_src[i] * p.max_pages;
      int32_t* to = p.table + (size_t)s_seq[i] * p.max_pages;
      for (int j = lane; j < s_old[i]; j += 32) {
        const int pg = from[j];
        to[j] = pg;
        if ((unsigned)pg < (unsigned)p.n_pages) atomicAdd(&p.refs[pg], 1);
        else atomicOr(p.status, NP_KV_S_PAGE);
      }
    }
  }
}

__global__ void __launch_bounds__(256)
k_kv_free(Pool p, const int32_t* __restrict__ seqs, int n) {
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int i = blockIdx.x, tid = threadIdx.x;
  const int seq = seqs ? seqs[i] : i;
  bool again = false;
  if (seqs)
    for (int j = tid; j < i; j += blockDim.x) again |= seqs[j] == seq;
  again = __syncthreads_or(again);
  if (again || seq < 0 || seq >= p.max_seqs) {
    if (tid == 0) atomicOr(p.status, NP_KV_S_SEQ);
    return;
  }
  const int m = pages_of(p, p.lens[seq]);
  __syncthreads();  // every thread has read the length
  if (m < 0) {
    if (tid == 0) atomicOr(p.status, NP_KV_S_LENGTH);
    return;
  }
  int32_t* row = p.table + (size_t)seq * p.max_pages;
  for (int j = tid; j < m; j += blockDim.x) {
    const int pg = row[j];
    row[j] = -1;
    if ((unsigned)pg < (unsigned)p.n_pages) atomicSub(&p.refs[pg], 1);
    else atomicOr(p.status, NP_KV_S_PAGE);
  }
  if (tid == 0) p.lens[seq] = 0;
}

// compact, first half: the map from old page numbers to new ones, the pairs to copy, the new reference counts.
__global__ void __launch_bounds__(kPlanThreads, 1)
k_kv_compact_plan(Pool p, int32_t* refs_out, int32_t* __restrict__ n_live) {
  __shared__ int red[34];
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int tid = threadIdx.x;
  int mine = 0;
  for (int q = tid; q < p.n_pages; q += kPlanThreads) mine += p.refs[q] > 0;
  const int live = npd::block_sum_int(mine, red);
  int32_t* map = p.pages();
  __syncthreads();
  auto moving = [live](int r, int q) { return r > 0 && q >= live; };
  auto hole = [](int r, int) { return r <= 0; };
  const int moves = list_pages(p.refs, p.n_pages, p.n_pages, pages_taken(p.refs, p.n_pages, 0, moving), p.pair_src(), red, moving);
  list_pages(p.refs, live, moves, pages_taken(p.refs, live, 0, hole), p.pair_dst(), red, hole);
  for (int q = tid; q < p.n_pages; q += kPlanThreads) {
    map[q] = q;
    const int r = p.refs[q];
    refs_out[q] = r > 0 && q < live ? r : (refs_out == p.refs ? r : 0);
  }
  __syncthreads();
  for (int i = tid; i < moves; i += kPlanThreads) {
    const int from = p.pair_src()[i], to = p.pair_dst()[i];
    map[from] = to;
    refs_out[to] = p.refs[from];
    refs_out[from] = 0;
  }
  if (tid == 0) {
    *p.pair_count() = moves;
    if (n_live) *n_live = live;
  }
}

// Copies pages (src[i] -> dst[i], in every layer) and, where `lens_out` is set, rewrites the page tables by `map`.
struct CopyArgs {
  char* dst;
  const char* src;
  const int32_t* from;
  const int32_t* to;
  const int32_t* count;   // device count of pairs; NULL: n_pairs
  int n_pairs;
  int n_pages, n_layers;
  int64_t page_bytes, layer_bytes;
  int32_t* status;        // NULL: pairs outside the pool are passed over silently (a fork's sequences without a copy)
};
struct RewriteArgs {
  const int32_t* table;
  const int32_t* lens;
  const int32_t* map;
  int32_t* table_out;
  int32_t* lens_out;      // NULL: no tables to rewrite
  int shift, n_pages, max_seqs, max_pages;
};

constexpr int kCopyThreads = 256;
constexpr int kUnit = 16384;  // bytes of a unit: four 16-byte loads per lane

__device__ __forceinline__ void copy_and_rewrite(const CopyArgs& a, const RewriteArgs& w) {
  const int tid = threadIdx.x;
  if (w.lens_out) {
    for (int s = blockIdx.x; s < w.max_seqs; s += gridDim.x) {
      const int len = w.lens[s];
      int used = len < 0 ? 0 : (int)(((int64_t)len + (1 << w.shift) - 1) >> w.shift);
      if (len < 0 || used > w.max_pages) {
        used = 0;
        if (tid == 0) atomicOr(a.status, NP_KV_S_LENGTH);
      }
      const int32_t* row = w.table + (size_t)s * w.max_pages;
      int32_t* out = w.table_out + (size_t)s * w.max_pages;
      for (int j = tid; j < w.max_pages; j += kCopyThreads) {
        int pg = -1;
        if (j < used) {
          pg = row[j];
          if ((unsigned)pg < (unsigned)w.n_pages) pg = w.map[pg];
          else {
            pg = -1;
            atomicOr(a.status, NP_KV_S_PAGE);
          }
        }
        out[j] = pg;
      }
      if (tid == 0) w.lens_out[s] = len;
    }
  }
  const int pairs = a.count ? min(*a.count, a.n_pairs) : a.n_pairs;
  const int per_page = (int)((a.page_bytes + kUnit - 1) / kUnit);
  const int64_t units = (int64_t)pairs * a.n_layers * per_page;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int piece = (int)(u % per_page);
    const int64_t r = u / per_page;
    const int i = (int)(r % pairs), layer = (int)(r / pairs);
    const int from = a.from[i], to = a.to[i];
    if ((unsigned)from >= (unsigned)a.n_pages || (unsigned)to >= (unsigned)a.n_pages) {
      if (a.status && tid == 0) atomicOr(a.status, NP_KV_S_PAGE);
      continue;
    }
    const int64_t off = (int64_t)layer * a.layer_bytes + (int64_t)piece * kUnit;
    const char* src = a.src + off + (int64_t)from * a.page_bytes;
    char* dst = a.dst + off + (int64_t)to * a.page_bytes;
    const int bytes = (int)min((int64_t)kUnit, a.page_bytes - (int64_t)piece * kUnit);
    uint4 v[kUnit / (16 * kCopyThreads)];
#pragma unroll
    for (int k = 0; k < kUnit / (16 * kCopyThreads); ++k) {
      const int at = (k * kCopyThreads + tid) * 16;
      if (at < bytes) v[k] = *reinterpret_cast<const uint4*>(src + at);
    }
#pragma unroll
    for (int k = 0; k < kUnit / (16 * kCopyThreads); ++k) {
      const int at = (k * kCopyThreads + tid) * 16;
      if (at < bytes) *reinterpret_cast<uint4*>(dst + at) = v[k];
    }
  }
}

__global__ void __launch_bounds__(kCopyThreads)
k_kv_copy(CopyArgs a, RewriteArgs w) {
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  copy_and_rewrite(a, w);
}

// compact of a small pool into other tables, in one launch: every block works the plan out for itself, a few loads and two scans, and
// nothing that it reads is written.  In a stream of calls 9.1 us with two launches for a pool of 28 pages, 7.0 with one; 148.5 and
// 146.5 for 96 pages of 80 layers.  The plan in memory (k_kv_compact_plan) is for larger pools, and for tables that are rewritten in place.
constexpr int kSmallPool = kCopyThreads * kPerThread;

__global__ void __launch_bounds__(kCopyThreads)
k_kv_compact_small(Pool p, int32_t* refs_out, int32_t* __restrict__ n_live, CopyArgs a, RewriteArgs w) {
  __shared__ int32_t s_map[kSmallPool], s_from[kSmallPool / 2], s_to[kSmallPool / 2];
  __shared__ int s_sum[2][kCopyThreads / 32];
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, first = tid * kPerThread;
  // what a block's threads before this one have, and (total) all of them
  auto scan = [&](int mine, int* sums, int& total) {
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane == 31) sums[wid] = inc;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kCopyThreads / 32; ++i) {
      if (i < wid) before += sums[i];
      total += sums[i];
    }
    return before + inc - mine;
  };
  int refs[kPerThread], alive = 0, live;
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    refs[j] = first + j < p.n_pages ? p.refs[first + j] : 0;
    alive += refs[j] > 0;
    s_map[first + j] = first + j;
  }
  scan(alive, s_sum[0], live);
  int both = 0, all;  // holes below `live`, and (from bit 16 on) pages that move
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) both += first + j < live ? (refs[j] <= 0) : (refs[j] > 0) << 16;
  const int before = scan(both, s_sum[1], all);
  int hole = before & 0xffff, mover = before >> 16;
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    if (first + j < live && refs[j] <= 0) s_to[hole++] = first + j;
    if (first + j >= live && refs[j] > 0) s_from[mover++] = first + j;
  }
  __syncthreads();
  const int moves = all >> 16;
  for (int i = tid; i < moves; i += kCopyThreads) s_map[s_from[i]] = s_to[i];
  __syncthreads();
  if (blockIdx.x == 0) {
#pragma unroll
    for (int j = 0; j < kPerThread; ++j)
      if (first + j < p.n_pages) {
        if (first + j >= live) refs_out[first + j] = 0;
        else if (refs[j] > 0) refs_out[first + j] = refs[j];
        if (refs[j] > 0 && first + j >= live) refs_out[s_map[first + j]] = refs[j];
      }
    if (tid == 0 && n_live) *n_live = live;
  }
  a.from = s_from;
  a.to = s_to;
  a.count = nullptr;
  a.n_pairs = moves;
  w.map = s_map;
  copy_and_rewrite(a, w);
}

struct AppendArgs {
  char* cache;               // of the layer
  const char* k;
  const char* v;
  int64_t k_token, k_head, v_token, v_head;  // bytes
  const int32_t* seqs;
  const int32_t* cu;
  const int32_t* start;
  int n, n_tokens, n_kv_heads, vec_shift;    // a head's row is 1 << vec_shift pieces of 16 bytes
};

constexpr int kAppendThreads = 256, kAppendVecs = 4;
constexpr int kAppendPerBlock = kAppendThreads * kAppendVecs;

// A piece of 16 bytes per lane and turn; the rows a block touches are looked up once (sequence by binary search in cu, then
// the page), by one lane each.
__global__ void __launch_bounds__(kAppendThreads)
k_kv_append(Pool p, AppendArgs a) {
  // a token has at least 16 pieces (one head of 64), so a block's pieces belong to 65 tokens at most
  __shared__ int64_t s_dst[kAppendPerBlock / 16 + 2];
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int tid = threadIdx.x;
  const int per_token = 2 * a.n_kv_heads << a.vec_shift;
  const int64_t total = (int64_t)a.n_tokens * per_token, first = (int64_t)blockIdx.x * kAppendPerBlock;
  const int64_t last = min(total, first + kAppendPerBlock) - 1;
  const int t0 = (int)(first / per_token), t1 = (int)(last / per_token);
  const int row_bytes = 16 << a.vec_shift;
  const int64_t head_bytes = (int64_t)row_bytes << p.shift;
  for (int t = t0 + tid; t <= t1; t += kAppendThreads) {
    int i = -1, off = 0;
    if (!a.cu) {
      i = t < a.n ? t : -1;
    } else if (t >= a.cu[0] && t < a.cu[a.n]) {
      int lo = 0, hi = a.n - 1;  // the last i with cu[i] <= t
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.cu[mid] <= t) lo = mid;
        else hi = mid - 1;
      }
      i = lo;
      off = t - a.cu[lo];
    }
    int64_t dst = -1;
    if (i >= 0) {
      const int seq = a.seqs ? a.seqs[i] : i, st = a.start[i];
      if (seq < 0 || seq >= p.max_seqs) {
        if (st >= 0) atomicOr(p.status, NP_KV_S_SEQ);
      } else if (st >= 0 && off >= 0) {
        const int64_t pos = (int64_t)st + off;
        if (pos < p.lens[seq]) {
          const int64_t j = pos >> p.shift;
          const int pg = j < p.max_pages ? p.table[(size_t)seq * p.max_pages + j] : -1;
          if ((unsigned)pg < (unsigned)p.n_pages)
            dst = (int64_t)pg * 2 * a.n_kv_heads * head_bytes + (pos & ((1 << p.shift) - 1)) * row_bytes;
          else atomicOr(p.status, NP_KV_S_PAGE);
        }
      }
    }
    s_dst[t - t0] = dst;
  }
  __syncthreads();
  uint4 v[kAppendVecs];
  char* to[kAppendVecs];
#pragma unroll
  for (int j = 0; j < kAppendVecs; ++j) {
    const int64_t at = first + j * kAppendThreads + tid;
    to[j] = nullptr;
    if (at < total) {
      const int t = (int)(at / per_token), r = (int)(at - (int64_t)t * per_token);
      const int64_t base = s_dst[t - t0];
      if (base >= 0) {
        const int piece = r & ((1 << a.vec_shift) - 1), row = r >> a.vec_shift;  // row: keys' heads, then values' heads
        const int head = row < a.n_kv_heads ? row : row - a.n_kv_heads;
        const char* src = row < a.n_kv_heads ? a.k + t * a.k_token + head * a.k_head : a.v + t * a.v_token + head * a.v_head;
        v[j] = *reinterpret_cast<const uint4*>(src + piece * 16);
        to[j] = a.cache + base + row * head_bytes + piece * 16;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kAppendVecs; ++j)
    if (to[j]) *reinterpret_cast<uint4*>(to[j]) = v[j];
}

__global__ void __launch_bounds__(256)
k_kv_reset(Pool p, int64_t scratch) {
  npp::pdl_wait_prior();
  npp::pdl_launch_dependents();
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t j = i; j < (int64_t)p.max_seqs * p.max_pages; j += step) p.table[j] = -1;
  for (int64_t j = i; j < p.max_seqs; j += step) p.lens[j] = 0;
  for (int64_t j = i; j < p.n_pages; j += step) p.refs[j] = 0;
  for (int64_t j = i; j < scratch; j += step) p.scratch[j] = 0;
  if (i == 0) *p.status = 0;
}

int64_t page_bytes(const np_kv_desc* d) { return (int64_t)2 * d->n_kv_heads * d->page_tokens * d->head_dim * 2; }

CopyArgs copy_args(const np_kv_desc* d, void* dst, const void* src, const int32_t* from, const int32_t* to, const int32_t* count, int n,
                   int32_t* status) {
  const int64_t pb = page_bytes(d);
  return CopyArgs{static_cast<char*>(dst), static_cast<const char*>(src), from, to, count, n, d->n_pages, d->n_layers, pb, pb * d->n_pages, status};
}

unsigned copy_blocks(const CopyArgs& a, const RewriteArgs& w, int sms) {
  const int64_t units = (int64_t)a.n_pairs * a.n_layers * ((a.page_bytes + kUnit - 1) / kUnit);
  const int64_t blocks = std::max<int64_t>(units, w.lens_out ? w.max_seqs : 1);
  return (unsigned)std::min<int64_t>(blocks, 8ll * sms);
}
cudaError_t launch_copy(const CopyArgs& a, const RewriteArgs& w, int sms, cudaStream_t s) {
  return launch_early(k_kv_copy, dim3(copy_blocks(a, w, sms)), kCopyThreads, 0, s, a, w);
}

// Checks what every call with tables takes.
int enter(const np_kv_desc* d, const np_kv_tables* t) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  return tables_ok(t) ? NP_OK : fail(NP_E_INVAL, "a table pointer is NULL");
}

int device(int* sms) { return device_sms(sms) ? NP_OK : fail(NP_E_CUDA, "no CUDA device"); }

int count_error(const np_kv_desc* d, int32_t n) { return n < 0 || n > d->max_seqs ? fail(NP_E_INVAL, "n outside [0, max_seqs]") : NP_OK; }

int done(cudaError_t e) { return e == cudaSuccess ? NP_OK : fail_cuda(e); }

}  // namespace
}  // namespace npa

using namespace npa;

extern "C" {

const char* np_attn_last_error(void) { return g_err; }

int np_attn_check(const int32_t* status, void* stream) {
  if (!status) return fail(NP_E_INVAL, "NULL argument");
  int32_t bits = 0;
  cudaError_t e = cudaMemcpyAsync(&bits, status, sizeof bits, cudaMemcpyDeviceToHost, static_cast<cudaStream_t>(stream));
  if (e == cudaSuccess) e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return fail_cuda(e);
  if (!bits) return NP_OK;
  snprintf(g_err, sizeof g_err, "status bits %d:%s%s%s%s%s", bits, bits & NP_KV_S_PAGE ? " page number outside the pool;" : "",
           bits & NP_KV_S_SEQ ? " sequence number outside the tables, listed twice or in use;" : "",
           bits & NP_KV_S_LENGTH ? " length outside its table row;" : "", bits & NP_KV_S_TIMEOUT ? " a bounded wait ran out;" : "",
           bits & NP_KV_S_FULL ? " not enough free pages;" : "");
  return NP_E_DEVICE;
}

int np_kv_sizes(const np_kv_desc* d, np_kv_sizes_out* out) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  if (!out) return fail(NP_E_INVAL, "NULL argument");
  out->page_bytes = page_bytes(d);
  out->cache_bytes = out->page_bytes * d->n_pages * d->n_layers;
  out->table_bytes = (uint64_t)d->max_seqs * d->max_pages * 4;
  out->scratch_bytes = scratch_ints(d) * 4;
  return NP_OK;
}

int np_kv_reset(const np_kv_desc* d, const np_kv_tables* t, void* stream) {
  if (int rc = enter(d, t)) return rc;
  int sms;
  if (int rc = device(&sms)) return rc;
  const int64_t most = std::max<int64_t>((int64_t)d->max_seqs * d->max_pages, (int64_t)scratch_ints(d));
  return done(launch_early(k_kv_reset, dim3((unsigned)std::min<int64_t>((most + 255) / 256, 8ll * sms)), 256, 0,
                           static_cast<cudaStream_t>(stream), pool_of(d, t), (int64_t)scratch_ints(d)));
}

int np_kv_reserve(const np_kv_desc* d, const np_kv_tables* t, const int32_t* seqs, const int32_t* n_new, int32_t n, int32_t* start_out,
                  void* stream) {
  if (int rc = enter(d, t)) return rc;
  if (int rc = count_error(d, n)) return rc;
  if (n == 0) return NP_OK;
  if (!n_new) return fail(NP_E_INVAL, "NULL argument");
  int sms;
  if (int rc = device(&sms)) return rc;
  return done(launch_early(k_kv_take<false>, dim3(1), kPlanThreads, 0, static_cast<cudaStream_t>(stream), pool_of(d, t), seqs, n_new, (int)n,
                           start_out));
}

int np_kv_append(const np_kv_desc* d, void* cache, int32_t layer, const np_kv_tables* t, const np_rows* k, const np_rows* v, int32_t n_tokens,
                 const int32_t* seqs, const int32_t* cu, const int32_t* start, int32_t n, void* stream) {
  if (int rc = enter(d, t)) return rc;
  if (int rc = count_error(d, n)) return rc;
  if (n_tokens < 0) return fail(NP_E_INVAL, "n_tokens must not be negative");
  if (!cu && n_tokens != n) return fail(NP_E_INVAL, "without cu there is one token for each sequence");
  if (n == 0 || n_tokens == 0) return NP_OK;
  if (!cache || !start) return fail(NP_E_INVAL, "NULL argument");
  if ((uintptr_t)cache % 16) return fail(NP_E_INVAL, "cache must be 16-byte aligned");
  if (layer < 0 || layer >= d->n_layers) return fail(NP_E_INVAL, "layer outside the cache");
  if (const char* m = rows_error(k)) return fail(NP_E_INVAL, m);
  if (const char* m = rows_error(v)) return fail(NP_E_INVAL, m);
  AppendArgs a = {};
  a.cache = static_cast<char*>(cache) + (int64_t)layer * d->n_pages * page_bytes(d);
  a.k = static_cast<const char*>(k->data);
  a.v = static_cast<const char*>(v->data);
  a.k_token = 2 * k->token_stride;
  a.k_head = 2 * k->head_stride;
  a.v_token = 2 * v->token_stride;
  a.v_head = 2 * v->head_stride;
  a.seqs = seqs;
  a.cu = cu;
  a.start = start;
  a.n = n;
  a.n_tokens = n_tokens;
  a.n_kv_heads = d->n_kv_heads;
  a.vec_shift = d->head_dim == 64 ? 3 : 4;
  const int64_t vecs = (int64_t)n_tokens * 2 * d->n_kv_heads << a.vec_shift, blocks = (vecs + kAppendPerBlock - 1) / kAppendPerBlock;
  if (blocks > 0x7fffffffLL) return fail(NP_E_INVAL, "too many rows for one call");
  int sms;
  if (int rc = device(&sms)) return rc;
  return done(launch_early(k_kv_append, dim3((unsigned)blocks), kAppendThreads, 0, static_cast<cudaStream_t>(stream), pool_of(d, t), a));
}

int np_kv_fork(const np_kv_desc* d, void* cache, const np_kv_tables* t, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  if (int rc = enter(d, t)) return rc;
  if (int rc = count_error(d, n)) return rc;
  if (n == 0) return NP_OK;
  if (!cache || !src || !dst) return fail(NP_E_INVAL, "NULL argument");
  if ((uintptr_t)cache % 16) return fail(NP_E_INVAL, "cache must be 16-byte aligned");
  int sms;
  if (int rc = device(&sms)) return rc;
  const Pool p = pool_of(d, t);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = launch_early(k_kv_take<true>, dim3(1), kPlanThreads, 0, s, p, src, dst, (int)n, (int32_t*)nullptr);
  if (e == cudaSuccess) e = launch_copy(copy_args(d, cache, cache, p.pair_src(), p.pair_dst(), nullptr, n, nullptr), RewriteArgs{}, sms, s);
  return done(e);
}

int np_kv_free(const np_kv_desc* d, const np_kv_tables* t, const int32_t* seqs, int32_t n, void* stream) {
  if (int rc = enter(d, t)) return rc;
  if (int rc = count_error(d, n)) return rc;
  if (n == 0) return NP_OK;
  int sms;
  if (int rc = device(&sms)) return rc;
  return done(launch_early(k_kv_free, dim3(n), 256, 0, static_cast<cudaStream_t>(stream), pool_of(d, t), seqs, (int)n));
}

int np_kv_compact(const np_kv_desc* d, void* cache, const np_kv_tables* in, const np_kv_tables* out, int32_t* n_live, void* stream) {
  if (int rc = enter(d, in)) return rc;
  if (!cache || !out || !out->page_table || !out->lens || !out->refs) return fail(NP_E_INVAL, "NULL argument");
  if ((uintptr_t)cache % 16) return fail(NP_E_INVAL, "cache must be 16-byte aligned");
  const int same = (out->page_table == in->page_table) + (out->lens == in->lens) + (out->refs == in->refs);
  if (same != 0 && same != 3) return fail(NP_E_INVAL, "the new tables are the old ones or three others");
  int sms;
  if (int rc = device(&sms)) return rc;
  const Pool p = pool_of(d, in);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (!same && d->n_pages <= kSmallPool) {
    const CopyArgs a = copy_args(d, cache, cache, nullptr, nullptr, nullptr, std::max(1, d->n_pages / 2), in->status);
    const RewriteArgs w{p.table, p.lens, nullptr, out->page_table, out->lens, p.shift, p.n_pages, p.max_seqs, p.max_pages};
    return done(launch_early(k_kv_compact_small, dim3(copy_blocks(a, w, sms)), kCopyThreads, 0, s, p, out->refs, n_live, a, w));
  }
  cudaError_t e = launch_early(k_kv_compact_plan, dim3(1), kPlanThreads, 0, s, p, out->refs, n_live);
  const RewriteArgs w{p.table, p.lens, p.pages(), out->page_table, out->lens, p.shift, p.n_pages, p.max_seqs, p.max_pages};
  if (e == cudaSuccess)
    e = launch_copy(copy_args(d, cache, cache, p.pair_src(), p.pair_dst(), p.pair_count(), std::max(1, d->n_pages / 2), in->status), w, sms, s);
  return done(e);
}

int np_kv_copy_pages(const np_kv_desc* d, void* dst_cache, const void* src_cache, const int32_t* src, const int32_t* dst, int32_t n,
                     int32_t* status, void* stream) {
  if (const char* m = desc_error(d)) return fail(NP_E_INVAL, m);
  if (n < 0 || n > d->n_pages) return fail(NP_E_INVAL, "n outside [0, n_pages]");
  if (n == 0) return NP_OK;
  if (!dst_cache || !src_cache || !src || !dst || !status) return fail(NP_E_INVAL, "NULL argument");
  if ((uintptr_t)dst_cache % 16 || (uintptr_t)src_cache % 16) return fail(NP_E_INVAL, "caches must be 16-byte aligned");
  int sms;
  if (int rc = device(&sms)) return rc;
  return done(launch_copy(copy_args(d, dst_cache, src_cache, src, dst, nullptr, n, status), RewriteArgs{}, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
