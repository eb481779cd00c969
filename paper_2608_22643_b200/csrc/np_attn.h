// Shared by the translation units of the paged cache and its attention (np_kv.cu, np_kv_rows.cu, np_attn_decode.cu, np_attn_prompt.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <cfloat>
#include <cmath>

#include "np.h"

namespace npa {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// scale * log2(e): scores are kept in base two.  Below the normal numbers, which the kernels flush to 0 (and 0 * -inf is no number), the
// least of them: either way products of finite scores this small are 0 to an exponential.  False: no scale.
inline bool scale_base2(float scale, float* out) {
  *out = scale * kLog2e;
  if (!(scale > 0.f) || !std::isfinite(*out)) return false;
  if (*out < FLT_MIN) *out = FLT_MIN;
  return true;
}
constexpr const char* kScaleError = "scale must be positive, and times log2(e) finite";

// Keeps the text for np_attn_last_error and returns the code.
int fail(int code, const char* msg);
int fail_cuda(cudaError_t e);

// Text of what is wrong with a description; NULL: nothing.
const char* desc_error(const np_kv_desc* d);
inline bool held_in_8(const np_kv_desc* d) { return (d->dtype & NP_KV_E4M3) != 0; }
inline int row_type(const np_kv_desc* d) { return d->dtype & ~NP_KV_E4M3; }
// Bytes of one page of one layer.
inline int64_t page_bytes(const np_kv_desc* d) {
  return (int64_t)2 * d->n_kv_heads * d->page_tokens * (held_in_8(d) ? d->head_dim + 1 : d->head_dim * 2);
}
const char* rows_error(const np_rows* r);
bool tables_ok(const np_kv_tables* t);  // no pointer NULL

inline int log2_of(int pow2) {
  int s = 0;
  while ((1 << s) < pow2) ++s;
  return s;
}

// The driver's cuTensorMapEncodeTiled; NULL without a driver.
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess
               ? reinterpret_cast<EncodeFn>(p)
               : nullptr;
  }();
  return fn;
}

// SM count of the current device; false: no device.
bool device_sms(int* sms);

// np_kv_append into a cache of 8 bits, behind the checks (np_kv_rows.cu).
int append_held(const np_kv_desc* d, void* cache, int32_t layer, const np_kv_tables* t, const np_rows* k, const np_rows* v, int32_t n_tokens,
                const int32_t* seqs, const int32_t* cu, const int32_t* start, int32_t n, void* stream);

// np_attn_decode behind its checks, and these (np_attn_decode.cu); shared: rows begin behind what their groups share.
struct SharedArgs;
int decode(const np_kv_desc* d, const void* cache, int32_t layer, const np_kv_tables* t, const np_rows* q, int32_t n_heads, const int32_t* seqs,
           int32_t n, float scale2, const np_rows* out, float* lse, void* workspace, const SharedArgs* shared, int sms, cudaStream_t s);
// The rows' own tokens behind shared ones, and the join (np_attn_rest.cu).  cache: of the layer.
int decode_rest(const np_kv_desc* d, const char* cache, const np_kv_tables* t, const np_rows* q, int32_t n_heads, const int32_t* seqs, int32_t n, float scale2,
                const np_rows* out, float* lse, const SharedArgs& shared, int sms, cudaStream_t s);
uint64_t decode_parts_bytes();  // of the workspace's first part, the same for all calls
const char* decode_heads_error(const np_kv_desc* d, int n_heads, int n);
const char* decode_error(const np_kv_desc* d, const void* cache, int32_t layer, const np_kv_tables* t, const np_rows* q, int32_t n_heads, int32_t n,
                         float scale, const np_rows* out, const void* workspace, float* scale2);

// A launch whose blocks may be scheduled while the kernel before it in the stream ends; the kernel begins with
// npp::pdl_wait_prior().
template <class K, class... Args>
cudaError_t launch_early(K kernel, dim3 grid, int threads, size_t smem, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace npa
