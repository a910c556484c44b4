// fastav_cache_weigh as its kernels see it.
#pragma once

#include "cache.cuh"
#include "sm100_ptx.cuh"

namespace fastav {

struct WeighCall {
  CacheView cache;
  float* weights;  // [num_pages, hkv, page tokens]
  float decay;
  int batch, total_q, max_qlen, hq, group, max_len, table_stride;
  long long q_st, q_sh;
  float scale_log2;
  bool causal;
  const uint16_t* q;
  const float* lse;
  const int32_t *cu_qlens, *table, *lens, *weighed;
  int32_t* device_status;
  int head_wait;
};
inline void mark_head(WeighCall& c, bool head) { c.head_wait = head ? 1 : 0; }

// The kernel for many stacked rows.  `*used` is false when the queries could not be described to the tensor-memory-accelerator; nothing was launched then.
bool weigh_many_applies(const WeighCall& c);
cudaError_t launch_weigh_many(const WeighCall& c, cudaStream_t stream, bool* used);

#ifdef __CUDACC__
// A sequence's query rows and tokens, cut down to what the host promised.
struct WeighSpan {
  int row0, rows, len;
  bool bad;
};
__device__ __forceinline__ WeighSpan weigh_span(const WeighCall& c, int b) {
  const Span rows = checked_span<true>(c.cu_qlens, b, c.total_q, c.max_qlen);
  const int len = chain_load_cached(c.lens + b);
  WeighSpan s{rows.first, rows.count, min(max(len, 0), c.max_len), rows.bad};
  s.bad |= s.len != len;
  return s;
}
#endif

}  // namespace fastav
