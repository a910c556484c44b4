// The 8-bit K/V cache as the kernels see it.
#pragma once

#include "common.cuh"

namespace fastav {

struct CacheView {
  uint8_t *k, *v;             // [num_pages, hkv, page tokens, dim] codes
  float *k_scale, *v_scale;   // [num_pages, hkv, page tokens]
  int num_pages, page_shift;  // page tokens: 1 << page_shift
  int hkv, dim;
  bool fp8;
};

// Everything fastav_cache has to satisfy by itself.
int32_t check_cache(const fastav_cache* c);
CacheView make_view(const fastav_cache& c);

#ifdef __CUDACC__
// A page table's entry for token `token` >= 0 of row `row`; -1 if it names no page of the pool.  `token` lies inside the table.
__device__ __forceinline__ int page_of(const CacheView& c, const int32_t* table, int stride, int row, int token) {
  const int page = chain_load_cached(table + (long long)row * stride + (token >> c.page_shift));
  return (unsigned)page < (unsigned)c.num_pages ? page : -1;
}
// Row of the pool (in units of dim codes, or of one scale) at which token `token` of KV head `head` lies.
__device__ __forceinline__ long long pool_row(const CacheView& c, int page, int head, int token) {
  return ((long long)page * c.hkv + head << c.page_shift) + (token & ((1 << c.page_shift) - 1));
}
#endif

}  // namespace fastav
