// fastav_cache_evict: the lightest tokens of a cached sequence go, the others move together.
//
// A thread-block cluster per sequence and KV head does both steps in one launch; one set for all heads is selected by a cluster per sequence first, since rows that
// move in place take their weights with them.  Selection: the k-th largest weight by its 32-bit key, 8 bits at a time, each block
// counting a slice of the tokens into a histogram of its own that all blocks of the cluster then add up; ranks by one sum over threads and blocks; the
// survivors' list goes to the workspace.  Moving: rounds of kMoved rows a block, in the survivors' order.  Bound by the rows that move (codes and scales of K and V, weights:
// 2 (d + 4) + 4 bytes each way), for one sequence by the selection's chain.
//
// In place.  Survivor i comes from a place >= i, and sources ascend.  So a round's rows may be written as soon as all of that round have been read: what later
// rounds read lies behind their own targets.
#include <limits.h>

#include "cache.cuh"
#include "cluster.cuh"

namespace fastav {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kHeld = 8192;  // keys that a block holds in shared memory; those of a longer slice are looked up again

struct EvictCall {
  CacheView cache;
  float* weights;
  int batch, max_len, max_keep, table_stride, out_stride, first, recent, blocks;
  const int32_t *table, *lens, *counts, *out_table;
  int32_t *lens_out, *keep_idx, *list;
  int32_t* device_status;
  int head_wait;
};
inline void mark_head(EvictCall& c, bool head) { c.head_wait = head ? 1 : 0; }

// Larger keys rank higher: NaN, then numbers in their order (-0 as 0), then tokens that always stay.
constexpr unsigned kStays = 0xFFFFFFFFu;
__device__ __forceinline__ unsigned key_of(float w) {
  if (w != w) return 0;
  const unsigned bits = __float_as_uint(w + 0.f);
  return bits ^ (bits >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

template <int DIM, bool SELECT, bool MOVE>
__global__ void __launch_bounds__(kThreads)
evict_kernel(EvictCall c) {
  constexpr int kPieces = DIM / 16, kAtOnce = kThreads / kPieces, kUnroll = 2;  // 16-byte pieces of a row; rows that the threads take at once
  constexpr int kMoved = kAtOnce * kUnroll;                                     // rows of a round
  constexpr int kSmall = (3 * kMoved + kThreads - 1) / kThreads;                // scales and weights of a round, per thread
  extern __shared__ unsigned held[];  // [kHeld]
  __shared__ unsigned hist[2][256];
  __shared__ unsigned warp_a[kWarps], warp_b[kWarps], found[4];
  __shared__ unsigned counts[2];  // of this block: keys above the threshold, keys equal to it
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
  constexpr bool kJoint = SELECT && !MOVE;  // one set for all heads: a cluster per sequence here
  const int blocks = c.blocks, rank = blocks > 1 ? (int)cluster_rank() : 0, job = blockIdx.x / blocks, b = kJoint ? job : job / c.cache.hkv;
  const int head = kJoint ? 0 : job - b * c.cache.hkv;
  auto sync_all = [&] { if (blocks > 1) cluster_sync(); else __syncthreads(); };
  if (c.head_wait) pdl_wait();
  pdl_trigger();
  pdl_wait();

  const int given_len = chain_load_cached(c.lens + b), given_keep = chain_load_cached(c.counts + b);
  const int n = min(max(given_len, 0), c.max_len), wanted = min(max(given_keep, 0), n), k = min(wanted, c.max_keep);
  const bool all = k == n;
  if (SELECT && rank == 0 && head == 0 && tid == 0) {
    c.lens_out[b] = k;
    const int stay = min(n, c.first) + min(max(n - c.first, 0), c.recent);
    const int bits = (n != given_len || k != wanted ? FASTAV_DEV_SHAPE_MISMATCH : 0) | (wanted != given_keep ? FASTAV_DEV_K_CLAMPED : 0) |
                     (stay > k ? FASTAV_DEV_PROTECT_OVERFLOW : 0);
    if (bits && c.device_status) atomicOr(c.device_status, bits);
  }
  int32_t* const list = c.list + (long long)(MOVE && !SELECT ? b : job) * c.max_keep;  // rows of the pool, of head 0; -1: in no page
  if constexpr (SELECT) {
  const int slice = (n + blocks - 1) / blocks, t0 = min(n, rank * slice), t1 = min(n, t0 + slice);

  auto look_up = [&](int t) {
    const int page = page_of(c.cache, c.table, c.table_stride, b, t);
    unsigned key = 0;
    if (page >= 0) {
      float w;
      if (kJoint) {
        double sum = 0.;
        for (int h = 0; h < c.cache.hkv; ++h) sum += (double)chain_load(c.weights + pool_row(c.cache, page, h, t));
        w = (float)sum;
      } else {
        w = chain_load(c.weights + pool_row(c.cache, page, head, t));
      }
      key = key_of(w);
    } else if (c.device_status) {
      atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
    }
    return t < c.first || t >= n - c.recent ? kStays : key;
  };
  auto key_at = [&](int t) { return t - t0 < kHeld ? held[t - t0] : look_up(t); };

  // ---- the threshold: the k-th largest key, and how many of those equal to it stay (the first ones) ----
  unsigned threshold = 0, equal_stay = 0;
  for (int t = t0 + tid; t < min(t1, t0 + kHeld); t += kThreads) held[t - t0] = look_up(t);
  if (tid < 256) hist[0][tid] = 0;
  __syncthreads();
  if (!all && k > 0) {
    unsigned remaining = k, prefix = 0;
    for (int pass = 0; pass < 4; ++pass) {
      const int shift = 24 - 8 * pass;
      unsigned* const mine = hist[pass & 1];
      for (int t = t0 + tid; t < t1; t += kThreads) {
        const unsigned key = key_at(t);
        if (pass == 0 || key >> (shift + 8) == prefix) atomicAdd(&mine[key >> shift & 255u], 1u);
      }
      sync_all();
      if (tid < 256) hist[pass & 1 ^ 1][tid] = 0;  // (everybody has read it: ahead of the barrier)
      unsigned total = 0;
      const int digit = 255 - tid;  // thread 0 has the highest
      if (tid < 256) {
        if (blocks == 1) total = mine[digit];
        else
          for (int r = 0; r < blocks; ++r) {
            unsigned v;
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote(&mine[digit], r)) : "memory");
            total += v;
          }
      }
      const unsigned above = sum_before<kWarps>(total, pass & 1 ? warp_b : warp_a, lane, warp);
      if (tid < 256 && above < remaining && remaining <= above + total) {
        found[0] = digit;
        found[1] = remaining - above;
        found[2] = total;
      }
      __syncthreads();
      prefix = prefix << 8 | found[0];
      remaining = found[1];
      if (remaining == found[2]) {  // all of them stay: no need to tell them apart
        threshold = shift == 0 ? prefix : prefix << shift;
        equal_stay = 0xFFFFFFFFu;
        break;
      }
      threshold = prefix;
      equal_stay = remaining;
      __syncthreads();  // `found` is written again
    }
  } else if (all) {
    equal_stay = 0xFFFFFFFFu;
  } else {
    threshold = kStays;  // nobody stays
    equal_stay = 0;
  }
  const bool from_threshold = equal_stay == 0xFFFFFFFFu;  // every key from the threshold on stays

  // ---- the survivors' list ----
  const int each = (t1 - t0 + kThreads - 1) / kThreads, mine0 = min(t1, t0 + tid * each), mine1 = min(t1, mine0 + each);
  unsigned above = 0, equal = 0;
  for (int t = mine0; t < mine1; ++t) {
    const unsigned key = key_at(t);
    above += from_threshold ? key >= threshold : key > threshold;
    equal += !from_threshold && key == threshold;
  }
  __syncthreads();
  const unsigned above_before = sum_before<kWarps>(above, warp_a, lane, warp), equal_before = sum_before<kWarps>(equal, warp_b, lane, warp);
  if (tid == kThreads - 1) {
    counts[0] = above_before + above;
    counts[1] = equal_before + equal;
  }
  sync_all();
  unsigned above_ahead = 0, equal_ahead = 0;
  for (int r = 0; r < rank; ++r) {
    unsigned x, y;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(remote(&counts[0], r)) : "memory");
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(y) : "r"(remote(&counts[1], r)) : "memory");
    above_ahead += x;
    equal_ahead += y;
  }
  {
    int32_t* const idx = c.keep_idx ? c.keep_idx + (long long)job * (kJoint ? c.cache.hkv : 1) * c.max_keep : nullptr;
    unsigned a = above_ahead + above_before, e = equal_ahead + equal_before;
    for (int t = mine0; t < mine1; ++t) {
      const unsigned key = key_at(t);
      const bool over = from_threshold ? key >= threshold : key > threshold, same = !from_threshold && key == threshold;
      if (over || (same && e < equal_stay)) {
        const unsigned at = a + min(e, from_threshold ? 0u : equal_stay);
        if (at < (unsigned)k) {
          const int page = page_of(c.cache, c.table, c.table_stride, b, t);
          list[at] = page < 0 ? -1 : (int)pool_row(c.cache, page, 0, t);
          if (idx)
            for (int h = 0; h < (kJoint ? c.cache.hkv : 1); ++h) idx[(long long)h * c.max_keep + at] = t;
        }
      }
      a += over;
      e += same;
    }
  }
  sync_all();  // the list is there for all blocks; nobody's shared memory is read by another any more
  }
  if constexpr (!MOVE) return;

  // ---- the rows ----
  const int32_t* const to_table = c.out_table ? c.out_table : c.table;
  const int to_stride = c.out_table ? c.out_stride : c.table_stride, of_head = head << c.cache.page_shift;
  // Survivor i comes from `from` and goes to `to`; false: it stays where it is, or is left out.
  auto moves = [&](int i, int& from, int& to) {
    if (i >= k) return false;
    from = chain_load(list + i);
    const int page = page_of(c.cache, to_table, to_stride, b, i);
    if (page < 0 && c.device_status) atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
    if (from < 0 || page < 0) return false;
    from += of_head;
    to = (int)pool_row(c.cache, page, head, i);
    return from != to;
  };
  const int piece = tid % kPieces, row_of = tid / kPieces;
  for (int r0 = 0; r0 < k; r0 += blocks * kMoved) {
    const int i0 = r0 + rank * kMoved;
    uint4 x[kUnroll], y[kUnroll];
    int to[kUnroll], small_to[kSmall];
    float value[kSmall];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      int from;
      if (!moves(i0 + u * kAtOnce + row_of, from, to[u])) { to[u] = -1; continue; }
      x[u] = chain_load(reinterpret_cast<const uint4*>(c.cache.k + (long long)from * DIM) + piece);
      y[u] = chain_load(reinterpret_cast<const uint4*>(c.cache.v + (long long)from * DIM) + piece);
    }
    auto small_pool = [&](int j) { const int which = (j * kThreads + tid) / kMoved; return which == 0 ? c.cache.k_scale : which == 1 ? c.cache.v_scale : c.weights; };
#pragma unroll
    for (int j = 0; j < kSmall; ++j) {
      const int item = j * kThreads + tid;
      int from;
      if (item >= 3 * kMoved || !moves(i0 + item % kMoved, from, small_to[j])) { small_to[j] = -1; continue; }
      value[j] = chain_load(small_pool(j) + from);
    }
    if (!c.out_table) sync_all();
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (to[u] >= 0) {
        reinterpret_cast<uint4*>(c.cache.k + (long long)to[u] * DIM)[piece] = x[u];
        reinterpret_cast<uint4*>(c.cache.v + (long long)to[u] * DIM)[piece] = y[u];
      }
#pragma unroll
    for (int j = 0; j < kSmall; ++j)
      if (small_to[j] >= 0) small_pool(j)[small_to[j]] = value[j];
  }
}

int32_t check_evict(const fastav_evict_params* p, const fastav_cache* cache) {
  const int32_t rc = check_cache(cache);
  if (rc != FASTAV_OK) return rc;
  if (!p || p->batch < 1 || p->max_kv_len < 0 || p->max_keep < 0 || p->first < 0 || p->recent < 0) return FASTAV_ERR_INVALID_ARG;
  if ((long long)p->batch * cache->num_kv_heads > INT_MAX / kMaxCluster || (long long)p->max_kv_len + p->first > INT_MAX) return FASTAV_ERR_UNSUPPORTED;
  return FASTAV_OK;
}

}  // namespace
}  // namespace fastav

using namespace fastav;

extern "C" int32_t fastav_evict_workspace_bytes(const fastav_evict_params* p, const fastav_cache* cache, size_t* out_bytes) {
  const int32_t rc = check_evict(p, cache);
  if (rc != FASTAV_OK) return rc;
  if (!out_bytes) return FASTAV_ERR_INVALID_ARG;
  *out_bytes = align_up((size_t)p->batch * cache->num_kv_heads * (size_t)(p->max_keep > 0 ? p->max_keep : 1) * sizeof(int32_t), 256);
  return FASTAV_OK;
}

extern "C" int32_t fastav_cache_evict(const fastav_evict_params* p, const fastav_cache* cache, float* weights, const int32_t* page_table, const int32_t* kv_lens,
                                      const int32_t* keep_counts, const int32_t* out_table_opt, int32_t* kv_lens_out, int32_t* keep_idx_out_opt, void* workspace,
                                      size_t workspace_bytes, int32_t* device_status, void* stream) {
  size_t need = 0;
  const int32_t rc = fastav_evict_workspace_bytes(p, cache, &need);
  if (rc != FASTAV_OK) return rc;
  if (!weights || !kv_lens || !keep_counts || !kv_lens_out) return FASTAV_ERR_INVALID_ARG;
  if (kv_lens_out < kv_lens + p->batch && kv_lens < kv_lens_out + p->batch) return FASTAV_ERR_INVALID_ARG;
  const long long page = cache->page_tokens;
  if (p->max_kv_len > 0 && (!page_table || p->table_stride < 1 || p->max_kv_len > p->table_stride * page)) return FASTAV_ERR_INVALID_ARG;
  if (out_table_opt && p->max_keep > 0 && (out_table_opt == page_table || p->out_table_stride < 1 || p->max_keep > p->out_table_stride * page)) return FASTAV_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(weights) & 15u) return FASTAV_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < need) return FASTAV_ERR_WORKSPACE;
  chain_begin(p->flags);
  EvictCall c{};
  c.cache = make_view(*cache);
  c.weights = weights;
  c.batch = p->batch; c.max_len = p->max_kv_len; c.max_keep = p->max_keep; c.table_stride = p->table_stride; c.out_stride = p->out_table_stride;
  c.first = p->first; c.recent = p->recent;
  c.table = page_table; c.lens = kv_lens; c.counts = keep_counts; c.out_table = out_table_opt;
  c.lens_out = kv_lens_out; c.keep_idx = keep_idx_out_opt; c.list = static_cast<int32_t*>(workspace);
  c.device_status = device_status;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto go = [&](auto kernel, int jobs, size_t smem) {
    c.blocks = cluster_blocks(jobs, p->max_kv_len, 256, kPortableCluster);
    count_launches(1);
    return launch_chained_cluster(kernel, dim3((unsigned)(jobs * c.blocks)), dim3(kThreads), c.blocks > 1 ? c.blocks : 0, smem, st, c);
  };
  constexpr size_t kKeys = kHeld * sizeof(unsigned);
  const int heads = p->batch * cache->num_kv_heads;
  cudaError_t e;
  if (p->flags & FASTAV_EVICT_JOINT) {
    e = go(evict_kernel<64, true, false>, p->batch, kKeys);
    if (e == cudaSuccess) e = c.cache.dim == 128 ? go(evict_kernel<128, false, true>, heads, 0) : go(evict_kernel<64, false, true>, heads, 0);
  } else {
    e = c.cache.dim == 128 ? go(evict_kernel<128, true, true>, heads, kKeys) : go(evict_kernel<64, true, true>, heads, kKeys);
  }
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}
