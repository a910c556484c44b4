// fastav_cache_evict: the lightest tokens of a cached sequence go, the others move together.
//
// Selection: a thread-block cluster per sequence and KV head (or per sequence, for one set of all heads), a slice of the tokens per block, eight in a row per thread (which lie in one
// page: one look-up, two loads), their keys in registers.  The
// k-th largest weight by its 32-bit key, 8 bits at a time: each block counts its keys into a histogram and sends it to all blocks of the cluster, where one warp adds
// them up and finds the digit.  Ranks by one sum over threads and blocks; the survivors' list goes to the workspace.  (Sums over all 1,024 threads of a block for
// each digit, histograms fetched from the others: 2 us a digit instead of 0.7; tokens kThreads apart per thread, ranks from ballots: 2.3 us for the list.)
//
// Moving: the same clusters go on with it in place and where there is little to move (one launch), in rounds of kMoved rows a block in the survivors' order; else a
// kernel with a block per kChunk rows, that many in flight.  Bound by the rows that move (codes and scales of K and V, weights: 2 (d + 4) + 4 bytes each
// way), for one sequence by the selection's chain.  32 sequences of 512 to 4,096 tokens, half of them kept, to other pages: 21.4 us a call, 7 of them selection (69 MB: 10.8 us
// at a copy's rate); 32 x 4,096 tokens of 4 heads to 2,048: 33 us a call to other pages, 39 alone in place; 819 of 1,024 tokens 8.7 us (8.5 when a thread's tokens lay kThreads
// apart, and the 32 sequences 22.0: eight in a row keep fewer threads of a short slice busy).
//
// In place.  Survivor i comes from a place >= i, and sources ascend.  So a round's rows may be written as soon as all of that round have been read: what later
// rounds read lies behind their own targets.  (The rows of the round after are asked for ahead of that.)  One set for all heads is selected by a launch of its own, since rows
// that move take the weights with them.
#include <limits.h>

#include "cache.cuh"
#include "cluster.cuh"

namespace fastav {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kChunk = 128, kChunkThreads = 256;  // rows of a block that only moves
constexpr int kEach = 8, kHeld = kEach * kThreads;  // keys that a thread, a block holds; those of a longer slice are looked up again
// Tokens of a block's slice, at least.  More blocks move rows sooner where the selecting clusters go on with it, and cost a cluster barrier a digit.  us with 512 / 1,024 /
// 2,048 / 4,096.  In place (and a copy of the weights): one sequence of 4,096 tokens to 2,048 15.5 / 17.4 / 22.6 / 22.6, eight of 4,000 less one 22.5 / 22.5 / 30.9 / 34.9, one of 16,384
// to 16,000 34.4 / 34.4 / 34.4 / 53.5.  To other pages: 1,500 to 1,200 11.9 / 11.5 / 9.5 / 9.1, eight of 4,000 to 2,000 15.5 / 15.5 / 15.0 / 12.6, 16,384 to 6,553 16.6 / 16.6 / 16.6 / 15.6;
// four of 16,384 jointly 30.9 / 31.0 / 30.9 / 31.4.
constexpr int kLeastSlice = 1024;
// A block's survivors up to which the selecting clusters move them, one or two rounds of theirs; beyond, another launch with more blocks is quicker (4 heads, by the selecting
// clusters / by another launch: 240 of 300 tokens 7.2 / 7.8 us, 819 of 1,024 11.2 / 8.7, 1,638 of 2,048 17.8 / 11.0; but 750 of 32 x 1,500 12.5 / 13.6).
constexpr int kFewRows = 256;

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

template <int DIM, bool SELECT, bool MOVE, bool JOINT>
__global__ void __launch_bounds__(kThreads, 1)
evict_kernel(EvictCall c) {
  constexpr int kPieces = DIM / 16, kAtOnce = kThreads / kPieces, kUnroll = 4;  // 16-byte pieces of a row; rows that the threads take at once
  constexpr int kMoved = kAtOnce * kUnroll;                                     // rows of a round
  static_assert(kMoved <= kThreads);
  __shared__ int pages[kHeld / 16 + 1];                              // of the first kHeld tokens of the slice; -1: none
  __shared__ int2 places[2][MOVE ? kMoved : 1];
  __shared__ unsigned hist[2][256];
  __shared__ __align__(16) unsigned inbox[2][kPortableCluster][256];  // the histograms of all blocks
  __shared__ unsigned warp_a[kWarps], totals[2], found[2][3];  // totals: of the blocks before this one, keys above the threshold and equal to it
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tid = threadIdx.x;
  constexpr bool kPerSequence = JOINT && SELECT;  // one set for all heads
  static_assert(!(JOINT && SELECT && MOVE));
  const int blocks = c.blocks, rank = blocks > 1 ? (int)cluster_rank() : 0, job = blockIdx.x / blocks, b = kPerSequence ? job : job / c.cache.hkv;
  const int head = kPerSequence ? 0 : job - b * c.cache.hkv;
  auto sync_all = [&] { if (blocks > 1) cluster_sync(); else __syncthreads(); };
  if constexpr (SELECT) {
    if (tid < 2) totals[tid] = 0;
    if (blocks > 1) cluster_arrive();  // "this block runs": waited for before the first remote access
  }
  if (c.head_wait) pdl_wait();
  pdl_trigger();
  pdl_wait();

  if constexpr (SELECT) {
    if (tid < 256) hist[0][tid] = hist[1][tid] = 0;
    if (blocks == 1)  // (the slice is known; entries behind the sequence's end are looked at and not used)
      for (int p = tid; p << c.cache.page_shift < min(c.max_len, kHeld); p += kThreads) pages[p] = page_of(c.cache, c.table, c.table_stride, b, p << c.cache.page_shift);
  }
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
  int32_t* const list = c.list + (long long)(JOINT ? b : job) * c.max_keep;  // rows of the pool, of head 0; -1: in no page
  if constexpr (SELECT) {
  const int slice = ((n + blocks - 1) / blocks + kEach - 1) / kEach * kEach, t0 = min(n, rank * slice), t1 = min(n, t0 + slice);
  const int shift = c.cache.page_shift, first_page = t0 >> shift;
  if (blocks > 1)
    for (int p = first_page + tid; p <= (min(t1, t0 + kHeld) - 1) >> shift; p += kThreads) pages[p - first_page] = page_of(c.cache, c.table, c.table_stride, b, p << shift);
  __syncthreads();
  // The page of a token that is a multiple of kEach and inside the slice.
  auto page_at = [&](int t) { return t - t0 < kHeld ? pages[(t >> shift) - first_page] : page_of(c.cache, c.table, c.table_stride, b, t); };

  // ---- keys of the thread's tokens g0 + kEach tid ..; behind the slice's end 0, and not counted anywhere ----
  auto look_up = [&](int g0, unsigned (&keys)[kEach]) {
    const int t = g0 + tid * kEach;
    float w[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) w[j] = __uint_as_float(0x7FC00000u);
    if (t < t1) {
      const int page = page_at(t);
      if (page >= 0) {
        const float* const from = c.weights + pool_row(c.cache, page, kPerSequence ? 0 : head, t);
        if (!kPerSequence) {
          const float4 lo = chain_load(reinterpret_cast<const float4*>(from)), hi = chain_load(reinterpret_cast<const float4*>(from) + 1);
          w[0] = lo.x; w[1] = lo.y; w[2] = lo.z; w[3] = lo.w; w[4] = hi.x; w[5] = hi.y; w[6] = hi.z; w[7] = hi.w;
        } else {
          double sum[kEach] = {};
          constexpr int kHeads = 8;  // at once
          for (int h0 = 0; h0 < c.cache.hkv; h0 += kHeads) {
            float4 lo[kHeads], hi[kHeads];
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
              const float4* const of_head = reinterpret_cast<const float4*>(from + ((long long)min(h0 + h, c.cache.hkv - 1) << shift));
              lo[h] = chain_load(of_head);
              hi[h] = chain_load(of_head + 1);
            }
#pragma unroll
            for (int h = 0; h < kHeads; ++h) {
              if (h0 + h < c.cache.hkv) {
                sum[0] += lo[h].x; sum[1] += lo[h].y; sum[2] += lo[h].z; sum[3] += lo[h].w;
                sum[4] += hi[h].x; sum[5] += hi[h].y; sum[6] += hi[h].z; sum[7] += hi[h].w;
              }
            }
          }
#pragma unroll
          for (int j = 0; j < kEach; ++j) w[j] = (float)sum[j];
        }
      } else if (c.device_status) {
        atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
      }
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) keys[j] = t + j >= t1 ? 0u : t + j < c.first || t + j >= n - c.recent ? kStays : key_of(w[j]);
  };
  unsigned keys[kEach];
  look_up(t0, keys);
  // f(key) for every key of the thread
  auto for_keys = [&](auto f) {
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (t0 + tid * kEach + j < t1) f(keys[j]);
    for (int g0 = t0 + kHeld; g0 < t1; g0 += kHeld) {
      unsigned more[kEach];
      look_up(g0, more);
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        if (g0 + tid * kEach + j < t1) f(more[j]);
    }
  };
  if (blocks > 1) cluster_wait();

  // ---- the threshold: the k-th largest key, and how many of those equal to it stay (the first ones) ----
  unsigned threshold = all ? 0 : kStays, equal_stay = 0;
  bool from_threshold = all;  // every key from the threshold on stays
  if (!all && k > 0) {
    unsigned remaining = k, prefix = 0;
    for (int pass = 0; pass < 4; ++pass) {
      const int low = 24 - 8 * pass, buffer = pass & 1;
      for_keys([&](unsigned key) {
        if (pass == 0 || key >> (low + 8) == prefix) atomicAdd(&hist[buffer][key >> low & 255u], 1u);
      });
      __syncthreads();
      if (tid < 256) {
        const unsigned mine = hist[buffer][tid];
        hist[buffer][tid] = 0;  // for the pass after the next
        if (blocks == 1) inbox[buffer][0][tid] = mine;
        else
          for (int r = 0; r < blocks; ++r) remote_store(remote(&inbox[buffer][rank][tid], r), mine);
      }
      sync_all();
      if (warp == 0) {  // lane l has the digits 255 - 8 l - j
        unsigned bins[8], sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) bins[j] = 0;
        for (int r = 0; r < blocks; ++r) {
          const uint4 lo = reinterpret_cast<const uint4*>(inbox[buffer][r])[62 - 2 * lane], hi = reinterpret_cast<const uint4*>(inbox[buffer][r])[63 - 2 * lane];
          bins[0] += hi.w; bins[1] += hi.z; bins[2] += hi.y; bins[3] += hi.x;
          bins[4] += lo.w; bins[5] += lo.z; bins[6] += lo.y; bins[7] += lo.x;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += bins[j];
        unsigned above = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const unsigned x = __shfl_up_sync(0xFFFFFFFFu, above, d);
          if (lane >= d) above += x;
        }
        above -= sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (above < remaining && remaining <= above + bins[j]) {
            found[buffer][0] = 255 - 8 * lane - j;
            found[buffer][1] = remaining - above;
            found[buffer][2] = bins[j];
          }
          above += bins[j];
        }
      }
      __syncthreads();
      prefix = prefix << 8 | found[buffer][0];
      remaining = found[buffer][1];
      threshold = prefix << low;
      equal_stay = remaining;
      from_threshold = remaining == found[buffer][2];  // all of them stay: no need to tell them apart
      if (from_threshold) break;
    }
  }
  auto is_above = [&](unsigned key) { return from_threshold ? key >= threshold : key > threshold; };
  auto is_equal = [&](unsigned key) { return !from_threshold && key == threshold; };

  // ---- what the blocks before this one keep ----
  unsigned above_ahead = all ? t0 : 0, equal_ahead = 0;
  if (blocks > 1 && !all && k > 0) {
    unsigned both_above = 0, both_equal = 0;
    for_keys([&](unsigned key) {
      both_above += is_above(key);
      both_equal += is_equal(key);
    });
    both_above = __reduce_add_sync(0xFFFFFFFFu, both_above);
    both_equal = __reduce_add_sync(0xFFFFFFFFu, both_equal);
    if (lane < blocks && lane > rank) {
      asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(remote(&totals[0], lane)), "r"(both_above) : "memory");
      asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(remote(&totals[1], lane)), "r"(both_equal) : "memory");
    }
    cluster_sync();
    above_ahead = totals[0];
    equal_ahead = totals[1];
  }

  // ---- the survivors' list, kHeld tokens at a time ----
  int32_t* const idx = c.keep_idx ? c.keep_idx + (long long)job * (kPerSequence ? c.cache.hkv : 1) * c.max_keep : nullptr;
  for (int g0 = t0; g0 < t1; g0 += kHeld) {
    if (g0 > t0) look_up(g0, keys);
    const int t = g0 + tid * kEach, there = min(kEach, t1 - t);
    unsigned above = 0, equal = 0;  // a bit per token
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (j < there) {
        above |= (is_above(keys[j]) ? 1u : 0u) << j;
        equal |= (is_equal(keys[j]) ? 1u : 0u) << j;
      }
    __syncthreads();
    const unsigned own = __popc(above) | __popc(equal) << 16, before = sum_before<kWarps>(own, warp_a, lane, warp);  // (4,096 at most)
    if (tid == kThreads - 1) found[0][0] = before + own;  // of all threads
    const unsigned e = equal_ahead + (before >> 16), quota = equal_stay > e ? equal_stay - e : 0u;  // of the equal ones the first stay
#pragma unroll 1
    while (__popc(equal) > quota) equal &= ~(0x80000000u >> __clz(equal));
    unsigned at = above_ahead + (before & 0xFFFFu) + (from_threshold ? 0u : min(e, equal_stay));  // in the list: the thread's survivors lie side by side
    if (unsigned stay = above | equal) {
      const int page = page_at(t), row = page < 0 ? -1 : (page * c.cache.hkv << shift) + (t & (1 << shift) - 1);  // (a pool has fewer than 2^31 rows)
#pragma unroll 1
      for (; stay && at < (unsigned)k; stay &= stay - 1, ++at) {
        const int j = __ffs(stay) - 1;
        list[at] = row < 0 ? -1 : row + j;
        if (idx)
          for (int h = 0; h < (kPerSequence ? c.cache.hkv : 1); ++h) idx[(long long)h * c.max_keep + at] = t + j;
      }
    }
    __syncthreads();
    above_ahead += found[0][0] & 0xFFFFu;
    equal_ahead += found[0][0] >> 16;
  }
  sync_all();  // the list is there for all blocks; nobody's shared memory is written by another any more
  }
  if constexpr (!MOVE) return;

  // ---- the rows ----
  const int32_t* const to_table = c.out_table ? c.out_table : c.table;
  const int to_stride = c.out_table ? c.out_stride : c.table_stride, of_head = head << c.cache.page_shift;
  const int piece = tid % kPieces, row_of = tid / kPieces, step = blocks * kMoved;
  // Thread t < kMoved finds where row t of a round comes from and goes to; -1: it stays where it is, is left out, or does not exist.
  auto locate = [&](int r0) {
    const int i = r0 + rank * kMoved + tid;
    int from = -1, to = -1;
    if (i < k) {
      from = chain_load(list + i);
      const int page = page_of(c.cache, to_table, to_stride, b, i);
      if (page < 0 && c.device_status) atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
      to = page < 0 ? -1 : (int)pool_row(c.cache, page, head, i);
      if (from >= 0) from += of_head;
      if (from < 0 || to < 0 || from == to) from = to = -1;
    }
    return make_int2(from, to);
  };
  struct Round {
    uint4 x[kUnroll], y[kUnroll];
    int to[kUnroll], small_to;
    float ks, vs, w;
  };
  auto read = [&](const int2* places, Round& r) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int2 at = places[u * kAtOnce + row_of];
      r.to[u] = at.y;
      if (at.y < 0) continue;
      r.x[u] = chain_load(reinterpret_cast<const uint4*>(c.cache.k + (long long)at.x * DIM) + piece);
      r.y[u] = chain_load(reinterpret_cast<const uint4*>(c.cache.v + (long long)at.x * DIM) + piece);
    }
    r.small_to = -1;
    if (tid < kMoved) {
      const int2 at = places[tid];
      r.small_to = at.y;
      if (at.y >= 0) {
        r.ks = chain_load(c.cache.k_scale + at.x);
        r.vs = chain_load(c.cache.v_scale + at.x);
        r.w = chain_load(c.weights + at.x);
      }
    }
  };
  auto write = [&](const Round& r) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (r.to[u] >= 0) {
        reinterpret_cast<uint4*>(c.cache.k + (long long)r.to[u] * DIM)[piece] = r.x[u];
        reinterpret_cast<uint4*>(c.cache.v + (long long)r.to[u] * DIM)[piece] = r.y[u];
      }
    if (r.small_to >= 0) {
      c.cache.k_scale[r.small_to] = r.ks;
      c.cache.v_scale[r.small_to] = r.vs;
      c.weights[r.small_to] = r.w;
    }
  };
  if (k == 0) return;  // (all blocks of the cluster)
  Round now, next;
  if (tid < kMoved) places[0][tid] = locate(0);
  if (tid < kMoved) places[1][tid] = locate(step);
  __syncthreads();
  read(places[0], now);
  int buffer = 0;
  for (int r0 = 0; r0 < k; r0 += step, buffer ^= 1) {
    sync_all();  // this round's rows have been read, and the next one's are located
    if (r0 + step < k) read(places[buffer ^ 1], next);
    if (r0 + 2 * step < k && tid < kMoved) places[buffer][tid] = locate(r0 + 2 * step);
    write(now);
    now = next;
  }
}

// Rows to pages of their own, kChunk survivors of a sequence's KV head a block.
template <int DIM>
__global__ void __launch_bounds__(kChunkThreads)
evict_rows_kernel(EvictCall c, int chunks, bool joint) {
  constexpr int kPieces = DIM / 16, kAtOnce = kChunkThreads / kPieces, kUnroll = kChunk / kAtOnce;
  __shared__ int source[kChunk], place[kChunk];  // rows of the pool; -1: left out
  const int job = blockIdx.x / chunks, b = job / c.cache.hkv, head = job - b * c.cache.hkv, i0 = (blockIdx.x - job * chunks) * kChunk, tid = threadIdx.x;
  if (c.head_wait) pdl_wait();
  pdl_trigger();
  pdl_wait();
  const int n = min(max(chain_load_cached(c.lens + b), 0), c.max_len), k = min(min(max(chain_load_cached(c.counts + b), 0), n), c.max_keep);
  if (i0 >= k) return;
  float ks = 0.f, vs = 0.f, w = 0.f;
  int from = -1, to = -1;
  if (tid < kChunk) {
    const int i = i0 + tid;
    if (i < k) {
      from = chain_load(c.list + (long long)(joint ? b : job) * c.max_keep + i);
      const int page = page_of(c.cache, c.out_table, c.out_stride, b, i);
      if (page >= 0) to = (int)pool_row(c.cache, page, head, i);
      else if (c.device_status) atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
      if (from < 0 || to < 0) from = to = -1;
      else from += head << c.cache.page_shift;
    }
    source[tid] = from;
    place[tid] = to;
  }
  __syncthreads();
  if (to >= 0) {
    ks = chain_load(c.cache.k_scale + from);
    vs = chain_load(c.cache.v_scale + from);
    w = chain_load(c.weights + from);
  }
  const int piece = tid % kPieces, row_of = tid / kPieces;
  uint4 x[kUnroll], y[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int at = source[u * kAtOnce + row_of];
    if (at < 0) continue;
    x[u] = chain_load(reinterpret_cast<const uint4*>(c.cache.k + (long long)at * DIM) + piece);
    y[u] = chain_load(reinterpret_cast<const uint4*>(c.cache.v + (long long)at * DIM) + piece);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int at = place[u * kAtOnce + row_of];
    if (at < 0) continue;
    reinterpret_cast<uint4*>(c.cache.k + (long long)at * DIM)[piece] = x[u];
    reinterpret_cast<uint4*>(c.cache.v + (long long)at * DIM)[piece] = y[u];
  }
  if (to >= 0) {
    c.cache.k_scale[to] = ks;
    c.cache.v_scale[to] = vs;
    c.weights[to] = w;
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
  auto go = [&](auto kernel, int jobs) {
    c.blocks = cluster_blocks(jobs, p->max_kv_len, kLeastSlice, kPortableCluster);
    count_launches(1);
    return launch_chained_cluster(kernel, dim3((unsigned)(jobs * c.blocks)), dim3(kThreads), c.blocks > 1 ? c.blocks : 0, 0, st, c);
  };
  const bool joint = (p->flags & FASTAV_EVICT_JOINT) != 0, wide = c.cache.dim == 128;
  const int jobs = p->batch * cache->num_kv_heads;
  const long long chunks = ((long long)p->max_keep + kChunk - 1) / kChunk;
  const bool apart = out_table_opt && p->max_keep > 0 && chunks * jobs <= INT_MAX && (joint || p->max_keep > kFewRows * cluster_blocks(jobs, p->max_kv_len, kLeastSlice, kPortableCluster));
  cudaError_t e;
  if (joint) e = go(evict_kernel<64, true, false, true>, p->batch);
  else if (apart) e = go(evict_kernel<64, true, false, false>, jobs);
  else e = wide ? go(evict_kernel<128, true, true, false>, jobs) : go(evict_kernel<64, true, true, false>, jobs);
  if (e == cudaSuccess && apart) {
    count_launches(1);
    const dim3 grid((unsigned)(chunks * jobs));
    e = wide ? launch_chained(evict_rows_kernel<128>, grid, dim3(kChunkThreads), 0, st, c, (int)chunks, joint)
             : launch_chained(evict_rows_kernel<64>, grid, dim3(kChunkThreads), 0, st, c, (int)chunks, joint);
  } else if (e == cudaSuccess && joint) {
    e = wide ? go(evict_kernel<128, false, true, true>, jobs) : go(evict_kernel<64, false, true, true>, jobs);
  }
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}
