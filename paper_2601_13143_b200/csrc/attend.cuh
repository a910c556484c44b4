// Attention over the 8-bit cache (fastav_attend): what its kernels share.
//
// The work of a call is a list of jobs.  An ENTRY is a set of query rows that see the same keys of the same page-table row: the rows of a
// sequence with the sequence's own tokens, or the rows of all sequences that share a prefix with the prefix.  Its query rows times the
// G query heads of a KV head are stacked (row i of the stack: query row i / G, head i % G) and cut into tiles; a JOB is one (entry, KV head,
// tile), its keys cut into granules, the UNITS.  All units of a launch form one list, keys innermost, and every worker takes an equal run
// of it, whatever the lengths.  A run that begins or ends inside a job leaves a part (its keys' log-sum-exp in base 2, and the output they alone would
// give: sums that are not divided yet pass fp32's range where values are near bf16's); the parts of a job lie with consecutive blocks, and the kernel that joins them works out which from the list alone.  A job begins with
// `job_cost` units that hold nothing: what its queries, its output and its first logits cost, in granules; short jobs would else
// all fall to a few workers.
#pragma once

#include <limits.h>

#include "cache.cuh"

namespace fastav {

struct AttendCall {
  CacheView cache;
  int batch, total_q, max_qlen, hq, group;
  unsigned group_magic;  // ceil(2^32 / group); 0: group is 1
  int max_len, table_stride;
  int prefixes, max_prefix_len, prefix_stride, max_prefix_q;
  long long q_st, q_sh, o_st, o_sh;
  float scale_log2;  // softmax scale * log2(e): logits are kept in base-2 units
  bool causal;
  const int32_t *cu_qlens, *table, *lens, *cu_prefix, *prefix_table, *prefix_lens;
  const uint16_t* q;
  uint16_t* out;
  float* lse_out;
  int32_t* device_status;
  // results of jobs that one block finished, where another level's are still to be joined: [2][total_q, Hq]
  float* whole_out;
  float* whole_lse;
  int beside;  // both kernels run, side by side on SMs of their own
  // ... and how the second knows that earlier work has ended, of which its own wait (for the first kernel's end) comes too late to tell it: the first
  // kernel writes the call's ticket here behind its wait and ahead of letting the second start; the join takes it away.
  uint64_t* ended;
  uint64_t ticket;
  int head_wait;
};
inline void mark_head(AttendCall& c, bool head) { c.head_wait = head ? 1 : 0; }

// One launch's list: the prefixes' entries (from_prefix of them), then the sequences' own (from_own).
struct AttendList {
  int from_prefix, from_own;
  int tile_rows, unit_keys;  // of a tile; of a granule
  int job_cost;              // units ahead of a job's granules
  int grid;                  // blocks that share the list
  int32_t* ahead;            // [entries + 1] units before an entry, left for the kernel that joins
  float* part_out;           // [grid][2][tile_rows][dim]
  float* part_lse;           // [grid][2][tile_rows], base 2
  float* scratch;            // few: parts that warps of one block exchange
  int32_t* copies;           // many: the blocks' own `ahead`, where there are more entries than shared memory has room for
  int through_l2;            // index arrays always: the kernel has no wait of its own ahead of its reads
  __host__ __device__ int entries() const { return from_prefix + from_own; }
};

// Few rows per KV head: mma.sync, a granule per warp, tiles of 8 or 16 rows (attend_few.cu).
constexpr int kFewKeys = 32, kFewJobCost = 3;
size_t few_scratch_floats(const AttendList& list, int dim);
cudaError_t launch_attend_few(const AttendCall& c, const AttendList& list, cudaStream_t stream);

// Many: tcgen05, a granule per step of a block (attend_many.cu).
constexpr int kManyTile = 256, kManyKeys = 128, kManyJobCost = 4;
constexpr int many_listed(int dim) { return dim == 128 ? 2000 : 3000; }  // entries whose `ahead` has room in shared memory
cudaError_t launch_attend_many(const AttendCall& c, const AttendList& list, cudaStream_t stream);

#ifdef __CUDACC__
// The query row of a stacked row, i / group (the host sees to it that i * group < 2^32).
__device__ __forceinline__ int query_row(const AttendCall& c, int i) { return c.group_magic ? (int)__umulhi((unsigned)i, c.group_magic) : i; }

struct Entry {
  int row0, rows;  // query rows
  int len;         // keys
  const int32_t* table;
  bool own;
};
// Reads of index arrays: after the kernel's wait through L1, ahead of it (or without one, AttendList::through_l2) through L2.
__device__ __forceinline__ int index_load(const int32_t* p, bool cached) { return cached ? chain_load_cached(p) : chain_load(p); }
__device__ __forceinline__ Entry entry_of(const AttendCall& c, const AttendList& list, int e, bool& bad, bool cached = true) {
  Entry x;
  x.own = e >= list.from_prefix;
  if (x.own) {
    const int b = e - list.from_prefix;
    const Span rows = checked_words(index_load(c.cu_qlens + b, cached), index_load(c.cu_qlens + b + 1, cached), c.total_q, c.max_qlen);
    x.row0 = rows.first;
    x.rows = rows.count;
    x.len = index_load(c.lens + b, cached);
    x.table = c.table + (long long)b * c.table_stride;
    bad |= rows.bad;
  } else {
    const int from = index_load(c.cu_prefix + e, cached), to = index_load(c.cu_prefix + e + 1, cached);
    const bool fits = from >= 0 && from <= to && to <= c.batch;
    const Span rows = fits ? checked_words(index_load(c.cu_qlens + from, cached), index_load(c.cu_qlens + to, cached), c.total_q, c.max_prefix_q)
                           : Span{0, 0, true};
    x.row0 = rows.first;
    x.rows = rows.count;
    x.len = index_load(c.prefix_lens + e, cached);
    x.table = c.prefix_table + (long long)e * c.prefix_stride;
    bad |= rows.bad;
  }
  const long long room = (long long)(x.own ? c.table_stride : c.prefix_stride) << c.cache.page_shift;
  const int most = (int)min((long long)(x.own ? c.max_len : c.max_prefix_len), room);
  if (x.len < 0 || x.len > most) {
    bad = true;
    x.len = max(0, min(x.len, most));
  }
  return x;
}
__device__ __forceinline__ int tiles_of(const AttendCall& c, const AttendList& list, const Entry& x) {
  return (x.rows * c.group + list.tile_rows - 1) / list.tile_rows;
}
__device__ __forceinline__ int granules_of(const AttendList& list, const Entry& x) { return (x.len + list.unit_keys - 1) / list.unit_keys; }
__device__ __forceinline__ int units_of(const AttendCall& c, const AttendList& list, const Entry& x) {
  const int granules = granules_of(list, x);
  return granules ? c.cache.hkv * tiles_of(c, list, x) * (list.job_cost + granules) : 0;
}

// Blocks that have units: all, or the first of them, one unit each.
__device__ __forceinline__ int workers_of(const AttendList& list, int total) { return max(1, min(list.grid, total)); }
// Worker w of `workers` takes the units [run_start(w), run_start(w + 1)) of `total`; worker_of is the one that has unit u.
// (32 bits wherever they do: a 64-bit division is a hundred instructions.)
__device__ __forceinline__ int scaled(int x, int times, int by) {
  return x <= INT_MAX / kNumSMs ? (int)((unsigned)x * (unsigned)times / (unsigned)by) : (int)((long long)x * times / by);
}
__device__ __forceinline__ int run_start(int w, int workers, int total) { return scaled(total, w, workers); }
__device__ __forceinline__ int worker_of(int u, int workers, int total) {
  return u < INT_MAX / kNumSMs ? (int)(((unsigned)(u + 1) * (unsigned)workers - 1u) / (unsigned)total) : (int)(((long long)(u + 1) * workers - 1) / total);
}

// The list, all threads of the block: ahead[e] in shared memory, [entries + 1]; the total.  Reads the index arrays only.
template <int THREADS>
__device__ int open_list(const AttendCall& c, const AttendList& list, int* ahead, int* warp_sum) {
  const int entries = list.entries(), each = (entries + THREADS - 1) / THREADS;
  const int e0 = min(entries, (int)threadIdx.x * each), e1 = min(entries, e0 + each);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int sum = 0;
  bool bad = false;
#pragma unroll 1
  for (int e = e0; e < e1; ++e) {
    ahead[e] = sum;
    sum += units_of(c, list, entry_of(c, list, e, bad, c.head_wait && !list.through_l2));
  }
  int upto = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int t = __shfl_up_sync(0xFFFFFFFFu, upto, d);
    if (lane >= d) upto += t;
  }
  if (lane == 31) warp_sum[warp] = upto;
  __syncthreads();
  int before = upto - sum, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += warp_sum[w];
    total += warp_sum[w];
  }
#pragma unroll 1
  for (int e = e0; e < e1; ++e) ahead[e] += before;
  if (threadIdx.x == 0) ahead[entries] = total;
  if (blockIdx.x == 0 && bad && c.device_status) atomicOr(c.device_status, FASTAV_DEV_SHAPE_MISMATCH);
  __syncthreads();
  return total;
}
// ... and block 0 leaves a copy for the kernel that joins (after the kernel's wait: an earlier call may still read what lies there).
template <int THREADS>
__device__ __forceinline__ void leave_list(const AttendList& list, const int* ahead) {
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e <= list.entries(); e += THREADS) list.ahead[e] = ahead[e];
}

// A walk along the list: the granule it stands at.
struct Walk {
  Entry x;
  int e, head, tile, granule;
  int tiles, granules;
  int unit;  // of the granule
  __device__ __forceinline__ int job_first() const { return unit - granule; }             // the unit of the job's first granule
  __device__ __forceinline__ int job_end() const { return unit - granule + granules; }
  __device__ __forceinline__ void load(const AttendCall& c, const AttendList& list) {
    bool bad = false;  // (reported by open_list)
    x = entry_of(c, list, e, bad, !list.through_l2);
    tiles = tiles_of(c, list, x);
    granules = granules_of(list, x);
  }
  // To the first granule at or behind unit u, which is less than the total.
  __device__ void seek(const AttendCall& c, const AttendList& list, const int* ahead, int u) {
    int lo = 0, hi = list.entries();  // the last entry that begins at or before u: one with units
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (ahead[mid] <= u) lo = mid; else hi = mid;
    }
    e = lo;
    load(c, list);
    const int r = u - ahead[e], each = list.job_cost + granules, job = r / each;
    granule = max(0, r - job * each - list.job_cost);
    head = job / tiles;
    tile = job - head * tiles;
    unit = ahead[e] + job * each + list.job_cost + granule;
  }
  // To the next granule, whose unit is less than `end`, the end of a run; false if there is none.
  __device__ __forceinline__ bool step(const AttendCall& c, const AttendList& list, const int* ahead, int end) {
    ++unit;
    if (++granule < granules) return unit < end;
    unit += list.job_cost;
    if (unit >= end) return false;
    granule = 0;
    if (++tile < tiles) return true;
    tile = 0;
    if (++head < c.cache.hkv) return true;
    head = 0;
    do ++e; while (ahead[e + 1] < unit);  // (its first granule stands job_cost units behind its beginning)
    load(c, list);
    return true;
  }
};
#endif

}  // namespace fastav
