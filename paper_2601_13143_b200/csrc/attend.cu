// fastav_attend: the call's plan, and the kernel that joins the parts of its jobs.
#include <cmath>
#include <limits.h>

#include <cuda.h>

#include "attend.cuh"
#include "sm100_ptx.cuh"

namespace fastav {
namespace {

constexpr int kJoinThreads = 256;

// The parts of one row and head at one level: which job, which blocks.
struct Parts {
  const float* out = nullptr;
  const float2* ml = nullptr;
  int first = 0, count = 0;  // blocks
  int row = 0;               // of the tile
  bool whole = false;
};

template <int DIM>
__device__ __forceinline__ const float* part_row(const AttendList& list, const Parts& p, int i) {  // part i: a job's first block has it second
  return list.part_out + ((long long)((p.first + i) * 2 + (i == 0 ? 1 : 0)) * list.tile_rows + p.row) * DIM;
}
__device__ __forceinline__ float2 part_stat(const AttendList& list, const Parts& p, int i) {
  return chain_load(list.part_ml + ((long long)((p.first + i) * 2 + (i == 0 ? 1 : 0)) * list.tile_rows + p.row));
}

__device__ Parts find_parts(const AttendCall& c, const AttendList& list, int e, int row, int head) {
  Parts p;
  bool bad = false;
  const Entry x = entry_of(c, list, e, bad);
  const int r = row - x.row0, granules = granules_of(list, x);
  if (r < 0 || r >= x.rows || granules == 0) return p;
  const int kv = head / c.group, i = r * c.group + head - kv * c.group, tile = i / list.tile_rows;
  const int start = chain_load_cached(list.ahead + e) + (kv * tiles_of(c, list, x) + tile) * (list.job_cost + granules) + list.job_cost;
  const int total = chain_load_cached(list.ahead + list.entries());
  if (start < 0 || start + granules > total) return p;  // (the arrays changed meanwhile)
  p.row = i - tile * list.tile_rows;
  const int workers = workers_of(list, total);
  p.first = worker_of(start, workers, total);
  p.count = worker_of(start + granules - 1, workers, total) - p.first + 1;
  p.whole = p.count == 1;
  return p;
}

// A warp per (query row, head): joins what the levels' blocks left.  With m the largest of the parts' maxima,
//   out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i,  lse = ln 2 (m + log2 sum).
// Rows of one level that one block finished are there already; a row that sees no key gets 0 and -inf.
template <int DIM>
__global__ void __launch_bounds__(kJoinThreads) attend_join_kernel(AttendCall c, AttendList own, AttendList shared) {
  constexpr int kEach = DIM / 32;
  chain_enter(c);
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int at = blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5), row = at / c.hq, head = at - row * c.hq;
  if (row >= c.total_q) return;
  int lo = 0, hi = c.batch;  // the row's sequence: the last one that begins at or before it
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (chain_load_cached(c.cu_qlens + mid) <= row) lo = mid; else hi = mid;
  }
  if (row < chain_load_cached(c.cu_qlens + lo) || row >= chain_load_cached(c.cu_qlens + lo + 1)) return;  // nobody's row
  Parts level[2];
  level[0] = find_parts(c, own, own.from_prefix + lo, row, head);
  if (c.prefixes > 0) {
    int a = 0, z = c.prefixes;  // the last prefix that begins at or before the sequence
    while (z - a > 1) {
      const int mid = (a + z) >> 1;
      if (chain_load_cached(c.cu_prefix + mid) <= lo) a = mid; else z = mid;
    }
    if (lo >= chain_load_cached(c.cu_prefix + a) && lo < chain_load_cached(c.cu_prefix + a + 1)) level[1] = find_parts(c, shared, a, row, head);
  } else if (level[0].whole) {
    return;
  }
  float top = -INFINITY;
  const long long flat = (long long)row * c.hq + head;
  auto stat = [&](int l, int i) {
    return level[l].whole ? chain_load(c.whole_ml + (long long)l * c.total_q * c.hq + flat) : part_stat(l ? shared : own, level[l], i);
  };
#pragma unroll
  for (int l = 0; l < 2; ++l)
    for (int i = lane; i < level[l].count; i += 32) top = fmaxf(top, stat(l, i).x);
#pragma unroll
  for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
  const float base = top == -INFINITY ? 0.f : top;
  float acc[kEach] = {}, sum = 0.f;
#pragma unroll
  for (int l = 0; l < 2; ++l) {
#pragma unroll 4
    for (int i = 0; i < level[l].count; ++i) {
      const float2 ml = stat(l, i);
      const float weight = exp2f(ml.x - base);
      const float* const o = (level[l].whole ? c.whole_out + ((long long)l * c.total_q * c.hq + flat) * DIM : part_row<DIM>(l ? shared : own, level[l], i)) + lane * kEach;
      sum += weight * ml.y;
      if (kEach == 4) {
        const float4 v = chain_load(reinterpret_cast<const float4*>(o));
        acc[0] += weight * v.x; acc[1] += weight * v.y; acc[2 % kEach] += weight * v.z; acc[3 % kEach] += weight * v.w;
      } else {
        const float2 v = chain_load(reinterpret_cast<const float2*>(o));
        acc[0] += weight * v.x; acc[1] += weight * v.y;
      }
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint32_t packed[kEach / 2];
#pragma unroll
  for (int i = 0; i < kEach / 2; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(packed[i]) : "f"(acc[2 * i + 1] * inv), "f"(acc[2 * i] * inv));
  uint16_t* const to = c.out + (long long)row * c.o_st + (long long)head * c.o_sh + lane * kEach;
  if (kEach == 4) *reinterpret_cast<uint2*>(to) = make_uint2(packed[0], packed[kEach / 2 - 1]);
  else *reinterpret_cast<uint32_t*>(to) = packed[0];
  if (c.lse_out && lane == 0) c.lse_out[flat] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// The levels' entries go to the kernel that suits their rows: few (mma.sync) up to kMostFew stacked rows, else many (tcgen05).
constexpr int kMostFew = 48;

struct Plan {
  AttendList few{}, many{};   // lists of the two kernels; without entries: not launched
  bool own_many, shared_many;
  size_t ahead[2], out[2], ml[2], whole_out, whole_ml, total = 0;  // offsets into the workspace: few, many
  bool fits = true;
};

// Most units of `entries` entries of at most `rows` query rows and `len` keys.
long long most_units(const fastav_attend_params& p, const fastav_cache& cache, const AttendList& list, long long entries, long long rows, long long len) {
  const long long group = p.num_q_heads / cache.num_kv_heads;
  return entries * cache.num_kv_heads * ((rows * group + list.tile_rows - 1) / list.tile_rows) * (list.job_cost + (len + list.unit_keys - 1) / list.unit_keys);
}

Plan make_plan(const fastav_attend_params& p, const fastav_cache& cache) {
  Plan w;
  size_t off = 0;
  auto carve = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return at; };
  const long long group = p.num_q_heads / cache.num_kv_heads;
  w.own_many = p.max_qlen * group > kMostFew;
  w.shared_many = p.num_prefixes > 0 && p.max_prefix_q * group > kMostFew;
  w.few.tile_rows = kFewTile;
  w.few.unit_keys = kFewKeys;
  w.many.tile_rows = kManyTile;
  w.many.unit_keys = kManyKeys;
  w.few.job_cost = kFewJobCost;
  w.many.job_cost = kManyJobCost;
  (w.own_many ? w.many : w.few).from_own = p.batch;
  (w.shared_many ? w.many : w.few).from_prefix = p.num_prefixes;
  AttendList* const lists[2] = {&w.few, &w.many};
  for (int i = 0; i < 2; ++i) {
    AttendList& list = *lists[i];
    const long long units = most_units(p, cache, list, list.from_own, p.max_qlen, p.max_kv_len) +
                            most_units(p, cache, list, list.from_prefix, p.max_prefix_q, p.max_prefix_len);
    w.fits &= units < INT_MAX;
    list.grid = (int)(units < 1 ? 1 : units < kNumSMs ? units : kNumSMs);
    const size_t parts = list.entries() > 0 ? (size_t)list.grid * 2 * list.tile_rows : 0;
    w.ahead[i] = carve((size_t)(list.entries() + 1) * sizeof(int32_t));
    w.out[i] = carve(parts * cache.head_dim * sizeof(float));
    w.ml[i] = carve(parts * sizeof(float2));
  }
  const size_t rows = p.num_prefixes > 0 ? (size_t)2 * p.total_q * p.num_q_heads : 0;
  w.whole_out = carve(rows * cache.head_dim * sizeof(float));
  w.whole_ml = carve(rows * sizeof(float2));
  w.total = off;
  return w;
}

int32_t check_shapes(const fastav_attend_params* p, const fastav_cache* cache) {
  int32_t rc = check_cache(cache);
  if (rc != FASTAV_OK) return rc;
  if (!p || p->batch < 1 || p->total_q < 0 || p->max_qlen < 0 || p->max_qlen > p->total_q || p->max_kv_len < 0) return FASTAV_ERR_INVALID_ARG;
  if (p->num_q_heads < 1 || p->num_q_heads % cache->num_kv_heads != 0 || p->table_stride < 0) return FASTAV_ERR_INVALID_ARG;
  if (p->num_prefixes < 0 || p->max_prefix_len < 0 || p->max_prefix_q < 0 || p->max_prefix_q > p->total_q) return FASTAV_ERR_INVALID_ARG;
  if (p->num_prefixes > 0 && p->prefix_table_stride < 0) return FASTAV_ERR_INVALID_ARG;
  if ((long long)p->batch + p->num_prefixes > FASTAV_ATTEND_MAX_BATCH) return FASTAV_ERR_UNSUPPORTED;
  // a stack of query rows and the rows of all heads are 32-bit counts
  if ((long long)p->total_q * p->num_q_heads > INT_MAX / 2) return FASTAV_ERR_UNSUPPORTED;
  return make_plan(*p, *cache).fits ? FASTAV_OK : FASTAV_ERR_UNSUPPORTED;
}

}  // namespace

bool encode_pool_map(const CacheView& c, const void* pool, int box_rows, void* map) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  const Encode encode = reinterpret_cast<Encode>(tensor_map_encode_entry());
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)c.dim, (cuuint64_t)c.num_pages * c.hkv << c.page_shift};
  const cuuint64_t strides[1] = {(cuuint64_t)c.dim};
  const cuuint32_t box[2] = {(cuuint32_t)c.dim, (cuuint32_t)box_rows};
  const cuuint32_t elem[2] = {1, 1};
  return encode(static_cast<CUtensorMap*>(map), CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(pool), dims, strides, box, elem,
                CU_TENSOR_MAP_INTERLEAVE_NONE, c.dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace fastav

using namespace fastav;

extern "C" int32_t fastav_attend_workspace_bytes(const fastav_attend_params* p, const fastav_cache* cache, size_t* out_bytes) {
  const int32_t rc = check_shapes(p, cache);
  if (rc != FASTAV_OK) return rc;
  if (!out_bytes) return FASTAV_ERR_INVALID_ARG;
  *out_bytes = make_plan(*p, *cache).total;
  return FASTAV_OK;
}

extern "C" int32_t fastav_attend(const fastav_attend_params* p, const fastav_cache* cache, const void* q, const int32_t* cu_qlens, const int32_t* page_table,
                                 const int32_t* kv_lens, const int32_t* cu_prefix, const int32_t* prefix_table, const int32_t* prefix_lens, void* out,
                                 float* lse_out_opt, void* workspace, size_t workspace_bytes, int32_t* device_status, void* stream) {
  int32_t rc = check_shapes(p, cache);
  if (rc != FASTAV_OK) return rc;
  if (!cu_qlens || !kv_lens || (p->max_kv_len > 0 && (!page_table || p->table_stride < 1))) return FASTAV_ERR_INVALID_ARG;
  if (p->num_prefixes > 0 && (!cu_prefix || !prefix_lens || (p->max_prefix_len > 0 && (!prefix_table || p->prefix_table_stride < 1)))) return FASTAV_ERR_INVALID_ARG;
  if (p->total_q > 0 && (!q || !out)) return FASTAV_ERR_INVALID_ARG;
  if ((rc = check_strides(p->q_stride_tok, p->q_stride_head, p->num_q_heads, cache->head_dim)) != FASTAV_OK) return rc;
  if ((rc = check_strides(p->o_stride_tok, p->o_stride_head, p->num_q_heads, cache->head_dim)) != FASTAV_OK) return rc;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15u) return FASTAV_ERR_UNSUPPORTED;
  const Plan w = make_plan(*p, *cache);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < w.total) return FASTAV_ERR_WORKSPACE;
  if (p->total_q == 0) return FASTAV_OK;
  chain_begin(p->flags);

  AttendCall c{};
  c.cache = make_view(*cache);
  c.batch = p->batch; c.total_q = p->total_q; c.max_qlen = p->max_qlen; c.hq = p->num_q_heads; c.group = p->num_q_heads / cache->num_kv_heads;
  c.max_len = p->max_kv_len; c.table_stride = p->table_stride;
  c.prefixes = p->num_prefixes; c.max_prefix_len = p->max_prefix_len; c.prefix_stride = p->prefix_table_stride; c.max_prefix_q = p->max_prefix_q;
  c.q_st = p->q_stride_tok; c.q_sh = p->q_stride_head; c.o_st = p->o_stride_tok; c.o_sh = p->o_stride_head;
  c.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / std::sqrt((float)cache->head_dim)) * kLog2e;
  c.causal = (p->flags & FASTAV_CAUSAL) != 0;
  c.cu_qlens = cu_qlens; c.table = page_table; c.lens = kv_lens;
  c.cu_prefix = cu_prefix; c.prefix_table = prefix_table; c.prefix_lens = prefix_lens;
  c.q = static_cast<const uint16_t*>(q);
  c.out = static_cast<uint16_t*>(out);
  c.lse_out = lse_out_opt;
  c.device_status = device_status;
  unsigned char* const ws = static_cast<unsigned char*>(workspace);
  c.whole_out = reinterpret_cast<float*>(ws + w.whole_out);
  c.whole_ml = reinterpret_cast<float2*>(ws + w.whole_ml);
  AttendList lists[2] = {w.few, w.many};
  for (int i = 0; i < 2; ++i) {
    lists[i].ahead = reinterpret_cast<int32_t*>(ws + w.ahead[i]);
    lists[i].part_out = reinterpret_cast<float*>(ws + w.out[i]);
    lists[i].part_ml = reinterpret_cast<float2*>(ws + w.ml[i]);
  }
  const AttendList &own = lists[w.own_many], &shared = lists[w.shared_many];
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (lists[1].entries() > 0) e = launch_attend_many(c, lists[1], st);
  if (e == cudaSuccess && lists[0].entries() > 0) e = launch_attend_few(c, lists[0], st);
  if (e != cudaSuccess) return cuda_failed(e);
  const int warps = kJoinThreads / 32;
  const dim3 grid((unsigned)(((long long)c.total_q * c.hq + warps - 1) / warps));
  count_launches(1);
  e = c.cache.dim == 128 ? launch_chained(attend_join_kernel<128>, grid, dim3(kJoinThreads), 0, st, c, own, shared)
                         : launch_chained(attend_join_kernel<64>, grid, dim3(kJoinThreads), 0, st, c, own, shared);
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}
