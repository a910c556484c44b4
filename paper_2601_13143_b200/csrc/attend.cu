// fastav_attend: the call's plan, and the kernel that joins the parts of its jobs.
#include <algorithm>
#include <cmath>
#include <limits.h>

#include "attend.cuh"
#include "sm100_ptx.cuh"

namespace fastav {
namespace {

constexpr int kJoinWarps = 8;
constexpr float kShare = 1.f / 1024;  // on every weight: the sum of some hundred parts near bf16's largest value stays in fp32

// The parts of one row and head at one level: which job, which blocks.
struct Parts {
  int first = 0, count = 0;  // blocks
  int row = 0;               // of the tile
  bool whole = false;
};
// Part i of a row: a job's first block has it in its second place.
__device__ __forceinline__ int part_of(int tile_rows, const Parts& p, int i) { return ((p.first + i) * 2 + (i == 0 ? 1 : 0)) * tile_rows + p.row; }

// Where the parts of one row and head of the entry e lie: x, with `ahead` units before it of `total`.
__device__ __forceinline__ Parts find_parts(const AttendCall& c, const AttendList& list, const Entry& x, int ahead, int total, int row, int head) {
  Parts p;
  const int r = row - x.row0, granules = granules_of(list, x);
  if (r < 0 || r >= x.rows || granules == 0) return p;
  const int kv = head / c.group, i = r * c.group + head - kv * c.group, tile = i / list.tile_rows;
  const int start = ahead + (kv * tiles_of(c, list, x) + tile) * (list.job_cost + granules) + list.job_cost;
  if (start < 0 || start + granules > total) return p;  // (the arrays changed meanwhile)
  const int workers = workers_of(list, total);
  p.row = i - tile * list.tile_rows;
  p.first = worker_of(start, workers, total);
  p.count = worker_of(start + granules - 1, workers, total) - p.first + 1;
  p.whole = p.count == 1;
  return p;
}

__device__ __forceinline__ Parts from_lane(const Parts& mine, int lane) {
  Parts p;
  p.first = __shfl_sync(0xFFFFFFFFu, mine.first, lane);
  p.count = __shfl_sync(0xFFFFFFFFu, mine.count, lane);
  p.row = __shfl_sync(0xFFFFFFFFu, mine.row, lane);
  p.whole = p.count == 1;
  return p;
}

// The last of n ascending numbers that is at most x (0 if none is); the whole warp, 32 looks at a time.
template <bool CACHED>
__device__ __forceinline__ int last_upto(const int32_t* a, int n, int x, int lane) {
  int lo = 0;
  while (n > 1) {
    const int step = (n + 31) / 32;
    const unsigned upto = __ballot_sync(0xFFFFFFFFu, lane * step < n && index_load(a + lo + min(lane * step, n - 1), CACHED) <= x);
    const int k = upto ? 31 - __clz(upto) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// What a row belongs to: sequence b, and prefix a (-1: none) at the levels.
struct Belongs {
  int b, a;
  bool somebody;
  Entry x[2];
};
template <bool CACHED>
__device__ __forceinline__ Belongs belongs_to(const AttendCall& c, const AttendList& own, const AttendList& shared, int row, int lane) {
  Belongs f;
  bool bad = false;  // (reported by open_list)
  f.b = last_upto<CACHED>(c.cu_qlens, c.batch, row, lane);
  f.somebody = row >= index_load(c.cu_qlens + f.b, CACHED) && row < index_load(c.cu_qlens + f.b + 1, CACHED);
  f.x[0] = entry_of(c, own, own.from_prefix + f.b, bad, CACHED);
  f.a = -1;
  if (c.prefixes > 0) {
    const int a = last_upto<CACHED>(c.cu_prefix, c.prefixes, f.b, lane);
    if (f.b >= index_load(c.cu_prefix + a, CACHED) && f.b < index_load(c.cu_prefix + a + 1, CACHED)) f.a = a;
    f.x[1] = entry_of(c, shared, a, bad, CACHED);
  }
  return f;
}

// Joins what the levels' blocks left.  With m the largest of the parts' log-sum-exps (base 2),
//   out = sum_i 2^(lse_i - m) out_i / sum_i 2^(lse_i - m),  lse = ln 2 (m + log2 sum).
// Rows of one level that one block finished are there already; a row that sees no key gets 0 and -inf.
//
// Bound by latency: a few trips to memory one after the other (the row's sequence; its bounds; the parts' statistics; the parts).  So a lane
// asks for one part's statistics each, and where rows are few and parts many, WARPS warps share those of a (row, head), eight at a time
// each (1 x 1,024 keys, 28 heads of up to 32 parts: the call in 13.3 us instead of 23.7 with a warp that went through them four at a time, in a step that
// also spared 64-bit divisions).  Many rows: a warp takes HEADS heads of a row and finds their jobs in as many lanes (41,000 (row, head): 36 us
// instead of 51).
template <int DIM, int WARPS, int HEADS>
__global__ void __launch_bounds__(32 * kJoinWarps) attend_join_kernel(AttendCall c, AttendList own, AttendList shared) {
  static_assert(WARPS == 1 || HEADS == 1);
  constexpr int kEach = DIM / 32, kHeads = kJoinWarps / WARPS * HEADS, kAtOnce = WARPS > 1 ? 8 : 2;
  __shared__ float part_acc[WARPS > 1 ? kJoinWarps : 1][DIM];
  __shared__ float2 part_sum[kJoinWarps];  // their maximum and sum
  __shared__ Belongs f;  // a block has one row
  chain_enter(c);
  // Where all blocks are there at once, this is looked up while the kernel before still runs.
  constexpr bool kEarly = HEADS == 1;
  if (!kEarly) pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % WARPS;
  const int head_blocks = (c.hq + kHeads - 1) / kHeads, row = blockIdx.x / head_blocks, head0 = (blockIdx.x - row * head_blocks) * kHeads + warp / WARPS * HEADS;
  if (warp == 0) {
    const Belongs mine = belongs_to<!kEarly>(c, own, shared, row, lane);
    if (lane == 0) f = mine;
  }
  __syncthreads();
  if (kEarly) pdl_wait();
  if (c.beside && blockIdx.x == 0 && threadIdx.x == 0) *c.ended = 0;
  if (!f.somebody) return;
  Parts found[2];  // of head head0 + lane
  const int lane_head = head0 + lane;
  const bool lane_there = lane < HEADS && lane_head < c.hq;
  const int own_ahead = chain_load_cached(own.ahead + own.from_prefix + f.b), own_total = chain_load_cached(own.ahead + own.entries());
  const int shared_ahead = f.a >= 0 ? chain_load_cached(shared.ahead + f.a) : 0, shared_total = f.a >= 0 ? chain_load_cached(shared.ahead + shared.entries()) : 0;
  if (lane_there) {
    found[0] = find_parts(c, own, f.x[0], own_ahead, own_total, row, lane_head);
    if (f.a >= 0) found[1] = find_parts(c, shared, f.x[1], shared_ahead, shared_total, row, lane_head);
  }
#pragma unroll 1
  for (int h = 0; h < HEADS; ++h) {
    const int head = head0 + h;
    const bool there = head < c.hq, done = c.prefixes == 0 && __shfl_sync(0xFFFFFFFFu, found[0].whole, h);
    const long long flat = (long long)row * c.hq + head, flats = (long long)c.total_q * c.hq;
    float top = -INFINITY, acc[kEach] = {}, sum = 0.f;
    // The parts of both levels are one list, own first.
    const Parts p0 = from_lane(found[0], h), p1 = from_lane(found[1], h);
    const int parts_all = done ? 0 : p0.count + p1.count;
#pragma unroll 1
    for (int i0 = 0; i0 < parts_all; i0 += 32 * WARPS) {  // a lane's part: WARPS lane + sub
      const int mine = i0 + lane * WARPS + sub;
      const bool is_shared = mine >= p0.count;
      const bool whole = is_shared ? p1.whole : p0.whole;
      Parts p;
      p.first = is_shared ? p1.first : p0.first;
      p.row = is_shared ? p1.row : p0.row;
      const long long at = whole ? (is_shared ? flats : 0) + flat
                                 : part_of(is_shared ? shared.tile_rows : own.tile_rows, p, mine - (is_shared ? p0.count : 0));
      const float lse = mine < parts_all ? chain_load((whole ? c.whole_lse : is_shared ? shared.part_lse : own.part_lse) + at) : -INFINITY;
      const float* const outs = (whole ? c.whole_out : is_shared ? shared.part_out : own.part_out) + at * DIM;
      float to = lse;
#pragma unroll
      for (int d = 16; d; d >>= 1) to = fmaxf(to, __shfl_xor_sync(0xFFFFFFFFu, to, d));
      to = fmaxf(to, top);
      const float base = to == -INFINITY ? 0.f : to, before = exp2f(top - base), weight = exp2f(lse - base) * kShare;
      top = to;
      sum = sum * before + weight;  // (a lane's own; added up below)
#pragma unroll
      for (int e = 0; e < kEach; ++e) acc[e] *= before;
      const int parts = min(32, (parts_all - i0 - sub + WARPS - 1) / WARPS);  // of this warp
      for (int j0 = 0; j0 < parts; j0 += kAtOnce) {
        float v[kAtOnce][kEach];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          const float* const from = reinterpret_cast<const float*>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(outs), (j0 + j) & 31)) + lane * kEach;
#pragma unroll
          for (int e = 0; e < kEach; ++e) v[j][e] = 0.f;
          if (j0 + j < parts) {
            if (kEach == 4) {
              const float4 x = chain_load(reinterpret_cast<const float4*>(from));
              v[j][0] = x.x; v[j][1] = x.y; v[j][2 % kEach] = x.z; v[j][3 % kEach] = x.w;
            } else {
              const float2 x = chain_load(reinterpret_cast<const float2*>(from));
              v[j][0] = x.x; v[j][1] = x.y;
            }
          }
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          const float w = __shfl_sync(0xFFFFFFFFu, weight, (j0 + j) & 31);
          if (j0 + j < parts)
#pragma unroll
            for (int e = 0; e < kEach; ++e) acc[e] = fmaf(w, v[j][e], acc[e]);
        }
      }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (WARPS > 1) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) part_acc[warp][lane * kEach + e] = acc[e];
      if (lane == 0) part_sum[warp] = make_float2(top, sum);
      __syncthreads();
      if (sub != 0) return;
      float to = -INFINITY;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) to = fmaxf(to, part_sum[warp + w].x);
      const float base = to == -INFINITY ? 0.f : to;
      top = to;
      sum = 0.f;
#pragma unroll
      for (int e = 0; e < kEach; ++e) acc[e] = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float weight = exp2f(part_sum[warp + w].x - base);
        sum += weight * part_sum[warp + w].y;
#pragma unroll
        for (int e = 0; e < kEach; ++e) acc[e] = fmaf(weight, part_acc[warp + w][lane * kEach + e], acc[e]);
      }
    }
    if (!there || done) continue;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint32_t packed[kEach / 2];
#pragma unroll
    for (int i = 0; i < kEach / 2; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(packed[i]) : "f"(acc[2 * i + 1] * inv), "f"(acc[2 * i] * inv));
    uint16_t* const to = c.out + (long long)row * c.o_st + (long long)head * c.o_sh + lane * kEach;
    if (kEach == 4) *reinterpret_cast<uint2*>(to) = make_uint2(packed[0], packed[kEach / 2 - 1]);
    else *reinterpret_cast<uint32_t*>(to) = packed[0];
    if (c.lse_out && lane == 0) c.lse_out[flat] = sum == 0.f ? -INFINITY : (top + log2f(sum * (1.f / kShare))) * kLn2;
  }
}

template <int DIM, int WARPS, int HEADS>
cudaError_t launch_join(const AttendCall& c, const AttendList& own, const AttendList& shared, cudaStream_t stream) {
  constexpr int kHeads = kJoinWarps / WARPS * HEADS;
  const long long blocks = (long long)c.total_q * ((c.hq + kHeads - 1) / kHeads);
  count_launches(1);
  return launch_chained(attend_join_kernel<DIM, WARPS, HEADS>, dim3((unsigned)blocks), dim3(32 * kJoinWarps), 0, stream, c, own, shared);
}
template <int DIM>
cudaError_t launch_join(const AttendCall& c, const AttendList& own, const AttendList& shared, cudaStream_t stream) {
  // As many warps per row and head as are resident at once (two blocks an SM; two warps: four blocks, 64 answers on a shared prefix 43.1 us
  // instead of 45.1; four warps were no quicker than two); many rows: several heads per warp.
  const long long flats = (long long)c.total_q * c.hq, room = kNumSMs * 2 * kJoinWarps;
  if (flats * 8 <= room) return launch_join<DIM, 8, 1>(c, own, shared, stream);
  if (flats <= room) return launch_join<DIM, 2, 1>(c, own, shared, stream);
  return flats <= 4 * room ? launch_join<DIM, 1, 1>(c, own, shared, stream) : launch_join<DIM, 1, 4>(c, own, shared, stream);
}

// The levels' entries go to the kernel that suits their stacked rows: few (mma.sync) up to 16, which an instruction pair takes at once, many (tcgen05)
// beyond.  us, few / many, when the rule was made: one sequence of 60 keys of 8 heads, 48 rows 15.3 / 13.5, of 1,000, 24 rows 17.9 / 16.0; 28 rows on 4 heads: 4,000 keys
// 19.8 / 17.5, 8 x 3,000 keys 35.5 / 26.3, a prefix of 4,000 for seven rows each of four sequences with few rows of their own 21.2 / 22.5;
// 8 sequences of 500 to 744 keys, up to 32 rows on 2 heads of 64, 14.4 / 14.9; 16 rows of 8 heads, 16 x 2,000 keys 39.3 / 43.3, one of 4,000 19.9 / 18.7.
constexpr int kMostFew = 16;
constexpr double kFewUnitCost = 0.13, kManyUnitCost = 1.7;  // us of an SM (many at 1.2 / 1.7 / 2.2 / 3, then: 32 answers 37.7 / 37.5 / 38.9 / 42.8, 64 44.4 / 42.0 / 42.2 / 40.5)

struct Plan {
  AttendList few{}, many{};   // lists of the two kernels; without entries: not launched
  bool own_many, shared_many;
  size_t ahead[2], out[2], lse[2], scratch, copies, whole_out, whole_lse, ended, total = 0;  // offsets into the workspace: few, many
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
  w.many.tile_rows = kManyTile;
  w.few.unit_keys = kFewKeys;
  w.many.unit_keys = kManyKeys;
  w.few.job_cost = kFewJobCost;
  w.many.job_cost = kManyJobCost;
  auto takes_many = [&](long long rows) { return rows * group > kMostFew; };
  w.own_many = takes_many(p.max_qlen);
  w.shared_many = p.num_prefixes > 0 && takes_many(p.max_prefix_q);
  const long long own_rows = w.own_many ? 0 : p.max_qlen * group, shared_rows = p.num_prefixes == 0 || w.shared_many ? 0 : p.max_prefix_q * group;
  w.few.tile_rows = std::max(own_rows, shared_rows) <= 8 ? 8 : 16;
  (w.own_many ? w.many : w.few).from_own = p.batch;
  (w.shared_many ? w.many : w.few).from_prefix = p.num_prefixes;
  AttendList* const lists[2] = {&w.few, &w.many};
  long long units[2];
  for (int i = 0; i < 2; ++i) {
    units[i] = most_units(p, cache, *lists[i], lists[i]->from_own, p.max_qlen, p.max_kv_len) +
               most_units(p, cache, *lists[i], lists[i]->from_prefix, p.max_prefix_q, p.max_prefix_len);
    w.fits &= units[i] < INT_MAX;
  }
  // Where both kernels run, they do so side by side, the SMs shared out by what their units cost by the host's bounds (one behind the other, each is a start of
  // 6 to 8 us and an end: 32 answers on a shared 16,384-token prefix 46.5 us instead of 40.4 at that step; 41.6 now).
  int sms[2] = {kNumSMs, kNumSMs};
  if (units[0] > 0 && units[1] > 0) {
    const double few = (double)units[0] * kFewUnitCost, many = (double)units[1] * kManyUnitCost;
    sms[0] = std::min(kNumSMs - 8, std::max(8, (int)(kNumSMs * few / (few + many))));
    sms[1] = kNumSMs - sms[0];
  }
  for (int i = 0; i < 2; ++i) {
    AttendList& list = *lists[i];
    list.grid = (int)std::max(1ll, std::min(units[i], (long long)sms[i]));
    const size_t parts = list.entries() > 0 ? (size_t)list.grid * 2 * list.tile_rows : 0;
    w.ahead[i] = carve((size_t)(list.entries() + 1) * sizeof(int32_t));
    w.out[i] = carve(parts * cache.head_dim * sizeof(float));
    w.lse[i] = carve(parts * sizeof(float));
  }
  w.copies = carve(w.many.entries() > many_listed(cache.head_dim) ? (size_t)w.many.grid * (w.many.entries() + 1) * sizeof(int32_t) : 0);
  w.scratch = carve(w.few.entries() > 0 ? few_scratch_floats(w.few, cache.head_dim) * sizeof(float) : 0);
  const size_t rows = p.num_prefixes > 0 ? (size_t)2 * p.total_q * p.num_q_heads : 0;
  w.whole_out = carve(rows * cache.head_dim * sizeof(float));
  w.whole_lse = carve(rows * sizeof(float));
  w.ended = carve(sizeof(uint64_t));
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
  // a stack of query rows and the rows of all heads are 32-bit counts, and a stacked row times G is (query_row)
  const long long group = p->num_q_heads / cache->num_kv_heads;
  if ((long long)p->total_q * p->num_q_heads > INT_MAX / 2 || (double)p->total_q * group * group >= 4294967296.0) return FASTAV_ERR_UNSUPPORTED;
  return make_plan(*p, *cache).fits ? FASTAV_OK : FASTAV_ERR_UNSUPPORTED;
}

}  // namespace

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
  c.group_magic = c.group > 1 ? (unsigned)((0x100000000ull + c.group - 1) / c.group) : 0;
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
  c.whole_lse = reinterpret_cast<float*>(ws + w.whole_lse);
  AttendList lists[2] = {w.few, w.many};
  for (int i = 0; i < 2; ++i) {
    lists[i].ahead = reinterpret_cast<int32_t*>(ws + w.ahead[i]);
    lists[i].part_out = reinterpret_cast<float*>(ws + w.out[i]);
    lists[i].part_lse = reinterpret_cast<float*>(ws + w.lse[i]);
  }
  lists[0].scratch = reinterpret_cast<float*>(ws + w.scratch);
  lists[1].copies = reinterpret_cast<int32_t*>(ws + w.copies);
  const AttendList &own = lists[w.own_many], &shared = lists[w.shared_many];
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  c.beside = lists[0].entries() > 0 && lists[1].entries() > 0;
  lists[1].through_l2 = c.beside;
  c.ended = reinterpret_cast<uint64_t*>(ws + w.ended);
  c.ticket = 0xFA57A77E00000000ull + (uint64_t)fastav_kernel_launches();  // another for every call
  if (lists[0].entries() > 0) e = launch_attend_few(c, lists[0], st);
  if (e == cudaSuccess && lists[1].entries() > 0) e = launch_attend_many(c, lists[1], st);
  if (e != cudaSuccess) return cuda_failed(e);
  e = c.cache.dim == 128 ? launch_join<128>(c, own, shared, st) : launch_join<64>(c, own, shared, st);
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}
