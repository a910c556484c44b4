// fastav_cache_weigh: what query rows pay to each cached token, summed up per KV head.
//
// A token's weight is a sum over query rows of exp(scale q.k - lse): with the rows' log-sum-exp given, tokens are independent of one another, so K's codes
// are read once, and tokens of different blocks have nothing to join.  Bound by reading the codes where rows are few: 8 heads of 4 x 16,384 tokens, one query row of 32
// heads, 73 MB: 19.0 us a call (3.9 TB/s), of which some 15 the kernel; 32 sequences of 512 to 4,096 tokens 12.3 us.  Three blocks of 168 registers an SM; with
// more than 8 stacked rows of 128 elements the compiler spills 8 to 44 bytes a thread.
#include <limits.h>

#include <algorithm>
#include <cmath>

#include "attend_8bit.cuh"
#include "weigh.cuh"

namespace fastav {
namespace {

// Stacked rows that the kernel for few takes; beyond, the kernel for many (which then is as quick or quicker: us, this one with up to 32 rows / that one: 20 rows on
// 4 x 16,384 tokens of 8 heads 44 / 41, on one sequence of 1,000 14.4 / 12.4; 21 rows on 16 x 3,000 of 4 heads 22.6 / 24.6; 12 rows on 4 x 16,384 29 / 41).
constexpr int kMostFew = 16;
constexpr int kWarps = 4, kThreads = 32 * kWarps, kUnit = 32;  // keys of a unit

// 16 stacked rows (query rows times G) at once, more by turns.  mma.sync with the keys as rows, S^T = K Q^T, the codes from global memory straight to
// the registers of the operand: the contraction may run over head_dim in any order, so lane 4 n + t holds, of query row n and of keys n and n + 8, the
// elements DIM / 4 t ..
//
// A TASK is a run of units of one KV head; every warp has one (or, with many short sequences, several).  How long a run has to be for all of them to fit into one wave of
// blocks comes from the lengths themselves: by the host's bounds, ragged sequences leave warps without work (32 of 512 to 4,096 tokens: 12.6 us).
template <int DIM>
constexpr int kBlocksPerSm = DIM == 128 ? 3 : 4;  // (4 and 5 of up to 8 rows: no quicker, and registers spill)

// ONE_LOOK: 32 sequences or fewer, whose bounds a warp looks at once.
template <int DIM, bool FP8, int NT, bool ONE_LOOK>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm<DIM>)
weigh_few_kernel(WeighCall c) {
  constexpr int kSteps = DIM / 16, kPieces = DIM / 64, kTile = 8 * NT;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n8 = lane >> 2, t4 = lane & 3;
  pdl_wait();  // everything may be what earlier work wrote

  // ---- the tasks: every warp finds its own, a lane per sequence, 32 sequences at a time ----
  auto units_at = [&](int b) { return b < c.batch ? (min(max(chain_load_cached(c.lens + b), 0), c.max_len) + kUnit - 1) / kUnit : 0; };
  auto fresh_at = [&](int b) { return c.decay == 0.f ? 0 : c.weighed ? chain_load_cached(c.weighed + b) : INT_MAX; };  // tokens from here on have no weight yet
  WeighSpan seq{0, 0, 0, false};  // up to 32 sequences: of sequence `lane`, asked for beside its length
  int seq_fresh = 0;
  if (ONE_LOOK && lane < c.batch) {
    seq = weigh_span(c, lane);
    seq_fresh = fresh_at(lane);
  }
  int units = ONE_LOOK ? (seq.len + kUnit - 1) / kUnit : units_at(lane);
  long long all = units;
  if (!ONE_LOOK)
#pragma unroll 4
    for (int b = 32 + lane; b < c.batch; b += 32) all += units_at(b);
#pragma unroll
  for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, d);
  if (blockIdx.x == 0 && warp == 0) {
    bool bad = seq.bad;
    if (!ONE_LOOK)
      for (int b = lane; b < c.batch; b += 32) bad |= weigh_span(c, b).bad;
    if (bad && c.device_status) atomicOr(c.device_status, FASTAV_DEV_SHAPE_MISMATCH);
  }
  const long long warps = (long long)gridDim.x * kWarps, room = max(warps - (long long)c.batch * c.cache.hkv, (warps + 1) / 2);
  const int run = (int)max(1ll, (all * c.cache.hkv + room - 1) / room);  // tasks: units / run, and less than one more for each sequence and head
  int b0 = 0, ahead = 0;  // tasks of the sequences before b0
  for (int task = blockIdx.x * kWarps + warp;; task += gridDim.x * kWarps) {
    int own_tasks, upto;
    unsigned behind;
    for (;;) {  // to the 32 sequences one of which has the task
      own_tasks = c.cache.hkv * ((units + run - 1) / run);
      upto = own_tasks;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= d) upto += x;
      }
      behind = __ballot_sync(0xFFFFFFFFu, ahead + upto > task);
      if (behind) break;
      ahead += __shfl_sync(0xFFFFFFFFu, upto, 31);
      b0 += 32;
      if (ONE_LOOK || b0 >= c.batch) return;
      units = units_at(b0 + lane);
    }
    const int at = __ffs(behind) - 1, b = b0 + at;
    WeighSpan s{__shfl_sync(0xFFFFFFFFu, seq.row0, at), __shfl_sync(0xFFFFFFFFu, seq.rows, at), __shfl_sync(0xFFFFFFFFu, seq.len, at), false};
    int fresh = __shfl_sync(0xFFFFFFFFu, seq_fresh, at);
    if (!ONE_LOOK) {
      s = weigh_span(c, b);
      fresh = fresh_at(b);
    }
    const int all_units = __shfl_sync(0xFFFFFFFFu, units, at), per_head = (all_units + run - 1) / run, in_seq = task - ahead - __shfl_sync(0xFFFFFFFFu, upto - own_tasks, at);
    const int head = in_seq / per_head, u0 = (in_seq - head * per_head) * run, u1 = min(u0 + run, all_units);
    pdl_trigger();
    const int stacked = s.rows * c.group;

    // Lane's key of a unit is key0 + lane for page, scale and weight; pages hold 16 tokens or more, so sixteen lanes have one page.
    struct Unit {
      uint4 a[2][kPieces], d[2][kPieces];  // of 16 keys h: key n8, key n8 + 8
      long long at;                        // row of the pool; -1: none
      float scale, before;
    };
    const int32_t* const pages = c.table + (long long)b * c.table_stride;
    auto page_entry = [&](int u) { return u < u1 && u * kUnit + lane < s.len ? chain_load_cached(pages + (u * kUnit + lane >> c.cache.page_shift)) : -1; };
    auto ask = [&](int u, int page, bool again, Unit& x) {
      const int key = u * kUnit + lane;
      const bool there = (unsigned)page < (unsigned)c.cache.num_pages;
      if (!there && key < s.len && c.device_status) atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
      x.at = there ? pool_row(c.cache, page, head, key) : -1;
      const long long at = there ? x.at : 0;  // (keys that are none read the pool's first rows: in bounds)
      x.scale = chain_load(c.cache.k_scale + at);
      x.before = there && (again || key < fresh) ? chain_load(c.weights + at) : 0.f;
      const long long half_row[2] = {__shfl_sync(0xFFFFFFFFu, at, 0), __shfl_sync(0xFFFFFFFFu, at, 16)};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          const uint8_t* const from = c.cache.k + (half_row[h] + n8) * DIM + (t4 * kPieces + p) * 16;
          x.a[h][p] = chain_load(reinterpret_cast<const uint4*>(from));
          x.d[h][p] = chain_load(reinterpret_cast<const uint4*>(from + 8 * DIM));
        }
    };

    for (int row0 = 0; row0 == 0 || row0 < stacked; row0 += kTile) {
      int page = page_entry(u0);
      // The query rows, asked for beside the first page; the first keys are on their way while they become operands.
      uint32_t x[NT][kSteps * 2];
      float own_lse[NT];
#pragma unroll
      for (int g = 0; g < NT; ++g) {
        const int i = row0 + 8 * g + n8;
        const bool there = i < stacked;
        const int r = there ? i / c.group : 0, query_head = head * c.group + i - r * c.group;
        const uint4* const from = reinterpret_cast<const uint4*>(c.q + (long long)(s.row0 + r) * c.q_st + (long long)query_head * c.q_sh + t4 * (DIM / 4));
#pragma unroll
        for (int j = 0; j < kSteps / 2; ++j) {
          const uint4 v = there ? chain_load(from + j) : make_uint4(0, 0, 0, 0);
          x[g][4 * j] = v.x; x[g][4 * j + 1] = v.y; x[g][4 * j + 2] = v.z; x[g][4 * j + 3] = v.w;
        }
        own_lse[g] = there ? chain_load(c.lse + (long long)(s.row0 + r) * c.hq + query_head) : -INFINITY;
      }
      Unit now, next;
      ask(u0, page, row0 > 0, now);
      page = page_entry(u0 + 1);
      uint32_t qf[NT][kSteps][2];
      float row_scale[NT][2], lse[NT][2];  // of rows 2 t4 + (0, 1)
      int sees[NT][2];
#pragma unroll
      for (int g = 0; g < NT; ++g) {
        const int i = row0 + 8 * g + n8, r = i < stacked ? i / c.group : 0;
        unsigned top = 0;  // bf16 bits of the largest magnitude; what is not a number is larger still
#pragma unroll
        for (int j = 0; j < kSteps * 2; ++j) top = __vmaxu2(top, x[g][j] & 0x7FFF7FFFu);
        top = max(top >> 16, top & 0xFFFFu);
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const float to = query_power(top);
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t v = x[g][2 * k + half];
            qf[g][k][half] = two_f16(__uint_as_float(v << 16) * to, __uint_as_float(v & 0xFFFF0000u) * to);
          }
        const int own_sees = own_lse[g] == -INFINITY ? 0 : c.causal ? max(0, s.len - s.rows + r + 1) : s.len;
#pragma unroll
        for (int e = 0; e < 2; ++e) {  // of row n8 -> of rows 2 t4 + e
          const int of = 4 * (2 * t4 + e);
          row_scale[g][e] = query_scale(c.scale_log2, __shfl_sync(0xFFFFFFFFu, to, of));
          lse[g][e] = __shfl_sync(0xFFFFFFFFu, own_lse[g], of) * kLog2e;
          sees[g][e] = __shfl_sync(0xFFFFFFFFu, own_sees, of);
        }
      }

      auto weigh = [&](int u, const Unit& k) {
        const int key0 = u * kUnit;
        float z[NT][2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int g = 0; g < NT; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[g][h][i] = 0.f;
#pragma unroll
          for (int p = 0; p < kPieces; ++p) {
            const uint32_t wa[4] = {k.a[h][p].x, k.a[h][p].y, k.a[h][p].z, k.a[h][p].w}, wb[4] = {k.d[h][p].x, k.d[h][p].y, k.d[h][p].z, k.d[h][p].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t a0, a1, a2, a3;
              four_codes<FP8>(wa[i], a0, a2);
              four_codes<FP8>(wb[i], a1, a3);
#pragma unroll
              for (int g = 0; g < NT; ++g) mma_f16(z[g][h], a0, a1, a2, a3, qf[g][4 * p + i][0], qf[g][4 * p + i][1]);
            }
          }
        }
        const float own_scale = k.scale * kKeyScaleFactor;
        float paid[4];  // to keys n8 + 8 i by the rows of this lane
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float scale = __shfl_sync(0xFFFFFFFFu, own_scale, 8 * i + n8);
          paid[i] = 0.f;
#pragma unroll
          for (int g = 0; g < NT; ++g)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float p = ptx::ex2_approx(fmaf(z[g][i / 2][i % 2 * 2 + e] * scale, row_scale[g][e], -lse[g][e]));
              paid[i] += key0 + 8 * i + n8 < sees[g][e] ? p : 0.f;
            }
          paid[i] += __shfl_xor_sync(0xFFFFFFFFu, paid[i], 1);
          paid[i] += __shfl_xor_sync(0xFFFFFFFFu, paid[i], 2);
        }
        // lane 4 n + t has the sums of keys n + 8 i: lane 8 i + n takes its own from lane 4 n
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = __shfl_sync(0xFFFFFFFFu, paid[i], 4 * (lane & 7));
          if (lane >> 3 == i) sum = x;
        }
        if (k.at >= 0) c.weights[k.at] = fmaf(row0 > 0 ? 1.f : c.decay, k.before, sum);
      };
      // A unit is asked for while the one before is weighed, its page a unit earlier still.
      for (int u = u0;;) {
        if (u + 1 < u1) {
          ask(u + 1, page, row0 > 0, next);
          page = page_entry(u + 2);
        }
        weigh(u, now);
        if (++u >= u1) break;
        if (u + 1 < u1) {
          ask(u + 1, page, row0 > 0, now);
          page = page_entry(u + 2);
        }
        weigh(u, next);
        if (++u >= u1) break;
      }
    }
  }
}

template <int DIM, bool FP8, int NT>
cudaError_t launch_few(const WeighCall& c, cudaStream_t stream) {
  const long long units = ((long long)c.max_len + kUnit - 1) / kUnit, blocks = (units * c.cache.hkv * c.batch + kWarps - 1) / kWarps, most = (long long)kNumSMs * kBlocksPerSm<DIM>;
  count_launches(1);
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  return c.batch <= 32 ? launch_chained(weigh_few_kernel<DIM, FP8, NT, true>, grid, dim3(kThreads), 0, stream, c)
                       : launch_chained(weigh_few_kernel<DIM, FP8, NT, false>, grid, dim3(kThreads), 0, stream, c);
}
template <int NT>
cudaError_t launch_few(const WeighCall& c, cudaStream_t stream) {
  if (c.cache.dim == 128) return c.cache.fp8 ? launch_few<128, true, NT>(c, stream) : launch_few<128, false, NT>(c, stream);
  return c.cache.fp8 ? launch_few<64, true, NT>(c, stream) : launch_few<64, false, NT>(c, stream);
}

}  // namespace
}  // namespace fastav

using namespace fastav;

extern "C" int32_t fastav_cache_weigh(const fastav_attend_params* p, const fastav_cache* cache, float* weights, float decay, const void* q, const float* lse,
                                      const int32_t* cu_qlens, const int32_t* page_table, const int32_t* kv_lens, const int32_t* weighed_lens_opt,
                                      int32_t* device_status, void* stream) {
  int32_t rc = check_cache(cache);
  if (rc != FASTAV_OK) return rc;
  if (!p || p->batch < 1 || p->total_q < 0 || p->max_qlen < 0 || p->max_qlen > p->total_q || p->max_kv_len < 0) return FASTAV_ERR_INVALID_ARG;
  if (p->num_q_heads < 1 || p->num_q_heads % cache->num_kv_heads != 0) return FASTAV_ERR_INVALID_ARG;
  if (!(decay >= 0.f && std::isfinite(decay))) return FASTAV_ERR_INVALID_ARG;
  if (!weights || !cu_qlens || !kv_lens) return FASTAV_ERR_INVALID_ARG;
  if (p->max_kv_len > 0 && (!page_table || p->table_stride < 1)) return FASTAV_ERR_INVALID_ARG;
  if (p->total_q > 0 && (!q || !lse)) return FASTAV_ERR_INVALID_ARG;
  if (p->batch > FASTAV_ATTEND_MAX_BATCH || (long long)p->total_q * p->num_q_heads > INT_MAX / 2) return FASTAV_ERR_UNSUPPORTED;
  if ((rc = check_strides(p->q_stride_tok, p->q_stride_head, p->num_q_heads, cache->head_dim)) != FASTAV_OK) return rc;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(weights)) & 15u) return FASTAV_ERR_UNSUPPORTED;
  if (p->max_kv_len == 0) return FASTAV_OK;
  chain_begin(p->flags);
  WeighCall c{};
  c.cache = make_view(*cache);
  c.weights = weights;
  c.decay = decay;
  c.batch = p->batch; c.total_q = p->total_q; c.max_qlen = p->max_qlen; c.hq = p->num_q_heads; c.group = p->num_q_heads / cache->num_kv_heads;
  c.max_len = (int)std::min((long long)p->max_kv_len, (long long)p->table_stride << c.cache.page_shift); c.table_stride = p->table_stride;
  c.q_st = p->q_stride_tok; c.q_sh = p->q_stride_head;
  c.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / std::sqrt((float)cache->head_dim)) * kLog2e;
  c.causal = (p->flags & FASTAV_CAUSAL) != 0;
  c.q = static_cast<const uint16_t*>(q);
  c.lse = lse;
  c.cu_qlens = cu_qlens; c.table = page_table; c.lens = kv_lens; c.weighed = weighed_lens_opt;
  c.device_status = device_status;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const long long stacked = (long long)c.max_qlen * c.group;
  cudaError_t e = cudaSuccess;
  bool used = false;
  if (stacked > kMostFew && weigh_many_applies(c)) e = launch_weigh_many(c, st, &used);
  if (!used) e = stacked <= 8 ? launch_few<1>(c, st) : launch_few<2>(c, st);
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}
