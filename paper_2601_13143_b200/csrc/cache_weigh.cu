// fastav_cache_weigh: what query rows pay to each cached token, summed up per KV head.
//
// A token's weight is a sum over query rows of exp(scale q.k - lse): with the rows' log-sum-exp given, tokens are independent of one another, so K's codes
// are read once, nothing is joined and sums have one order.  Bound by reading the codes where rows are few.
#include <limits.h>

#include <algorithm>
#include <cmath>

#include "attend_8bit.cuh"
#include "weigh.cuh"

namespace fastav {
namespace {

constexpr int kMostFew = 16;  // stacked rows; beyond, the kernel for many
constexpr int kWarps = 4, kThreads = 32 * kWarps, kUnit = 32;  // keys of a unit

// Up to 16 stacked rows (query rows times G) at once, more by turns.  A warp has a run of units of one KV head; mma.sync with the keys as rows, S^T = K Q^T, the codes
// from global memory straight to the registers of the operand: the contraction may run over head_dim in any order, so lane 4 n + t holds, of query row
// n and of keys n and n + 8, the elements DIM / 4 t ..
template <int DIM, bool FP8, int NT>
__global__ void __launch_bounds__(kThreads)
weigh_few_kernel(WeighCall c, int run) {
  constexpr int kSteps = DIM / 16, kPieces = DIM / 64, kTile = 8 * NT;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n8 = lane >> 2, t4 = lane & 3;
  const int b = blockIdx.z, head = blockIdx.y;
  if (c.head_wait) pdl_wait();
  pdl_trigger();
  pdl_wait();
  const WeighSpan s = weigh_span(c, b);
  if (s.bad && blockIdx.x == 0 && head == 0 && threadIdx.x == 0 && c.device_status) atomicOr(c.device_status, FASTAV_DEV_SHAPE_MISMATCH);
  const int u0 = (blockIdx.x * kWarps + warp) * run, u1 = min(u0 + run, (s.len + kUnit - 1) / kUnit);
  if (u0 >= u1) return;
  const int stacked = s.rows * c.group;
  const int fresh = c.decay == 0.f ? 0 : c.weighed ? chain_load_cached(c.weighed + b) : s.len;  // tokens from here on have no weight yet

  for (int row0 = 0; row0 == 0 || row0 < stacked; row0 += kTile) {
    uint32_t qf[NT][kSteps][2];
    float row_scale[NT][2], lse[NT][2];  // of rows 2 t4 + (0, 1)
    int sees[NT][2];
#pragma unroll
    for (int g = 0; g < NT; ++g) {
      const int i = row0 + 8 * g + n8;
      const bool there = i < stacked;
      const int r = there ? i / c.group : 0, query_head = head * c.group + i - r * c.group;
      uint32_t x[kSteps * 2];
      const uint4* const from = reinterpret_cast<const uint4*>(c.q + (long long)(s.row0 + r) * c.q_st + (long long)query_head * c.q_sh + t4 * (DIM / 4));
      unsigned top = 0;  // bf16 bits of the largest magnitude; what is not a number is larger still
#pragma unroll
      for (int j = 0; j < kSteps / 2; ++j) {
        const uint4 v = there ? chain_load(from + j) : make_uint4(0, 0, 0, 0);
        x[4 * j] = v.x; x[4 * j + 1] = v.y; x[4 * j + 2] = v.z; x[4 * j + 3] = v.w;
      }
#pragma unroll
      for (int j = 0; j < kSteps * 2; ++j) top = __vmaxu2(top, x[j] & 0x7FFF7FFFu);
      top = max(top >> 16, top & 0xFFFFu);
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      const float to = query_power(top);
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t v = x[2 * k + half];
          qf[g][k][half] = two_f16(__uint_as_float(v << 16) * to, __uint_as_float(v & 0xFFFF0000u) * to);
        }
      const float own_lse = there ? chain_load(c.lse + (long long)(s.row0 + r) * c.hq + query_head) : -INFINITY;
      const int own_sees = own_lse == -INFINITY ? 0 : c.causal ? max(0, s.len - s.rows + r + 1) : s.len;
#pragma unroll
      for (int e = 0; e < 2; ++e) {  // of row n8 -> of rows 2 t4 + e
        const int of = 4 * (2 * t4 + e);
        row_scale[g][e] = query_scale(c.scale_log2, __shfl_sync(0xFFFFFFFFu, to, of));
        lse[g][e] = __shfl_sync(0xFFFFFFFFu, own_lse, of) * kLog2e;
        sees[g][e] = __shfl_sync(0xFFFFFFFFu, own_sees, of);
      }
    }

    for (int u = u0; u < u1; ++u) {
      const int key0 = u * kUnit;
      // Lane's key is key0 + lane for page, scale and weight; pages hold 16 tokens or more, so sixteen lanes have one page.
      const bool mine = key0 + lane < s.len;
      const int page = mine ? page_of(c.cache, c.table, c.table_stride, b, key0 + lane) : -1;
      if (mine && page < 0 && c.device_status) atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
      const long long at = page < 0 ? 0 : pool_row(c.cache, page, head, key0 + lane);
      const float own_scale = page < 0 ? 0.f : chain_load(c.cache.k_scale + at) * kKeyScaleFactor;
      const float before = page >= 0 && (row0 > 0 || key0 + lane < fresh) ? chain_load(c.weights + at) : 0.f;
      const long long half_row[2] = {__shfl_sync(0xFFFFFFFFu, at, 0), __shfl_sync(0xFFFFFFFFu, at, 16)};
      uint4 a[2][kPieces], d[2][kPieces];  // of 16 keys h: key n8, key n8 + 8
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          const uint8_t* const from = c.cache.k + (half_row[h] + n8) * DIM + (t4 * kPieces + p) * 16;
          a[h][p] = chain_load(reinterpret_cast<const uint4*>(from));
          d[h][p] = chain_load(reinterpret_cast<const uint4*>(from + 8 * DIM));
        }
      float z[NT][2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int g = 0; g < NT; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) z[g][h][i] = 0.f;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
          const uint32_t wa[4] = {a[h][p].x, a[h][p].y, a[h][p].z, a[h][p].w}, wb[4] = {d[h][p].x, d[h][p].y, d[h][p].z, d[h][p].w};
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
      if (page >= 0) c.weights[at] = fmaf(row0 > 0 ? 1.f : c.decay, before, sum);
    }
  }
}

template <int NT>
cudaError_t launch_few(const WeighCall& c, cudaStream_t stream) {
  // Runs as short as fill the SMs with 16 warps each.
  const long long units = (c.max_len + kUnit - 1) / kUnit, all = units * c.cache.hkv * c.batch;
  const int run = (int)max(1ll, min(all / (kNumSMs * 16), 64ll));
  const dim3 grid((unsigned)((units + (long long)run * kWarps - 1) / ((long long)run * kWarps)), c.cache.hkv, c.batch);
  auto go = [&](auto kernel) { return launch_chained(kernel, grid, dim3(kThreads), 0, stream, c, run); };
  count_launches(1);
  if (c.cache.dim == 128) return c.cache.fp8 ? go(weigh_few_kernel<128, true, NT>) : go(weigh_few_kernel<128, false, NT>);
  return c.cache.fp8 ? go(weigh_few_kernel<64, true, NT>) : go(weigh_few_kernel<64, false, NT>);
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
