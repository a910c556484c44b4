// K and V rows into the 8-bit cache and back (fastav_cache_write, fastav_cache_read).
//
// Both are bound by HBM: a row of d values moves 2 d bytes on one side and d + 4 on the other.  A block takes a few consecutive rows
// of the packed side: one thread per token finds its sequence, its token on either side and its page; then d / 8 lanes take a head of K
// or V each, eight values of a row per lane, several tokens' loads in flight.
#include <limits.h>

#include "cache.cuh"

namespace fastav {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;     // rows that a thread has in flight
constexpr int kMostTokens = 32;  // of a block

struct RowsCall {
  CacheView cache;
  int batch, total_src, total_dst, max_src;  // packed source rows; rows that move (at most); longest sequence of the source
  int table_stride, tokens;                  // tokens per block
  long long k_st, k_sh, v_st, v_sh;          // of the bf16 side
  bool global_idx;
  int head_wait;
};
inline void mark_head(RowsCall& c, bool head) { c.head_wait = head ? 1 : 0; }

// The largest magnitude of eight bf16 values, twice; what is not a number is larger than everything else.
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) {
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
  return a;
}
__device__ __forceinline__ unsigned magnitudes(unsigned a) {
  asm("abs.bf16x2 %0, %0;" : "+r"(a));
  return a;
}
__device__ __forceinline__ unsigned top_of(const uint4& x) { return larger(larger(magnitudes(x.x), magnitudes(x.y)), larger(magnitudes(x.z), magnitudes(x.w))); }

// code_i = round(x_i L / top) to nearest, ties to even, exactly.  x_i L has at most 15 bits, so it is exact in fp32, and the quotient of a
// 15-bit and an 8-bit number that is no tie is at least 2^-16 of itself away from one.  Everything is scaled by a power of two that brings
// `top` near 1 (and leaves room for L), so that nothing overflows and 1 / top is normal.
//
// An approximate quotient corrected once by its remainder (q + (n - q t) / t: an ulp off at most, and exact where the quotient is short)
// rounds as the true one does.
struct Quotient {
  float2 to, less, r;  // L times the power of two; -top times it; the reciprocal of that
  __device__ Quotient(unsigned top, float largest) {
    const int e = (int)(top >> 7);
    const float power = __uint_as_float((unsigned)min(max(254 - e, 1), 240) << 23), t = top ? __uint_as_float(top << 16) * power : 1.f, inv = __fdividef(1.f, t);
    to = make_float2(power * largest, power * largest);
    less = make_float2(-t, -t);
    r = make_float2(inv, inv);
  }
  __device__ float2 operator()(const float2& two) const {
    const float2 n = __fmul2_rn(two, to), q = __fmul2_rn(n, r);
    return __ffma2_rn(__ffma2_rn(q, less, n), r, q);
  }
};
// int8, in one step: x times L / top rounded UP.  A quotient that is no tie is not moved across one.  A tie, 254 x = (2 k + 1) top, needs 127
// to divide 2 k + 1 or top's eight bits: then it is 63.5, which goes up to 64, or top is 254 times a power of two and 127 / top and
// every product are exact.  So one fused multiply-add with 1.5 * 2^23 leaves the code in the sum's low bits.  (Not where L / top is too large.)
constexpr unsigned kLeastTop = 0x1000;  // 2^-95
__device__ __forceinline__ float inverse_up(unsigned top) {
  const int e = (int)(top >> 7);
  const float power = __uint_as_float((unsigned)max(254 - e, 1) << 23), t = __uint_as_float(top << 16) * power, inv = __fdividef(1.f, t);
  float x = 127.f * inv;
  x = fmaf(fmaf(-x, t, 127.f), inv, x);                                           // within an ulp
  const float below = __uint_as_float(__float_as_uint(x) - 1);
  if (fmaf(-x, t, 127.f) > 0.f) x = __uint_as_float(__float_as_uint(x) + 1);      // (the remainders are exact)
  else if (fmaf(-below, t, 127.f) <= 0.f) x = below;
  return x * power;
}
// top / L, to nearest: a quotient within an ulp, corrected by its exact remainder times the nearest reciprocal (Markstein), where the remainder is normal.
template <bool FP8>
__device__ __forceinline__ float scale_of(unsigned top) {
  constexpr float kLargest = FP8 ? 448.f : 127.f, kInverse = 1.f / kLargest;
  const float t = __uint_as_float(top << 16);
  if (top < kLeastTop) return __fdiv_rn(t, kLargest);
  const float q = t * kInverse;
  return fmaf(fmaf(-q, kLargest, t), kInverse, q);
}

__device__ __forceinline__ unsigned low_bytes(const float2& a, const float2& b) {
  return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
}
__device__ __forceinline__ unsigned pack_e4m3(const float2& a, const float2& b) {
  unsigned short lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(a.y), "f"(a.x));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(b.y), "f"(b.x));
  return (unsigned)lo | (unsigned)hi << 16;
}

__device__ __forceinline__ float2 both(unsigned two) { return make_float2(__uint_as_float(two << 16), __uint_as_float(two & 0xFFFF0000u)); }
template <bool FP8>
__device__ __forceinline__ uint2 quantise8(const uint4& x, unsigned top) {
  if (FP8) {
    const Quotient q(top, 448.f);
    return make_uint2(pack_e4m3(q(both(x.x)), q(both(x.y))), pack_e4m3(q(both(x.z)), q(both(x.w))));
  }
  const float2 round = make_float2(12582912.f, 12582912.f);
  if (top < kLeastTop) {
    const Quotient q(top, 127.f);
    return make_uint2(low_bytes(__fadd2_rn(q(both(x.x)), round), __fadd2_rn(q(both(x.y)), round)), low_bytes(__fadd2_rn(q(both(x.z)), round), __fadd2_rn(q(both(x.w)), round)));
  }
  const float up = inverse_up(top);
  const float2 r = make_float2(up, up);
  return make_uint2(low_bytes(__ffma2_rn(both(x.x), r, round), __ffma2_rn(both(x.y), r, round)), low_bytes(__ffma2_rn(both(x.z), r, round), __ffma2_rn(both(x.w), r, round)));
}

// Two e4m3 codes as floats.
__device__ __forceinline__ float2 two_e4m3(unsigned short pair) {
  unsigned h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(pair));
  float lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
  return make_float2(lo, hi);
}
__device__ __forceinline__ unsigned two_bf16(float lo, float hi) {
  unsigned r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool FP8>
__device__ __forceinline__ uint4 dequantise8(const uint2& x, float scale) {
  unsigned out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned w = (i < 2 ? x.x : x.y) >> (i % 2 * 16);
    const float2 c = FP8 ? two_e4m3((unsigned short)w) : make_float2((float)(signed char)w, (float)(signed char)(w >> 8));
    out[i] = two_bf16(c.x * scale, c.y * scale);
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

// WRITE: bf16 rows -> cache; else back.  `cu`: prefix sums of the rows that move (the keep list's, or the sequences' own).
template <int DIM, bool FP8, bool WRITE>
__global__ void __launch_bounds__(kThreads, WRITE ? 4 : 5)
cache_rows_kernel(RowsCall c, uint16_t* __restrict__ k, uint16_t* __restrict__ v, const int32_t* __restrict__ cu_seqlens,
                  const int32_t* __restrict__ keep_idx, const int32_t* __restrict__ cu, const int32_t* __restrict__ table,
                  const int32_t* __restrict__ start, int32_t* device_status) {
  constexpr int kLanes = DIM / 8, kRows = kThreads / kLanes;  // lanes of a row; rows at a time
  __shared__ long long packed_row[kMostTokens];  // of the bf16 side, -1: left out
  __shared__ long long cache_row[kMostTokens];   // of the pool, head 0
  chain_enter(c);
  pdl_wait();  // everything may be what earlier work wrote
  pdl_acquire(k);
  pdl_acquire(v);
  pdl_acquire(cu_seqlens);
  pdl_acquire(keep_idx);
  pdl_acquire(cu);
  pdl_acquire(table);
  pdl_acquire(start);
  const int first = blockIdx.x * c.tokens, tokens = min(c.tokens, min(c.total_dst, chain_load_cached(cu + c.batch)) - first);
  if (blockIdx.x == 0 && threadIdx.x == 0 && device_status && chain_load_cached(cu + c.batch) > c.total_dst) atomicOr(device_status, FASTAV_DEV_SHAPE_MISMATCH);
  if ((int)threadIdx.x < tokens) {
    const int row = first + threadIdx.x;
    int lo = 0, hi = c.batch;  // largest b with cu[b] <= row
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (chain_load_cached(cu + mid) <= row) lo = mid; else hi = mid;
    }
    const int i = row - chain_load_cached(cu + lo);
    long long src = row;
    int bad = 0;
    if (keep_idx) {
      const Span seq = checked_span<true>(cu_seqlens, lo, c.total_src, c.max_src);
      const int idx = chain_load(keep_idx + row);
      src = (c.global_idx ? 0ll : (long long)seq.first) + idx;
      if (src < seq.first || src >= seq.first + seq.count) bad = FASTAV_DEV_BAD_INDEX;
    }
    const long long token = (long long)(start ? chain_load_cached(start + lo) : 0) + i;
    long long at = 0;
    if (i < 0 || token < 0 || token >= (long long)c.table_stride << c.cache.page_shift || token > INT_MAX) {
      bad |= FASTAV_DEV_SHAPE_MISMATCH;
    } else {
      const int page = page_of(c.cache, table, c.table_stride, lo, (int)token);
      if (page < 0) bad |= FASTAV_DEV_BAD_INDEX;
      else at = pool_row(c.cache, page, 0, (int)token);
    }
    packed_row[threadIdx.x] = bad ? -1 : src;
    cache_row[threadIdx.x] = at;
    if (bad && device_status) atomicOr(device_status, bad);
  }
  __syncthreads();

  // A group of kLanes lanes keeps to one head of K or V and walks over the block's tokens, so that all of an address but the token's row is
  // known beforehand; with fewer heads than groups several of these share a head's tokens.  (Survivors of 4 x 16,384 tokens, int8, 163 MB: 40.5
  // us; without the arithmetic 37: what takes the time is issued per row and address, 0.7 instructions a cycle and scheduler, some 140 of a warp for two
  // rows of 128.  Tried: rows copied into shared memory ahead of their use, 94 us for the ragged batch instead of 65; a
  // warp per few tokens with eight rows unrolled, 102; the scales gathered in shared memory and written head by head, 48.8.)
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes, heads = 2 * c.cache.hkv;
  const int sharing = max(1, kRows / heads), step = min(kRows, heads);
  const bool active = group < sharing * heads;
  // (all lanes of a warp make the same number of turns: they shuffle)
#pragma unroll 1
  for (int h0 = 0; h0 < heads; h0 += step) {
    const int h = h0 + group % step, first_token = group / step;
    const bool is_v = h >= c.cache.hkv, mine = active && h < heads;
    const int head = is_v ? h - c.cache.hkv : h;
    uint16_t* const packed = (is_v ? v : k) + (long long)head * (is_v ? c.v_sh : c.k_sh) + lane * 8;
    const long long stride = is_v ? c.v_st : c.k_st, head_row = (long long)head << c.cache.page_shift;
    uint8_t* const codes = (is_v ? c.cache.v : c.cache.k) + head_row * DIM + lane * 8;
    float* const scales = (is_v ? c.cache.v_scale : c.cache.k_scale) + head_row;
#pragma unroll 1
    for (int t0 = 0; t0 < tokens; t0 += sharing * kUnroll) {
      uint4 wide[kUnroll];
      uint2 narrow[kUnroll];
      float scale[kUnroll];
      long long from[kUnroll], to[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int token = t0 + first_token + u * sharing;
        from[u] = mine && token < tokens ? packed_row[token] : -1;
        if (from[u] < 0) continue;
        to[u] = cache_row[token];
        if (WRITE) {
          wide[u] = chain_load(reinterpret_cast<const uint4*>(packed + from[u] * stride));
        } else {
          narrow[u] = chain_load(reinterpret_cast<const uint2*>(codes + to[u] * DIM));
          scale[u] = chain_load(scales + to[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (WRITE) {
          unsigned top = from[u] < 0 ? 0u : top_of(wide[u]);
#pragma unroll
          for (int d = 1; d < kLanes; d <<= 1) top = larger(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
          if (from[u] < 0) continue;
          top = larger(top, __byte_perm(top, top, 0x1032)) & 0xFFFFu;
          const bool finite = top < 0x7F80u;  // else the codes are 0 (a NaN among them would reach rows that do not see it) and the scale is NaN
          const uint2 c8 = quantise8<FP8>(wide[u], top);
          *reinterpret_cast<uint2*>(codes + to[u] * DIM) = finite ? c8 : make_uint2(0, 0);
          if (lane == 0) scales[to[u]] = finite ? scale_of<FP8>(top) : __uint_as_float(0x7FC00000u);
        } else {
          if (from[u] < 0) continue;
          *reinterpret_cast<uint4*>(packed + from[u] * stride) = dequantise8<FP8>(narrow[u], scale[u]);
        }
      }
    }
  }
}

template <bool WRITE>
cudaError_t launch_rows(RowsCall c, uint16_t* k, uint16_t* v, const int32_t* cu_seqlens, const int32_t* keep_idx, const int32_t* cu, const int32_t* table,
                        const int32_t* start, int32_t* device_status, cudaStream_t stream) {
  // Few rows: a token per block, so that more SMs take part.  Many: as many as keep a group of lanes busy for four turns.
  const int groups = kThreads / (c.cache.dim / 8), sharing = groups > 2 * c.cache.hkv ? groups / (2 * c.cache.hkv) : 1;
  const int most = 4 * kUnroll * sharing < kMostTokens ? 4 * kUnroll * sharing : kMostTokens;
  c.tokens = 1;
  while (2 * c.tokens <= most && c.total_dst / (2 * c.tokens) >= kNumSMs * 2) c.tokens *= 2;
  const dim3 grid((unsigned)((c.total_dst + c.tokens - 1) / c.tokens));
  auto go = [&](auto kernel) { return launch_chained(kernel, grid, dim3(kThreads), 0, stream, c, k, v, cu_seqlens, keep_idx, cu, table, start, device_status); };
  count_launches(1);
  if (c.cache.dim == 128) return c.cache.fp8 ? go(cache_rows_kernel<128, true, WRITE>) : go(cache_rows_kernel<128, false, WRITE>);
  return c.cache.fp8 ? go(cache_rows_kernel<64, true, WRITE>) : go(cache_rows_kernel<64, false, WRITE>);
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// What both directions ask of the shapes.
int32_t check_rows(const fastav_params* p, const fastav_cache* cache, const int32_t* cu_seqlens, const int32_t* page_table, int32_t table_stride,
                   const void* k, const void* v, int64_t k_st, int64_t k_sh, int64_t v_st, int64_t v_sh) {
  int32_t rc = check_cache(cache);
  if (rc != FASTAV_OK) return rc;
  if (!p || p->batch < 1 || p->total_tokens < 0 || p->max_seqlen < 0 || p->max_seqlen > p->total_tokens) return FASTAV_ERR_INVALID_ARG;
  if (p->num_kv_heads != cache->num_kv_heads || p->head_dim != cache->head_dim) return FASTAV_ERR_INVALID_ARG;
  if (!cu_seqlens || !page_table || table_stride < 1) return FASTAV_ERR_INVALID_ARG;
  if (p->total_tokens > 0 && (!k || !v)) return FASTAV_ERR_INVALID_ARG;
  if ((rc = check_strides(k_st, k_sh, p->num_kv_heads, p->head_dim)) != FASTAV_OK) return rc;
  if ((rc = check_strides(v_st, v_sh, p->num_kv_heads, p->head_dim)) != FASTAV_OK) return rc;
  return aligned(k, 16) && aligned(v, 16) ? FASTAV_OK : FASTAV_ERR_UNSUPPORTED;
}

}  // namespace

int32_t check_cache(const fastav_cache* c) {
  if (!c) return FASTAV_ERR_INVALID_ARG;
  if (c->num_pages < 1 || c->num_kv_heads < 1 || !c->k || !c->v || !c->k_scale || !c->v_scale) return FASTAV_ERR_INVALID_ARG;
  if (c->format != FASTAV_CACHE_INT8 && c->format != FASTAV_CACHE_FP8) return FASTAV_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return FASTAV_ERR_UNSUPPORTED;
  if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return FASTAV_ERR_UNSUPPORTED;
  // (128 bytes: a row of codes lies in one line, which fastav_attend calls into L2 by one prefetch per row)
  if (!aligned(c->k, 128) || !aligned(c->v, 128) || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16)) return FASTAV_ERR_UNSUPPORTED;
  // fastav_attend's kernel for many rows counts rows of the pool in 32 bits; with the heads bounded no product of counts here overflows
  if (c->num_kv_heads > 1024 || (long long)c->num_pages * c->num_kv_heads * c->page_tokens > INT_MAX) return FASTAV_ERR_UNSUPPORTED;
  return FASTAV_OK;
}

CacheView make_view(const fastav_cache& c) {
  int shift = 4;
  while ((1 << shift) < c.page_tokens) ++shift;
  return CacheView{static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.k_scale, c.v_scale, c.num_pages, shift, c.num_kv_heads, c.head_dim,
                   c.format == FASTAV_CACHE_FP8};
}

}  // namespace fastav

using namespace fastav;

extern "C" int32_t fastav_cache_write(const fastav_params* p, const fastav_cache* cache, const void* k, const void* v, const int32_t* cu_seqlens,
                                      const int32_t* keep_idx_opt, const int32_t* cu_keep_opt, const int32_t* page_table, int32_t table_stride,
                                      const int32_t* start_opt, int32_t* device_status, void* stream) {
  int32_t rc = p ? check_rows(p, cache, cu_seqlens, page_table, table_stride, k, v, p->k_stride_tok, p->k_stride_head, p->v_stride_tok, p->v_stride_head)
                 : FASTAV_ERR_INVALID_ARG;
  if (rc != FASTAV_OK) return rc;
  if ((keep_idx_opt == nullptr) != (cu_keep_opt == nullptr)) return FASTAV_ERR_INVALID_ARG;
  if (keep_idx_opt && (p->total_keep < 0 || p->total_keep > p->total_tokens)) return FASTAV_ERR_INVALID_ARG;
  const int rows = keep_idx_opt ? p->total_keep : p->total_tokens;
  if (rows == 0) return FASTAV_OK;
  chain_begin(p->flags);
  RowsCall c{};
  c.cache = make_view(*cache);
  c.batch = p->batch; c.total_src = p->total_tokens; c.total_dst = rows; c.max_src = p->max_seqlen; c.table_stride = table_stride;
  c.k_st = p->k_stride_tok; c.k_sh = p->k_stride_head; c.v_st = p->v_stride_tok; c.v_sh = p->v_stride_head;
  c.global_idx = (p->flags & FASTAV_KEEP_IDX_GLOBAL) != 0;
  const cudaError_t e = launch_rows<true>(c, static_cast<uint16_t*>(const_cast<void*>(k)), static_cast<uint16_t*>(const_cast<void*>(v)), cu_seqlens, keep_idx_opt,
                                          keep_idx_opt ? cu_keep_opt : cu_seqlens, page_table, start_opt, device_status, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}

extern "C" int32_t fastav_cache_read(const fastav_params* p, const fastav_cache* cache, const int32_t* page_table, int32_t table_stride, const int32_t* start_opt,
                                     const int32_t* cu_seqlens, void* k_out, void* v_out, int32_t* device_status, void* stream) {
  const int32_t rc = p ? check_rows(p, cache, cu_seqlens, page_table, table_stride, k_out, v_out, p->ko_stride_tok, p->ko_stride_head, p->vo_stride_tok,
                                    p->vo_stride_head)
                       : FASTAV_ERR_INVALID_ARG;
  if (rc != FASTAV_OK) return rc;
  if (p->total_tokens == 0) return FASTAV_OK;
  chain_begin(p->flags);
  RowsCall c{};
  c.cache = make_view(*cache);
  c.batch = p->batch; c.total_src = c.total_dst = p->total_tokens; c.max_src = p->max_seqlen; c.table_stride = table_stride;
  c.k_st = p->ko_stride_tok; c.k_sh = p->ko_stride_head; c.v_st = p->vo_stride_tok; c.v_sh = p->vo_stride_head;
  const cudaError_t e = launch_rows<false>(c, static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out), cu_seqlens, nullptr, cu_seqlens, page_table, start_opt,
                                           device_status, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}
