// Queries and keys in their positions (fastav_rotate), new tokens straight into the cache (fastav_rotate_write).
//
// y = x w / sqrt(mean x^2 + eps) per head, then pairs of elements turned by the angle position * frequency.  Bound by HBM: a row of d values is read and
// written once (2 d bytes each way; d + 4 bytes to the cache).  A block takes a few consecutive tokens.  Their sines and cosines depend on token and pair only,
// so they are made once into shared memory, in the order in which lanes read them; then d / 16 lanes take a head's row each, a lane two pieces of 8
// elements: pieces that hold the two halves of the same pairs, so that a rotation needs no other lane.
//
// Angles.  frequency / (2 pi) as a 64-bit binary fraction of a turn times the position, modulo 2^64, IS the angle modulo a turn: integers wrap where floats
// lose bits (fp32 is 0.06 rad off at position 10^6).
#include <limits.h>

#include <cmath>
#include <cstring>

#include "cache.cuh"
#include "cache_quantise.cuh"

namespace fastav {
namespace {

constexpr int kThreads = 256;
constexpr int kMostTokens = 8;  // of a block
constexpr int kPairs = FASTAV_ROTATE_MAX_PAIRS;

struct RotateCall {
  CacheView cache;
  int batch, total, hq, hkv, rows;   // rows of a token: query heads, then K heads, then (to the cache) V heads
  int rotary, table_stride, tokens;  // tokens per block
  bool interleaved;
  float eps;
  long long q_st, q_sh, k_st, k_sh, v_st, v_sh, qo_st, qo_sh, ko_st, ko_sh, pos_st, pos_sa;
  const uint16_t *q, *k, *v, *q_norm, *k_norm;
  uint16_t *q_out, *k_out;
  const int32_t *pos, *cu, *table, *start;
  int32_t* device_status;
  int head_wait;
  uint8_t axis[kPairs];
  unsigned long long turn[kPairs];  // of a pair per position, in 2^-64 turns
};
inline void mark_head(RotateCall& c, bool head) { c.head_wait = head ? 1 : 0; }

enum { kToRows, kToInt8, kToFp8 };

__device__ __forceinline__ float max_nan2(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

__device__ __forceinline__ uint4 to_bf16(const float* x) {
  uint4 r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.x) : "f"(x[1]), "f"(x[0]));
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.y) : "f"(x[3]), "f"(x[2]));
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.z) : "f"(x[5]), "f"(x[4]));
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w) : "f"(x[7]), "f"(x[6]));
  return r;
}
__device__ __forceinline__ void to_floats(const uint4& x, float* f) {
  const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// Eight codes of a row whose largest magnitude is laid on L: x * power is exact (a power of two that brings the largest into [1, 2)), times L / that.
template <bool FP8>
__device__ __forceinline__ uint2 codes_of(const float* x, float power, float factor) {
  float2 y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = make_float2(x[2 * i] * power * factor, x[2 * i + 1] * power * factor);
  if (FP8) {
    return make_uint2(pack_e4m3(y[0], y[1]), pack_e4m3(y[2], y[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = make_float2(y[i].x + 12582912.f, y[i].y + 12582912.f);  // 1.5 * 2^23: the code in the low bits
    return make_uint2(low_bytes(y[0], y[1]), low_bytes(y[2], y[3]));
  }
}

template <int DIM, int TO>
__global__ void __launch_bounds__(kThreads, 3)
rotate_kernel(const __grid_constant__ RotateCall c) {
  constexpr int kLanes = DIM / 16, kGroups = kThreads / kLanes, kUnroll = 2;
  constexpr bool kFp8 = TO == kToFp8;
  __shared__ __align__(16) float2 table[kMostTokens][kPairs];  // (cos, sin): of lane l's i-th pair at ((i / 2) * 8 + l) * 2 + i % 2
  __shared__ __align__(16) float norm[2][DIM];                 // of lane l's i-th element at ((i / 4) * kLanes + l) * 4 + i % 4
  __shared__ long long place[kMostTokens];                     // row of the pool, head 0; -1: left out
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int turned = c.rotary / 16;  // lanes whose pieces are turned
  const int piece0 = lane < turned ? lane : 2 * lane, piece1 = lane < turned ? lane + turned : piece0 + 1;

  if (c.head_wait) pdl_wait();
  pdl_trigger();
  pdl_wait();
  const int first = blockIdx.x * c.tokens, listed = TO == kToRows ? c.total : min(c.total, chain_load_cached(c.cu + c.batch));
  const int tokens = max(0, min(c.tokens, listed - first));
  if (TO != kToRows && blockIdx.x == 0 && threadIdx.x == 0 && c.device_status && chain_load_cached(c.cu + c.batch) > c.total)
    atomicOr(c.device_status, FASTAV_DEV_SHAPE_MISMATCH);
  const int total_rows = tokens * c.rows;

  const int half = c.rotary / 2;
  for (int e = threadIdx.x; e < tokens * half; e += kThreads) {
    const int token = e / half, slot = e - token * half, l = slot / 8, i = slot % 8;
    const int pair = !c.interleaved ? slot : i < 4 ? 4 * l + i : 4 * (l + turned) + i - 4;
    const int pos = chain_load(c.pos + (first + token) * c.pos_st + c.axis[pair] * c.pos_sa);
    const unsigned long long angle = c.turn[pair] * (unsigned long long)(long long)pos;
    float s, co;
    sincospif((float)(int)(angle >> 32) * (1.f / 2147483648.f), &s, &co);
    table[token][((i >> 1) * 8 + l) * 2 + (i & 1)] = make_float2(co, s);
  }
  if (threadIdx.x < 2 * DIM) {
    const int side = threadIdx.x / DIM, at = threadIdx.x % DIM, piece = at / 8;
    const int l = piece < 2 * turned ? piece % max(turned, 1) : turned + (piece - 2 * turned) / 2;
    const int i = (piece < 2 * turned ? piece / max(turned, 1) : (piece - 2 * turned) % 2) * 8 + at % 8;
    const uint16_t* const w = side ? c.k_norm : c.q_norm;
    norm[side][((i >> 2) * kLanes + l) * 4 + (i & 3)] = w ? __uint_as_float((unsigned)chain_load(w + at) << 16) : 1.f;
  }
  if (TO != kToRows && (int)threadIdx.x < tokens) {
    const int row = first + threadIdx.x;
    int lo = 0, hi = c.batch;  // largest b with cu[b] <= row
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (chain_load_cached(c.cu + mid) <= row) lo = mid; else hi = mid;
    }
    const int i = row - chain_load_cached(c.cu + lo);
    const long long token = (long long)(c.start ? chain_load_cached(c.start + lo) : 0) + i;
    int bad = 0;
    long long at = -1;
    if (i < 0 || token < 0 || token >= (long long)c.table_stride << c.cache.page_shift || token > INT_MAX) {
      bad = FASTAV_DEV_SHAPE_MISMATCH;
    } else {
      const int page = page_of(c.cache, c.table, c.table_stride, lo, (int)token);
      if (page < 0) bad = FASTAV_DEV_BAD_INDEX;
      else at = pool_row(c.cache, page, 0, (int)token);
    }
    place[threadIdx.x] = at;
    if (bad && c.device_status) atomicOr(c.device_status, bad);
  }
  __syncthreads();

  int token = group / c.rows, head = group - token * c.rows;
  const int token_step = kGroups / c.rows, head_step = kGroups - token_step * c.rows;
  // (all lanes of a warp make the same number of turns: they shuffle)
#pragma unroll 1
  for (int r0 = 0; r0 < total_rows; r0 += kGroups * kUnroll) {
    uint4 in0[kUnroll], in1[kUnroll];
    int of_token[kUnroll], of_head[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      of_token[u] = token;
      of_head[u] = head;
      in0[u] = in1[u] = make_uint4(0, 0, 0, 0);
      if (token < tokens) {
        const long long row = first + token;
        const uint16_t* const from = head < c.hq ? c.q + row * c.q_st + head * c.q_sh
                                     : TO == kToRows || head < c.hq + c.hkv ? c.k + row * c.k_st + (head - c.hq) * c.k_sh
                                                                           : c.v + row * c.v_st + (head - c.hq - c.hkv) * c.v_sh;
        in0[u] = chain_load(reinterpret_cast<const uint4*>(from + piece0 * 8));
        in1[u] = chain_load(reinterpret_cast<const uint4*>(from + piece1 * 8));
      }
      token += token_step;
      head += head_step;
      if (head >= c.rows) { head -= c.rows; ++token; }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool there = of_token[u] < tokens, is_q = of_head[u] < c.hq, is_v = TO != kToRows && of_head[u] >= c.hq + c.hkv;
      const long long row = first + of_token[u];
      float x[16];
      to_floats(in0[u], x);
      to_floats(in1[u], x + 8);
      if (c.q_norm || c.k_norm) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (__any_sync(0xFFFFFFFFu, !(sum < INFINITY))) {  // squares beyond fp32: once more, of what is 2^-64 as large (eps is nothing beside them)
          float small = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) small = fmaf(x[i] * 0x1p-64f, x[i] * 0x1p-64f, small);
#pragma unroll
          for (int d = 1; d < kLanes; d <<= 1) small += __shfl_xor_sync(0xFFFFFFFFu, small, d);
          sum = sum < INFINITY ? rsqrtf(fmaf(sum, 1.f / DIM, c.eps)) : rsqrtf(small * (1.f / DIM)) * 0x1p-64f;
        } else {
          sum = rsqrtf(fmaf(sum, 1.f / DIM, c.eps));
        }
        if (!is_v && (is_q ? c.q_norm : c.k_norm)) {
          const float4* const w = reinterpret_cast<const float4*>(norm[is_q ? 0 : 1]) + lane;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 f = w[i * kLanes];
            x[4 * i] *= sum * f.x;
            x[4 * i + 1] *= sum * f.y;
            x[4 * i + 2] *= sum * f.z;
            x[4 * i + 3] *= sum * f.w;
          }
        }
      }
      if (lane < turned && there && !is_v) {
        const float4* const t = reinterpret_cast<const float4*>(table[of_token[u]]) + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 f = t[i * 8];  // (cos, sin) of two pairs
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float co = j ? f.z : f.x, s = j ? f.w : f.y;
            const int p = 2 * i + j;
            if (c.interleaved) {
              const float y = x[2 * p], z = x[2 * p + 1];
              x[2 * p] = y * co - z * s;
              x[2 * p + 1] = z * co + y * s;
            } else {
              const float y = x[p], z = x[p + 8];
              x[p] = y * co - z * s;
              x[p + 8] = z * co + y * s;
            }
          }
        }
      }
      if (TO == kToRows || is_q) {
        if (there) {
          uint16_t* const to = is_q ? c.q_out + row * c.qo_st + of_head[u] * c.qo_sh : c.k_out + row * c.ko_st + (of_head[u] - c.hq) * c.ko_sh;
          *reinterpret_cast<uint4*>(to + piece0 * 8) = to_bf16(x);
          *reinterpret_cast<uint4*>(to + piece1 * 8) = to_bf16(x + 8);
        }
      }
      if (TO != kToRows) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max_nan2(top, fabsf(x[i]));
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) top = max_nan2(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const long long at = there ? place[of_token[u]] : -1;
        if (!is_q && at >= 0) {
          const int kv = of_head[u] - c.hq - (is_v ? c.hkv : 0);
          const long long to = at + ((long long)kv << c.cache.page_shift);
          uint8_t* const codes = (is_v ? c.cache.v : c.cache.k) + to * DIM;
          const bool finite = top < INFINITY;  // else the codes are 0 and the scale is NaN, as fastav_cache_write leaves them
          uint2 c0, c1;
          float scale;
          if (is_v) {  // exactly as fastav_cache_write rounds
            const unsigned bits = __float_as_uint(top) >> 16;
            c0 = quantise8<kFp8>(in0[u], bits);
            c1 = quantise8<kFp8>(in1[u], bits);
            scale = scale_of<kFp8>(bits);
          } else {
            constexpr float kLargest = kFp8 ? 448.f : 127.f;
            const int e = (int)(__float_as_uint(top) >> 23);
            const float power = __uint_as_float((unsigned)min(max(254 - e, 1), 253) << 23), t = top * power;
            const float factor = t > 0.f ? __fdiv_rn(kLargest, t) : 0.f;
            c0 = codes_of<kFp8>(x, power, factor);
            c1 = codes_of<kFp8>(x + 8, power, factor);
            scale = __fdiv_rn(top, kLargest);
          }
          *reinterpret_cast<uint2*>(codes + piece0 * 8) = finite ? c0 : make_uint2(0, 0);
          *reinterpret_cast<uint2*>(codes + piece1 * 8) = finite ? c1 : make_uint2(0, 0);
          if (lane == 0) (is_v ? c.cache.v_scale : c.cache.k_scale)[to] = finite ? scale : __uint_as_float(0x7FC00000u);
        }
      }
    }
  }
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// radians -> 2^-64 turns, modulo a turn: the mantissa times 2^66 / (2 pi) in integers.
unsigned long long turns(double radians) {
  constexpr unsigned long long kInverse = 0xa2f9836e4e44152aull;  // 2^66 / (2 pi), to nearest
  unsigned long long bits;
  std::memcpy(&bits, &radians, sizeof bits);
  const int exponent = (int)(bits >> 52 & 2047);
  const unsigned long long mantissa = (bits & ((1ull << 52) - 1)) | (exponent ? 1ull << 52 : 0);
  const int shift = (exponent ? exponent : 1) - 1075 - 2;  // radians = mantissa 2^(shift + 2)
  const unsigned __int128 product = (unsigned __int128)mantissa * kInverse;
  unsigned long long t = 0;
  if (shift < 0 && shift > -128) t = (unsigned long long)(product >> -shift);
  else if (shift >= 0 && shift < 64) t = (unsigned long long)product << shift;
  return bits >> 63 ? 0ull - t : t;
}

int32_t check_side(const void* in, const void* out, int64_t in_st, int64_t in_sh, int64_t out_st, int64_t out_sh, int heads, int dim) {
  if (!in != !out) return FASTAV_ERR_INVALID_ARG;
  if (!in) return FASTAV_OK;
  int32_t rc;
  if (heads < 1) return FASTAV_ERR_INVALID_ARG;
  if ((rc = check_strides(in_st, in_sh, heads, dim)) != FASTAV_OK || (rc = check_strides(out_st, out_sh, heads, dim)) != FASTAV_OK) return rc;
  if (in == out && (in_st != out_st || (heads > 1 && in_sh != out_sh))) return FASTAV_ERR_INVALID_ARG;
  return aligned(in, 16) && aligned(out, 16) ? FASTAV_OK : FASTAV_ERR_UNSUPPORTED;
}

// What both entry points ask of the rotation.
int32_t check_turns(const fastav_rotate_params* p, const int32_t* pos, bool normed) {
  if (!p || p->total_tokens < 0) return FASTAV_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return FASTAV_ERR_UNSUPPORTED;
  if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim) return FASTAV_ERR_INVALID_ARG;
  if (p->rotary_dim % 16 != 0) return FASTAV_ERR_UNSUPPORTED;
  if (normed && !(p->norm_eps >= 1e-20f && std::isfinite(p->norm_eps))) return FASTAV_ERR_INVALID_ARG;
  if (p->rotary_dim == 0) return FASTAV_OK;
  if (p->num_axes < 1 || p->num_axes > FASTAV_ROTATE_MAX_AXES || (p->total_tokens > 0 && !pos)) return FASTAV_ERR_INVALID_ARG;
  if (!aligned(pos, 4)) return FASTAV_ERR_UNSUPPORTED;
  for (int i = 0; i < p->rotary_dim / 2; ++i)
    if (p->axis[i] >= p->num_axes || !std::isfinite(p->frequency[i])) return FASTAV_ERR_INVALID_ARG;
  return FASTAV_OK;
}

RotateCall make_call(const fastav_rotate_params& p, const void* q, const void* k, const int32_t* pos, const void* q_norm, const void* k_norm, void* q_out) {
  RotateCall c{};
  c.total = p.total_tokens;
  c.hq = q ? p.num_q_heads : 0;
  c.hkv = k ? p.num_kv_heads : 0;
  c.rotary = p.rotary_dim;
  c.interleaved = (p.flags & FASTAV_ROTATE_INTERLEAVED) != 0;
  c.eps = p.norm_eps;
  c.q_st = p.q_stride_tok; c.q_sh = p.q_stride_head; c.k_st = p.k_stride_tok; c.k_sh = p.k_stride_head;
  c.qo_st = p.qo_stride_tok; c.qo_sh = p.qo_stride_head;
  c.pos_st = p.pos_stride_tok; c.pos_sa = p.pos_stride_axis;
  c.q = static_cast<const uint16_t*>(q); c.k = static_cast<const uint16_t*>(k);
  c.q_norm = q ? static_cast<const uint16_t*>(q_norm) : nullptr;
  c.k_norm = k ? static_cast<const uint16_t*>(k_norm) : nullptr;
  c.q_out = static_cast<uint16_t*>(q_out);
  c.pos = pos;
  for (int i = 0; i < p.rotary_dim / 2; ++i) {
    c.axis[i] = p.axis[i];
    c.turn[i] = turns(p.frequency[i]);
  }
  return c;
}

template <int TO>
int32_t launch(RotateCall& c, int dim, cudaStream_t stream) {
  // Few tokens: one per block, so that more SMs take part.  Many: the block's start is shared by more rows.
  c.tokens = 1;
  while (2 * c.tokens <= kMostTokens && c.total / (2 * c.tokens) >= kNumSMs * 3) c.tokens *= 2;
  const dim3 grid((unsigned)((c.total + c.tokens - 1) / c.tokens));
  count_launches(1);
  const cudaError_t e = dim == 128 ? launch_chained(rotate_kernel<128, TO>, grid, dim3(kThreads), 0, stream, c)
                                   : launch_chained(rotate_kernel<64, TO>, grid, dim3(kThreads), 0, stream, c);
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}

}  // namespace
}  // namespace fastav

using namespace fastav;

extern "C" int32_t fastav_rotate(const fastav_rotate_params* p, const void* q, const void* k, const int32_t* pos, const void* q_norm_opt, const void* k_norm_opt,
                                 void* q_out, void* k_out, void* stream) {
  int32_t rc = check_turns(p, pos, (q && q_norm_opt) || (k && k_norm_opt));
  if (rc != FASTAV_OK) return rc;
  if ((rc = check_side(q, q_out, p->q_stride_tok, p->q_stride_head, p->qo_stride_tok, p->qo_stride_head, p->num_q_heads, p->head_dim)) != FASTAV_OK) return rc;
  if ((rc = check_side(k, k_out, p->k_stride_tok, p->k_stride_head, p->ko_stride_tok, p->ko_stride_head, p->num_kv_heads, p->head_dim)) != FASTAV_OK) return rc;
  if (p->total_tokens == 0) return FASTAV_OK;
  if (!q && !k) return FASTAV_ERR_INVALID_ARG;
  chain_begin(p->flags);
  RotateCall c = make_call(*p, q, k, pos, q_norm_opt, k_norm_opt, q_out);
  c.rows = c.hq + c.hkv;
  c.ko_st = p->ko_stride_tok; c.ko_sh = p->ko_stride_head;
  c.k_out = static_cast<uint16_t*>(k_out);
  return launch<kToRows>(c, p->head_dim, static_cast<cudaStream_t>(stream));
}

extern "C" int32_t fastav_rotate_write(const fastav_rotate_params* p, const fastav_cache* cache, const void* q, const void* k, const void* v, const int32_t* pos,
                                       const void* q_norm_opt, const void* k_norm_opt, const int32_t* cu_seqlens, const int32_t* page_table, int32_t table_stride,
                                       const int32_t* start_opt, void* q_out, int32_t* device_status, void* stream) {
  int32_t rc = check_turns(p, pos, (q && q_norm_opt) || k_norm_opt);
  if (rc != FASTAV_OK) return rc;
  if ((rc = check_cache(cache)) != FASTAV_OK) return rc;
  if (p->batch < 1 || p->num_kv_heads != cache->num_kv_heads || p->head_dim != cache->head_dim) return FASTAV_ERR_INVALID_ARG;
  if (!cu_seqlens || !page_table || table_stride < 1) return FASTAV_ERR_INVALID_ARG;
  if (p->total_tokens > 0 && (!k || !v)) return FASTAV_ERR_INVALID_ARG;
  if ((rc = check_side(q, q_out, p->q_stride_tok, p->q_stride_head, p->qo_stride_tok, p->qo_stride_head, p->num_q_heads, p->head_dim)) != FASTAV_OK) return rc;
  if ((rc = check_strides(p->k_stride_tok, p->k_stride_head, p->num_kv_heads, p->head_dim)) != FASTAV_OK) return rc;
  if ((rc = check_strides(p->v_stride_tok, p->v_stride_head, p->num_kv_heads, p->head_dim)) != FASTAV_OK) return rc;
  if (!aligned(k, 16) || !aligned(v, 16)) return FASTAV_ERR_UNSUPPORTED;
  if (p->total_tokens == 0) return FASTAV_OK;
  chain_begin(p->flags);
  RotateCall c = make_call(*p, q, k, pos, q_norm_opt, k_norm_opt, q_out);
  c.cache = make_view(*cache);
  c.batch = p->batch;
  c.rows = c.hq + 2 * c.hkv;
  c.table_stride = table_stride;
  c.v_st = p->v_stride_tok; c.v_sh = p->v_stride_head;
  c.v = static_cast<const uint16_t*>(v);
  c.cu = cu_seqlens; c.table = page_table; c.start = start_opt;
  c.device_status = device_status;
  return c.cache.fp8 ? launch<kToFp8>(c, p->head_dim, static_cast<cudaStream_t>(stream)) : launch<kToInt8>(c, p->head_dim, static_cast<cudaStream_t>(stream));
}
