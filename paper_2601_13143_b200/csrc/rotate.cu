// Queries and keys in their positions (fastav_rotate), new tokens straight into the cache (fastav_rotate_write).
//
// y = x w / sqrt(mean x^2 + eps) per head, then pairs of elements turned by the angle position * frequency.  Bound by HBM: a row of d values is read and
// written once (2 d bytes each way; d + 4 bytes to the cache).  A block takes a few consecutive tokens.  Their sines and cosines depend on token and pair only,
// so they are made once into shared memory, in the order in which lanes read them.  d / 16 lanes take a row, a lane two pieces of 8
// elements: pieces that hold the two halves of the same pairs, so that a rotation needs no other lane.  A group of lanes keeps to one head and walks over
// the block's tokens, so that addresses, the norm's weights and what becomes of the row are known beforehand, and a block has as many threads as that
// takes.  65,536 tokens of 40 rows: 220 us, 6.1 TB/s, 95 % of a copy.  16 x 900 tokens of 48 rows into the cache: 72 us, 3.9 TB/s, 177 instructions of a warp
// for four rows; with norms 80 us and 260, 0.57 of them a cycle and scheduler.  (Groups that walk over the heads of a token instead: 324 instructions, 102 us.)  With pairs
// of neighbours (INTERLEAVED) four blocks an SM leave the compiler 64 registers, and it spills 4 to 20 bytes a thread.
//
// Angles.  frequency / (2 pi) as a 64-bit binary fraction of a turn times the position, modulo 2^64, IS the angle modulo a turn: integers wrap where floats
// lose bits (fp32 is 0.06 rad off at position 10^6).
#include <limits.h>

#include <cmath>
#include <cstring>

#include "cache.cuh"
#include "cache_quantise.cuh"
#include "sm100_ptx.cuh"

namespace fastav {
namespace {

constexpr int kMostThreads = 256;
constexpr int kMostTokens = 4;  // of a block: what all blocks have in flight should lie close together (65,536 tokens of 40 rows: 4 or 8 tokens 223 and 229 us, 16 249, 32 272)
constexpr int kPairs = FASTAV_ROTATE_MAX_PAIRS;
constexpr int kMostHeads = 1 << 26;  // of a side: the lanes of a token's rows are counted in 32 bits

struct RotateCall {
  CacheView cache;
  int batch, total, hq, hkv, rows;   // rows of a token: query heads, then K heads, then (to the cache) V heads
  int heads, at_once;                // rows that a block's groups take in one pass, tokens at a time
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

// Sixteen values of a row, as they lie in memory: a lane's two pieces.
struct Row {
  uint4 lo, hi;
};

__device__ __forceinline__ float2 two(float x) { return make_float2(x, x); }

// Eight codes of a row whose largest magnitude is laid on L, given factor = L / that.
template <bool FP8>
__device__ __forceinline__ uint2 codes_of(const float2* x, float factor) {
  float2 y[4];
  if (FP8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __fmul2_rn(x[i], two(factor));
    return make_uint2(pack_e4m3(y[0], y[1]), pack_e4m3(y[2], y[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __ffma2_rn(x[i], two(factor), two(12582912.f));  // 1.5 * 2^23: the code in the low bits
    return make_uint2(low_bytes(y[0], y[1]), low_bytes(y[2], y[3]));
  }
}

template <int DIM, int TO, bool NORMED, bool INTERLEAVED>
__global__ void __launch_bounds__(kMostThreads, 4)
rotate_kernel(const __grid_constant__ RotateCall c) {
  constexpr int kLanes = DIM / 16;
  constexpr bool kFp8 = TO == kToFp8;
  // Halves: (cos, cos, sin, sin) of lane l's pairs 2 j and 2 j + 1 at [j * 8 + l]; neighbours: (cos, cos, -sin, sin) of its j-th.
  __shared__ __align__(16) float4 table[kMostTokens][INTERLEAVED ? kPairs : kPairs / 2];
  __shared__ __align__(16) float4 weights[NORMED ? 2 : 1][NORMED ? DIM / 4 : 1];  // the norm's, of lane l's four j at [j * kLanes + l]
  __shared__ long long place[kMostTokens];  // row of the pool, head 0; -1: left out
  const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const unsigned mates = ((1u << kLanes) - 1u) << (threadIdx.x & 31 & ~(kLanes - 1));  // the group's lanes of the warp
  const int turned = c.rotary / 16;  // lanes whose pieces are turned
  const int piece0 = lane < turned ? lane : 2 * lane, piece1 = lane < turned ? lane + turned : piece0 + 1;

  if (c.head_wait) pdl_wait();
  pdl_trigger();
  pdl_wait();
  const int first = blockIdx.x * c.tokens, listed = TO == kToRows ? c.total : min(c.total, chain_load_cached(c.cu + c.batch));
  const int tokens = max(0, min(c.tokens, listed - first));
  if (TO != kToRows && blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0 && c.device_status && chain_load_cached(c.cu + c.batch) > c.total)
    atomicOr(c.device_status, FASTAV_DEV_SHAPE_MISMATCH);

  // The rows that this group takes in a pass: where the first one lies, and how far apart they are.
  struct Head {
    const uint16_t *from, *norm;
    long long step;
  };
  const int phase = group / c.heads;
  auto head_of = [&](int h) {
    Head x;
    if (h < c.hq) x = Head{c.q + (first + phase) * c.q_st + h * c.q_sh, c.q_norm, c.q_st};
    else if (TO == kToRows || h < c.hq + c.hkv) x = Head{c.k + (first + phase) * c.k_st + (h - c.hq) * c.k_sh, c.k_norm, c.k_st};
    else x = Head{c.v + (first + phase) * c.v_st + (h - c.hq - c.hkv) * c.v_sh, nullptr, c.v_st};
    x.step *= c.at_once;
    return x;
  };
  Row next;
  auto ask = [&](Head& x, int token) {
    if (token < tokens) {
      next.lo = chain_load(reinterpret_cast<const uint4*>(x.from) + piece0);
      next.hi = chain_load(reinterpret_cast<const uint4*>(x.from) + piece1);
    }
    x.from += x.step;
  };
  // The first rows are on their way while the table is made.
  const bool active = group < c.heads * c.at_once;
  int h = active ? blockIdx.y * c.heads + group - phase * c.heads : c.rows;
  Head head{};
  if (h < c.rows) {
    head = head_of(h);
    ask(head, phase);
  }

  if (NORMED)
    for (int i = threadIdx.x; i < 2 * DIM; i += blockDim.x) {
      const uint16_t* const w = i < DIM ? c.q_norm : c.k_norm;
      const int at = i % DIM, piece = at / 8, second = piece < 2 * turned ? piece >= turned : piece & 1;
      const int l = piece < 2 * turned ? piece - (second ? turned : 0) : piece / 2, j = second * 8 + at % 8;
      reinterpret_cast<float*>(&weights[i / DIM][(j >> 2) * kLanes + l])[j & 3] = w ? __uint_as_float((unsigned)chain_load(w + at) << 16) : 1.f;
    }
  const int half = c.rotary / 2;
  for (int e = threadIdx.x; e < tokens * half; e += blockDim.x) {
    const int token = e / half, slot = e - token * half, l = slot / 8, i = slot % 8;
    const int pair = !INTERLEAVED ? slot : i < 4 ? 4 * l + i : 4 * (l + turned) + i - 4;
    const int pos = chain_load(c.pos + (first + token) * c.pos_st + c.axis[pair] * c.pos_sa);
    const unsigned long long angle = c.turn[pair] * (unsigned long long)(long long)pos;
    // The nearest quarter turn off in integers, so that what becomes a float is at most an eighth of a turn (its last bit 2^-25 of that); then turned back by it.
    const unsigned high = (unsigned)(angle >> 32), quarters = (high + 0x20000000u) >> 30;
    float s, co;
    sincospif((float)(int)(high - (quarters << 30)) * (1.f / 2147483648.f), &s, &co);
    if (quarters & 1) {
      const float was = s;
      s = co;
      co = -was;
    }
    if (quarters & 2) {
      s = -s;
      co = -co;
    }
    if (INTERLEAVED) {
      table[token][i * 8 + l] = make_float4(co, co, -s, s);
    } else {
      float* const at = reinterpret_cast<float*>(&table[token][(i >> 1) * 8 + l]) + (i & 1);
      at[0] = co;
      at[2] = s;
    }
  }
  if (TO != kToRows)
    for (int t = threadIdx.x; t < tokens; t += blockDim.x) {
      const int row = first + t;
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
      place[t] = at;
      if (bad && c.device_status) atomicOr(c.device_status, bad);
    }
  __syncthreads();

  // A row normed and rotated, as pairs of neighbours: x[0..3] the first piece, x[4..7] the second.
  auto turn = [&](const Row& r, int token, bool normed, int side, float2 (&x)[8]) {
    const unsigned in[8] = {r.lo.x, r.lo.y, r.lo.z, r.lo.w, r.hi.x, r.hi.y, r.hi.z, r.hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = both(in[i]);
    if (NORMED && normed) {
      float2 squares = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) squares = __ffma2_rn(x[i], x[i], squares);
      float sum = squares.x + squares.y;
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor_sync(mates, sum, d);
      const float mean = fmaf(sum, 1.f / DIM, c.eps);
      float inverse = __frsqrt_rn(mean);
      if (!(mean < INFINITY)) {  // beyond fp32 (the whole group's): once more, of what is 2^-80 as large, 2^103 in all at most
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 small = __fmul2_rn(x[i], two(0x1p-80f));
          sum = fmaf(small.x, small.x, fmaf(small.y, small.y, sum));
        }
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor_sync(mates, sum, d);
        // (2^-128 at least: where it is subnormal, it is still good to 2^-22.  To leave the row alone here is 1 us of 107 for 16 x 900 tokens into the cache.)
        inverse = __frsqrt_rn(fmaf(sum, 1.f / DIM, c.eps * 0x1p-80f * 0x1p-80f)) * 0x1p-80f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 w = weights[NORMED ? side : 0][NORMED ? i * kLanes + lane : 0];
        x[2 * i] = __fmul2_rn(__fmul2_rn(x[2 * i], two(inverse)), make_float2(w.x, w.y));  // (w / rms alone may leave fp32; x / rms is 11.4 at most)
        x[2 * i + 1] = __fmul2_rn(__fmul2_rn(x[2 * i + 1], two(inverse)), make_float2(w.z, w.w));
      }
    }
    if (lane >= turned) return;
    const float4* const t = table[token] + lane;
    if (INTERLEAVED) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 f = t[i * 8];
        x[i] = __ffma2_rn(x[i], make_float2(f.x, f.y), __fmul2_rn(make_float2(x[i].y, x[i].x), make_float2(f.z, f.w)));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 f = t[i * 8];
        const float2 co = make_float2(f.x, f.y), s = make_float2(f.z, f.w), a = x[i], b = x[i + 4];
        x[i] = __ffma2_rn(a, co, __fmul2_rn(b, __fmul2_rn(s, two(-1.f))));
        x[i + 4] = __ffma2_rn(b, co, __fmul2_rn(a, s));
      }
    }
  };
  auto put_rows = [&](uint16_t* to, const float2 (&x)[8]) {
    *reinterpret_cast<uint4*>(to + piece0 * 8) = make_uint4(two_bf16(x[0].x, x[0].y), two_bf16(x[1].x, x[1].y), two_bf16(x[2].x, x[2].y), two_bf16(x[3].x, x[3].y));
    *reinterpret_cast<uint4*>(to + piece1 * 8) = make_uint4(two_bf16(x[4].x, x[4].y), two_bf16(x[5].x, x[5].y), two_bf16(x[6].x, x[6].y), two_bf16(x[7].x, x[7].y));
  };
  // Codes and scale of a row of K or V; what is not finite: codes 0 and a scale that is NaN, as fastav_cache_write leaves them.
  auto put_codes = [&](uint8_t* pool, float* scales, long long row, uint2 c0, uint2 c1, float scale, bool finite) {
    uint8_t* const to = pool + row * DIM;
    *reinterpret_cast<uint2*>(to + piece0 * 8) = finite ? c0 : make_uint2(0, 0);
    *reinterpret_cast<uint2*>(to + piece1 * 8) = finite ? c1 : make_uint2(0, 0);
    if (lane == 0) scales[row] = finite ? scale : __uint_as_float(0x7FC00000u);
  };

  // f(row, token) for the group's rows, the next one asked for ahead.
  auto walk = [&](auto f) {
    for (int token = phase; token < tokens; token += c.at_once) {
      const Row now = next;
      ask(head, token + c.at_once);
      f(now, token);
    }
  };
  while (h < c.rows) {
    if (h < c.hq || TO == kToRows) {
      const bool is_q = h < c.hq, normed = head.norm != nullptr;
      uint16_t* const out = is_q ? c.q_out + first * c.qo_st + h * c.qo_sh : c.k_out + first * c.ko_st + (h - c.hq) * c.ko_sh;
      const long long stride = is_q ? c.qo_st : c.ko_st;
      walk([&](const Row& r, int token) {
        float2 x[8];
        turn(r, token, normed, is_q ? 0 : 1, x);
        put_rows(out + token * stride, x);
      });
    } else if (h < c.hq + c.hkv) {
      const bool normed = head.norm != nullptr;
      const long long of_head = (long long)(h - c.hq) << c.cache.page_shift;
      walk([&](const Row& r, int token) {
        float2 x[8];
        turn(r, token, normed, 1, x);
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = ptx::max_nan(top, fabsf(x[i].x), fabsf(x[i].y));
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) {
          const float other = __shfl_xor_sync(mates, top, d);
          top = ptx::max_nan(top, other, other);
        }
        const long long at = place[token];
        if (at < 0) return;
        constexpr float kLargest = kFp8 ? 448.f : 127.f;
        float factor = __fdiv_rn(kLargest, top);
        if (top < 0x1p-100f) {  // L / top leaves fp32: everything by 2^100 first (exact)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __fmul2_rn(x[i], two(0x1p100f));
          factor = top > 0.f ? __fdiv_rn(kLargest, top * 0x1p100f) : 0.f;
        }
        put_codes(c.cache.k, c.cache.k_scale, at + of_head, codes_of<kFp8>(x, factor), codes_of<kFp8>(x + 4, factor), __fdiv_rn(top, kLargest), top < INFINITY);
      });
    } else {
      const long long of_head = (long long)(h - c.hq - c.hkv) << c.cache.page_shift;
      walk([&](const Row& r, int token) {  // exactly as fastav_cache_write rounds
        unsigned top = larger(top_of(r.lo), top_of(r.hi));
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) top = larger(top, __shfl_xor_sync(mates, top, d));
        top = larger(top, __byte_perm(top, top, 0x1032)) & 0xFFFFu;
        const long long at = place[token];
        if (at < 0) return;
        put_codes(c.cache.v, c.cache.v_scale, at + of_head, quantise8<kFp8>(r.lo, top), quantise8<kFp8>(r.hi, top), scale_of<kFp8>(top), top < 0x7F80u);
      });
    }
    h += c.heads * gridDim.y;
    if (h < c.rows) {
      head = head_of(h);
      ask(head, phase);
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
  if (heads > kMostHeads) return FASTAV_ERR_UNSUPPORTED;
  if ((rc = check_strides(in_st, in_sh, heads, dim)) != FASTAV_OK || (rc = check_strides(out_st, out_sh, heads, dim)) != FASTAV_OK) return rc;
  if (in == out && (in_st != out_st || (heads > 1 && in_sh != out_sh))) return FASTAV_ERR_INVALID_ARG;
  return aligned(in, 16) && aligned(out, 16) ? FASTAV_OK : FASTAV_ERR_UNSUPPORTED;
}

// What both entry points ask of the rotation.
int32_t check_turns(const fastav_rotate_params* p, const int32_t* pos, const void* q_norm, const void* k_norm) {
  if (!p || p->total_tokens < 0) return FASTAV_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return FASTAV_ERR_UNSUPPORTED;
  if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim) return FASTAV_ERR_INVALID_ARG;
  if (p->rotary_dim % 16 != 0) return FASTAV_ERR_UNSUPPORTED;
  if ((q_norm || k_norm) && !(p->norm_eps >= 1e-20f && std::isfinite(p->norm_eps))) return FASTAV_ERR_INVALID_ARG;
  if (!aligned(q_norm, 16) || !aligned(k_norm, 16)) return FASTAV_ERR_UNSUPPORTED;
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
  const int lanes = dim / 16, passes = (c.rows * lanes + kMostThreads - 1) / kMostThreads;
  c.heads = (c.rows + passes - 1) / passes;
  c.at_once = kMostThreads / (c.heads * lanes);
  c.at_once = c.at_once < 1 ? 1 : c.at_once < kMostTokens ? c.at_once : kMostTokens;
  const int threads = (c.heads * c.at_once * lanes + 31) / 32 * 32;
  // Few tokens: one per block (or as many as it takes at once), so that more SMs take part.  Many: the block's start is shared by more rows; in
  // whole waves of blocks, four to an SM.
  const long long resident = kNumSMs * 4, waves = (c.total + resident * kMostTokens - 1) / (resident * kMostTokens);
  c.tokens = (int)((c.total + resident * waves - 1) / (resident * waves));
  if (c.tokens < c.at_once) c.tokens = c.at_once;
  // The passes over a token's rows: one behind the other, or side by side where that leaves no SM without room (32 tokens of 36 rows 6.1 -> 4.9 us).
  const long long blocks = ((long long)c.total + c.tokens - 1) / c.tokens;
  const dim3 grid((unsigned)blocks, blocks * passes <= resident ? passes : 1);
  count_launches(1);
  auto go = [&](auto kernel) { return launch_chained(kernel, grid, dim3(threads), 0, stream, c); };
  const bool normed = c.q_norm || c.k_norm;
  cudaError_t e;
  if (dim == 128) e = c.interleaved ? (normed ? go(rotate_kernel<128, TO, true, true>) : go(rotate_kernel<128, TO, false, true>))
                                    : (normed ? go(rotate_kernel<128, TO, true, false>) : go(rotate_kernel<128, TO, false, false>));
  else e = c.interleaved ? (normed ? go(rotate_kernel<64, TO, true, true>) : go(rotate_kernel<64, TO, false, true>))
                         : (normed ? go(rotate_kernel<64, TO, true, false>) : go(rotate_kernel<64, TO, false, false>));
  return e == cudaSuccess ? FASTAV_OK : cuda_failed(e);
}

}  // namespace
}  // namespace fastav

using namespace fastav;

extern "C" int32_t fastav_rotate(const fastav_rotate_params* p, const void* q, const void* k, const int32_t* pos, const void* q_norm_opt, const void* k_norm_opt,
                                 void* q_out, void* k_out, void* stream) {
  int32_t rc = check_turns(p, pos, q ? q_norm_opt : nullptr, k ? k_norm_opt : nullptr);
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
  int32_t rc = check_turns(p, pos, q ? q_norm_opt : nullptr, k_norm_opt);
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
