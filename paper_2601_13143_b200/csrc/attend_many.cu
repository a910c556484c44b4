// Attention over the 8-bit cache for many query rows per KV head: a prefix that a batch shares, a question's tokens at once.
//
// Dense contractions, so they run on the fifth-generation tensor cores: S = Q K^T and O += P V (tcgen05.mma, f16 operands, fp32 sums in
// tensor memory).  A unit is 128 keys of one KV head for up to 256 stacked query rows.  Per block, one per SM:
//
//   warps 0-7    softmax, a thread per row: warps 0-3 and 4-7 are two STREAMS with an S and an O of their own, so that the matrix pipe
//                works on one while the exponentials of the other are taken.  With more than 128 rows the streams are the two halves of
//                the rows and share every tile of keys; with fewer they take the tiles in turn and their sums are joined at the end.
//   warps 8-15   codes -> f16, 16 keys of every tile each: straight from global memory (one tile ahead in registers) to the operand
//                tiles in shared memory
//   warp 16      issues the MMAs: QK of a visit goes out before PV of the visit before it (warps 17-19 fill its warpgroup)
//
// Registers move from the warps that need few to the softmax's, which hold a visit's weights.
//
// A value's scale is folded into its f16 operand relative to the power of two E of the largest scale of 16 keys, and E joins the exponent:
// w = 2^(z + E - m + kOffset) is rounded to f16 for the matrix pipe, l = sum w 2^(-E - kOffset) stays in fp32.  So no weight is
// multiplied by a scale, and values of very different size keep their bits.  The keys' scales multiply the logits in fp32.
//
// The weights of a visit are taken with the maximum of the visits before; only where one comes out above 2^15 (or a row meets its first keys)
// the visit's own maximum is taken first, and O rescaled.
#include <limits.h>

#include <cuda.h>

#include "attend.cuh"
#include "attend_8bit.cuh"
#include "sm100_ptx.cuh"

namespace fastav {
namespace {

constexpr int kSub = 128;  // rows of a stream
constexpr int kSoftWarps = 8, kConvWarps = 8, kIssueWarp = kSoftWarps + kConvWarps, kWarps = kIssueWarp + 4;
constexpr int kSoftThreads = 32 * kSoftWarps, kThreads = 32 * kWarps;
// Registers a thread has per role.  What the three take together has to fit into what the block is launched with (checked before the launch).
constexpr int kSoftRegs = 152, kConvRegs = 72, kIssueRegs = 24;
constexpr int kRegsNeeded = 32 * (kSoftWarps * kSoftRegs + kConvWarps * kConvRegs + 4 * kIssueRegs);
constexpr int kGroups = kManyKeys / 16;          // of 16 keys: a converting warp's
constexpr int kScaleRing = 4;
constexpr int kOffset = 11;                      // the largest weight of a row's first visit is 2^kOffset ...
constexpr unsigned kMostWeight = 0x7800;          // ... and of any visit at most this: 2^15 as f16 bits (f16 ends at 65,504)
constexpr int kValuePower = 7;                   // a value operand is code * (scale / 2^E) * 2^kValuePower, below 2^15
constexpr int kTmemCols = 512;
static_assert(kConvWarps == kGroups);

template <int DIM>
struct Many {
  static constexpr int kHalves = DIM / 64;               // 128-byte column blocks of an operand tile
  static constexpr int kHalfBytes = 128 * 128;           // 128 rows of 128 bytes
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kOperands = 6 * kTileBytes;       // Q twice, K twice, V twice
};

struct Control {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], pv_done[2], scale_full[kScaleRing], q_full, last;
  uint32_t tmem_base;
  int abort;
  int warp_sum[kWarps];
  alignas(16) float k_scale[kScaleRing][kManyKeys];
  float exponent[kScaleRing][kGroups], unscale[kScaleRing][kGroups];  // E; 2^(-E - kOffset)
  float2 row_ml[2][kSub];                                             // the streams' statistics, to be joined
};

__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kSoftThreads) : "memory"); }

// What a block does of its run in one job: `tiles` tiles of keys from `first` on.
struct Segment {
  int first, tiles;
  bool two;  // more than 128 rows: two streams of rows
};
__device__ __forceinline__ int rows_of(const AttendCall& c, const Walk& at) { return min(kManyTile, at.x.rows * c.group - at.tile * kManyTile); }
__device__ __forceinline__ Segment segment_of(const AttendCall& c, const Walk& at, int u1) {
  return Segment{at.granule, min(u1, at.job_end()) - at.unit, rows_of(c, at) > kSub};
}
// To what is behind the segment; false if that is the run's end.
__device__ __forceinline__ bool skip(const AttendCall& c, const AttendList& list, const int* ahead, Walk& at, const Segment& s, int u1) {
  at.granule += s.tiles - 1;
  at.unit += s.tiles - 1;
  return at.step(c, list, ahead, u1);
}

// ---- codes to f16 ----------------------------------------------------------------------------------------------------
// One warp's 16 keys of a tile: lane's 16-byte pieces of K or V.  DIM 128: rows 4 j + lane / 8, piece lane % 8; DIM 64: rows 8 j + lane / 4, piece lane % 4.
template <int DIM>
struct Piece {
  static constexpr int kLoads = DIM / 32, kRowLanes = DIM / 16;
  static __device__ __forceinline__ int row(int j, int lane) { return j * (32 / kRowLanes) + lane / kRowLanes; }
};

// 16 codes -> 32 bytes of a swizzled operand row.  `times`: f16x2 factor (values only).
template <int DIM, bool FP8, bool VALUES>
__device__ __forceinline__ void convert_piece(const uint4& x, uint32_t tile, int row, int lane, uint32_t times) {
  const int piece = lane & (Piece<DIM>::kRowLanes - 1);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    four_codes<FP8>(w[i], h[2 * i], h[2 * i + 1]);
    if (VALUES) {
      asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(h[2 * i]) : "r"(times));
      asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(h[2 * i + 1]) : "r"(times));
    }
  }
  const uint32_t at = tile + (piece >> 2) * Many<DIM>::kHalfBytes + row * 128;
  const int chunk = 2 * (piece & 3), turn = DIM == 128 ? piece >> 2 : 0;  // (lanes of the second half the other way round: no two on one bank)
  const uint32_t first = at + ((chunk ^ turn ^ (row & 7)) << 4), second = at + ((chunk ^ turn ^ 1 ^ (row & 7)) << 4);
  if (turn) {
    ptx::st_shared4(first, h[4], h[5], h[6], h[7]);
    ptx::st_shared4(second, h[0], h[1], h[2], h[3]);
  } else {
    ptx::st_shared4(first, h[0], h[1], h[2], h[3]);
    ptx::st_shared4(second, h[4], h[5], h[6], h[7]);
  }
}

template <int DIM, bool FP8>
__device__ __forceinline__ void convert_keys(const AttendCall& c, const AttendList& list, const int* ahead, Control& ctl, uint32_t k_tiles, uint32_t v_tiles, int u0,
                                             int u1, int warp, int lane) {
  using P = Piece<DIM>;
  Walk at;
  at.seek(c, list, ahead, u0);
  if (at.unit >= u1) return;
  uint4 k[P::kLoads], v[P::kLoads];
  float ks = 0.f, vs = 0.f;  // of key `lane` of this warp's 16
  int pool = 0;              // row of the pool of the first of them
  int have = 0;              // how many exist
  int page = 0;              // the page of the tile that `at` stands at, asked for a tile ahead of its keys
  auto find_page = [&] {
    const int key0 = at.granule * kManyKeys + 16 * warp;
    if (key0 < at.x.len) page = chain_load_cached(at.x.table + (key0 >> c.cache.page_shift));
  };
  auto find_keys = [&] {
    const int key0 = at.granule * kManyKeys + 16 * warp;
    have = min(16, at.x.len - key0);
    if ((unsigned)page >= (unsigned)c.cache.num_pages) {
      if (have > 0 && lane == 0 && c.device_status) atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
      page = 0;  // (its keys are as wrong as any)
    }
    pool = (int)pool_row(c.cache, page, at.head, key0);
  };
  const int piece = lane & (P::kRowLanes - 1);
  auto ask = [&](const uint8_t* codes, uint4 (&to)[P::kLoads]) {
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j)
      to[j] = P::row(j, lane) < have ? chain_load(reinterpret_cast<const uint4*>(codes + ((long long)pool + P::row(j, lane)) * DIM + piece * 16)) : make_uint4(0, 0, 0, 0);
  };
  auto ask_scales = [&] {
    ks = lane < have ? chain_load(c.cache.k_scale + pool + lane) : 0.f;
    vs = lane < have ? chain_load(c.cache.v_scale + pool + lane) : 0.f;
  };
  find_page();
  find_keys();
  ask(c.cache.k, k);
  ask_scales();
  ask(c.cache.v, v);
  bool more = at.step(c, list, ahead, u1);
  if (more) find_page();
  for (int i = 0;; ++i) {  // `at` stands a tile further on
    const int slot = i & 1, ring = i & (kScaleRing - 1);
    const uint32_t free_parity = ((i >> 1) & 1) ^ 1u;
    // values' scales: a value row that is not finite makes the weights of the rows that see it NaN, not everybody's sums
    const bool good = fabsf(vs) < INFINITY;
    float top = good ? fabsf(vs) : 0.f;
#pragma unroll
    for (int d = 8; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const int e = top > 0.f ? min(max((int)(__float_as_uint(top) >> 23) - 126, -100), 118) : 0;  // top <= 2^e (lanes 0 to 15)
    const float times = good ? vs * __uint_as_float((unsigned)(127 + kValuePower - e) << 23) : 0.f;
    const float key_scale = good ? ks : __uint_as_float(0x7FC00000u);

    ptx::mbar_wait_warp(ptx::smem_u32(&ctl.k_empty[slot]), free_parity, &ctl.abort);  // (a wait that gives up only marks the results as invalid)
    if (lane < 16) ctl.k_scale[ring][16 * warp + lane] = key_scale;
    if (lane == 0) {
      ctl.exponent[ring][warp] = (float)e;
      ctl.unscale[ring][warp] = __uint_as_float((unsigned)(127 - e - kOffset) << 23);
    }
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j)
      convert_piece<DIM, FP8, false>(k[j], k_tiles + slot * Many<DIM>::kTileBytes, 16 * warp + P::row(j, lane), lane, 0);
    ptx::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      ptx::mbar_arrive(ptx::smem_u32(&ctl.scale_full[ring]));
      ptx::mbar_arrive(ptx::smem_u32(&ctl.k_full[slot]));
    }
    if (more) {
      find_keys();
      ask(c.cache.k, k);
      ask_scales();
    }
    ptx::mbar_wait_warp(ptx::smem_u32(&ctl.v_empty[slot]), free_parity, &ctl.abort);
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j) {
      const float f = __shfl_sync(0xFFFFFFFFu, times, P::row(j, lane));
      convert_piece<DIM, FP8, true>(v[j], v_tiles + slot * Many<DIM>::kTileBytes, 16 * warp + P::row(j, lane), lane, two_f16(f, f));
    }
    ptx::fence_proxy_async_smem();
    ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.v_full[slot]), lane);
    if (!more) break;
    ask(c.cache.v, v);
    more = at.step(c, list, ahead, u1);
    if (more) find_page();
  }
}

// ---- the MMAs -----------------------------------------------------------------------------------------------------------
template <int DIM>
__device__ __forceinline__ void issue_mmas(const AttendCall& c, const AttendList& list, const int* ahead, Control& ctl, uint32_t q_tiles, uint32_t k_tiles, uint32_t v_tiles, int u0,
                           int u1, int lane) {
  using M = Many<DIM>;
  constexpr uint32_t kScores = ptx::umma_idesc_f16(kSub, kManyKeys, false), kOutput = ptx::umma_idesc_f16(kSub, DIM, true);
  const uint32_t tmem = ctl.tmem_base;
  Walk at;
  at.seek(c, list, ahead, u0);
  int visits[2] = {0, 0};  // weights consumed, per stream
  int segments = 0, done = 0;  // tiles before the segment
  for (bool more = at.unit < u1; more;) {
    const Segment seg = segment_of(c, at, u1);
    ptx::mbar_wait_warp(ptx::smem_u32(&ctl.q_full), segments & 1, &ctl.abort);
    ptx::tc_fence_after_sync();
    const int total = seg.two ? 2 * seg.tiles : seg.tiles;
    for (int v = 0; v <= total; ++v) {
      if (v < total) {  // S = Q K^T
        const int tile = seg.two ? v >> 1 : v, i = done + tile, slot = i & 1, stream = v & 1;
        if (!seg.two || stream == 0) {
          ptx::mbar_wait_warp(ptx::smem_u32(&ctl.k_full[slot]), (i >> 1) & 1, &ctl.abort);
          ptx::tc_fence_after_sync();
        }
        const uint64_t a = ptx::umma_desc_sw128(q_tiles + (seg.two ? stream : 0) * M::kTileBytes, 0), b = ptx::umma_desc_sw128(k_tiles + slot * M::kTileBytes, 0);
        ptx::umma_bf16_steps<DIM / 16, M::kHalfBytes, M::kHalfBytes>(tmem + stream * kManyKeys, a, b, kScores, false);
        ptx::umma_commit(ptx::smem_u32(&ctl.s_full[stream]));
        if (!seg.two || stream == 1) ptx::umma_commit(ptx::smem_u32(&ctl.k_empty[slot]));
      }
      if (v > 0) {  // O += P V of the visit before
        const int w = v - 1, tile = seg.two ? w >> 1 : w, i = done + tile, slot = i & 1, stream = w & 1;
        if (!seg.two || stream == 0) ptx::mbar_wait_warp(ptx::smem_u32(&ctl.v_full[slot]), (i >> 1) & 1, &ctl.abort);
        ptx::mbar_wait_warp(ptx::smem_u32(&ctl.p_full[stream]), visits[stream] & 1, &ctl.abort);
        ++visits[stream];
        ptx::tc_fence_after_sync();
        const uint32_t values = v_tiles + slot * M::kTileBytes;
#pragma unroll
        for (int ks = 0; ks < kManyKeys / 16; ++ks)  // 16 keys: 16 rows of 128 bytes further on
          ptx::umma_ts(tmem + 2 * kManyKeys + stream * 128, tmem + stream * kManyKeys + ks * 8, ptx::umma_desc_sw128_mn(values + ks * 2048, M::kHalfBytes), kOutput,
                       w > 1 || ks > 0 ? 1u : 0u);  // (the first visit of either stream begins anew)
        ptx::umma_commit(ptx::smem_u32(&ctl.pv_done[stream]));
        if (!seg.two || stream == 1) ptx::umma_commit(ptx::smem_u32(&ctl.v_empty[slot]));
      }
    }
    done += seg.tiles;
    ++segments;
    more = skip(c, list, ahead, at, seg, u1);
  }
  ptx::umma_commit(ptx::smem_u32(&ctl.last));
  int never = 0;  // the columns are given back behind this: not before the last MMA is done
  ptx::mbar_wait_bounded(ptx::smem_u32(&ctl.last), 0, &never);
  __syncwarp();
}

// ---- softmax ------------------------------------------------------------------------------------------------------------
struct Visit {
  uint32_t s;       // tensor memory address of the logits
  const float* ks;  // scales of the keys, exponents of the groups, and what undoes them
  const float *exponent, *unscale;
};

// One visit's weights with the maximum `m` (base 2): f16 pairs, and their fp32 sum.  `limit`: columns from there on are hidden.
template <bool MASKED>
__device__ __forceinline__ float visit_weights(const Visit& x, float row_scale, float m, int limit, uint32_t (&p)[kManyKeys / 2]) {
  float l = 0.f;
  const float2 rs = make_float2(row_scale, row_scale);
  uint32_t v[2][32];
  ptx::tmem_ld32(x.s, v[0]);
#pragma unroll
  for (int b = 0; b < kManyKeys / 32; ++b) {
    uint32_t(&z)[32] = v[b & 1];
    ptx::tmem_ld_wait_for(z);
    if (b + 1 < kManyKeys / 32) ptx::tmem_ld32(x.s + (b + 1) * 32, v[(b + 1) & 1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int g = 2 * b + h;
      const float add = x.exponent[g] - m + kOffset;
      const float2 plus = make_float2(add, add);
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        const float4 ks = *reinterpret_cast<const float4*>(x.ks + g * 16 + j);
        const uint32_t* const t = z + h * 16 + j;
        float2 t0 = __fmul2_rn(make_float2(__uint_as_float(t[0]), __uint_as_float(t[1])), make_float2(ks.x, ks.y));
        float2 t1 = __fmul2_rn(make_float2(__uint_as_float(t[2]), __uint_as_float(t[3])), make_float2(ks.z, ks.w));
        t0 = __ffma2_rn(t0, rs, plus);
        t1 = __ffma2_rn(t1, rs, plus);
        float2 w0 = make_float2(ptx::ex2_approx(t0.x), ptx::ex2_approx(t0.y)), w1 = make_float2(ptx::ex2_approx(t1.x), ptx::ex2_approx(t1.y));
        if (MASKED) {
          const int k = g * 16 + j;
          w0.x = k < limit ? w0.x : 0.f;
          w0.y = k + 1 < limit ? w0.y : 0.f;
          w1.x = k + 2 < limit ? w1.x : 0.f;
          w1.y = k + 3 < limit ? w1.y : 0.f;
        }
        sum = __fadd2_rn(sum, __fadd2_rn(w0, w1));
        p[(g * 16 + j) / 2] = two_f16(w0.x, w0.y);
        p[(g * 16 + j) / 2 + 1] = two_f16(w1.x, w1.y);
      }
      l = fmaf(sum.x + sum.y, x.unscale[g], l);
    }
  }
  return l;
}

// The largest z + E of the visit's visible keys (-inf: none).
__device__ __forceinline__ float visit_top(const Visit& x, float row_scale, int limit) {
  float top = -INFINITY;
#pragma unroll 1
  for (int b = 0; b < kManyKeys / 32; ++b) {
    uint32_t z[32];
    ptx::tmem_ld32(x.s + b * 32, z);
    ptx::tmem_ld_wait_for(z);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float most = -INFINITY;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float t = __uint_as_float(z[h * 16 + j]) * x.ks[b * 32 + h * 16 + j];
        most = fmaxf(most, b * 32 + h * 16 + j < limit ? t : -INFINITY);
      }
      top = fmaxf(top, fmaf(most, row_scale, x.exponent[2 * b + h]));
    }
  }
  return top;
}

template <int DIM>
__device__ __forceinline__ void rescale_output(uint32_t o, float factor) {
#pragma unroll 1
  for (int i = 0; i < DIM; i += 32) {
    uint32_t v[32];
    ptx::tmem_ld32(o + i, v);
    ptx::tmem_ld_wait_for(v);
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * factor);
    ptx::tmem_st32(o + i, v);
  }
  ptx::tmem_st_wait();
}

// Where a stacked row lies: query row and head.
struct Place {
  long long q_row;
  int head, r;
};
__device__ __forceinline__ Place place_of(const AttendCall& c, const Walk& at, int tile_row) {
  const int i = at.tile * kManyTile + tile_row, r = i / c.group;
  return Place{(long long)at.x.row0 + r, at.head * c.group + i - r * c.group, r};
}

// 32 query rows of a warp into their operand tile, DIM / 8 lanes to a row, scaled by a power of two that makes their bf16 values exact in f16;
// for the lane's own row what takes that back, times the softmax scale.
template <int DIM>
__device__ __forceinline__ float load_queries(const AttendCall& c, const Walk& at, int first_row, uint32_t tile, int row_in_tile, int lane) {
  constexpr int kLanes = DIM / 8, kRows = 32 / kLanes, kAtOnce = 8;  // rows of a load; loads in flight
  const int sub = lane / kLanes, piece = lane % kLanes;
  float mine = 0.f;
#pragma unroll
  for (int j0 = 0; j0 < 32 / kRows; j0 += kAtOnce) {
    uint4 x[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int tile_row = first_row + (j0 + j) * kRows + sub;
      const Place q = place_of(c, at, tile_row);
      x[j] = q.r < at.x.rows ? chain_load_cached(reinterpret_cast<const uint4*>(c.q + q.q_row * c.q_st + (long long)q.head * c.q_sh + piece * 8)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const unsigned m = 0x7FFF7FFFu;
      unsigned top = __vmaxu2(__vmaxu2(x[j].x & m, x[j].y & m), __vmaxu2(x[j].z & m, x[j].w & m));  // what is not a number is larger than the rest
      top = max(top >> 16, top & 0xFFFFu);
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
      const float to = to_one(__uint_as_float(top << 16));
      const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
      uint32_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = two_f16(__uint_as_float(w[i] << 16) * to, __uint_as_float(w[i] & 0xFFFF0000u) * to);
      const int row = row_in_tile + (j0 + j) * kRows + sub;
      ptx::st_shared4(tile + (piece >> 3) * Many<DIM>::kHalfBytes + row * 128 + (((piece & 7) ^ (row & 7)) << 4), h[0], h[1], h[2], h[3]);
      const float of_row = __shfl_sync(0xFFFFFFFFu, to, lane % kRows * kLanes);
      if (lane / kRows == j0 + j) mine = c.scale_log2 / of_row;
    }
  }
  return mine;
}

template <int DIM>
__device__ __forceinline__ void softmax(const AttendCall& c, const AttendList& list, const int* ahead, Control& ctl, uint32_t q_tiles, int u0, int u1, int warp, int lane) {
  using M = Many<DIM>;
  const int stream = warp >> 2, row = (warp & 3) * 32 + lane;
  const uint32_t lanes = ctl.tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
  const uint32_t s = lanes + stream * kManyKeys, o = lanes + 2 * kManyKeys + stream * 128;
  Walk at;
  at.seek(c, list, ahead, u0);
  int visits = 0, done = 0;  // of this stream; tiles before the segment
  for (bool more = at.unit < u1; more;) {
    const Segment seg = segment_of(c, at, u1);
    // With two streams of rows a thread's row is of its stream's half; else threads of both streams have the same one.
    const int warp_row = (seg.two ? stream * kSub : 0) + (warp & 3) * 32;
    const float row_scale = load_queries<DIM>(c, at, warp_row, q_tiles + stream * M::kTileBytes, (warp & 3) * 32, lane);
    ptx::fence_proxy_async_smem();
    ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.q_full), lane);
    int sees, all_see;
    bool there;
    {
      const Place q = place_of(c, at, warp_row + lane);
      there = q.r < at.x.rows;
      sees = !there ? 0 : at.x.own && c.causal ? max(0, at.x.len - at.x.rows + q.r + 1) : at.x.len;
      all_see = __reduce_min_sync(0xFFFFFFFFu, there ? sees : INT_MAX);
    }

    float m = -INFINITY, l = 0.f;
    bool first = true;
#pragma unroll 1
    for (int tile = seg.two ? 0 : stream; tile < seg.tiles; tile += seg.two ? 1 : 2) {
      const int n = done + tile, ring = n & (kScaleRing - 1);
      const Visit x{s, ctl.k_scale[ring], ctl.exponent[ring], ctl.unscale[ring]};
      ptx::mbar_wait_warp(ptx::smem_u32(&ctl.scale_full[ring]), (n / kScaleRing) & 1, &ctl.abort);
      ptx::mbar_wait_warp(ptx::smem_u32(&ctl.s_full[stream]), visits & 1, &ctl.abort);
      ptx::tc_fence_after_sync();
      const int key0 = (seg.first + tile) * kManyKeys;
      const int limit = sees - key0;  // columns of this row that are visible
      uint32_t p[kManyKeys / 2];
      float sum = 0.f;
      bool redo = first, masked = key0 + kManyKeys > all_see;
      if (!first && !masked) {
        sum = visit_weights<false>(x, row_scale, m == -INFINITY ? 0.f : m, limit, p);
        uint32_t most[2] = {p[0], p[1]};
#pragma unroll
        for (int j = 2; j < kManyKeys / 2; ++j) asm("max.f16x2 %0, %0, %1;" : "+r"(most[j & 1]) : "r"(p[j]));
        asm("max.f16x2 %0, %0, %1;" : "+r"(most[0]) : "r"(most[1]));
        const unsigned top = max(most[0] >> 16, most[0] & 0xFFFFu);  // (not negative: bits compare as values)
        redo = __any_sync(0xFFFFFFFFu, there && (top > kMostWeight || m == -INFINITY));
      }
      if (redo || masked) {  // the visit's own maximum first
        const float top = visit_top(x, row_scale, limit);
        if (first) {
          m = top;
        } else if (__any_sync(0xFFFFFFFFu, top > m)) {  // the sums so far
          const float to = fmaxf(top, m), factor = m == -INFINITY ? 0.f : ptx::ex2_approx(m - to);
          l *= factor;
          m = to;
          ptx::mbar_wait_warp(ptx::smem_u32(&ctl.pv_done[stream]), (visits - 1) & 1, &ctl.abort);
          ptx::tc_fence_after_sync();
          rescale_output<DIM>(o, factor);
        }
        sum = visit_weights<true>(x, row_scale, m == -INFINITY ? 0.f : m, limit, p);
      }
      l += sum;
      __syncwarp();
      ptx::tmem_st32(s, p);
      ptx::tmem_st32(s + 32, p + 32);
      ptx::tmem_st_wait();
      ptx::tc_fence_before_sync();
      ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.p_full[stream]), lane);
      first = false;
      ++visits;
    }
    if (!first) ptx::mbar_wait_warp(ptx::smem_u32(&ctl.pv_done[stream]), (visits - 1) & 1, &ctl.abort);

    // The end of the segment.  O is sum 2^(z - m) v times 2^(kOffset + kValuePower).
    const bool both = !seg.two && seg.tiles > 1;  // the other stream has a part of the row, too
    float other = 0.f, back = __uint_as_float((unsigned)(127 - kOffset - kValuePower) << 23);
    if (both) {
      ctl.row_ml[stream][row] = make_float2(m, l);
      ptx::tc_fence_before_sync();
      soft_sync();
      const float2 ml = ctl.row_ml[stream ^ 1][row];
      const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.f : top;
      const float mine = ptx::ex2_approx(m - base), theirs = ptx::ex2_approx(ml.x - base);
      l = l * mine + ml.y * theirs;
      other = back * theirs;
      back *= mine;
      m = top;
    }
    ptx::tc_fence_after_sync();
    const bool whole = at.job_first() >= u0 && at.job_end() <= u1, final = whole && c.prefixes == 0;
    const long long level = at.x.own ? 0ll : (long long)c.total_q * c.hq;
    const long long part = ((long long)blockIdx.x * 2 + (at.job_first() < u0 ? 0 : 1)) * kManyTile;  // the block's place for what it did not finish
    if (final) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      back *= inv;
      other *= inv;
    }
    // A stream writes its rows; where both have the same rows, half of the columns each.  By 64 columns through this warp's part of the
    // stream's query tile, which nobody needs any more, so that rows are written in whole lines.
    const int from = both ? stream * (DIM / 2) : 0, to = seg.two ? DIM : both ? from + DIM / 2 : stream == 0 ? DIM : 0;
    constexpr int kWide = DIM == 128 ? 64 : 32, kLanes = kWide / 4, kRows = 32 / kLanes;
    const uint32_t stage = q_tiles + stream * M::kTileBytes + (warp & 3) * (32 * kWide * 4);
#pragma unroll 1
    for (int d = from; d < to; d += kWide) {
#pragma unroll
      for (int h = 0; h < kWide; h += 32) {
        uint32_t v[32], y[32];
        ptx::tmem_ld32(o + d + h, v);
        if (both) ptx::tmem_ld32(lanes + 2 * kManyKeys + (stream ^ 1) * 128 + d + h, y);
        ptx::tmem_ld_wait_for(v);
        if (both) ptx::tmem_ld_wait_for(y);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          float f = __uint_as_float(v[j]) * back;
          if (both) f = fmaf(__uint_as_float(y[j]), other, f);
          v[j] = __float_as_uint(f);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          ptx::st_shared4(stage + lane * (kWide * 4) + (((h / 4 + j) ^ (lane & 7)) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
      }
      __syncwarp();
      const int piece = lane % kLanes;
#pragma unroll 4
      for (int j = 0; j < 32 / kRows; ++j) {
        const int r = j * kRows + lane / kLanes;
        const uint4 x = ptx::ld_shared4(stage + r * (kWide * 4) + ((piece ^ (r & 7)) << 4));
        const Place q = place_of(c, at, warp_row + r);
        if (q.r >= at.x.rows) continue;
        if (final) {
          *reinterpret_cast<uint2*>(c.out + q.q_row * c.o_st + (long long)q.head * c.o_sh + d + piece * 4) =
              make_uint2(pair_bf16(__uint_as_float(x.x), __uint_as_float(x.y)), pair_bf16(__uint_as_float(x.z), __uint_as_float(x.w)));
        } else {
          float* const out = whole ? c.whole_out + (level + q.q_row * c.hq + q.head) * DIM : list.part_out + (part + warp_row + r) * DIM;
          *reinterpret_cast<uint4*>(out + d + piece * 4) = x;
        }
      }
      __syncwarp();
    }
    if (there && (seg.two || stream == 0)) {
      const Place q = place_of(c, at, warp_row + lane);
      if (final) {
        if (c.lse_out) c.lse_out[q.q_row * c.hq + q.head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      } else {
        *(whole ? c.whole_ml + level + q.q_row * c.hq + q.head : list.part_ml + part + warp_row + lane) = make_float2(m, l);
      }
    }
    ptx::tc_fence_before_sync();
    soft_sync();  // the other stream has read this one's O, and Q is free
    done += seg.tiles;
    more = skip(c, list, ahead, at, seg, u1);
  }
}

template <int DIM, bool FP8>
__global__ void __launch_bounds__(kThreads, 1) attend_many_kernel(AttendCall c, AttendList list) {
  using M = Many<DIM>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(16) Control ctl;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned char* const smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t q_tiles = ptx::smem_u32(smem), k_tiles = q_tiles + 2 * M::kTileBytes, v_tiles = k_tiles + 2 * M::kTileBytes;
  int* const ahead = reinterpret_cast<int*>(smem + M::kOperands);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(ptx::smem_u32(&ctl.k_full[i]), kConvWarps);
      ptx::mbar_init(ptx::smem_u32(&ctl.v_full[i]), kConvWarps);
      ptx::mbar_init(ptx::smem_u32(&ctl.k_empty[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.v_empty[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.s_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.p_full[i]), kSoftWarps / 2);
      ptx::mbar_init(ptx::smem_u32(&ctl.pv_done[i]), 1);
    }
    for (int i = 0; i < kScaleRing; ++i) ptx::mbar_init(ptx::smem_u32(&ctl.scale_full[i]), kConvWarps);
    ptx::mbar_init(ptx::smem_u32(&ctl.q_full), kSoftWarps);
    ptx::mbar_init(ptx::smem_u32(&ctl.last), 1);
    ctl.abort = 0;
    ptx::fence_barrier_init();
  }
  chain_enter_late(c);
  pdl_wait();  // everything may be what earlier work wrote; and tensor memory is taken when all earlier work has ended
  if (warp == kIssueWarp) {
    ptx::tmem_alloc(ptx::smem_u32(&ctl.tmem_base), kTmemCols);
    ptx::tmem_relinquish();
    ptx::tc_fence_before_sync();
  }
  const int total = open_list<kThreads>(c, list, ahead, ctl.warp_sum);  // (two block-wide barriers)
  ptx::tc_fence_after_sync();
  const int workers = workers_of(list, total), u0 = run_start(min((int)blockIdx.x, workers), workers, total), u1 = run_start(min((int)blockIdx.x + 1, workers), workers, total);
  if (warp < kSoftWarps) {
    ptx::more_registers<kSoftRegs>();
    if (u0 < u1) softmax<DIM>(c, list, ahead, ctl, q_tiles, u0, u1, warp, lane);
  } else if (warp < kIssueWarp) {
    ptx::fewer_registers<kConvRegs>();
    if (u0 < u1) convert_keys<DIM, FP8>(c, list, ahead, ctl, k_tiles, v_tiles, u0, u1, warp - kSoftWarps, lane);
  } else {
    ptx::fewer_registers<kIssueRegs>();
    if (u0 < u1 && warp == kIssueWarp) issue_mmas<DIM>(c, list, ahead, ctl, q_tiles, k_tiles, v_tiles, u0, u1, lane);
  }
  pdl_trigger();
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  if (warp == kIssueWarp) ptx::tmem_dealloc(ctl.tmem_base, kTmemCols);
  if (threadIdx.x == 0 && ctl.abort && c.device_status) atomicOr(c.device_status, FASTAV_DEV_WAIT_EXPIRED);
}

template <int DIM>
size_t many_smem(int entries) { return 1024 + Many<DIM>::kOperands + (size_t)(entries + 1) * 4; }

template <int DIM, bool FP8>
cudaError_t run(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  const cudaError_t e = once_per_context([] {
    cudaFuncAttributes a;
    const cudaError_t got = cudaFuncGetAttributes(&a, attend_many_kernel<DIM, FP8>);
    if (got != cudaSuccess) return got;
    if (a.numRegs * kThreads < kRegsNeeded) return cudaErrorInvalidConfiguration;  // the softmax's warps would wait for registers for ever
    return cudaFuncSetAttribute(attend_many_kernel<DIM, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)many_smem<DIM>(FASTAV_ATTEND_MAX_BATCH));
  });
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_chained(attend_many_kernel<DIM, FP8>, dim3(list.grid), dim3(kThreads), many_smem<DIM>(list.entries()), stream, c, list);
}

}  // namespace

cudaError_t launch_attend_many(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  if (c.cache.dim == 128) return c.cache.fp8 ? run<128, true>(c, list, stream) : run<128, false>(c, list, stream);
  return c.cache.fp8 ? run<64, true>(c, list, stream) : run<64, false>(c, list, stream);
}

}  // namespace fastav
