// Attention over the 8-bit cache for many query rows per KV head: a prefix that a batch shares, a question's tokens at once.
//
// More than 16 rows.  Dense contractions, so they run on the fifth-generation tensor cores: S = Q K^T and O += P V (tcgen05.mma, f16 operands, fp32 sums in
// tensor memory).  A unit is 128 keys of one KV head for up to 256 stacked query rows.  Per block, one per SM:
//
//   warps 0-7    softmax, a thread per row.  Warps 0-3 and 4-7 are two STREAMS with an S, an O and two P of their own.  With more than 128
//                rows the streams are the two halves of the rows and share every key; with fewer they take 64 keys of every tile each and
//                their sums are joined at the end.  A VISIT is 64 keys of a stream.
//   warps 8-15   codes -> f16, 16 keys of every tile each, to the operand tiles in shared memory.  What a tile ahead is asked for stays in
//                flight: K's codes in 16 KB of shared memory (asynchronous copies), V's in registers, and V's rows are called into L2 when
//                K's are.  (Both in registers: each was asked for only half a tile ahead, 2.4 us a tile from HBM instead of 1.65;
//                16 sequences of 3,000 keys, 64 rows: 71 us instead of 60.)
//   warps 16-19  issue the MMAs: the S of a stream's next visit as soon as the logits of this one are in registers, PV when its weights are
//                there
//
// Tensor memory is used up: 2 x 64 columns of S, 4 x 32 of P, 2 x 128 of O.  (128 keys at a time with P in the place of S: the next S had to
// wait for PV, and a stream stood still for the way to the issuing warp, PV, QK and back; 16 questions on 16,384 keys, Mistral-7B shapes,
// 597 us instead of 579 at that step.)  Registers move from the warps that need few to the softmax's, which hold a visit's logits.
//
// The keys' scales multiply the logits in fp32.  The values' scales are looked at sixteen keys at a time.  Where they lie within a factor of 2^kEven of
// each other (EVEN groups), a value's operand is code * scale / 2^E * 2^kValuePower, rounded once, with 2^E the least power of two above all sixteen, and E
// joins the exponent: w = 2^(z + E - m + kOffset) is rounded to f16 for the matrix pipe, l = sum w 2^(-E - kOffset) stays in fp32.  m is the row's largest
// z + E.  So f16 sees one rounding of the weight and one of the value (2^-11 each), and what it cannot hold, 2^-25 of a unit, is 2^-36 of the row's
// largest product of weight and scale where the scales of sixteen neighbours are alike, 2^-30 where they differ by 2^kEven.
//
// Other groups (a row of zeros, an outlier, a hidden key's large value) would lose the smaller values that way: f16 has no room for both.  There
// a value's operand is its code alone, its own scale's exponent e counts for m, log2 of the scale joins its logit, and the weights are summed up ahead of that.  That
// takes the exponentials twice: 16 questions on 16,384 keys with every eighth group uneven 611 us instead of 527 at that step.  (The scales multiplying
// the weights in fp32 in every group: 607 us.  What it takes is not the products, 12 us, but two 16-byte loads per eight logits, which every lane of a warp gets.)
//
// 16 questions of 64 to 128 tokens on 16,384 keys (346 GFLOP): 523 us, 0.66 PFLOP/s.  Bound by the chains of the converting and softmax warps per
// tile (5,200 cycles, of which the MMAs take 2,600 and the exponentials 2,000).  Taking the weights with the maximum so far first, and a new one
// only where f16 overflows, spills: 619 us instead of 500 at that step.
//
// O is rescaled only when a row's maximum has grown by kSlack: until then its weights are larger than 2^kOffset, which f16 has room for.
#include <limits.h>

#include "attend.cuh"
#include "attend_8bit.cuh"
#include "sm100_ptx.cuh"

namespace fastav {
namespace {

constexpr int kSub = 128;  // rows of a stream
constexpr int kVisit = 64;  // keys of a visit
constexpr int kSoftWarps = 8, kConvWarps = 8, kIssueWarp = kSoftWarps + kConvWarps, kWarps = kIssueWarp + 4;
constexpr int kSoftThreads = 32 * kSoftWarps, kThreads = 32 * kWarps;
// Registers a thread has per role.  What the three take together has to fit into what the block is launched with (checked before the launch).
constexpr int kSoftRegs = 144, kConvRegs = 72, kIssueRegs = 48;
constexpr int kRegsNeeded = 32 * (kSoftWarps * kSoftRegs + kConvWarps * kConvRegs + 4 * kIssueRegs);
constexpr int kGroups = kManyKeys / 16;          // of 16 keys: a converting warp's
constexpr int kScaleRing = 4;
constexpr int kValuePower = 7;                   // a value operand is below 2^16
constexpr int kEven = 6;
constexpr int kOffset = 12;                      // the largest weight of a row's first visit is up to 2^kOffset ...
constexpr float kSlack = 3.9f;                   // ... and the maximum is moved when one would be this much (log2) above that (f16 ends at 2^16)
// Bounds of the exponents.  A key's from kLeastExponent on: 2^(z - m) stays below 2^74 (value rows that are smaller, 10^-19 and less, keep fewer bits).
// E of an uneven group up to kMostGroup: its weights without their scales stay below 2^116, and above 2^-80 where all scales are as large as can be.
constexpr int kLeastExponent = -70, kMostGroup = 30;
constexpr int kTmemCols = 512, kWeightsAt = 2 * kVisit, kOutputAt = kWeightsAt + 4 * (kVisit / 2);  // columns: S, P, O
static_assert(kConvWarps == kGroups && kOutputAt + 2 * 128 <= kTmemCols);

template <int DIM>
struct Many {
  static constexpr int kHalves = DIM / 64;               // 128-byte column blocks of an operand tile
  static constexpr int kHalfBytes = 128 * 128;           // 128 rows of 128 bytes
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kOperands = 6 * kTileBytes;       // Q twice, K twice, V twice
  static constexpr int kCodes = kManyKeys * DIM;         // K's codes of the tile after
};

struct Control {
  // [stream], [slot of a tile] or [stream][buffer of the weights]
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], s_free[2], p_full[2][2], pv_done[2][2], scale_full[kScaleRing], q_full, last;
  uint32_t tmem_base;
  int abort;
  int warp_sum[kWarps];
  alignas(16) float k_scale[kScaleRing][kManyKeys];
  alignas(16) float v_exponent[kScaleRing][kManyKeys], v_log[kScaleRing][kManyKeys];  // of values in groups that are not even: e, the least with scale <= 2^e; log2 scale - E
  float exponent[kScaleRing][kGroups];                                                // E
  float bound[kScaleRing][kGroups], unscale[kScaleRing][kGroups];                     // of even groups E and 2^(-E - kOffset), else -inf and 0
  alignas(4) uint8_t even[kScaleRing][kGroups];
  float row_scale[2][kSub];                                           // of a stream's query rows
  float2 row_ml[2][kSub];                                             // the streams' statistics, to be joined
};

// Whether all three phases are over (a whole warp's answer).
__device__ __forceinline__ bool wait_all(uint32_t a, uint32_t a_parity, uint32_t b, uint32_t b_parity, uint32_t c, uint32_t c_parity) {
  const bool x = ptx::mbar_try_wait(a, a_parity), y = ptx::mbar_try_wait(b, b_parity), z = ptx::mbar_try_wait(c, c_parity);
  return __all_sync(0xFFFFFFFFu, x && y && z);
}
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

// 2^e for e of -126 and more, up to 127.
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(127 + e) << 23); }

// ---- codes to f16 ----------------------------------------------------------------------------------------------------
// One warp's 16 keys of a tile, 16 codes per lane and load.  DIM 128: a load is 4 keys of 8 pieces; lane bits 0, 1 and 3 name the piece, 2 and 4 the
// key, so that the eight lanes of a phase store to eight different banks' quarters.  DIM 64: 8 keys of 4 pieces.
template <int DIM>
struct Piece {
  static constexpr int kLoads = DIM / 32, kRows = 16 / kLoads;  // loads; keys of one
  int piece, row;
  uint32_t to[2];  // where the first half of the piece goes in an operand tile, from the tile's start: keys of even and of odd loads
  __device__ __forceinline__ Piece(int warp, int lane) {
    piece = DIM == 128 ? (lane & 3) | (lane >> 1 & 4) : lane & 3;
    row = DIM == 128 ? (lane >> 2 & 1) | (lane >> 3 & 2) : lane >> 2;
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
      const int r = 16 * warp + row + odd * kRows;
      to[odd] = (piece >> 2) * Many<DIM>::kHalfBytes + (16 * warp + row) * 128 + (((2 * (piece & 3)) ^ (r & 7)) << 4);
    }
  }
  __device__ __forceinline__ int key(int j) const { return j * kRows + row; }
};

// 16 codes -> 32 bytes of a swizzled operand row.  Values only: times a factor in two f16 parts (twice each), rounded once.
template <bool FP8, bool VALUES>
__device__ __forceinline__ void convert_piece(const uint4& x, uint32_t at, uint32_t times, uint32_t rest) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    four_codes<FP8>(w[i], h[2 * i], h[2 * i + 1]);
    if (VALUES)
#pragma unroll
      for (int j = 2 * i; j < 2 * i + 2; ++j) {
        uint32_t small;
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(small) : "r"(h[j]), "r"(rest));
        asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(h[j]) : "r"(times), "r"(small));
      }
  }
  ptx::st_shared4(at, h[0], h[1], h[2], h[3]);
  ptx::st_shared4(at ^ 16, h[4], h[5], h[6], h[7]);
}

template <int DIM, bool FP8>
__device__ __forceinline__ void convert_keys(const AttendCall& c, const AttendList& list, const int* ahead, Control& ctl, uint32_t k_tiles, uint32_t v_tiles, uint32_t codes_at,
                                             int u0, int u1, int warp, int lane) {
  using P = Piece<DIM>;
  const P mine(warp, lane);
  Walk at;
  at.seek(c, list, ahead, u0);
  if (at.unit >= u1) return;
  uint4 v[P::kLoads];
  const uint32_t my_codes = codes_at + warp * P::kLoads * 512 + lane * 16;  // of K: what a lane copies there is what it reads
  float ks = 0.f, vs = 0.f;  // of key `lane` of this warp's 16
  int pool = 0;              // row of the pool of the first of them
  int have = 0;              // how many exist
  int page = 0;              // the page of the tile that `at` stands at, asked for a tile ahead of its keys
  auto find_page = [&] {
    const int key0 = at.granule * kManyKeys + 16 * warp;
    if (key0 < at.x.len) page = index_load(at.x.table + (key0 >> c.cache.page_shift), !list.through_l2);
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
  // (What lies behind a sequence's end in its last page may be anything: the logits of such keys are hidden, and values are zeroed below.)
  auto ask = [&](const uint8_t* codes, uint4 (&to)[P::kLoads]) {
    const uint8_t* const from = codes + (long long)pool * DIM + mine.row * DIM + mine.piece * 16;
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j) to[j] = chain_load(reinterpret_cast<const uint4*>(from + j * P::kRows * DIM));
  };
  auto copy_keys = [&] {
    const uint8_t* const from = c.cache.k + (long long)pool * DIM + mine.row * DIM + mine.piece * 16;
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j) ptx::copy_async<16>(my_codes + j * 512, from + j * P::kRows * DIM);
    ptx::copies_commit();
  };
  auto ask_scales = [&] {
    ks = lane < have ? chain_load(c.cache.k_scale + pool + lane) : 0.f;
    vs = lane < have ? chain_load(c.cache.v_scale + pool + lane) : 0.f;
  };
  find_page();
  find_keys();
  copy_keys();
  ask_scales();
  ask(c.cache.v, v);
  bool more = at.step(c, list, ahead, u1);
  if (more) find_page();
  for (int i = 0;; ++i) {  // `at` stands a tile further on
    const int slot = i & 1, ring = i & (kScaleRing - 1);
    const uint32_t free_parity = ((i >> 1) & 1) ^ 1u;
    ptx::mbar_wait_warp(ptx::smem_u32(&ctl.k_empty[slot]), free_parity, &ctl.abort);  // (a wait that gives up only marks the results as invalid)
    ptx::copies_wait<0>();
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j)
      convert_piece<FP8, false>(ptx::ld_shared4(my_codes + j * 512), k_tiles + slot * Many<DIM>::kTileBytes + mine.to[j & 1] + j * P::kRows * 128, 0, 0);
    ptx::fence_proxy_async_smem();
    ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.k_full[slot]), lane);
    const float key = ks, value = vs;  // the scales are looked at when what comes next is under way: nobody needs them before the logits
    const int exist = have;
    if (more) {
      find_keys();
      copy_keys();
      ask_scales();
      if (lane < 16) ptx::prefetch_l2(c.cache.v + (long long)(pool + lane) * DIM);
    }
    // values' scales: a value row that is not finite makes the weights of the rows that see it NaN, not everybody's sums
    const bool good = fabsf(value) < INFINITY;
    const int own = max(good ? (int)(__float_as_uint(fabsf(value)) >> 23) - 126 : kLeastExponent, kLeastExponent);  // |value| <= 2^own
    unsigned both = (unsigned)own << 16 | (lane < exist && good ? -own : -1000) & 0xFFFF;  // the largest; the least, negated
#pragma unroll
    for (int d = 8; d; d >>= 1) both = __vmaxs2(both, __shfl_xor_sync(0xFFFFFFFFu, both, d));
    const int largest = (int)both >> 16;
    const bool even = largest + (int)(short)both <= kEven;  // (lanes 0 to 15)
    const int e = even ? largest : min(largest, kMostGroup);
    const float factor = !good ? 0.f : even ? value * power_of_two(kValuePower - e) : copysignf(1 << kValuePower, value), coarse = __uint_as_float(__float_as_uint(factor) & 0xFFFFE000u);
    const uint32_t factors = two_f16(coarse, factor - coarse);
    const float key_scale = good ? key * kKeyScaleFactor : __uint_as_float(0x7FC00000u);
    if (lane < 16) ctl.k_scale[ring][16 * warp + lane] = key_scale;
    if (!even && lane < 16) {
      ctl.v_exponent[ring][16 * warp + lane] = (float)own;
      ctl.v_log[ring][16 * warp + lane] = good ? log2f(fabsf(value)) - (float)e : 0.f;
    }
    if (lane == 0) {
      ctl.exponent[ring][warp] = (float)e;
      ctl.even[ring][warp] = even;
      ctl.bound[ring][warp] = even ? (float)e : -INFINITY;
      ctl.unscale[ring][warp] = even ? power_of_two(-e) * (1.f / (1 << kOffset)) : 0.f;
    }
    ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.scale_full[ring]), lane);
    ptx::mbar_wait_warp(ptx::smem_u32(&ctl.v_empty[slot]), free_parity, &ctl.abort);
    if (exist < 16)
#pragma unroll
      for (int j = 0; j < P::kLoads; ++j)
        if (mine.key(j) >= exist) v[j] = make_uint4(0, 0, 0, 0);  // (e4m3 has NaN, which a weight of 0 does not take away)
#pragma unroll
    for (int j = 0; j < P::kLoads; ++j) {
      const uint32_t two = __shfl_sync(0xFFFFFFFFu, factors, mine.key(j));
      convert_piece<FP8, true>(v[j], v_tiles + slot * Many<DIM>::kTileBytes + mine.to[j & 1] + j * P::kRows * 128, __byte_perm(two, two, 0x1010), __byte_perm(two, two, 0x3232));
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
// Four warps issue, QK and PV of either stream each, on a scheduler of their own: what lies between two visits' MMAs (waits that are over
// already, addresses, commits) is some hundred cycles of a warp among busy ones, and one warp for all of it left the matrix pipe idle half of the
// time.  S and P being apart, the four need not know of each other; tiles of keys are given back by two arrivals.
template <int DIM, bool SCORES>
__device__ __forceinline__ void issue_mmas(const AttendCall& c, const AttendList& list, const int* ahead, Control& ctl, uint32_t q_tiles, uint32_t k_tiles, uint32_t v_tiles, int u0,
                                           int u1, int stream) {
  using M = Many<DIM>;
  constexpr uint32_t kScores = ptx::umma_idesc_f16(kSub, kVisit, false), kOutput = ptx::umma_idesc_f16(kSub, DIM, true);
  constexpr uint32_t kHalfTile = kVisit * 128 >> 4, kTile = M::kTileBytes >> 4;  // in units of a descriptor's address
  const uint32_t tmem = ctl.tmem_base;
  const uint64_t q_desc = ptx::umma_desc_sw128(q_tiles, 0), tile_desc = SCORES ? ptx::umma_desc_sw128(k_tiles, 0) : ptx::umma_desc_sw128_mn(v_tiles, M::kHalfBytes);
  const uint32_t full = ptx::smem_u32(SCORES ? &ctl.k_full[0] : &ctl.v_full[0]), empty = ptx::smem_u32(SCORES ? &ctl.k_empty[0] : &ctl.v_empty[0]);
  const uint32_t s_full = ptx::smem_u32(&ctl.s_full[stream]), s_free = ptx::smem_u32(&ctl.s_free[stream]);
  const uint32_t p_full = ptx::smem_u32(&ctl.p_full[stream][0]), pv_done = ptx::smem_u32(&ctl.pv_done[stream][0]);
  Walk at;
  at.seek(c, list, ahead, u0);
  int segments = 0, tile = 0, visit = 0;  // of the run
  for (bool more = at.unit < u1; more; ++segments) {
    const Segment seg = segment_of(c, at, u1);
    const int halves = seg.two ? 2 : 1;
    if (SCORES) ptx::mbar_wait_warp(ptx::smem_u32(&ctl.q_full), segments & 1, &ctl.abort);
    const uint64_t a_desc = q_desc + (seg.two ? stream * kTile : 0);
#pragma unroll 1
    for (int t = 0; t < seg.tiles; ++t, ++tile) {
      const int slot = tile & 1;
      ptx::mbar_wait_warp(full + slot * 8, (tile >> 1) & 1, &ctl.abort);
#pragma unroll 1
      for (int h = 0; h < halves; ++h, ++visit) {
        const uint64_t b_desc = tile_desc + (slot * kTile + (seg.two ? h : stream) * kHalfTile);
        if (SCORES) {  // S = Q K^T
          if (t + h > 0) ptx::mbar_wait_warp(s_free, (visit - 1) & 1, &ctl.abort);
          ptx::tc_fence_after_sync();
          ptx::umma_bf16_steps<DIM / 16, M::kHalfBytes, M::kHalfBytes>(tmem + stream * kVisit, a_desc, b_desc, kScores, false);
          ptx::umma_commit(s_full);
        } else {  // O += P V
          const int buffer = visit & 1;
          ptx::mbar_wait_warp(p_full + buffer * 8, (visit >> 1) & 1, &ctl.abort);
          ptx::tc_fence_after_sync();
          const uint32_t d = tmem + kOutputAt + stream * 128, a = tmem + kWeightsAt + (stream * 2 + buffer) * (kVisit / 2);
#pragma unroll
          for (int ks = 0; ks < kVisit / 16; ++ks)  // 16 keys: 8 columns of weights, 16 rows of 128 bytes of values
            ptx::umma_ts(d, a + ks * 8, b_desc + ks * (16 * 128 >> 4), kOutput, t + h + ks > 0 ? 1u : 0u);
          ptx::umma_commit(pv_done + buffer * 8);
        }
      }
      ptx::umma_commit(empty + slot * 8);
    }
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
  const float *ks, *ve, *log_vs, *bound, *exponent, *unscale;  // as in Control
  const uint8_t* even_at;
};

// A visit's logits times the scales of their keys (and not yet of the row), and the largest z + e of the groups whose scales are even; `limit`: columns from there on are hidden.
__device__ __forceinline__ float visit_logits(const Visit& x, float row_scale, bool masked, int limit, float2 (&t)[kVisit / 2]) {
  uint32_t (&v)[kVisit / 32][32] = reinterpret_cast<uint32_t(&)[kVisit / 32][32]>(t);
#pragma unroll
  for (int b = 0; b < kVisit / 32; ++b) ptx::tmem_ld32(x.s + b * 32, v[b]);
#pragma unroll
  for (int b = 0; b < kVisit / 32; ++b) ptx::tmem_ld_wait_for(v[b]);
#pragma unroll
  for (int j = 0; j < kVisit / 2; j += 2) {
    const float4 ks = *reinterpret_cast<const float4*>(x.ks + 2 * j);
    t[j] = __fmul2_rn(t[j], make_float2(ks.x, ks.y));
    t[j + 1] = __fmul2_rn(t[j + 1], make_float2(ks.z, ks.w));
  }
  if (masked) {
#pragma unroll
    for (int j = 0; j < kVisit / 2; ++j) {
      if (2 * j >= limit) t[j].x = -INFINITY;
      if (2 * j + 1 >= limit) t[j].y = -INFINITY;
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int g = 0; g < kVisit / 16; ++g) {
    float most = -INFINITY;
#pragma unroll
    for (int j = g * 8; j < g * 8 + 8; ++j) most = ptx::max3(most, t[j].x, t[j].y);
    top = fmaxf(top, fmaf(most, row_scale, x.bound[g]));
  }
  return top;
}
// ... and of the others.
__device__ __forceinline__ float uneven_top(const Visit& x, uint32_t even, float row_scale, float top, const float2 (&t)[kVisit / 2]) {
  const float2 rs = make_float2(row_scale, row_scale);
#pragma unroll
  for (int g = 0; g < kVisit / 16; ++g) {
    if (even >> 8 * g & 1) continue;
#pragma unroll
    for (int j = g * 8; j < g * 8 + 8; j += 2) {
      const float4 ve = *reinterpret_cast<const float4*>(x.ve + 2 * j);
      const float2 a = __ffma2_rn(t[j], rs, make_float2(ve.x, ve.y)), b = __ffma2_rn(t[j + 1], rs, make_float2(ve.z, ve.w));
      top = ptx::max3(ptx::max3(top, a.x, a.y), b.x, b.y);
    }
  }
  return top;
}
// For these, ahead of the weights: their fp32 sum; and the logits, times the row's scale, get the logarithms of their values' scales.
__device__ __forceinline__ float uneven_weights(const Visit& x, uint32_t even, float row_scale, float m, float2 (&t)[kVisit / 2]) {
  float l = 0.f;
  const float2 rs = make_float2(row_scale, row_scale);
#pragma unroll
  for (int g = 0; g < kVisit / 16; ++g) {
    if (even >> 8 * g & 1) continue;
    const float add = x.exponent[g] - m;
    float sum = 0.f;
#pragma unroll
    for (int j = g * 8; j < g * 8 + 8; j += 2) {
      const float4 log_vs = *reinterpret_cast<const float4*>(x.log_vs + 2 * j);
      sum += ptx::ex2_approx(fmaf(t[j].x, row_scale, add)) + ptx::ex2_approx(fmaf(t[j].y, row_scale, add)) + ptx::ex2_approx(fmaf(t[j + 1].x, row_scale, add)) +
             ptx::ex2_approx(fmaf(t[j + 1].y, row_scale, add));
      t[j] = __ffma2_rn(t[j], rs, make_float2(log_vs.x, log_vs.y));
      t[j + 1] = __ffma2_rn(t[j + 1], rs, make_float2(log_vs.z, log_vs.w));
    }
    l = fmaf(sum, power_of_two(-(int)x.exponent[g]), l);
  }
  return l;
}
// The weights of a visit with the maximum `m` (base 2) as f16 pairs to tensor memory; the fp32 sum of the even groups'.
__device__ __forceinline__ float visit_weights(const Visit& x, uint32_t even, uint32_t to, float row_scale, float m, float2 (&t)[kVisit / 2]) {
  float l = 0.f;
  uint32_t p[kVisit / 2];
#pragma unroll
  for (int g = 0; g < kVisit / 16; ++g) {
    const float add = x.exponent[g] - m + kOffset, r = even >> 8 * g & 1 ? row_scale : 1.f;
    const float2 plus = make_float2(add, add), rs = make_float2(r, r);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = g * 8; j < g * 8 + 8; ++j) {
      const float2 z = __ffma2_rn(t[j], rs, plus), w = make_float2(ptx::ex2_approx(z.x), ptx::ex2_approx(z.y));
      sum = __fadd2_rn(sum, w);
      p[j] = two_f16(w.x, w.y);
    }
    l = fmaf(sum.x + sum.y, x.unscale[g], l);
  }
  ptx::tmem_st32(to, p);
  return l;
}

template <int DIM>
__device__ __forceinline__ void rescale_output(uint32_t o, float factor) {  // (few registers: the visit's logits are held meanwhile)
#pragma unroll 1
  for (int i = 0; i < DIM; i += 8) {
    uint32_t v[8];
    ptx::tmem_ld8(o + i, v);
    ptx::tmem_ld_wait_for(v);
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(v[j]) * factor;
    ptx::tmem_st8(o + i, f);
  }
  ptx::tmem_st_wait();
}

// Where a stacked row lies: query row and head.
struct Place {
  long long q_row;
  int head, r;
};
__device__ __forceinline__ Place place_of(const AttendCall& c, const Walk& at, int tile_row) {
  const int i = at.tile * kManyTile + tile_row, r = query_row(c, i);
  return Place{(long long)at.x.row0 + r, at.head * c.group + i - r * c.group, r};
}

// `rows` query rows into an operand tile, DIM / 8 lanes to a row, scaled by a power of two each (query_power); to `scale` what takes that back, times
// the softmax scale.  Every lane copies its pieces to where they belong and turns them into f16 there: the
// loads are all in flight, and the code is short (unrolled it took 7 us the first time, most of it instruction fetch).  Rows that do not
// exist keep what lies there: whatever it is, it stays in their own row of S and O, which nobody reads.
template <int DIM>
__device__ __forceinline__ void load_queries(const AttendCall& c, const Walk& at, int first_row, int rows, uint32_t tile, int row_in_tile, float* scale, int lane) {
  constexpr int kLanes = DIM / 8, kRows = 32 / kLanes;  // rows of a load
  const int sub = lane / kLanes, piece = lane % kLanes;
  const uint32_t to = tile + (piece >> 3) * Many<DIM>::kHalfBytes;
#pragma unroll 1
  for (int j = sub; j < rows; j += kRows) {
    const Place q = place_of(c, at, first_row + j);
    const int row = row_in_tile + j;
    if (q.r < at.x.rows) ptx::copy_async<16>(to + row * 128 + (((piece & 7) ^ (row & 7)) << 4), c.q + q.q_row * c.q_st + (long long)q.head * c.q_sh + piece * 8);
  }
  ptx::copies_commit();
  ptx::copies_wait<0>();
#pragma unroll 4
  for (int j0 = 0; j0 < rows; j0 += kRows) {  // (four rows' ways through the shuffles side by side: one by one they took 8,500 cycles)
    const int row = row_in_tile + j0 + sub;
    const uint32_t at_piece = to + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
    const uint4 x = ptx::ld_shared4(at_piece);
    const unsigned m = 0x7FFF7FFFu;
    unsigned top = __vmaxu2(__vmaxu2(x.x & m, x.y & m), __vmaxu2(x.z & m, x.w & m));  // what is not a number is larger than the rest
    top = max(top >> 16, top & 0xFFFFu);
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    const float by = query_power(top);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = two_f16(__uint_as_float(w[i] << 16) * by, __uint_as_float(w[i] & 0xFFFF0000u) * by);
    ptx::st_shared4(at_piece, h[0], h[1], h[2], h[3]);
    if (piece == 0) scale[row] = query_scale(c.scale_log2, by);
  }
}

template <int DIM>
__device__ __forceinline__ void softmax(const AttendCall& c, const AttendList& list, const int* ahead, Control& ctl, uint32_t q_tiles, int u0, int u1, int warp, int lane) {
  using M = Many<DIM>;
  const int stream = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
  const uint32_t lanes = ctl.tmem_base + ((uint32_t)(quarter * 32) << 16), outputs = lanes + kOutputAt;
  const uint32_t s = lanes + stream * kVisit, weights = lanes + kWeightsAt + stream * kVisit;
  const uint32_t s_full = ptx::smem_u32(&ctl.s_full[stream]), s_free = ptx::smem_u32(&ctl.s_free[stream]);
  const uint32_t p_full = ptx::smem_u32(&ctl.p_full[stream][0]), pv_done = ptx::smem_u32(&ctl.pv_done[stream][0]);
  Walk at;
  at.seek(c, list, ahead, u0);
  int visits = 0, done = 0;  // of this stream; tiles before the segment
  for (bool more = at.unit < u1; more;) {
    const Segment seg = segment_of(c, at, u1);
    // With two streams of rows a thread's row is of its stream's half; else threads of both streams have the same one.
    const int warp_row = (seg.two ? stream * kSub : 0) + quarter * 32;
    {  // every row once: a stream its own, or both streams half of them each
      const int first = seg.two ? warp_row : warp * 16, most = seg.two ? 32 : 16, rows = min(most, max(0, rows_of(c, at) - first));
      load_queries<DIM>(c, at, first, rows, q_tiles + (seg.two ? stream : 0) * M::kTileBytes, first - (seg.two ? stream * kSub : 0), ctl.row_scale[seg.two ? stream : 0], lane);
    }
    ptx::fence_proxy_async_smem();
    ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.q_full), lane);
    if (!seg.two) soft_sync();
    const float row_scale = ctl.row_scale[seg.two ? stream : 0][row];
    int sees, all_see;
    bool there;
    {
      const Place q = place_of(c, at, warp_row + lane);
      there = q.r < at.x.rows;
      sees = !there ? 0 : at.x.own && c.causal ? max(0, at.x.len - at.x.rows + q.r + 1) : at.x.len;
      all_see = __reduce_min_sync(0xFFFFFFFFu, there ? sees : INT_MAX);
    }

    float m = -INFINITY, l = 0.f;
    const int count = seg.two ? 2 * seg.tiles : seg.tiles;
#pragma unroll 1
    for (int v = 0; v < count; ++v, ++visits) {
      const int tile = seg.two ? v >> 1 : v, half = seg.two ? v & 1 : stream, n = done + tile, ring = n & (kScaleRing - 1);
      const Visit x{s, ctl.k_scale[ring] + half * kVisit, ctl.v_exponent[ring] + half * kVisit, ctl.v_log[ring] + half * kVisit, ctl.bound[ring] + half * (kGroups / 2),
                    ctl.exponent[ring] + half * (kGroups / 2), ctl.unscale[ring] + half * (kGroups / 2), ctl.even[ring] + half * (kGroups / 2)};
      const int buffer = visits & 1;
      // The tile's scales, the logits, and that the weights two visits before have been used: looked at together (one after the other, each look
      // is a hundred cycles and more of a visit's two thousand).
      const uint32_t scale_full = ptx::smem_u32(&ctl.scale_full[ring]), buffer_done = pv_done + buffer * 8, done_parity = ((visits >> 1) - 1) & 1;
      if (!wait_all(scale_full, (n / kScaleRing) & 1, s_full, visits & 1, buffer_done, done_parity)) {
        ptx::mbar_wait_warp(scale_full, (n / kScaleRing) & 1, &ctl.abort);
        ptx::mbar_wait_warp(s_full, visits & 1, &ctl.abort);
        ptx::mbar_wait_warp(buffer_done, done_parity, &ctl.abort);
      }
      ptx::tc_fence_after_sync();
      const int key0 = (seg.first + tile) * kManyKeys + half * kVisit;
      float2 t[kVisit / 2];
      const uint32_t even_groups = *reinterpret_cast<const uint32_t*>(x.even_at);  // a byte each
      const bool even = even_groups == 0x01010101u;
      float top = visit_logits(x, row_scale, key0 + kVisit > all_see, sees - key0, t);
      if (!even) top = uneven_top(x, even_groups, row_scale, top, t);
      ptx::tc_fence_before_sync();
      ptx::mbar_arrive_warp(s_free, lane);
      if (v == 0) {
        m = top;
      } else if (__any_sync(0xFFFFFFFFu, there && (top > m + kSlack || (m == -INFINITY && top > m)))) {  // the sums so far
        const float to = fmaxf(top, m), by = m == -INFINITY ? -INFINITY : m - to, factor = ptx::ex2_approx(by), root = ptx::ex2_approx(0.5f * by);
        l = l * root * root;  // (l may be as large as 2^74: it is not yet 0 where the factor is)
        m = to;
        ptx::mbar_wait_warp(pv_done + ((visits - 1) & 1) * 8, (visits - 1) >> 1 & 1, &ctl.abort);
        ptx::tc_fence_after_sync();
        rescale_output<DIM>(outputs + stream * 128, factor);
      }
      const float base = m == -INFINITY ? 0.f : m;
      if (!even) l += uneven_weights(x, even_groups, row_scale, base, t);
      l += visit_weights(x, even_groups, weights + buffer * (kVisit / 2), row_scale, base, t);
      ptx::tmem_st_wait();
      ptx::tc_fence_before_sync();
      ptx::mbar_arrive_warp(p_full + buffer * 8, lane);
    }
    ptx::mbar_wait_warp(pv_done + ((visits - 1) & 1) * 8, (visits - 1) >> 1 & 1, &ctl.abort);

    // The end of the segment; the streams' sums are joined where both have a part of the row.  O is sum 2^(z - m) v times 2^(kOffset + kValuePower).
    ctl.row_ml[stream][row] = make_float2(m, l);
    ptx::tc_fence_before_sync();
    soft_sync();
    ptx::tc_fence_after_sync();
    float other = 0.f, back = power_of_two(-kOffset - kValuePower);
    if (!seg.two) {
      const float2 a = ctl.row_ml[0][row], b = ctl.row_ml[1][row];
      m = fmaxf(a.x, b.x);
      const float base = m == -INFINITY ? 0.f : m, f0 = ptx::ex2_approx(0.5f * (a.x - base)), f1 = ptx::ex2_approx(0.5f * (b.x - base));
      l = a.y * f0 * f0 + b.y * f1 * f1;  // (roots, as above)
      other = back * f1 * f1;
      back *= f0 * f0;
    }
    const bool whole = at.job_first() >= u0 && at.job_end() <= u1, final = whole && c.prefixes == 0;
    const long long level = at.x.own ? 0ll : (long long)c.total_q * c.hq;
    const long long part = ((long long)blockIdx.x * 2 + (at.job_first() < u0 ? 0 : 1)) * kManyTile;  // the block's place for what it did not finish
    const float inv = l == 0.f ? 0.f : 1.f / l, lse = plus_log2(m, l);
    back *= inv;
    other *= inv;
    // A stream writes its rows; where both have the same ones, half of the columns each.  By kWide columns through shared memory (the query
    // tiles, which nobody needs any more), so that rows are written in whole lines.
    constexpr int kWide = DIM / 2, kLanes = kWide / 4, kRows = 32 / kLanes;
    const uint32_t stage = q_tiles + warp * (32 * kWide * 4), mine = outputs + (seg.two ? stream * 128 : 0);
#pragma unroll 1
    for (int d = seg.two ? 0 : stream * kWide; d < (seg.two ? DIM : (stream + 1) * kWide); d += kWide) {
#pragma unroll 1
      for (int h = 0; h < kWide; h += 32) {
        uint32_t x[32], y[32];
        ptx::tmem_ld32(mine + d + h, x);
        if (!seg.two) ptx::tmem_ld32(outputs + 128 + d + h, y);
        ptx::tmem_ld_wait_for(x);
        if (!seg.two) ptx::tmem_ld_wait_for(y);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          float f = __uint_as_float(x[j]) * back;
          if (!seg.two) f = fmaf(__uint_as_float(y[j]), other, f);
          x[j] = __float_as_uint(f);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          ptx::st_shared4(stage + lane * (kWide * 4) + (((h / 4 + j) ^ (lane & 7)) << 4), x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
      }
      __syncwarp();
      const int piece = lane % kLanes;
#pragma unroll 4
      for (int j = 0; j < 32 / kRows; ++j) {
        const int r = j * kRows + lane / kLanes;
        const uint4 x = ptx::ld_shared4(stage + r * (kWide * 4) + ((piece ^ (r & 7)) << 4));
        const Place q = place_of(c, at, warp_row + r);
        if (q.r >= at.x.rows) break;
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
        if (c.lse_out) c.lse_out[q.q_row * c.hq + q.head] = lse * kLn2;
      } else {
        *(whole ? c.whole_lse + level + q.q_row * c.hq + q.head : list.part_lse + part + warp_row + lane) = lse;
      }
    }
    ptx::tc_fence_before_sync();
    soft_sync();  // O has been read, and the query tiles are free
    done += seg.tiles;
    more = skip(c, list, ahead, at, seg, u1);
  }
}

// LISTED: the list's entries have room in shared memory (all others go through global memory: 500 -> 511 us with the choice made at run time).
template <int DIM, bool FP8, bool LISTED>
__global__ void __launch_bounds__(kThreads, 1) attend_many_kernel(AttendCall c, AttendList list) {
  using M = Many<DIM>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(16) Control ctl;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned char* const smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t q_tiles = ptx::smem_u32(smem), k_tiles = q_tiles + 2 * M::kTileBytes, v_tiles = k_tiles + 2 * M::kTileBytes;
  int* const ahead = LISTED ? reinterpret_cast<int*>(smem + M::kOperands + M::kCodes) : list.copies + (long long)blockIdx.x * (list.entries() + 1);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(ptx::smem_u32(&ctl.k_full[i]), kConvWarps);
      ptx::mbar_init(ptx::smem_u32(&ctl.v_full[i]), kConvWarps);
      ptx::mbar_init(ptx::smem_u32(&ctl.k_empty[i]), 2);
      ptx::mbar_init(ptx::smem_u32(&ctl.v_empty[i]), 2);
      ptx::mbar_init(ptx::smem_u32(&ctl.s_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.s_free[i]), kSoftWarps / 2);
      for (int b = 0; b < 2; ++b) {
        ptx::mbar_init(ptx::smem_u32(&ctl.p_full[i][b]), kSoftWarps / 2);
        ptx::mbar_init(ptx::smem_u32(&ctl.pv_done[i][b]), 1);
      }
    }
    for (int i = 0; i < kScaleRing; ++i) ptx::mbar_init(ptx::smem_u32(&ctl.scale_full[i]), kConvWarps);
    ptx::mbar_init(ptx::smem_u32(&ctl.q_full), kSoftWarps);
    ptx::mbar_init(ptx::smem_u32(&ctl.last), 4);
    ctl.abort = 0;
    ptx::fence_barrier_init();
  }
  chain_enter_late(c);
  // Beside the kernel for few rows: where its ticket is seen, so is all that the work before it wrote.  (It was written ahead of this kernel's start, so
  // it is seen; if not, this kernel waits until the other has ended, as any would.  Nothing spins.)
  if (c.beside && !__syncthreads_or(threadIdx.x == 0 && ptx::ld_acquire_gpu(c.ended) == c.ticket)) pdl_wait();
  if (!LISTED && !c.beside) pdl_wait();  // (earlier work may still read what lies there)
  const int total = open_list<kThreads>(c, list, ahead, ctl.warp_sum);
  if (!c.beside) pdl_wait();  // the rest may be what earlier work wrote; and tensor memory is taken when all earlier work has ended
  leave_list<kThreads>(list, ahead);
  if (warp == kIssueWarp) {
    ptx::tmem_alloc(ptx::smem_u32(&ctl.tmem_base), kTmemCols);
    ptx::tmem_relinquish();
    ptx::tc_fence_before_sync();
  }
  __syncthreads();
  ptx::tc_fence_after_sync();
  const int workers = workers_of(list, total), u0 = run_start(min((int)blockIdx.x, workers), workers, total), u1 = run_start(min((int)blockIdx.x + 1, workers), workers, total);
  if (warp < kSoftWarps) {
    ptx::more_registers<kSoftRegs>();
    if (u0 < u1) softmax<DIM>(c, list, ahead, ctl, q_tiles, u0, u1, warp, lane);
  } else if (warp < kIssueWarp) {
    ptx::fewer_registers<kConvRegs>();
    if (u0 < u1) convert_keys<DIM, FP8>(c, list, ahead, ctl, k_tiles, v_tiles, v_tiles + 2 * M::kTileBytes, u0, u1, warp - kSoftWarps, lane);
  } else {
    ptx::fewer_registers<kIssueRegs>();
    if (u0 < u1 && warp < kIssueWarp + 2) issue_mmas<DIM, true>(c, list, ahead, ctl, q_tiles, k_tiles, v_tiles, u0, u1, warp & 1);
    else if (u0 < u1) issue_mmas<DIM, false>(c, list, ahead, ctl, q_tiles, k_tiles, v_tiles, u0, u1, warp & 1);
  }
  pdl_trigger();
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  if (warp == kIssueWarp) ptx::tmem_dealloc(ctl.tmem_base, kTmemCols);
  if (threadIdx.x == 0 && ctl.abort && c.device_status) atomicOr(c.device_status, FASTAV_DEV_WAIT_EXPIRED);
  if (c.beside) pdl_wait();  // what waits for this kernel waits for the one beside it, too
}

template <int DIM>
size_t many_smem(int entries) { return 1024 + Many<DIM>::kOperands + Many<DIM>::kCodes + (entries <= many_listed(DIM) ? (size_t)(entries + 1) * 4 : 0); }

template <int DIM, bool FP8, bool LISTED>
cudaError_t run(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  const cudaError_t e = once_per_context([] {
    cudaFuncAttributes a;
    const cudaError_t got = cudaFuncGetAttributes(&a, attend_many_kernel<DIM, FP8, LISTED>);
    if (got != cudaSuccess) return got;
    if (a.numRegs * kThreads < kRegsNeeded) return cudaErrorInvalidConfiguration;  // the softmax's warps would wait for registers for ever
    return cudaFuncSetAttribute(attend_many_kernel<DIM, FP8, LISTED>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)many_smem<DIM>(many_listed(DIM)));
  });
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_chained(attend_many_kernel<DIM, FP8, LISTED>, dim3(list.grid), dim3(kThreads), many_smem<DIM>(list.entries()), stream, c, list);
}

template <bool LISTED>
cudaError_t run(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  if (c.cache.dim == 128) return c.cache.fp8 ? run<128, true, LISTED>(c, list, stream) : run<128, false, LISTED>(c, list, stream);
  return c.cache.fp8 ? run<64, true, LISTED>(c, list, stream) : run<64, false, LISTED>(c, list, stream);
}

}  // namespace

cudaError_t launch_attend_many(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  return list.entries() <= many_listed(c.cache.dim) ? run<true>(c, list, stream) : run<false>(c, list, stream);
}

}  // namespace fastav
