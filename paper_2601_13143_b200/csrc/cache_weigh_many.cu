// fastav_cache_weigh for many query rows: a question's tokens at once, all rows that share a prefix.
//
// More stacked rows (query rows times G) than the kernel for few takes.  S^T = K Q^T on the fifth-generation tensor cores (tcgen05.mma, bf16 operands, fp32 sums in tensor memory) with the KEYS as the
// accumulator's lanes: a token's weight is then a sum over one lane's columns, which one thread adds up by itself; only what the teams (below) have of a token's row tiles is
// joined.  Codes are exact in bf16 (int8 and e4m3 have at most eight significant bits), so queries go to the matrix pipe as they are, by TMA from the caller's tensor.
//
// A block, one per SM, takes an equal run of units (128 keys of a KV head, against all stacked rows of their sequence, 96 at a time), one or two units together.
// A PRODUCT is a unit against a row tile; with two units theirs alternate.
//
//   warps 0-15  four teams of four, a thread per key: exponentials of a product's columns from tensor memory, summed in a register.  The teams take the products
//               in turn, from five accumulators in turn: while four are summed up the fifth is made.
//   warps 16-23 codes -> bf16 operand tiles in shared memory, scales and weights so far beside them, a group of units ahead
//   warp 24     plans of the groups for those, as far ahead as there is room: rows of the pool, which it calls into L2
//   warp 25     query rows by TMA, their log-sum-exps and masks
//   warps 26-27 issue the MMAs, every other product each
//
// Bound by the exponentials (16 per clock and SM) and by power: 1,536 rows on 16,384 keys of 8 heads (206 GFLOP, 805 million exponentials) take 242 us, 0.85 PFLOP/s;
// call upon call, at the power limit and some 1.65 GHz, 252.  An eighth of the exponentials is made of multiplications instead: none 250 us, a sixteenth 246 (call upon call
// 4 and 2 % more than an eighth).  The compiler spills some 200 bytes a thread without them and nothing with them, which shows where row tiles are few (below).  Measured on the way:
// eight summing warps a block 296 us; four accumulators of 128 columns, each summed up and made in turn, 256; eight of 64 columns 267; a third stage of query rows the same.
// With few row tiles bound by the chain from a group's codes to its sums: 64 rows on 4 x 16,384 tokens 41 us (47 with spills, 55 where the converting warps look up pages and
// walk the list by themselves), 192 rows 57 (64), 96 rows on 8 x 3,000 27 (29).
#include <cuda.h>
#include <limits.h>

#include "attend_8bit.cuh"
#include "weigh.cuh"

namespace fastav {
namespace {

constexpr int kTile = 128;   // keys of a unit
constexpr int kTileRows = 96;    // stacked rows of a row tile, at most
constexpr int kBuffers = 5;  // accumulators of kTileRows columns: one more than there are teams
constexpr int kSumWarps = 16, kConvWarps = 8, kPlanWarp = kSumWarps + kConvWarps, kRowWarp = kPlanWarp + 1, kIssueWarp = kPlanWarp + 2, kWarps = kPlanWarp + 4, kThreads = 32 * kWarps;
// Registers a thread has per role.  What the three take together has to fit into what the block is launched with (checked before the launch).
constexpr int kSumRegs = 80, kConvRegs = 64, kLastRegs = 48;
constexpr int kRegsNeeded = 32 * (kSumWarps * kSumRegs + kConvWarps * kConvRegs + 4 * kLastRegs);
constexpr int kStages = 2, kRowSlots = 8, kKeySlots = 4, kPlans = 8;
constexpr int kTmemCols = 512;
constexpr int kPiece = 32;  // columns of tensor memory in registers at a time
constexpr int kHalfBytes = kTile * 128, kRowBytes = kTileRows * 128;  // rows of 128 bytes: 64 elements

template <int DIM>
struct Many {
  static constexpr int kTileBytes = DIM / 64 * kHalfBytes, kStageBytes = DIM / 64 * kRowBytes;
  static constexpr int kOperands = 4 * kTileBytes + kStages * kStageBytes;  // K: two units, twice; Q
};

struct RowSlot {
  alignas(16) float neg_lse[kTileRows];  // -log2(e) lse
  alignas(16) int sees[kTileRows];       // keys that the row sees; 0: it pays nothing
  int least[kTileRows / 32];             // the least of 32 of them
};
struct KeySlot {  // of a group of units
  int row[2 * kTile];  // of the pool; -1: no key, or in no page
  float scale[2 * kTile], before[2 * kTile];  // (of such, too: 0)
};
struct Plan {  // what the converting warps have to know of a group
  int row[2 * kTile / 16];  // of the pool, of each sixteen keys; -1: in no page
  int units, keys, fresh;   // units 0: there is no further group; keys that exist, and that have a weight so far
  int convert;              // there are query rows
};
struct Control {
  KeySlot keys[kKeySlots];
  Plan plans[kPlans];
  uint64_t plan_full[kPlans], plan_empty[kPlans], keys_full[kKeySlots], keys_empty[kKeySlots], k_full[2], k_empty[2], q_full[kStages], q_empty[kStages], rows_full[kRowSlots], rows_empty[kRowSlots], s_full[kBuffers], s_empty[kBuffers];
  RowSlot rows[kRowSlots];
  float join[2][4][kTile];
  long long warp_sum[kWarps];
  int first[2], unit[2];  // where the block's run begins and ends: sequence, unit of it
  uint32_t tmem_base;
  int abort;
};

struct ManyCall {
  WeighCall w;
  int rows_per_tile;  // query rows (not stacked) of a row tile
};
inline void mark_head(ManyCall& c, bool head) { c.w.head_wait = head ? 1 : 0; }

// A block's run, walked by every role for itself.
struct Run {
  int b, end_b, end_u, start_u;
  WeighSpan s;
  int row_tiles, head, tile, units;  // units: 1 or 2 from `tile` on
  int key_tiles = -1, left = 0;      // left: units of the sequence that are still to come
  __device__ __forceinline__ Run(const Control& ctl) : b(ctl.first[0]), end_b(ctl.first[1]), end_u(ctl.unit[1]), start_u(ctl.unit[0]) {}
  // To the next group; what it finds is meant to be short, every role goes through it once a group.
  __device__ __forceinline__ bool next(const ManyCall& c) {
    if (left > 0) {
      tile += units;
      if (tile >= key_tiles) {
        tile = 0;
        ++head;
      }
    } else {
      for (;; ++b, start_u = 0, key_tiles = -1) {
        if (key_tiles >= 0) continue;  // this one is done
        if (b > end_b || (b == end_b && start_u >= end_u)) return false;
        s = weigh_span(c.w, b);
        key_tiles = (s.len + kTile - 1) / kTile;
        row_tiles = (s.rows + c.rows_per_tile - 1) / c.rows_per_tile;
        left = (b == end_b ? end_u : key_tiles * c.w.cache.hkv) - start_u;
        if (left > 0) break;
      }
      head = start_u / key_tiles;
      tile = start_u - head * key_tiles;
    }
    units = min(2, min(key_tiles - tile, left));
    left -= units;
    return true;
  }
  __device__ __forceinline__ int stacked(const ManyCall& c, int row_tile) const {  // rows of a row tile
    return min(c.rows_per_tile, s.rows - row_tile * c.rows_per_tile) * c.w.group;
  }
};

// What a sequence costs per unit: its row tiles, and about as much as one more for what is done once.
__device__ __forceinline__ int unit_cost(const ManyCall& c, const WeighSpan& s) { return (s.rows + c.rows_per_tile - 1) / c.rows_per_tile + 1; }

// Finds the block's run: the units whose start, in the call's total cost, lies in the block's share.
__device__ __forceinline__ void find_run(const ManyCall& c, Control& ctl) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, batch = c.w.batch;
  if (batch <= 32) {  // one warp, one look
    if (warp != 0) return;
    int cost = 0, units = 0;
    if (lane < batch) {
      const WeighSpan s = weigh_span(c.w, lane);
      if (s.bad && blockIdx.x == 0 && c.w.device_status) atomicOr(c.w.device_status, FASTAV_DEV_SHAPE_MISMATCH);
      units = (s.len + kTile - 1) / kTile * c.w.cache.hkv;
      cost = unit_cost(c, s);
    }
    const long long own = (long long)units * cost;
    long long upto = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long x = __shfl_up_sync(0xFFFFFFFFu, upto, d);
      if (lane >= d) upto += x;
    }
    const long long total = __shfl_sync(0xFFFFFFFFu, upto, 31), start = upto - own, last = start + (long long)(units - 1) * cost;
    for (int e = 0; e < 2; ++e) {
      const long long edge = total * (blockIdx.x + e) / gridDim.x;
      const unsigned behind = __ballot_sync(0xFFFFFFFFu, units > 0 && edge <= last);
      if (behind && lane == __ffs(behind) - 1) {
        ctl.first[e] = lane;
        ctl.unit[e] = edge <= start ? 0 : (int)((edge - start + cost - 1) / cost);
      }
    }
    return;
  }
  long long total = 0;
  for (int pass = 0; pass < 2; ++pass) {
    long long ahead = 0;
    const long long from = pass ? total * blockIdx.x / gridDim.x : 0, to = pass ? total * (blockIdx.x + 1) / gridDim.x : 0;
    for (int b0 = 0; b0 < batch; b0 += kThreads) {
      const int b = b0 + tid;
      int cost = 0, units = 0;
      if (b < batch) {
        const WeighSpan s = weigh_span(c.w, b);
        if (s.bad && pass == 0 && blockIdx.x == 0 && c.w.device_status) atomicOr(c.w.device_status, FASTAV_DEV_SHAPE_MISMATCH);
        units = (s.len + kTile - 1) / kTile * c.w.cache.hkv;
        cost = unit_cost(c, s);
      }
      const long long own = (long long)units * cost;
      long long incl = own;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long x = __shfl_up_sync(0xFFFFFFFFu, incl, d);
        if (lane >= d) incl += x;
      }
      if (lane == 31) ctl.warp_sum[warp] = incl;
      __syncthreads();
      long long start = ahead + incl - own;
      for (int i = 0; i < kWarps; ++i) {
        if (i < warp) start += ctl.warp_sum[i];
        ahead += ctl.warp_sum[i];
      }
      // An edge's unit is the first one that starts there or behind: of the least sequence whose last unit does.
      const long long last = start + (long long)(units - 1) * cost;
      if (pass && units > 0)
        for (int e = 0; e < 2; ++e)
          if ((e ? to : from) <= last) atomicMin(&ctl.first[e], b);
      __syncthreads();
      if (pass && units > 0) {
        for (int e = 0; e < 2; ++e) {
          const long long edge = e ? to : from;
          if (ctl.first[e] == b) ctl.unit[e] = edge <= start ? 0 : (int)((edge - start + cost - 1) / cost);
        }
      }
    }
    total = ahead;
  }
  __syncthreads();
}

// 16 codes -> 32 bytes of a swizzled bf16 operand row.
template <bool FP8>
__device__ __forceinline__ void codes_to_bf16(const uint4& x, uint32_t at) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (FP8) {
      // s eeee mmm as the sign and the low end of bf16's exponent and mantissa is the value times 2^-120 (subnormals, too); exact
      const uint32_t a = __byte_perm(w[i], 0, 0x1404), b = __byte_perm(w[i], 0, 0x3424);  // a code in the upper byte of each half
      const uint32_t la = ((a >> 4) & 0x07F007F0u) | (a & 0x80008000u), lb = ((b >> 4) & 0x07F007F0u) | (b & 0x80008000u), up = 0x7B807B80u;  // 2^120, twice
      asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(h[2 * i]) : "r"(la), "r"(up));
      asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(h[2 * i + 1]) : "r"(lb), "r"(up));
    } else {
      // the code plus 128 as the low bits of 2^23, less 2^23 + 128: a whole number of at most eight bits, whose float ends in sixteen zeros
      const uint32_t u = w[i] ^ 0x80808080u;
      const float2 less = make_float2(-8388736.f, -8388736.f);
      const float2 a = __fadd2_rn(make_float2(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7441))), less);
      const float2 b = __fadd2_rn(make_float2(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7442)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7443))), less);
      h[2 * i] = __byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x7632);
      h[2 * i + 1] = __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x7632);
    }
  }
  ptx::st_shared4(at, h[0], h[1], h[2], h[3]);
  ptx::st_shared4(at ^ 16, h[4], h[5], h[6], h[7]);
}

__device__ __forceinline__ float2 two(float x) { return make_float2(x, x); }

// 2^x of two x by multiplications and additions, beside the special-function unit: x = n + f, n the nearest integer (whose sum with 127 ends up in the low
// bits of what the first addition gives), 2^f on [-1/2, 1/2] by the polynomial of degree 5 with the least largest relative error (by Remez' exchange; 2.2e-7 with
// all roundings, as the unit's own).  From 127.5 on infinite, below -126.5 zero; what is not a number stays none.
__device__ __forceinline__ float2 exp2_by_products(float2 x) {
  constexpr float kToInteger = 12582912.f + 127.f;  // 1.5 * 2^23, and the exponent's bias
  x = make_float2(ptx::clamp_nan(x.x, -127.f, 128.f), ptx::clamp_nan(x.y, -127.f, 128.f));
  const float2 t = __fadd2_rn(x, two(kToInteger)), n = __fadd2_rn(t, two(-kToInteger)), f = __ffma2_rn(n, two(-1.f), x);
  float2 p = __ffma2_rn(f, two(0.00132764725f), two(0.00967554096f));
  p = __ffma2_rn(p, f, two(0.0555071309f));
  p = __ffma2_rn(p, f, two(0.240221202f));
  p = __ffma2_rn(p, f, two(0.693146944f));
  p = __ffma2_rn(p, f, two(1.00000012f));
  return __fmul2_rn(p, make_float2(__uint_as_float(__float_as_uint(t.x) << 23), __uint_as_float(__float_as_uint(t.y) << 23)));
}

// What kPiece columns of rows add to the weight of the thread's key.  MASKED: a mask's edge, rows that pay nothing or do not exist (what stands in their
// columns may be anything).  An eighth of the exponentials goes without the special-function unit (of four columns in sixteen the second two).
template <bool MASKED>
__device__ __forceinline__ void add_columns(const uint32_t (&v)[kPiece], const float* neg_lse, const int* sees, int key, const float2& scale, float2 (&sum)[2]) {
  const float4* const nl = reinterpret_cast<const float4*>(neg_lse);
#pragma unroll
  for (int j = 0; j < kPiece / 4; ++j) {
    const float4 l = nl[j];
    const float2 a = __ffma2_rn(make_float2(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1])), scale, make_float2(l.x, l.y));
    const float2 b = __ffma2_rn(make_float2(__uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3])), scale, make_float2(l.z, l.w));
    float2 p = make_float2(ptx::ex2_approx(a.x), ptx::ex2_approx(a.y));
    float2 q = !MASKED && j % 4 == 1 ? exp2_by_products(b) : make_float2(ptx::ex2_approx(b.x), ptx::ex2_approx(b.y));
    if (MASKED) {
      const int4 n = reinterpret_cast<const int4*>(sees)[j];
      p = make_float2(key < n.x ? p.x : 0.f, key < n.y ? p.y : 0.f);
      q = make_float2(key < n.z ? q.x : 0.f, key < n.w ? q.y : 0.f);
    }
    sum[0] = __fadd2_rn(sum[0], p);
    sum[1] = __fadd2_rn(sum[1], q);
  }
}

template <int DIM, bool FP8>
__global__ void __launch_bounds__(kThreads, 1)
weigh_many_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ ManyCall c) {
  using M = Many<DIM>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t k_tiles = base, q_tiles = base + 4 * M::kTileBytes;
  Control& ctl = *reinterpret_cast<Control*>(smem_raw + (base - ptx::smem_u32(smem_raw)) + M::kOperands);
  volatile int* abort = &ctl.abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WeighCall& w = c.w;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(ptx::smem_u32(&ctl.k_full[i]), kConvWarps);
      ptx::mbar_init(ptx::smem_u32(&ctl.k_empty[i]), 2);
      ctl.first[i] = w.batch;
      ctl.unit[i] = 0;
    }
    for (int i = 0; i < kBuffers; ++i) {
      ptx::mbar_init(ptx::smem_u32(&ctl.s_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.s_empty[i]), kSumWarps / 4);
    }
    for (int i = 0; i < kStages; ++i) {
      ptx::mbar_init(ptx::smem_u32(&ctl.q_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.q_empty[i]), 2);
    }
    for (int i = 0; i < kRowSlots; ++i) {
      ptx::mbar_init(ptx::smem_u32(&ctl.rows_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.rows_empty[i]), kSumWarps / 2);
    }
    for (int i = 0; i < kPlans; ++i) {
      ptx::mbar_init(ptx::smem_u32(&ctl.plan_full[i]), 1);
      ptx::mbar_init(ptx::smem_u32(&ctl.plan_empty[i]), kConvWarps);
    }
    for (int i = 0; i < kKeySlots; ++i) {
      ptx::mbar_init(ptx::smem_u32(&ctl.keys_full[i]), kConvWarps);
      ptx::mbar_init(ptx::smem_u32(&ctl.keys_empty[i]), kSumWarps);
    }
    ctl.abort = 0;
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&q_map);
  }
  if (w.head_wait) pdl_wait();
  pdl_trigger();
  pdl_wait();
  if (warp == kIssueWarp) {
    ptx::tmem_alloc(ptx::smem_u32(&ctl.tmem_base), kTmemCols);
    ptx::tmem_relinquish();
  }
  __syncthreads();
  find_run(c, ctl);
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = ctl.tmem_base;
  Run run(ctl);

  // (A wait that gives up changes nothing in the way a warp goes: it only marks the results as invalid, and sums behind the mark are not stored.)
  if (warp < kSumWarps) {
    ptx::more_registers<kSumRegs>();
    const int team = warp >> 2, in_tile = threadIdx.x & (kTile - 1);
    const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    int tiles_before = 0, products = 0, group = 0;  // row tiles, and products, of the groups before
    const int tile_rows = c.rows_per_tile * w.group;
    while (run.next(c)) {
      const bool pair = run.units == 2;
      const int nth = (team - products) & 3, half = pair ? nth & 1 : 0;  // of the group's products the team takes nth, nth + 4, ..: all of one unit
      const int key0 = (run.tile + half) * kTile, key = key0 + in_tile, key_end = min(run.s.len, key0 + kTile), row_tiles = run.row_tiles;
      const int stacked = run.s.rows * w.group, of_group = half * kTile + in_tile, keys = group % kKeySlots;
      const bool known = ptx::mbar_wait_warp(ptx::smem_u32(&ctl.keys_full[keys]), group / kKeySlots & 1, abort);
      const int mine = known ? ctl.keys[keys].row[of_group] : -1;
      const float own_scale = ctl.keys[keys].scale[of_group], before = ctl.keys[keys].before[of_group];
      ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.keys_empty[keys]), lane);
      const float2 scale = make_float2(own_scale, own_scale);
      float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, other[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};  // other: see the swap
      const int of_run = row_tiles << (pair ? 1 : 0);
      for (int i = nth; i < of_run; i += 4) {
        const int t = pair ? i >> 1 : i, slot = (tiles_before + t) % kRowSlots, product = products + i, buffer = product % kBuffers;
        const RowSlot& rows = ctl.rows[slot];
        const uint32_t rows_bar = ptx::smem_u32(&ctl.rows_full[slot]), s_bar = ptx::smem_u32(&ctl.s_full[buffer]);
        const uint32_t rows_parity = (tiles_before + t) / kRowSlots & 1, s_parity = product / kBuffers & 1;
        const bool there = ptx::mbar_try_wait(rows_bar, rows_parity) & ptx::mbar_try_wait(s_bar, s_parity);
        if (!__all_sync(0xFFFFFFFFu, there)) {
          ptx::mbar_wait_warp(rows_bar, rows_parity, abort);
          ptx::mbar_wait_warp(s_bar, s_parity, abort);
        }
        ptx::tc_fence_after_sync();
        const int columns = min(tile_rows, stacked - t * tile_rows);
#pragma unroll 1
        for (int c0 = 0; c0 < columns; c0 += kPiece) {
          uint32_t v[kPiece];
          ptx::tmem_ld32(lanes + buffer * kTileRows + c0, v);
          ptx::tmem_ld_wait_for(v);
          if (rows.least[c0 / kPiece] >= key_end) add_columns<false>(v, rows.neg_lse + c0, rows.sees + c0, key, scale, sum);
          else add_columns<true>(v, rows.neg_lse + c0, rows.sees + c0, key, scale, sum);
          __syncwarp();
        }
        ptx::tc_fence_before_sync();
        ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.s_empty[buffer]), lane);
        if (pair) {  // of a pair's units a team has every other row tile: in turns to either sum, each four tiles apart as a single unit's
          const float2 s0 = sum[0], s1 = sum[1];
          sum[0] = other[0]; sum[1] = other[1];
          other[0] = s0; other[1] = s1;
        }
        if (lane == 0) {
          ptx::mbar_arrive(ptx::smem_u32(&ctl.rows_empty[slot]));
          if (!pair) ptx::mbar_arrive(ptx::smem_u32(&ctl.rows_empty[slot]));  // (for the team of another unit)
        }
        __syncwarp();
      }
      tiles_before += row_tiles;
      products += of_run;
      float total = ((sum[0].x + sum[0].y) + (sum[1].x + sum[1].y)) + ((other[0].x + other[0].y) + (other[1].x + other[1].y));
      // The teams' sums.  With s_i what the row tiles i, i + 4, .. come to, a token is paid (s_0 + s_2) + (s_1 + s_3), whether its unit is one of a pair or
      // not: that depends on where a block's run begins, hence on the rest of the batch.  (One sum for a pair's tiles, in another order: 250.3 instead of 252.4 us for
      // 1,536 rows on 16,384 tokens call upon call, but with the registers that this leaves 43.0 instead of 41.1 for 64 rows on 4 x 16,384.)
      const bool joins = nth == 0 || (pair && nth == 1);
      if (!joins) ctl.join[group & 1][nth][in_tile] = total;
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kSumWarps) : "memory");
      if (joins) {
        if (pair) total += ctl.join[group & 1][nth + 2][in_tile];
        else total = (total + ctl.join[group & 1][2][in_tile]) + (ctl.join[group & 1][1][in_tile] + ctl.join[group & 1][3][in_tile]);
        const bool valid = *abort == 0;  // whoever gave up left the flag before what came of it: no wrong sum is added to the weights
        if (mine >= 0 && valid) w.weights[mine] = fmaf(w.decay, before, total);
      }
      ++group;
    }
  } else if (warp < kPlanWarp) {
    ptx::fewer_registers<kConvRegs>();
    // Loads of 4 keys of 8 pieces (head_dim 64: 8 of 4); the eight lanes of a phase store to eight different quarters of the banks.
    constexpr int kLoads = DIM / 32, kKeysAtOnce = 16 / kLoads;
    const int cw = warp - kSumWarps;
    const int piece = DIM == 128 ? (lane & 3) | (lane >> 1 & 4) : lane & 3, row = DIM == 128 ? (lane >> 2 & 1) | (lane >> 3 & 2) : lane >> 2;
    // A warp has two sixteens of a group's keys (one of a single unit's), each in one page; a group is asked for as soon as the one before is in the tiles.
    uint4 x[2][kLoads];
    int at = -1;  // of key `lane` of the 32 (16)
    float scale = 0.f, before = 0.f;
    const uint8_t* const codes = w.cache.k + row * DIM + piece * 16;
    auto ask = [&](const Plan& g) {
      const int units = g.units, own = cw * units, key = own * 16 + lane;
      const int first[2] = {g.row[own], g.row[own + units - 1]};
      const int mine = lane < 16 ? first[0] : first[1];
      at = lane < 16 * units && key < g.keys && mine >= 0 ? mine + (lane & 15) : -1;
      scale = at >= 0 ? chain_load(w.cache.k_scale + at) : 0.f;
      before = at >= 0 && key < g.fresh ? chain_load(w.weights + at) : 0.f;
      if (!g.convert) return;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i >= units || (own + i) * 16 >= g.keys) continue;
        const uint8_t* const from = codes + (long long)max(first[i], 0) * DIM;  // (the weights of a page that is none are left out)
#pragma unroll
        for (int j = 0; j < kLoads; ++j) x[i][j] = chain_load(reinterpret_cast<const uint4*>(from + j * kKeysAtOnce * DIM));
      }
    };
    // (Where a plan's wait gives up there is no plan to go by.)
    bool more = ptx::mbar_wait_warp(ptx::smem_u32(&ctl.plan_full[0]), 0, abort) && ctl.plans[0].units > 0;
    if (more) ask(ctl.plans[0]);
    for (int group = 0, converted = 0; more; ++group) {
      const Plan& now = ctl.plans[group % kPlans];
      const int keys = group % kKeySlots, units = now.units;
      ptx::mbar_wait_warp(ptx::smem_u32(&ctl.keys_empty[keys]), (group / kKeySlots & 1) ^ 1u, abort);
      if (lane < 16 * units) {
        const int of_group = cw * units * 16 + lane;
        ctl.keys[keys].row[of_group] = at;
        ctl.keys[keys].scale[of_group] = scale * w.scale_log2;
        ctl.keys[keys].before[of_group] = before;
      }
      ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.keys_full[keys]), lane);
      if (now.convert) {
        const int slot = converted & 1;
        ptx::mbar_wait_warp(ptx::smem_u32(&ctl.k_empty[slot]), (converted >> 1 & 1) ^ 1u, abort);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int in_group = (cw * units + i) * 16;
          if (i >= units || in_group >= now.keys) continue;
          const uint32_t tile = k_tiles + (2 * slot + in_group / kTile) * M::kTileBytes + (piece >> 2) * kHalfBytes;
#pragma unroll
          for (int j = 0; j < kLoads; ++j) {
            const int r = in_group % kTile + j * kKeysAtOnce + row;
            codes_to_bf16<FP8>(x[i][j], tile + r * 128 + (((2 * (piece & 3)) ^ (r & 7)) << 4));
          }
        }
        ptx::fence_proxy_async_smem();
        ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.k_full[slot]), lane);
        ++converted;
      }
      ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.plan_empty[group % kPlans]), lane);
      const Plan& next = ctl.plans[(group + 1) % kPlans];
      more = ptx::mbar_wait_warp(ptx::smem_u32(&ctl.plan_full[(group + 1) % kPlans]), (group + 1) / kPlans & 1, abort) && next.units > 0;
      if (more) ask(next);
    }
  } else {
    ptx::fewer_registers<kLastRegs>();
  }
  if (warp == kPlanWarp) {
    // Plans of the groups, some groups ahead: a lane per sixteen keys, the pages of a group asked for a group earlier still.  Codes, scales and weights are called
    // into L2 by the way.
    int fresh = 0, fresh_of = -1;  // tokens of a sequence from there on have no weight yet
    int page = 0, keys = 0, planned = 0;
    bool last = !run.next(c), done = false;
    auto look_up = [&] {
      if (run.b != fresh_of) {
        fresh_of = run.b;
        fresh = w.decay == 0.f ? 0 : w.weighed ? chain_load_cached(w.weighed + run.b) : INT_MAX;
      }
      keys = min(run.units * kTile, run.s.len - run.tile * kTile);
      if (16 * lane < keys) page = chain_load_cached(w.table + (long long)run.b * w.table_stride + (run.tile * kTile + 16 * lane >> w.cache.page_shift));
    };
    if (!last) look_up();
    auto plan_next = [&] {
      const int slot = planned % kPlans;
      if (!ptx::mbar_wait_warp(ptx::smem_u32(&ctl.plan_empty[slot]), (planned / kPlans & 1) ^ 1u, abort)) {
        done = true;
        return;
      }
      Plan& g = ctl.plans[slot];
      if (last) {
        if (lane == 0) g.units = 0;
      } else {
        const int key0 = run.tile * kTile, weighed = min(max(fresh, key0) - key0, keys);
        int row = -1;
        if (16 * lane < keys) {
          if ((unsigned)page < (unsigned)w.cache.num_pages) {
            row = (int)pool_row(w.cache, page, run.head, key0 + 16 * lane);
            if (run.row_tiles > 0) ptx::prefetch_l2_bulk(w.cache.k + (long long)row * DIM, 16 * DIM);
            ptx::prefetch_l2(w.cache.k_scale + row);
            if (16 * lane < weighed) ptx::prefetch_l2(w.weights + row);
          } else if (w.device_status) {
            atomicOr(w.device_status, FASTAV_DEV_BAD_INDEX);
          }
        }
        if (lane < 2 * kTile / 16) g.row[lane] = row;
        if (lane == 0) {
          g.units = run.units;
          g.keys = keys;
          g.fresh = weighed;
          g.convert = run.row_tiles > 0;
        }
      }
      ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.plan_full[slot]), lane);
      ++planned;
      done = last;
      last = last || !run.next(c);
      if (!last) look_up();
    };
    while (!done) plan_next();
  } else if (warp == kRowWarp) {
    int tiles = 0, t = 0;
    const uint32_t box_bytes = (uint32_t)(c.rows_per_tile * w.group) * 128u;
    constexpr int kEach = kTileRows / 32;
    float lse[kEach];  // of the next row tile, asked for ahead of the wait for its place
    int sees[kEach];
    auto ask = [&] {
      const int stacked = run.stacked(c, t), first = t * c.rows_per_tile;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int x = 32 * i + lane, r = x / w.group, head = run.head * w.group + x - r * w.group;
        lse[i] = x < stacked ? chain_load(w.lse + (long long)(run.s.row0 + first + r) * w.hq + head) : -INFINITY;
        sees[i] = w.causal ? max(0, run.s.len - run.s.rows + first + r + 1) : run.s.len;
      }
    };
    auto advance = [&] {
      if (++t < run.row_tiles) return true;
      t = 0;
      do {
        if (!run.next(c)) return false;
      } while (run.row_tiles == 0);
      return true;
    };
    run.row_tiles = 0;
    bool more = advance();
    if (more) ask();
    for (; more; ++tiles) {
      const int slot = tiles % kRowSlots, stage = tiles % kStages;
      const uint32_t bar = ptx::smem_u32(&ctl.q_full[stage]);
      ptx::mbar_wait_warp(ptx::smem_u32(&ctl.q_empty[stage]), (tiles / kStages & 1) ^ 1u, abort);
      ptx::mbar_expect_tx_warp(bar, box_bytes * (DIM / 64));
#pragma unroll
      for (int sub = 0; sub < DIM / 64; ++sub)
        ptx::tma_load_3d_warp(q_tiles + stage * M::kStageBytes + sub * kRowBytes, &q_map, sub * 64, run.head * w.group, run.s.row0 + t * c.rows_per_tile, bar);
      ptx::mbar_wait_warp(ptx::smem_u32(&ctl.rows_empty[slot]), (tiles / kRowSlots & 1) ^ 1u, abort);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int n = lse[i] == -INFINITY ? 0 : sees[i], least = __reduce_min_sync(0xFFFFFFFFu, n);
        ctl.rows[slot].neg_lse[32 * i + lane] = -lse[i] * kLog2e;
        ctl.rows[slot].sees[32 * i + lane] = n;
        if (lane == 0) ctl.rows[slot].least[i] = least;
      }
      ptx::mbar_arrive_warp(ptx::smem_u32(&ctl.rows_full[slot]), lane);
      more = advance();
      if (more) ask();
    }
    // The copies write into this block's shared memory: they have to be waited for before it may exit.
    int never = 0;
    for (int i = max(0, tiles - kStages); i < tiles; ++i) ptx::mbar_wait_bounded(ptx::smem_u32(&ctl.q_full[i % kStages]), i / kStages & 1, &never);
    __syncwarp();
  } else if (warp >= kIssueWarp) {
    // Every other product each, so that neither waits for the other's sums.
    const int parity = warp - kIssueWarp;
    int tiles = 0, products = 0;
    for (int group = 0; run.next(c);) {
      if (run.row_tiles == 0) continue;
      const int slot = group & 1;
      const bool pair = run.units == 2;
      ptx::mbar_wait_warp(ptx::smem_u32(&ctl.k_full[slot]), group >> 1 & 1, abort);
      for (int t = 0; t < run.row_tiles; ++t, ++tiles) {
        const int stage = tiles % kStages;
        ptx::mbar_wait_warp(ptx::smem_u32(&ctl.q_full[stage]), tiles / kStages & 1, abort);
        const int unit = (parity - products) & 1, product = products + unit;
        products += run.units;
        if (pair || unit == 0) {
          const int buffer = product % kBuffers;
          ptx::mbar_wait_warp(ptx::smem_u32(&ctl.s_empty[buffer]), (product / kBuffers & 1) ^ 1u, abort);
          ptx::tc_fence_after_sync();
          ptx::umma_bf16_steps<DIM / 16, kHalfBytes, kRowBytes>(tmem + buffer * kTileRows, ptx::umma_desc_sw128(k_tiles + (2 * slot + unit) * M::kTileBytes, 0),
                                                                ptx::umma_desc_sw128(q_tiles + stage * M::kStageBytes, 0),
                                                                ptx::umma_idesc_bf16(kTile, (run.stacked(c, t) + 15) / 16 * 16), false);
          ptx::umma_commit(ptx::smem_u32(&ctl.s_full[buffer]));
        }
        ptx::umma_commit(ptx::smem_u32(&ctl.q_empty[stage]));
      }
      ptx::umma_commit(ptx::smem_u32(&ctl.k_empty[slot]));
      ++group;
    }
    if (tiles > 0) {  // the columns are given back below: not before the last MMA is done
      int never = 0;
      ptx::mbar_wait_bounded(ptx::smem_u32(&ctl.q_empty[(tiles - 1) % kStages]), (tiles - 1) / kStages & 1, &never);
      __syncwarp();
    }
  }

  // ---- everybody meets here, whatever happened above ----
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == kIssueWarp) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, kTmemCols);
  }
  if (threadIdx.x == 0 && ctl.abort && w.device_status) atomicOr(w.device_status, FASTAV_DEV_WAIT_EXPIRED);
}

template <int DIM, bool FP8>
cudaError_t launch(const ManyCall& c, const CUtensorMap& map, cudaStream_t stream) {
  constexpr size_t kSmem = Many<DIM>::kOperands + sizeof(Control) + 1024;
  const cudaError_t e = once_per_context([&] {
    cudaFuncAttributes a;
    const cudaError_t got = cudaFuncGetAttributes(&a, weigh_many_kernel<DIM, FP8>);
    if (got != cudaSuccess) return got;
    if (a.numRegs * kThreads < kRegsNeeded) return cudaErrorInvalidConfiguration;  // the summing warps would wait for registers for ever
    return cudaFuncSetAttribute(weigh_many_kernel<DIM, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  });
  if (e != cudaSuccess) return e;
  const long long units = (long long)c.w.batch * c.w.cache.hkv * (((long long)c.w.max_len + kTile - 1) / kTile);
  count_launches(1);
  return launch_chained(weigh_many_kernel<DIM, FP8>, dim3((unsigned)(units < kNumSMs ? units : kNumSMs)), dim3(kThreads), kSmem, stream, map, c);
}

}  // namespace

bool weigh_many_applies(const WeighCall& c) { return c.group <= kTileRows; }

cudaError_t launch_weigh_many(const WeighCall& w, cudaStream_t stream, bool* used) {
  ManyCall c{w, kTileRows / w.group};
  if (c.rows_per_tile > w.max_qlen) c.rows_per_tile = w.max_qlen;
  CUtensorMap map;
  *used = encode_rows_map(w.q, w.cache.dim, w.hq, w.total_q, w.q_st, w.q_sh, w.group, c.rows_per_tile, &map);
  if (!*used) return cudaSuccess;
  if (w.cache.dim == 128) return w.cache.fp8 ? launch<128, true>(c, map, stream) : launch<128, false>(c, map, stream);
  return w.cache.fp8 ? launch<64, true>(c, map, stream) : launch<64, false>(c, map, stream);
}

}  // namespace fastav
