// Attention over the 8-bit cache for few query rows per KV head (up to 16): decoding, a few drafted tokens.
//
// Bound by reading the cache once from HBM.  A unit is 32 keys of one KV head; every warp takes an equal run of the call's units, and has a
// ring of its own that it fills itself (no barrier between warps until the end).  mma.sync (f16, fp32 sums) with the keys as
// the rows: S^T = K Q^T, softmax in registers, O^T += V^T P^T, so that up to eight stacked query rows fill an instruction (sixteen: two, on the
// same operands from the cache).  Codes become f16 exactly on their way from shared memory; a query row is scaled by a power of two first
// and exact in f16 down to 2^-32 of its largest element (query_power); the keys' scales multiply the logits, the values' scales the weights.  The weights
// 2^(z - m) vs are rounded to f16 (11 bits; the output has 8) after another power of two per row.  Running maxima move only when a logit
// is 6 above them, so that the sums are hardly ever rescaled.
//
// Any order of the contractions will do as long as both operands have it.  Lane 4 n + t holds, of query row n and of keys n and n + 8 of
// sixteen, the elements DIM/4 t ..; of V the keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9 and the elements DIM/8 n ..: 16-byte reads (8 for head_dim 64),
// free of bank conflicts for head_dim 128: piece p of a key's row (16 bytes) lies at p ^ (key % 8).  The ring is filled by 16-byte asynchronous
// copies of all lanes; with TMA, four copies of one lane per unit, the issuing took a warp 900 of 4,000 cycles.
//
// The query rows as the rows of the instructions (half of each empty with 8 rows, 243 registers, 8 warps): 4 x 16,384 keys 48.9 us
// instead of 46.2 at that step.  Now: 36.6 us (138 MB, 3.8 TB/s; the loop about half of that time, at the copy's rate, the start of a block, its
// warps' join and the join kernel the rest), 32 sequences of 512 to 4,096 keys 29.0 us (83 MB).
#include <limits.h>

#include "attend.cuh"
#include "attend_8bit.cuh"
#include "sm100_ptx.cuh"

namespace fastav {
namespace {

constexpr int kWarps = 12, kThreads = 32 * kWarps, kFewKeysShift = 5;
static_assert(1 << kFewKeysShift == kFewKeys);
constexpr float kSlack = 6.f;        // log2 of what a weight may reach before the maximum is moved (times the largest scale it is below 2^128)
// A row's weights 2^(z - m) vs times a power of two that brings the largest to 2,048 .. 4,096; lowered when one is above 32,768 (f16 ends at
// 65,504), raised when the maximum moves.  So the largest so far has 2,048 at least, and f16's last step, 2^-24, is 2^-35 of it.
constexpr float kWeightPower = 2048, kMostWeight = 32768;
constexpr float kShare = 1.f / 32;   // on the weights of a block's parts, 24 at most: their sum stays in fp32 where values are near bf16's largest

template <int DIM>
struct Few {
  static constexpr int kStages = DIM == 128 ? 2 : 4;
  static constexpr int kHalf = kFewKeys * DIM, kStage = 2 * kHalf;  // bytes: K or V; both
  static constexpr int kScales = 2 * kFewKeys;                      // floats of a stage
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr size_t smem(int entries) { return kRing + (size_t)kWarps * kStages * kScales * 4 + (size_t)(entries + 1) * 4; }
};

// A part of a job that a warp leaves for the other warps of its block.
struct Left {
  int job_first, job_end, row0, rows, tile, head, own;
  int in_ring;  // where: the warp's ring, else its place in global memory
};

// Where four values of a part lie in shared memory: row-major, the pieces of a row turned by the row (no two lanes on one bank).
template <int DIM>
__device__ __forceinline__ int part_at(int row, int piece) { return row * DIM + (piece ^ (row >> 1 & 3)) * 4; }

// 8 x 8 f16 values, a row per four lanes -> a column per four lanes.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// NT: groups of eight stacked rows.
template <int DIM, bool FP8, int NT>
__global__ void __launch_bounds__(kThreads, 1)
attend_few_kernel(AttendCall c, AttendList list) {
  using F = Few<DIM>;
  constexpr int kTile = 8 * NT;      // stacked rows
  constexpr int kSteps = DIM / 16;   // of the contraction over head_dim, and groups of sixteen output elements
  constexpr int kRun = DIM / 8;      // output elements of a lane, per row
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ Left left[kWarps][2];
  __shared__ float left_lse[kWarps][2][kTile], part_weight[2 * kWarps][kTile];
  __shared__ int warp_sum[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n8 = lane >> 2, t4 = lane & 3;
  unsigned char* const my_ring = smem + warp * F::kStages * F::kStage;
  const float* const scales = reinterpret_cast<float*>(smem + F::kRing) + warp * F::kStages * F::kScales;
  int* const ahead = reinterpret_cast<int*>(smem + F::kRing) + kWarps * F::kStages * F::kScales;
  float* const scratch = list.scratch + (long long)blockIdx.x * kWarps * kTile * DIM;  // a warp's first part
  if (lane < 2) left[warp][lane].job_first = -1;
  chain_enter_late(c);
  if (c.beside) {
    pdl_wait();
    if (blockIdx.x == 0) {
      if (threadIdx.x == 0) ptx::st_release_gpu(c.ended, c.ticket);
      __syncthreads();  // (ahead of any thread's trigger)
    }
    pdl_trigger();  // the kernel for many rows starts beside this one
  }
  const int total = open_list<kThreads>(c, list, ahead, warp_sum);
  pdl_wait();  // the rest may be what earlier work wrote
  leave_list<kThreads>(list, ahead);
  const int workers = workers_of(list, total), block_u0 = run_start(min((int)blockIdx.x, workers), workers, total);
  const int block_u1 = run_start(min((int)blockIdx.x + 1, workers), workers, total);
  const int u0 = block_u0 + run_start(warp, kWarps, block_u1 - block_u0), u1 = block_u0 + run_start(warp + 1, kWarps, block_u1 - block_u0);

  const uint32_t ring = ptx::smem_u32(my_ring);
  Walk next;
  if (u0 < u1) next.seek(c, list, ahead, u0);
  if (u0 < u1 && next.unit < u1) {
    Walk at = next;
    bool more = true;  // `next` stands at a granule of the run
    // A unit's copies.  Lane: piece lane % kPieces of the rows lane / kPieces + kRows j; the unit's two halves of 16 keys may lie in two pages.
    constexpr int kPieces = DIM / 16, kRows = 32 / kPieces, kCopies = kFewKeys / kRows;
    const int row0 = lane / kPieces, piece = lane % kPieces;
    uint32_t to[2];  // rows of even and of odd copies lie differently
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) to[odd] = ring + row0 * DIM + ((DIM == 128 ? piece ^ (row0 + odd * kRows & 7) : piece ^ (row0 >> 1 & 3)) << 4);
    int page[2], stage_in = 0;
    auto look_up = [&] {  // the pages of the unit that `next` stands at
      const int key0 = next.granule * kFewKeys;
      page[0] = chain_load_cached(next.x.table + (key0 >> c.cache.page_shift));
      page[1] = page[0];
      if (c.cache.page_shift == 4 && next.x.len > key0 + 16) page[1] = chain_load_cached(next.x.table + (key0 + 16 >> 4));
    };
    auto issue = [&] {  // the copies of the unit that `next` stands at; then the one after it is looked up
      if (more) {
        const int key0 = next.granule * kFewKeys;
        if ((unsigned)max(page[0], page[1]) >= (unsigned)c.cache.num_pages || (page[0] | page[1]) < 0) {
          page[0] = page[1] = 0;  // (their keys are as wrong as any)
          if (lane == 0 && c.device_status) atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
        }
        const long long pool[2] = {pool_row(c.cache, page[0], next.head, key0), pool_row(c.cache, page[1], next.head, key0 + 16)};
        const int have = next.x.len - key0;  // copies of rows that no page has are left out; what a page has behind the sequence's end is harmless
        const uint32_t at_stage = stage_in * F::kStage;
#pragma unroll
        for (int j = 0; j < kCopies; ++j) {
          const int second = j >= kCopies / 2 ? 1 : 0;
          if (second && have <= 16) break;
          const long long from = (pool[second] + row0 + (j - second * (kCopies / 2)) * kRows) * DIM + piece * 16;
          ptx::copy_async<16>(to[j & 1] + at_stage + j * kRows * DIM, c.cache.k + from);
          ptx::copy_async<16>(to[j & 1] + at_stage + F::kHalf + j * kRows * DIM, c.cache.v + from);
        }
        if (lane < 16 || have > 16) {
          const long long row = (lane < 16 ? pool[0] : pool[1]) + (lane & 15);
          const uint32_t at_scale = ptx::smem_u32(scales) + (stage_in * F::kScales + lane) * 4;
          ptx::copy_async<4>(at_scale, c.cache.k_scale + row);
          ptx::copy_async<4>(at_scale + kFewKeys * 4, c.cache.v_scale + row);
        }
        stage_in = stage_in + 1 == F::kStages ? 0 : stage_in + 1;
        more = next.step(c, list, ahead, u1);
        if (more) look_up();
      }
      ptx::copies_commit();  // (a group per unit, empty ones too)
    };
    // The query rows of a job: stacked row 8 g + n8, elements DIM/4 t4 ...  Asked for ahead of the first copies, whose way is as long, if
    // there are registers for it.
    uint32_t x[NT][kSteps * 2];
    auto ask_queries = [&] {
#pragma unroll
      for (int g = 0; g < NT; ++g) {
        const int i = at.tile * kTile + 8 * g + n8, r = query_row(c, i);
        const uint4* const from = reinterpret_cast<const uint4*>(c.q + (long long)(at.x.row0 + r) * c.q_st + (long long)(at.head * c.group + i - r * c.group) * c.q_sh + t4 * (DIM / 4));
#pragma unroll
        for (int j = 0; j < kSteps / 2; ++j) {
          const uint4 v = r < at.x.rows ? chain_load_cached(from + j) : make_uint4(0, 0, 0, 0);
          x[g][4 * j] = v.x; x[g][4 * j + 1] = v.y; x[g][4 * j + 2] = v.z; x[g][4 * j + 3] = v.w;
        }
      }
    };
    look_up();
    if (NT == 1) ask_queries();
#pragma unroll 1
    for (int i = 0; i < F::kStages; ++i) issue();

    uint32_t qf[NT][kSteps][2];
    float o[NT][kSteps][4];                                        // elements kRun n8 + 2 i + (0, 1) of rows 2 t4 + (0, 1)
    float m[NT][2], l[NT][2], power[NT][2], row_scale[NT][2];      // of those rows
    int sees[NT][2], all_see = 0;
#pragma unroll 1
    for (int n = 0;; ++n) {
      const int key0 = at.granule * kFewKeys;
      if (n == 0 || at.granule == 0) {  // another job: its query rows
        if (NT > 1 || n > 0) ask_queries();
#pragma unroll
        for (int g = 0; g < NT; ++g) {
          const int i = at.tile * kTile + 8 * g + n8, r = query_row(c, i);
          const bool there = r < at.x.rows;
          unsigned top = 0;  // bf16 bits of the largest magnitude; what is not a number is larger still
#pragma unroll
          for (int j = 0; j < kSteps * 2; ++j) top = __vmaxu2(top, x[g][j] & 0x7FFF7FFFu);
          top = max(top >> 16, top & 0xFFFFu);
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
          const float to = query_power(top);
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t v = x[g][2 * s + half];
              qf[g][s][half] = two_f16(__uint_as_float(v << 16) * to, __uint_as_float(v & 0xFFFF0000u) * to);
            }
          const int own_sees = !there ? 0 : at.x.own && c.causal ? max(0, at.x.len - at.x.rows + r + 1) : at.x.len;
          const int least = __reduce_min_sync(0xFFFFFFFFu, there ? own_sees : INT_MAX);
          all_see = g == 0 ? least : min(all_see, least);
#pragma unroll
          for (int e = 0; e < 2; ++e) {  // of row n8 -> of rows 2 t4 + e
            row_scale[g][e] = query_scale(c.scale_log2, __shfl_sync(0xFFFFFFFFu, to, 4 * (2 * t4 + e)));
            sees[g][e] = __shfl_sync(0xFFFFFFFFu, own_sees, 4 * (2 * t4 + e));
            m[g][e] = -INFINITY;
            l[g][e] = power[g][e] = 0.f;
          }
#pragma unroll
          for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[g][j][e] = 0.f;
        }
      }
      const int stage = n % F::kStages;
      ptx::copies_wait<F::kStages - 1>();
      __syncwarp();  // ... of all lanes
      const uint32_t kt = ring + stage * F::kStage, vt = kt + F::kHalf;
      const float* const ks = scales + stage * F::kScales;

      float z[NT][2][4];  // of 16 keys h: key n8, rows 2 t4 + (0, 1); key n8 + 8, the same
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int g = 0; g < NT; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) z[g][h][i] = 0.f;
#pragma unroll
        for (int p = 0; p < kSteps / 4; ++p) {
          const int key = 16 * h + n8;
          const uint32_t piece = DIM == 128 ? ((2 * t4 + p) ^ n8) : (t4 ^ (n8 >> 1 & 3)), from = kt + key * DIM + piece * 16;
          const uint4 a = ptx::ld_shared4(from), b = ptx::ld_shared4(from + 8 * DIM);
          const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
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
      const bool masked = key0 + kFewKeys > all_see;
      float k_scale[4], v_scale[4];  // of keys n8, n8 + 8, n8 + 16, n8 + 24
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        k_scale[i] = ks[8 * i + n8] * kKeyScaleFactor;
        v_scale[i] = ks[kFewKeys + 8 * i + n8];
      }
      // The maxima and the powers of two are moved only when a lane meets a value above what they allow; only then the lanes of a row compare theirs.
      bool over = false;
#pragma unroll
      for (int g = 0; g < NT; ++g)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float& x = z[g][i / 2][i % 2 * 2 + e];
            x *= k_scale[i];
            top = fmaxf(top, x);
          }
          if (masked) {
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float& x = z[g][i / 2][i % 2 * 2 + e];
              if (key0 + 8 * i + n8 >= sees[g][e]) x = -INFINITY;
              top = fmaxf(top, x);
            }
          }
          over |= top * row_scale[g][e] > m[g][e] + kSlack;  // (no key yet: -inf)
        }
      if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
        for (int g = 0; g < NT; ++g) {
          float factor[2];  // of what has been summed up
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = fmaxf(fmaxf(z[g][0][e], z[g][0][2 + e]), fmaxf(z[g][1][e], z[g][1][2 + e])) * row_scale[g][e];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            // By whole bits, and the power of two goes up by what the weights so far go down by: the largest of these stays where it was, and nothing drifts.
            // (Else the power would remain that of values which count for nothing any more.)  What this unit's weights make of it is seen to below.
            const float before = m[g][e], to = before == -INFINITY ? top : before + fmaxf(ceilf(top - before), 0.f), by = to - before;
            factor[e] = before == -INFINITY ? 0.f : ptx::ex2_approx(-by);
            l[g][e] *= factor[e];
            if (before > -INFINITY && power[g][e] > 0.f) {
              const unsigned bits = __float_as_uint(power[g][e]);
              const int up = min((int)rintf(fminf(by, 300.f)), 251 - (int)(bits >> 23));
              power[g][e] = __uint_as_float(bits + ((unsigned)up << 23));
              factor[e] = ptx::ex2_approx((float)up - by);
            }
            m[g][e] = to;
          }
#pragma unroll
          for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[g][j][e] *= factor[e & 1];
        }
      }
      over = false;
#pragma unroll
      for (int g = 0; g < NT; ++g)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float base = m[g][e] == -INFINITY ? 0.f : m[g][e];
          float most = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float& x = z[g][i / 2][i % 2 * 2 + e];
            const float p = ptx::ex2_approx(fmaf(x, row_scale[g][e], -base));
            l[g][e] += p;
            x = p * v_scale[i];
            most = fmaxf(most, fabsf(x));
          }
          if (masked) {  // (a place that no key fills may hold any scale)
            most = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float& x = z[g][i / 2][i % 2 * 2 + e];
              if (key0 + 8 * i + n8 >= sees[g][e]) x = 0.f;
              most = fmaxf(most, fabsf(x));
            }
          }
          over |= most * power[g][e] > kMostWeight || (power[g][e] == 0.f && most > 0.f);
        }
      if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
        for (int g = 0; g < NT; ++g) {
          float factor[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float most = fmaxf(fmaxf(fabsf(z[g][0][e]), fabsf(z[g][0][2 + e])), fmaxf(fabsf(z[g][1][e]), fabsf(z[g][1][2 + e])));
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
            factor[e] = 1.f;
            if (most * power[g][e] > kMostWeight || (power[g][e] == 0.f && most > 0.f)) {
              const float to = to_one(most) * kWeightPower;
              factor[e] = power[g][e] == 0.f ? 0.f : to * inverse_power(power[g][e]);
              power[g][e] = to;
            }
          }
#pragma unroll
          for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[g][j][e] *= factor[e & 1];
        }
      }
      uint32_t weight[NT][4];  // keys 8 i + 2 t4 + (0, 1) of row n8
#pragma unroll
      for (int g = 0; g < NT; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) weight[g][i] = transposed(two_f16(z[g][i / 2][i % 2 * 2] * power[g][0], z[g][i / 2][i % 2 * 2 + 1] * power[g][1]));
      // Keys behind the sequence's end: what their places hold is multiplied by a weight of 0, so it must not be NaN or infinite.  e4m3 has NaN.
      const int have = at.x.len - key0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t v[4][DIM / 32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = 16 * h + 2 * t4 + (i & 1) + (i & 2) * 4;
          if (DIM == 128) {
            const uint4 x = ptx::ld_shared4(vt + key * DIM + ((n8 ^ (key & 7)) << 4));
            v[i][0] = x.x; v[i][1] = x.y; v[i][2 % (DIM / 32)] = x.z; v[i][3 % (DIM / 32)] = x.w;
          } else {
            const uint2 x = ptx::ld_shared2(vt + key * DIM + (((n8 >> 1) ^ (key >> 1 & 3)) << 4) + (n8 & 1) * 8);
            v[i][0] = x.x; v[i][1] = x.y;
          }
          if (FP8 && have < kFewKeys && key >= have)
#pragma unroll
            for (int j = 0; j < DIM / 32; ++j) v[i][j] = 0;
        }
#pragma unroll
        for (int j = 0; j < DIM / 32; ++j)
#pragma unroll
          for (int half = 0; half < 2; ++half) {  // elements kRun n8 + 4 j + 2 half + (0, 1)
            uint32_t a0, a1, a2, a3;
            four_codes<FP8>(__byte_perm(v[0][j], v[1][j], half ? 0x7362 : 0x5140), a0, a1);
            four_codes<FP8>(__byte_perm(v[2][j], v[3][j], half ? 0x7362 : 0x5140), a2, a3);
#pragma unroll
            for (int g = 0; g < NT; ++g) mma_f16(o[g][2 * j + half], a0, a1, a2, a3, weight[g][2 * h], weight[g][2 * h + 1]);
          }
      }
      __syncwarp();  // the stage has been read
      issue();

      const int job_first = at.job_first(), job_end = at.job_end();
      if (at.unit + 1 == u1 || at.unit + 1 == job_end) {  // the end of the job, or of the run
        const bool whole = job_first >= u0 && job_end <= u1, final = whole && c.prefixes == 0;
        // A part that no other warp of the block has a share in goes to the block's place at once.
        const bool alone = (job_first >= u0 || u0 == block_u0) && (job_end <= u1 || u1 == block_u1);
        const long long place = ((long long)blockIdx.x * 2 + (job_first < block_u0 ? 0 : 1)) * kTile;
        const int slot = job_first < u0 ? 0 : 1;
        // A run's last part lies where its ring was: nothing is in flight any more.
        const bool last = at.unit + 1 + (at.unit + 1 == job_end ? list.job_cost : 0) >= u1;
        float* const part = last ? reinterpret_cast<float*>(my_ring) : scratch + warp * kTile * DIM;
#pragma unroll
        for (int g = 0; g < NT; ++g)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[g][e] += __shfl_xor_sync(0xFFFFFFFFu, l[g][e], d);
            const int row = 8 * g + 2 * t4 + e, i = at.tile * kTile + row, r = query_row(c, i);
            if (r >= at.x.rows) continue;
            const float back = power[g][e] == 0.f ? 0.f : inverse_power(power[g][e]), inv = l[g][e] == 0.f ? 0.f : 1.f / l[g][e];
            const float lse = plus_log2(m[g][e], l[g][e]);
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {  // (in this order no product leaves fp32's range)
              o[g][j][e] = o[g][j][e] * inv * back;
              o[g][j][2 + e] = o[g][j][2 + e] * inv * back;
            }
            const long long q_row = at.x.row0 + r;
            const int head = at.head * c.group + i - r * c.group;
            const long long flat = (at.x.own ? 0ll : (long long)c.total_q * c.hq) + q_row * c.hq + head;
            if (final) {
              uint16_t* const to = c.out + q_row * c.o_st + (long long)head * c.o_sh + n8 * kRun;
#pragma unroll
              for (int j = 0; j < kRun / 8; ++j) {
                uint32_t x[4];
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) x[i4] = pair_bf16(o[g][4 * j + i4][e], o[g][4 * j + i4][2 + e]);
                *reinterpret_cast<uint4*>(to + 8 * j) = make_uint4(x[0], x[1], x[2], x[3]);
              }
              if (c.lse_out && n8 == 0) c.lse_out[flat] = lse * kLn2;
            } else {
              float* const to = whole ? c.whole_out + flat * DIM : alone ? list.part_out + (place + row) * DIM : part;
#pragma unroll
              for (int j = 0; j < kRun / 4; ++j) {
                const int piece = n8 * (kRun / 4) + j;
                *reinterpret_cast<float4*>(to + (whole || alone ? piece * 4 : part_at<DIM>(row, piece))) =
                    make_float4(o[g][2 * j][e], o[g][2 * j][2 + e], o[g][2 * j + 1][e], o[g][2 * j + 1][2 + e]);
              }
              if (n8 == 0) *(whole ? c.whole_lse + flat : alone ? list.part_lse + place + row : &left_lse[warp][slot][row]) = lse;
            }
          }
        if (!whole && !alone && lane == 0) left[warp][slot] = Left{job_first, job_end, at.x.row0, at.x.rows, at.tile, at.head, at.x.own, last};
      }
      if (!at.step(c, list, ahead, u1)) break;
    }
  }
  pdl_trigger();
  __syncthreads();

  // The parts of one job that several warps left, joined in their order: to the output if the block has the whole job, else to the block's place.
  // First what every part counts for (lane: slot), then the sums.
  static_assert(2 * kWarps <= 32);
  const int slot_first = lane < 2 * kWarps ? left[lane / 2][lane & 1].job_first : -1;
  const unsigned alike = __match_any_sync(0xFFFFFFFFu, slot_first), leaders = __ballot_sync(0xFFFFFFFFu, slot_first >= 0 && __ffs(alike) - 1 == lane);
  for (int row = warp; row < kTile; row += kWarps) {
    const float lse = slot_first >= 0 ? left_lse[lane / 2][lane & 1][row] : -INFINITY;
    float top = -INFINITY;  // of the lanes with the same job
#pragma unroll 1
    for (unsigned rest = leaders; rest; rest &= rest - 1) {
      const unsigned group = __shfl_sync(0xFFFFFFFFu, alike, __ffs(rest) - 1);
      float of_group = group >> lane & 1 ? lse : -INFINITY;
#pragma unroll
      for (int d = 16; d; d >>= 1) of_group = fmaxf(of_group, __shfl_xor_sync(0xFFFFFFFFu, of_group, d));
      if (group >> lane & 1) top = of_group;
    }
    if (lane < 2 * kWarps) {
      part_weight[lane][row] = ptx::ex2_approx(lse - (top == -INFINITY ? 0.f : top)) * kShare;
      left_lse[lane / 2][lane & 1][row] = top;
    }
  }
  __syncthreads();
#pragma unroll 1
  for (unsigned rest = leaders; rest; rest &= rest - 1) {
    const int first = __ffs(rest) - 1;
    const unsigned group = __shfl_sync(0xFFFFFFFFu, alike, first);
    const Left job = left[first / 2][first & 1];
    const bool whole = job.job_first >= block_u0 && job.job_end <= block_u1;
    const int slot = job.job_first < block_u0 ? 0 : 1;
    const int rows = min(kTile, job.rows * c.group - job.tile * kTile);
    for (int item = threadIdx.x; item < rows * (DIM / 4); item += kThreads) {
      const int row = item / (DIM / 4), piece = item % (DIM / 4);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
#pragma unroll 4
      for (unsigned of = group; of; of &= of - 1) {
        const int j = __ffs(of) - 1;
        const float w = part_weight[j][row];
        const float* const part = left[j / 2][j & 1].in_ring ? reinterpret_cast<float*>(smem + j / 2 * F::kStages * F::kStage) : scratch + j / 2 * kTile * DIM;
        const float4 v = *reinterpret_cast<const float4*>(part + part_at<DIM>(row, piece));
        sum += w;
        acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y); acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
      }
      const float lse = sum == 0.f ? -INFINITY : left_lse[first / 2][first & 1][row] + log2f(sum * (1.f / kShare)), inv = sum == 0.f ? 0.f : 1.f / sum;
      acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
      const int stacked = job.tile * kTile + row, r = query_row(c, stacked), head = job.head * c.group + stacked - r * c.group;
      const long long q_row = job.row0 + r, flat = (job.own ? 0ll : (long long)c.total_q * c.hq) + q_row * c.hq + head;
      if (whole && c.prefixes == 0) {
        *reinterpret_cast<uint2*>(c.out + q_row * c.o_st + (long long)head * c.o_sh + piece * 4) = make_uint2(pair_bf16(acc.x, acc.y), pair_bf16(acc.z, acc.w));
        if (c.lse_out && piece == 0) c.lse_out[flat] = lse * kLn2;
      } else {
        const long long place = ((long long)blockIdx.x * 2 + slot) * kTile + row;
        *reinterpret_cast<float4*>((whole ? c.whole_out + flat * DIM : list.part_out + place * DIM) + piece * 4) = acc;
        if (piece == 0) *(whole ? c.whole_lse + flat : list.part_lse + place) = lse;
      }
    }
  }
}

template <int DIM, bool FP8, int NT>
cudaError_t run(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  const cudaError_t e = once_per_context([] {
    return cudaFuncSetAttribute(attend_few_kernel<DIM, FP8, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Few<DIM>::smem(FASTAV_ATTEND_MAX_BATCH));
  });
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_chained(attend_few_kernel<DIM, FP8, NT>, dim3(list.grid), dim3(kThreads), Few<DIM>::smem(list.entries()), stream, c, list);
}
template <int DIM, bool FP8>
cudaError_t run(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  return list.tile_rows == 8 ? run<DIM, FP8, 1>(c, list, stream) : run<DIM, FP8, 2>(c, list, stream);
}

}  // namespace

size_t few_scratch_floats(const AttendList& list, int dim) { return (size_t)list.grid * kWarps * list.tile_rows * dim; }

cudaError_t launch_attend_few(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  if (c.cache.dim == 128) return c.cache.fp8 ? run<128, true>(c, list, stream) : run<128, false>(c, list, stream);
  return c.cache.fp8 ? run<64, true>(c, list, stream) : run<64, false>(c, list, stream);
}

}  // namespace fastav
