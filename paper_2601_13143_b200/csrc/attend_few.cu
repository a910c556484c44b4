// Attention over the 8-bit cache for few query rows per KV head: decoding, drafted tokens, and short questions.
//
// Bound by reading the cache once from HBM.  A unit is 32 keys of one KV head; every warp takes an equal run of the call's units, and has a
// ring of its own that it fills itself with TMA (no barrier between warps until the end).  Up to 16 stacked query rows are the A operand
// of mma.sync (f16, fp32 sums): S = Q K^T over 8 keys at a time, softmax in registers, O += P V.  Codes become f16 exactly on
// their way from shared memory; a query row is scaled by a power of two first, so that bf16 values are exact in f16 too; the keys'
// scales multiply the logits, the values' scales the weights.  The weights 2^(z - m) vs are rounded to f16 (11 bits; the output has 8) after
// another power of two per row.  Running maxima move only when a logit is 2^8 above them, so
// that the sums are hardly ever rescaled.
//
// Any order of the contractions will do as long as both operands have it.  Lane 4 n + t holds, of Q and of key n of a group of eight, the
// elements DIM/4 t ..; of V the keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9 and the elements DIM/8 n ..: 16-byte reads (8 for head_dim 64), free of bank
// conflicts for head_dim 128 in the swizzle that the copies write.
#include <limits.h>

#include <cuda.h>

#include "attend.cuh"
#include "attend_8bit.cuh"
#include "gather.cuh"
#include "sm100_ptx.cuh"

namespace fastav {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr float kSlack = 8.f;        // log2 of what a weight may reach before the maximum is moved
// A row's weights 2^(z - m) vs times a power of two that brings the largest to 2,048 .. 4,096, and moved when one is above 32,768 (f16 ends at
// 65,504): what lies under f16's normal numbers is less than 2^-25 of the largest.
constexpr float kWeightPower = 2048, kMostWeight = 32768;

template <int DIM>
struct Few {
  static constexpr int kStages = DIM == 128 ? 2 : 4;
  static constexpr int kHalf = kFewKeys * DIM, kStage = 2 * kHalf;  // bytes: K or V; both
  static constexpr int kScales = 2 * kFewKeys;                      // floats of a stage
  static constexpr int kRing = kWarps * kStages * kStage;
};

// A part of a job that a warp leaves for the other warps of its block.
struct Left {
  int job_first, job_end, row0, rows, tile, head, own;
};

template <int DIM>
struct FewSmem {
  using F = Few<DIM>;
  unsigned char* base;
  __device__ unsigned char* ring(int warp) const { return base + warp * F::kStages * F::kStage; }
  __device__ float* scales(int warp) const { return reinterpret_cast<float*>(base + F::kRing) + warp * F::kStages * F::kScales; }
  __device__ float* first_part(int warp, int rows) const {
    return reinterpret_cast<float*>(base + F::kRing) + kWarps * F::kStages * F::kScales + warp * rows * DIM;
  }
  __device__ int* ahead(int rows) const { return reinterpret_cast<int*>(first_part(kWarps, rows)); }
};
template <int DIM>
size_t few_smem(int rows, int entries) {
  using F = Few<DIM>;
  return 1024 + F::kRing + (size_t)kWarps * F::kStages * F::kScales * 4 + (size_t)kWarps * rows * DIM * 4 + (size_t)(entries + 1) * 4;
}

// Where four values of a part lie: row-major, the 16-byte pieces of a thread's run of DIM / 4 values turned by its lane.
template <int DIM>
__device__ __forceinline__ int part_at(int row, int piece) {  // piece: of four values, DIM / 4 of them
  constexpr int kRun = DIM / 16;
  const int t = piece / kRun, q = piece % kRun;
  return row * DIM + (t * kRun + (q ^ ((row * 4 + t) & (kRun - 1)))) * 4;
}

template <int DIM, bool FP8>
__global__ void __launch_bounds__(kThreads, 1)
attend_few_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, AttendCall c, AttendList list, int part_rows) {
  using F = Few<DIM>;
  constexpr int kSteps = DIM / 16;   // of the contraction over head_dim, and 8-column groups of a lane's two
  constexpr int kTiles = DIM / 8;    // groups of eight output columns
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t full[kWarps][F::kStages];
  __shared__ Left left[kWarps][2];
  __shared__ float2 left_ml[kWarps][2][kFewTile];
  __shared__ int warp_sum[kWarps], abort_flag;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n8 = lane >> 2, t4 = lane & 3;
  const FewSmem<DIM> smem{smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u)};
  int* const ahead = smem.ahead(part_rows);
  if (threadIdx.x == 0) {
    abort_flag = 0;
    ptx::prefetch_tensormap(&k_map);
    ptx::prefetch_tensormap(&v_map);
  }
  if (lane == 0) {
    for (int i = 0; i < F::kStages; ++i) ptx::mbar_init(ptx::smem_u32(&full[warp][i]), 1);
    ptx::fence_barrier_init();
  }
  if (lane < 2) left[warp][lane].job_first = -1;
  chain_enter_late(c);
  pdl_wait();  // everything may be what earlier work wrote
  const int total = open_list<kThreads>(c, list, ahead, warp_sum);
  const int workers = workers_of(list, total), block_u0 = run_start(min((int)blockIdx.x, workers), workers, total);
  const int block_u1 = run_start(min((int)blockIdx.x + 1, workers), workers, total);
  const int u0 = block_u0 + run_start(warp, kWarps, block_u1 - block_u0), u1 = block_u0 + run_start(warp + 1, kWarps, block_u1 - block_u0);

  const uint32_t ring = ptx::smem_u32(smem.ring(warp));
  const float* const scales = smem.scales(warp);
  bool ok = true;
  int issued = 0;  // granules asked for
  Walk next;
  if (u0 < u1) next.seek(c, list, ahead, u0);
  if (u0 < u1 && next.unit < u1) {
    Walk at = next;
    bool more = true;                                        // `next` stands at a granule of the run
    const int box = min(1 << c.cache.page_shift, kFewKeys);  // keys of a copy; lane i has copy i
    int page = 0;                                            // of this lane's copy of the next unit
    auto boxes = [&](const Walk& x) { return (min(kFewKeys, x.x.len - x.granule * kFewKeys) + box - 1) / box; };
    auto look_up = [&] {
      if (lane < boxes(next)) {
        page = chain_load_cached(next.x.table + (next.granule * kFewKeys + lane * box >> c.cache.page_shift));
        if ((unsigned)page >= (unsigned)c.cache.num_pages) {
          page = 0;  // (its keys are as wrong as any)
          if (c.device_status) atomicOr(c.device_status, FASTAV_DEV_BAD_INDEX);
        }
      }
    };
    auto issue = [&] {  // the unit that `next` stands at; then the one after it is looked up
      const int stage = issued % F::kStages, count = boxes(next);
      const uint32_t bar = ptx::smem_u32(&full[warp][stage]);
      __syncwarp();  // what the stage held has been read
      if (lane == 0) ptx::mbar_arrive_expect_tx(bar, count * box * 2 * (DIM + 4));
      __syncwarp();
      if (lane < count) {
        const long long row = pool_row(c.cache, page, next.head, next.granule * kFewKeys + lane * box);
        const uint32_t to = ring + stage * F::kStage + lane * box * DIM, to_scale = ptx::smem_u32(scales + stage * F::kScales + lane * box);
        ptx::tma_load_2d(to, &k_map, 0, (int)row, bar);
        ptx::tma_load_2d(to + F::kHalf, &v_map, 0, (int)row, bar);
        bulk_load(to_scale, c.cache.k_scale + row, box * 4, bar);
        bulk_load(to_scale + kFewKeys * 4, c.cache.v_scale + row, box * 4, bar);
      }
      ++issued;
      more = next.step(c, list, ahead, u1);
      if (more) look_up();
    };
    look_up();
    while (more && issued < F::kStages) issue();

    uint32_t qf[kSteps][4];
    float o[kTiles][4], m[2], l[2], power[2], row_scale[2];
    int sees[2], all_see = 0;
#pragma unroll 1
    for (int n = 0;; ++n) {
      const int key0 = at.granule * kFewKeys;
      if (n == 0 || at.granule == 0) {  // another job: its query rows
        all_see = INT_MAX;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int i = at.tile * kFewTile + n8 + 8 * e, r = i / c.group;
          const bool there = r < at.x.rows;
          sees[e] = !there ? 0 : at.x.own && c.causal ? max(0, at.x.len - at.x.rows + r + 1) : at.x.len;
          all_see = min(all_see, there ? sees[e] : INT_MAX);
          const uint4* const from = reinterpret_cast<const uint4*>(c.q + (long long)(at.x.row0 + r) * c.q_st + (long long)(at.head * c.group + i - r * c.group) * c.q_sh + t4 * (DIM / 4));
          uint32_t x[kSteps * 2];
#pragma unroll
          for (int j = 0; j < kSteps / 2; ++j) {
            const uint4 v = there ? chain_load_cached(from + j) : make_uint4(0, 0, 0, 0);
            x[4 * j] = v.x; x[4 * j + 1] = v.y; x[4 * j + 2] = v.z; x[4 * j + 3] = v.w;
          }
          unsigned top = 0;  // bf16 bits of the largest magnitude; what is not a number is larger still
#pragma unroll
          for (int j = 0; j < kSteps * 2; ++j) top = __vmaxu2(top, x[j] & 0x7FFF7FFFu);
          top = max(top >> 16, top & 0xFFFFu);
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
          const float to = to_one(__uint_as_float(top << 16));
          row_scale[e] = c.scale_log2 / to;
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t v = x[2 * s + half];
              qf[s][2 * half + e] = two_f16(__uint_as_float(v << 16) * to, __uint_as_float(v & 0xFFFF0000u) * to);
            }
          m[e] = -INFINITY;
          l[e] = power[e] = 0.f;
        }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) all_see = min(all_see, __shfl_xor_sync(0xFFFFFFFFu, all_see, d));
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
      }
      const int stage = n % F::kStages;
      ok = ptx::mbar_wait_warp(ptx::smem_u32(&full[warp][stage]), (n / F::kStages) & 1, &abort_flag);
      if (!ok) break;
      const uint32_t kt = ring + stage * F::kStage, vt = kt + F::kHalf;
      const float* const ks = scales + stage * F::kScales;

      float z[4][4];  // key 8 j + 2 t4 + (0, 1): row n8, row n8 + 8
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[j][i] = 0.f;
        const int key = 8 * j + n8;
#pragma unroll
        for (int p = 0; p < kSteps / 4; ++p) {
          const uint32_t piece = DIM == 128 ? ((2 * t4 + p) ^ (key & 7)) : (t4 ^ (key >> 1 & 3));
          const uint4 v = ptx::ld_shared4(kt + key * DIM + piece * 16);
          const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t lo, hi;
            four_codes<FP8>(word[i], lo, hi);
            const int s = 4 * p + i;
            mma_f16(z[j], qf[s][0], qf[s][1], qf[s][2], qf[s][3], lo, hi);
          }
        }
      }
      const bool masked = key0 + kFewKeys > all_see;
      float factor[2];
      bool moved = false;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 s = *reinterpret_cast<const float2*>(ks + 8 * j + 2 * t4);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float& x = z[j][2 * e + i];
            x = x * ((i ? s.y : s.x) * row_scale[e]);
            if (masked && key0 + 8 * j + 2 * t4 + i >= sees[e]) x = -INFINITY;
            top = fmaxf(top, x);
          }
        }
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        factor[e] = 1.f;
        if (top > m[e] + kSlack || (m[e] == -INFINITY && top > m[e])) {
          factor[e] = ptx::ex2_approx(m[e] - top);
          m[e] = top;
          l[e] *= factor[e];
          moved = true;
        }
      }
      uint32_t weight[4][2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float base = m[e] == -INFINITY ? 0.f : m[e];
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 s = *reinterpret_cast<const float2*>(ks + kFewKeys + 8 * j + 2 * t4);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float& x = z[j][2 * e + i];
            const float p = ptx::ex2_approx(x - base);
            l[e] += p;
            // (a place that no key fills may hold any scale)
            x = masked && key0 + 8 * j + 2 * t4 + i >= sees[e] ? 0.f : p * (i ? s.y : s.x);
            top = fmaxf(top, x);
          }
        }
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        if (top * power[e] > kMostWeight || (power[e] == 0.f && top > 0.f)) {
          const float to = to_one(top) * kWeightPower;
          factor[e] = power[e] == 0.f ? 0.f : factor[e] * (to / power[e]);
          power[e] = to;
          moved = true;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) weight[j][e] = two_f16(z[j][2 * e] * power[e], z[j][2 * e + 1] * power[e]);
      }
      if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          o[i][0] *= factor[0];
          o[i][1] *= factor[0];
          o[i][2] *= factor[1];
          o[i][3] *= factor[1];
        }
      }
      // Keys behind the sequence's end: what their places hold is multiplied by a weight of 0, so it must not be NaN or infinite.  e4m3 has NaN.
      const int have = at.x.len - key0;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint32_t v[4][DIM / 32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = 16 * s + 2 * t4 + (i & 1) + (i & 2) * 4;
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
          for (int half = 0; half < 2; ++half) {
            uint32_t b00, b01, b10, b11;  // (key pair, column)
            four_codes<FP8>(__byte_perm(v[0][j], v[1][j], half ? 0x7362 : 0x5140), b00, b01);
            four_codes<FP8>(__byte_perm(v[2][j], v[3][j], half ? 0x7362 : 0x5140), b10, b11);
            mma_f16(o[4 * j + 2 * half], weight[2 * s][0], weight[2 * s][1], weight[2 * s + 1][0], weight[2 * s + 1][1], b00, b10);
            mma_f16(o[4 * j + 2 * half + 1], weight[2 * s][0], weight[2 * s][1], weight[2 * s + 1][0], weight[2 * s + 1][1], b01, b11);
          }
      }
      if (more) issue();

      const int job_first = at.job_first(), job_end = at.job_end();
      if (at.unit + 1 == u1 || at.unit + 1 == job_end) {  // the end of the job, or of the run
        const bool whole = job_first >= u0 && job_end <= u1;
        const int slot = job_first < u0 ? 0 : 1;
        // (a run's last part may lie where its ring was: nothing is in flight any more)
        float* const part = slot == 0 ? smem.first_part(warp, part_rows) : reinterpret_cast<float*>(smem.ring(warp));
        if (!whole) __syncwarp();  // (the ring has been read)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 1);
          l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 2);
          const int row = n8 + 8 * e, i = at.tile * kFewTile + row, r = i / c.group;
          if (r >= at.x.rows) continue;
          const float back = power[e] == 0.f ? 0.f : 1.f / power[e];
          const long long q_row = at.x.row0 + r;
          const int head = at.head * c.group + i - r * c.group;
          if (whole && c.prefixes == 0) {
            const float inv = l[e] == 0.f ? 0.f : back / l[e];
            uint16_t* const to = c.out + q_row * c.o_st + (long long)head * c.o_sh + t4 * (DIM / 4);
#pragma unroll
            for (int col = 0; col < 2; ++col)  // columns 2 t4 + col of every group of eight: elements DIM / 8 (2 t4 + col) ..
#pragma unroll
              for (int j = 0; j < kTiles / 8; ++j) {
                uint32_t x[4];
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) x[i4] = pair_bf16(o[8 * j + 2 * i4][2 * e + col] * inv, o[8 * j + 2 * i4 + 1][2 * e + col] * inv);
                *reinterpret_cast<uint4*>(to + col * (DIM / 8) + 8 * j) = make_uint4(x[0], x[1], x[2], x[3]);
              }
            if (c.lse_out && t4 == 0) c.lse_out[q_row * c.hq + head] = l[e] == 0.f ? -INFINITY : (m[e] + log2f(l[e])) * kLn2;
          } else {
            const long long flat = (at.x.own ? 0ll : (long long)c.total_q * c.hq) + q_row * c.hq + head;
            float* const to = whole ? c.whole_out + flat * DIM : part;
#pragma unroll
            for (int col = 0; col < 2; ++col)
#pragma unroll
              for (int j = 0; j < kTiles / 4; ++j) {
                const int piece = t4 * (DIM / 16) + col * (DIM / 32) + j;
                *reinterpret_cast<float4*>(to + (whole ? piece * 4 : part_at<DIM>(row, piece))) =
                    make_float4(o[4 * j][2 * e + col] * back, o[4 * j + 1][2 * e + col] * back, o[4 * j + 2][2 * e + col] * back, o[4 * j + 3][2 * e + col] * back);
              }
            if (t4 == 0) {
              if (whole) c.whole_ml[flat] = make_float2(m[e], l[e]);
              else left_ml[warp][slot][row] = make_float2(m[e], l[e]);
            }
          }
        }
        if (!whole && lane == 0) left[warp][slot] = Left{job_first, job_end, at.x.row0, at.x.rows, at.tile, at.head, at.x.own};
      }
      if (!at.step(c, list, ahead, u1)) break;
    }
    if (!ok) {
      if (lane == 0 && c.device_status) atomicOr(c.device_status, FASTAV_DEV_WAIT_EXPIRED);
      // The copies in flight write into this block's shared memory: they are waited for before it may exit, also where another warp gave up.
      int never = 0;
      for (int n = max(0, issued - F::kStages); n < issued; ++n)
        ptx::mbar_wait_bounded(ptx::smem_u32(&full[warp][n % F::kStages]), (n / F::kStages) & 1, &never);
    }
  }
  pdl_trigger();
  __syncthreads();
  if (abort_flag) return;

  // The parts of one job that several warps left, joined in their order: to the output if the block has the whole job, else to the block's place.
  for (int i = 0; i < 2 * kWarps;) {
    const Left job = left[i / 2][i % 2];
    if (job.job_first < 0) {
      ++i;
      continue;
    }
    int end = i + 1;  // (unused slots lie between)
    for (int j = i + 1; j < 2 * kWarps; ++j) {
      const int start = left[j / 2][j % 2].job_first;
      if (start >= 0 && start != job.job_first) break;
      end = j + 1;
    }
    const bool whole = job.job_first >= block_u0 && job.job_end <= block_u1;
    const int slot = job.job_first < block_u0 ? 0 : 1;
    const int rows = min(kFewTile, job.rows * c.group - job.tile * kFewTile);
    for (int item = threadIdx.x; item < rows * (DIM / 4); item += kThreads) {
      const int row = item / (DIM / 4), piece = item % (DIM / 4);
      float top = -INFINITY;
      for (int j = i; j < end; ++j)
        if (left[j / 2][j % 2].job_first >= 0) top = fmaxf(top, left_ml[j / 2][j % 2][row].x);
      const float base = top == -INFINITY ? 0.f : top;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
      for (int j = i; j < end; ++j) {
        if (left[j / 2][j % 2].job_first < 0) continue;
        const float2 ml = left_ml[j / 2][j % 2][row];
        const float f = ptx::ex2_approx(ml.x - base);
        const float* const part = j % 2 == 0 ? smem.first_part(j / 2, part_rows) : reinterpret_cast<const float*>(smem.ring(j / 2));
        const float4 v = *reinterpret_cast<const float4*>(part + part_at<DIM>(row, piece));
        sum += f * ml.y;
        acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
      }
      const int stacked = job.tile * kFewTile + row, r = stacked / c.group, head = job.head * c.group + stacked - r * c.group;
      const long long q_row = job.row0 + r, flat = (job.own ? 0ll : (long long)c.total_q * c.hq) + q_row * c.hq + head;
      if (whole && c.prefixes == 0) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint2*>(c.out + q_row * c.o_st + (long long)head * c.o_sh + piece * 4) = make_uint2(pair_bf16(acc.x * inv, acc.y * inv), pair_bf16(acc.z * inv, acc.w * inv));
        if (c.lse_out && piece == 0) c.lse_out[flat] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
      } else {
        const long long place = ((long long)blockIdx.x * 2 + slot) * kFewTile + row;
        *reinterpret_cast<float4*>((whole ? c.whole_out + flat * DIM : list.part_out + place * DIM) + piece * 4) = acc;
        if (piece == 0) *(whole ? c.whole_ml + flat : list.part_ml + place) = make_float2(top, sum);
      }
    }
    i = end;
  }
}

template <int DIM, bool FP8>
cudaError_t run(const AttendCall& c, const AttendList& list, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t stream) {
  const long long most_rows = (long long)(c.prefixes > 0 && c.max_prefix_q > c.max_qlen ? c.max_prefix_q : c.max_qlen) * c.group;
  const int part_rows = most_rows < kFewTile ? (int)most_rows : kFewTile;
  const size_t smem = few_smem<DIM>(part_rows, list.entries());
  const cudaError_t e = once_per_context([] {
    return cudaFuncSetAttribute(attend_few_kernel<DIM, FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_smem<DIM>(kFewTile, FASTAV_ATTEND_MAX_BATCH));
  });
  if (e != cudaSuccess) return e;
  count_launches(1);
  return launch_chained(attend_few_kernel<DIM, FP8>, dim3(list.grid), dim3(kThreads), smem, stream, k_map, v_map, c, list, part_rows);
}

}  // namespace

cudaError_t launch_attend_few(const AttendCall& c, const AttendList& list, cudaStream_t stream) {
  CUtensorMap k_map, v_map;
  const int box = 1 << c.cache.page_shift < kFewKeys ? 1 << c.cache.page_shift : kFewKeys;
  if (!encode_pool_map(c.cache, c.cache.k, box, &k_map) || !encode_pool_map(c.cache, c.cache.v, box, &v_map)) return cudaErrorNotSupported;
  if (c.cache.dim == 128) return c.cache.fp8 ? run<128, true>(c, list, k_map, v_map, stream) : run<128, false>(c, list, k_map, v_map, stream);
  return c.cache.fp8 ? run<64, true>(c, list, k_map, v_map, stream) : run<64, false>(c, list, k_map, v_map, stream);
}

}  // namespace fastav
