// Grouped products of few tokens per group: out[r, n] = sum_k x[src(r), k] * W_e[n, k] for the rows r of group e, for bf16 and
// 8-bit integers, with the gated activation of two products (pair) or scales per token and channel behind it.
//
// Bound: the weights' bytes, read once per 64 tokens of a group.  (One token through six pairs of 2048 x 1408, 69 MB: 16.2 to 16.5
// us where calls follow one another, of which 10 are the stream at 6.9 TB/s; 18.6 alone.  Two matrices of 4096 x 14336, 235 MB: 40 us,
// 5.9 TB/s.)
//   * A unit is 128 rows of one group's weights (64 of W1 and 64 of W3 of a pair) and up to 64 of its tokens.  The weights are
//     the M = 128 operand of a tcgen05 MMA and the tokens its N columns, so that a single token costs 16 columns, not 128 rows.
//   * A cluster of 1 to 8 blocks takes a unit and splits K among its blocks; the partial sums meet through distributed shared
//     memory, added in rank order: no workspace, the same bits whatever the timing, and integers stay exact.
//   * Weights come by TMA in the 128-byte swizzle.  The tokens' rows, which may lie anywhere, come by 16-byte asynchronous copies
//     that put them where the swizzle wants them; nothing is packed beforehand.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "grouped.cuh"
#include "grouped_launch.h"

namespace zipmoe_dev {

constexpr uint32_t kFewTokens = 64, kFewThreads = 256, kFewMaxStages = 8, kFewLag = 3;
constexpr uint32_t kFewWeights = 128 * 128;      // bytes of a step's weights
constexpr uint32_t kFewPitch = 132;              // words between tokens of the partial sums: neighbours fall into other banks

// The unit that a cluster takes: group, its first row, rows in all, first of the unit's tokens and their number, block of weights.
struct FewUnit {
  uint32_t e, first, n, rows0;   // rows0: first weight row (output column) of the unit
};

template <bool kInt8, bool kPair>
__global__ void __launch_bounds__(kFewThreads, 2) grouped_few_kernel(const __grid_constant__ GroupedMaps maps, const GroupedArgs a,
                                                                    const uint32_t NT, const uint32_t stages, const uint32_t tmem_cols) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * kFewMaxStages + 1];
  __shared__ uint32_t words[3];   // tmem, dead, bad
  __shared__ FewUnit unit_at;
  __shared__ int32_t source[kFewTokens];
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = cluster_rank(), S = cluster_size();
  uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t ring0 = smem_addr(ring), stage_bytes = kFewWeights + NT * 128;
  const uint32_t full = smem_addr(bars), empty = full + 8 * kFewMaxStages, done = empty + 8 * kFewMaxStages;
  volatile uint32_t *dead = words + 1;
  const WaitLimit lim = {dead, a.status, a.limit_ns};
  constexpr uint32_t kCols = kPair ? 64 : 128;   // output columns of a unit
  const uint32_t NB = (a.N + kCols - 1) / kCols, unit = blockIdx.x / S;
  const uint32_t steps = (a.Kb + 127) / 128, s0 = rank * steps / S, s1 = (rank + 1) * steps / S;

  if (tid == 0) {
    for (uint32_t s = 0; s < stages; ++s) {
      mbar_init(full + 8 * s, 5);   // the weights' copy and four warps that bring tokens
      mbar_init(empty + 8 * s, 1);
    }
    mbar_init(done, 1);
    *dead = 0;
    words[2] = 0;
    if (a.even) {
      prefetch_map(&maps.w[kPair ? 2 : 0]);
      if constexpr (kPair) prefetch_map(&maps.w[3]);
    }
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(smem_addr(words), tmem_cols);
  if (a.offsets) wait_predecessor();
  if (warp == 0) {
    // units before each group: lane l has the groups from per * l on; all loads are asked for before any is looked at
    const uint32_t per = (a.E + 31) / 32, e0 = lane * per;
    int32_t at[9];
    uint32_t n[8], units = 0;
#pragma unroll
    for (uint32_t i = 0; i < 9; ++i) at[i] = a.offsets && i <= per ? __ldcg(a.offsets + min(e0 + i, a.E)) : 0;
    bool fine = true;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) n[i] = i < per && e0 + i < a.E ? rows_between(a, at[i], at[i + 1], fine) : 0;
    fine = __all_sync(0xFFFFFFFFu, fine);
    if (!fine && lane == 0 && blockIdx.x == 0) report(a.status, kStatusBadDescriptor);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      if (!fine) n[i] = 0;   // rows could belong to two groups: nothing is computed
      units += (n[i] + kFewTokens - 1) / kFewTokens * NB;
    }
    uint32_t before = units;
#pragma unroll
    for (uint32_t d = 1; d < 32; d <<= 1) {
      const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, before, d);
      if (lane >= d) before += v;
    }
    const uint32_t all = __shfl_sync(0xFFFFFFFFu, before, 31);
    before -= units;
    if (unit >= all) {
      if (lane == 0) unit_at = FewUnit{0, 0, 0, 0};
    } else if (unit >= before && unit < before + units) {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t tiles = (n[i] + kFewTokens - 1) / kFewTokens, mine = tiles * NB;
        if (unit >= before && unit < before + mine) {   // token tiles of the same weights stand next to one another
          const uint32_t in = unit - before, block = tiles == 1 ? in : in / tiles, tile = in - block * tiles;
          unit_at = FewUnit{e0 + i, (uint32_t)at[i] + tile * kFewTokens, min(kFewTokens, n[i] - tile * kFewTokens), block * kCols};
        }
        before += mine;
      }
    }
  }
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  const uint32_t tmem = words[0];
  const FewUnit u = unit_at;
  const bool work = u.n > 0;
  if (!a.offsets) wait_predecessor();   // (what is to be done was known without it)
  let_successor();

  if (work && warp == 0 && lane == 0) {
    // ---- weights ----
    const uint64_t policy = policy_evict_first();
    const void *m0 = &maps.w[kPair ? 2 : 0], *m1 = &maps.w[3];
    if (!a.even) {
      m0 = a.table + (size_t)u.e * ZIPMOE_GROUPED_ENTRY_BYTES + (kPair ? kPairMap : 0);
      m1 = a.table + (size_t)u.e * ZIPMOE_GROUPED_ENTRY_BYTES + kPairMap + 128;
      acquire_map(m0);
      if constexpr (kPair) acquire_map(m1);
    }
    const int32_t z = a.even ? (int32_t)u.e : 0;
    uint32_t st = 0, round = 0;
    for (uint32_t s = s0; s < s1; ++s) {
      if (round > 0 && !wait_bar(empty + 8 * st, (round - 1) & 1, lim)) break;
      const uint32_t dst = ring0 + st * stage_bytes, bar = full + 8 * st;
      const int32_t x = (int32_t)(s * (kInt8 ? 128 : 64));
      mbar_expect_tx(bar, kFewWeights + a.extra_tx);
      if constexpr (kPair) {
        tma_load_3d(dst, m0, x, (int32_t)u.rows0, z, bar, policy);
        tma_load_3d(dst + kFewWeights / 2, m1, x, (int32_t)u.rows0, z, bar, policy);
      } else {
        tma_load_3d(dst, m0, x, (int32_t)u.rows0, z, bar, policy);
      }
      if (++st == stages) {
        st = 0;
        ++round;
      }
    }
  } else if (work && warp == 1 && lane == 0) {
    // ---- products ----
    const uint32_t idesc = grouped_idesc<kInt8>((u.n + 15) & ~15u);
    uint32_t st = 0, round = 0;
    bool ok = true;
    for (uint32_t s = s0; s < s1; ++s) {
      ok = wait_bar(full + 8 * st, round & 1, lim);
      if (!ok) break;
      tc_after_sync();
      const uint64_t wd = swizzled_desc(ring0 + st * stage_bytes), xd = swizzled_desc(ring0 + st * stage_bytes + kFewWeights);
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) grouped_mma<kInt8>(tmem, wd + 2 * j, xd + 2 * j, idesc, s > s0 || j > 0);
      tc_commit(empty + 8 * st);
      if (++st == stages) {
        st = 0;
        ++round;
      }
    }
    if (ok) tc_commit(done);
  } else if (work && warp >= 4) {
    // ---- tokens: a thread has one 16-byte column of every 16th row ----
    const uint32_t t = tid - 128, c = t & 7, r0 = t >> 3;
    const uint8_t *row[kFewTokens / 16];
    bool there[kFewTokens / 16];
#pragma unroll
    for (uint32_t i = 0; i < kFewTokens / 16; ++i) {
      const uint32_t r = r0 + 16 * i;
      const int32_t src = r < u.n ? source_row(a, u.first + r) : -1;
      if (r < u.n && src < 0) words[2] = 1;
      if (c == 0) source[r] = src;
      there[i] = src >= 0;
      row[i] = a.x + (src >= 0 ? (uint64_t)src * a.x_pitch : 0);
    }
    uint32_t st = 0, round = 0, behind = 0, issued = 0;
    bool ok = true;
    auto publish = [&] {   // the oldest stage's rows are there: seen by the tensor core, then told
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive(full + 8 * behind);
      if (++behind == stages) behind = 0;
    };
    for (uint32_t s = s0; s < s1; ++s) {
      ok = __all_sync(0xFFFFFFFFu, round == 0 || wait_bar(empty + 8 * st, (round - 1) & 1, lim));
      if (!ok) break;
      const uint32_t at = s * 128 + c * 16, dst = ring0 + st * stage_bytes + kFewWeights + r0 * 128 + ((c ^ (r0 & 7)) << 4);
#pragma unroll
      for (uint32_t i = 0; i < kFewTokens / 16; ++i)
        if (r0 + 16 * i < u.n) copy16(dst + i * 2048, row[i] + (at < a.Kb ? at : 0), there[i] && at < a.Kb);
      copies_commit();
      if (++issued > kFewLag) {
        copies_wait<kFewLag>();
        publish();
      }
      if (++st == stages) {
        st = 0;
        ++round;
      }
    }
    copies_wait<0>();
    if (ok)
      for (uint32_t i = 0; i < min(issued, kFewLag); ++i) publish();
  }
  __syncwarp();

  // ---- partial sums into shared memory, over the ring (every product has read it); a warp has 32 rows of the weights ----
  uint32_t *part = reinterpret_cast<uint32_t *>(ring);
  if (work && warp >= 4) {
    const bool ok = __all_sync(0xFFFFFFFFu, wait_bar(done, 0, lim));
    tc_after_sync();
    if (ok) {
      const uint32_t w = warp & 3;
      for (uint32_t t0 = 0; t0 < u.n; t0 += 8) {
        uint32_t v[8];
        tmem_load8(tmem + ((32 * w) << 16) + t0, v);
        tmem_wait();
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) part[(t0 + i) * kFewPitch + 32 * w + lane] = v[i];
      }
    }
  }
  __syncwarp();
  tc_before_sync();
  cluster_sync();
  tc_after_sync();
  if (*dead)   // let the copies and MMAs that this block has under way end before its memory goes to somebody else
    for (uint32_t i = 0; i < 200; ++i) __nanosleep(1000);
  if (warp == 1) tmem_free(tmem, tmem_cols);

  // ---- the tokens of this rank: a warp per token, four neighbouring rows of the weights per lane ----
  if (work && !*dead) {
    uint32_t base[8];
#pragma unroll
    for (uint32_t r = 0; r < 8; ++r) base[r] = in_block(ring0, r < S ? r : 0);
    const uint32_t col = u.rows0 + (kPair ? lane & 15 : lane) * 4;   // (lanes 16-31 have W3's sums of a pair)
    const bool mine = (!kPair || lane < 16) && col < a.N;
    float scale[4] = {1.f, 1.f, 1.f, 1.f};
    if constexpr (kInt8) {
      const float *from = a.col_scales + (size_t)u.e * a.N + (kPair && lane >= 16 ? (size_t)a.E * a.N : 0);
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) scale[i] = col + i < a.N ? __ldcg(from + col + i) : 0.f;
    }
    for (uint32_t t = rank + S * warp; t < u.n; t += S * (kFewThreads / 32)) {
      float4 v[8];
#pragma unroll
      for (uint32_t r = 0; r < 8; ++r)
        if (r < S) v[r] = load_cluster(base[r] + (t * kFewPitch + lane * 4) * 4);
      float sum[4];
      if constexpr (kInt8) {
        int32_t acc[4] = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r)
          if (r < S) {
            acc[0] += __float_as_int(v[r].x);
            acc[1] += __float_as_int(v[r].y);
            acc[2] += __float_as_int(v[r].z);
            acc[3] += __float_as_int(v[r].w);
          }
        const float token = source[t] >= 0 ? __ldcg(a.row_scales + source[t]) : 0.f;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) sum[i] = scaled(acc[i], token, scale[i]);
      } else {
        sum[0] = sum[1] = sum[2] = sum[3] = 0.f;
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r)
          if (r < S) {
            sum[0] += v[r].x;
            sum[1] += v[r].y;
            sum[2] += v[r].z;
            sum[3] += v[r].w;
          }
      }
      if constexpr (kPair) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
          const float up = __shfl_down_sync(0xFFFFFFFFu, sum[i], 16);
          sum[i] = silu_product(sum[i], up);
        }
      }
      if (mine) {
        const uint64_t to = (uint64_t)(u.first + t) * a.out_pitch + col;
        if (a.out_f32) {
          float *out = reinterpret_cast<float *>(a.out) + to;
          if (a.wide && col + 4 <= a.N) *reinterpret_cast<float4 *>(out) = make_float4(sum[0], sum[1], sum[2], sum[3]);
          else
            for (uint32_t i = 0; i < 4 && col + i < a.N; ++i) out[i] = sum[i];
        } else {
          __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(a.out) + to;
          if (a.wide && col + 4 <= a.N) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(sum[0], sum[1]), hi = __floats2bfloat162_rn(sum[2], sum[3]);
            *reinterpret_cast<uint2 *>(out) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
          } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
              if (col + i < a.N) out[i] = __float2bfloat16_rn(sum[i]);
          }
        }
      }
    }
  }
  if (rank == 0 && tid == 0 && words[2]) report(a.status, kStatusBadDescriptor);
  __syncwarp();
  cluster_sync();   // nobody leaves while a neighbour may still read its shared memory
}

}  // namespace zipmoe_dev

namespace {

template <bool kInt8, bool kPair>
zipmoe_status launch(int dev, const zipmoe_dev::GroupedMaps &maps, const zipmoe_dev::GroupedArgs &a, uint32_t tiles, cudaStream_t stream) {
  using namespace zipmoe_dev;
  static bool ready[64];
  if (!ready[dev]) {
    if (cudaFuncSetAttribute(grouped_few_kernel<kInt8, kPair>, cudaFuncAttributeMaxDynamicSharedMemorySize, 112 * 1024) != cudaSuccess)
      return ZIPMOE_ERR_CUDA;
    ready[dev] = true;
  }
  const uint32_t NT = std::min(kFewTokens, (a.R + 15) / 16 * 16), stage = kFewWeights + NT * 128;
  const uint32_t stages = std::min(kFewMaxStages, 108u * 1024 / stage), steps = (a.Kb + 127) / 128;
  uint32_t cols = 32;
  while (cols < NT) cols <<= 1;
  const uint32_t blocks = (a.N + (kPair ? 63 : 127)) / (kPair ? 64 : 128);
  const uint64_t units = (uint64_t)tiles * blocks;
  // as many blocks per unit as fill the device (two to an SM), each with four steps at least
  const uint32_t at_once = zipmoe_host::current_sms() * 2;
  uint32_t S = 8;
  while (S > 1 && (4 * S > steps || units * S > at_once)) S >>= 1;
  if (units * S > 0x7FFFFFFFull) return ZIPMOE_ERR_UNSUPPORTED;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeClusterDimension;
  attrs[0].val.clusterDim.x = S;
  attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
  attrs[1] = zipmoe_host::overlapped_if_whole(units * S, at_once);
  cudaLaunchConfig_t cfg = {};
  cfg.stream = stream;
  cfg.attrs = attrs;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3((uint32_t)(units * S));
  cfg.blockDim = dim3(kFewThreads);
  cfg.dynamicSmemBytes = 1024 + std::max(stages * stage, NT * kFewPitch * 4);
  return cudaLaunchKernelEx(&cfg, grouped_few_kernel<kInt8, kPair>, maps, a, NT, stages, cols) == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}

}  // namespace

zipmoe_status zipmoe_host::launch_grouped_few(int dev, bool int8, bool pair, const zipmoe_dev::GroupedMaps &maps,
                                              const zipmoe_dev::GroupedArgs &a, cudaStream_t stream) {
  // the most tiles of 64 rows that R rows can make in E groups
  const uint32_t most = std::min(a.E, a.R);
  const uint32_t NT = std::min(zipmoe_dev::kFewTokens, (a.R + 15) / 16 * 16);
  const uint32_t tiles = (uint32_t)std::min<uint64_t>(a.R, ((uint64_t)a.R + (uint64_t)(NT - 1) * most) / NT);
  if (int8) return pair ? launch<true, true>(dev, maps, a, tiles, stream) : launch<true, false>(dev, maps, a, tiles, stream);
  return pair ? launch<false, true>(dev, maps, a, tiles, stream) : launch<false, false>(dev, maps, a, tiles, stream);
}
