// Grouped products of many tokens: the same product as grouped_few_kernel.cu's, in tiles of 512 rows of weights (256 of W1 and 256 of
// W3 of a pair) by up to 256 tokens of a group.
//
// Bound: what shared memory takes in and gives out beside the tensor cores.  A tcgen05 MMA reads its operands there at 64 of the 128
// bytes a cycle, so every byte that the copies bring costs.  (8192 x 8192 x 8192 in bf16: 661 to 710 us, 1.55 to 1.66 PFLOP/s; 8192
// tokens of 8-bit integers, 4096 x 14336: 297 to 305 us, 3.2 POP/s; 8192 tokens' six of 64 experts, pairs of 2048 x 1408, without the
// packing: 458 to 470 us, 1.22 PFLOP/s.  These are ten calls behind one another after a pause.  In calls that go on for 0.15 s and
// more the clock is at the power limit, and the last two take 360 and 544 us.  A tile of 512 x 256 x 2048 takes 34.9 K cycles, 32.8 K of
// them products.)
//   * Two blocks of a cluster share one MMA (cta_group::2): each brings 128 rows of either half of the weights and half of the
//     tokens, and keeps the sums of its own weights in its tensor memory, two halves of [128 x tokens] of 32 bits.  Per step of 128
//     bytes of K that is 48 KB for two MMAs' worth of 256 x 256 sums, where tiles of 256 x 256 would take in 64 KB.
//   * The halves fill all of tensor memory, so sums cannot be read back under the next tile's products - but for the order in which
//     the products are issued: the first half is three steps ahead of the second at either end of a tile.  While the second
//     catches up the first is read back; while the next tile's first half gets ahead, the second is.
//   * Of a pair the first half is W1's rows and the second W3's: both values of an output come back in the same lane, the first
//     waits in registers for the second.
//   * Tokens are the N operand: a tile has as many columns as it has tokens, rounded to 32; a group's tokens are spread evenly over
//     its tiles.  Few columns do not make a tile short, since its weights have to come all the same: a step takes 0.50 us up to 96
//     columns, 0.57 with 128, 0.72 with 192 and 0.90 with 256 (bf16, weights in the second-level cache).
//   * One persistent pair of blocks per two SMs walks over the tiles of all groups; a group's tiles follow one another with the
//     tokens inside, so that pairs at work at the same time read the same weights.  One thread of each block works the tiles out,
//     ahead of the others.
//   * Rows of x that are gathered are packed first, by a kernel of their own.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "grouped.cuh"
#include "grouped_launch.h"

namespace zipmoe_dev {

constexpr uint32_t kWideStages = 4, kWidePart = 16384, kWideStage = 3 * kWidePart;   // a block's part of a step: both halves' weights, tokens
constexpr uint32_t kWideAhead = 3;                                           // steps that the first half is ahead: fewer than stages
constexpr uint32_t kWideCols = 256;                                          // columns of a half's sums
constexpr uint32_t kWideBand = 8;                                            // token tiles that are done before the next ones are looked at
constexpr uint32_t kWideReaders = 8, kWideThreads = 128 + 32 * kWideReaders; // warps that read sums back: two per 32 lanes of tensor memory

// Registers per thread: at launch (what 384 threads can have), then of the first four warps and of the readers.
constexpr uint32_t kWideRegs = 168, kWideRegsFew = 56, kWideRegsMany = 224;
static_assert(128 * kWideRegsFew + 32 * kWideReaders * kWideRegsMany <= kWideThreads * kWideRegs, "the readers would wait for registers that nobody gives up");

// (one half of bf16 products in fp32 fits the registers of the launch)
__host__ __device__ constexpr bool splits_registers(bool int8, bool pair, bool f32) { return pair || int8 || !f32; }

struct WideMaps {
  CUtensorMap w[2];
  CUtensorMap x128, x16;   // boxes of 128 and of 16 rows of x
};

// ---- what takes part in a pair of blocks ----
__device__ __forceinline__ void pair_load_3d(uint32_t dst, const void *map, int32_t x, int32_t y, int32_t z, uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], "
      "[%1, {%2, %3, %4}], [%5], %6;" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
      : "memory");
}
template <bool kInt8>
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate) {
  if constexpr (kInt8)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// one arrival on both blocks' barriers at this place once every MMA so far has completed
__device__ __forceinline__ void pair_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
               : "memory");
}
// An arrival on a barrier that may be another block's.  It tells that sums have been read from tensor memory, which the wait for
// those loads ensures; nothing in memory has to be seen by the other block, and ordering memory between the blocks of a cluster
// would hold the warp up for more than a thousand cycles.
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// wait_bar without a call, across which nothing could stay in registers
__device__ __forceinline__ bool wait_pair(uint32_t bar, uint32_t parity, const WaitLimit &w) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
  for (;;) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*w.dead) return false;
    if (global_ns() - t0 > w.limit_ns) {
      *w.dead = 1;
      report(w.status, kStatusWaitTimeout);
      return false;
    }
  }
}
// 16 columns of the warp's 32 lanes.  kF32: the thread has its lane's 16 columns.  Else, lanes b * 16 ..: of the 8 x 8 pieces that
// stmatrix takes, v[8 b + 4 g + 2 r + i] is lane 16 b + 8 r + lane / 4, column 8 g + 2 * (lane % 4) + i.
template <bool kF32>
__device__ __forceinline__ void tmem_load_chunk(uint32_t addr, uint32_t *v) {
  if constexpr (kF32) {
    tmem_load8(addr, v);
    tmem_load8(addr + 8, v + 8);
  } else {
#pragma unroll
    for (uint32_t b = 0; b < 2; ++b)
      asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(v[8 * b]), "=r"(v[8 * b + 1]), "=r"(v[8 * b + 2]), "=r"(v[8 * b + 3]), "=r"(v[8 * b + 4]), "=r"(v[8 * b + 5]),
                     "=r"(v[8 * b + 6]), "=r"(v[8 * b + 7])
                   : "r"(addr + ((16 * b) << 16))
                   : "memory");
  }
}
// Which row (0..31) and which of the 16 columns the thread's i-th value of a chunk is.
template <bool kF32>
__device__ __forceinline__ uint32_t chunk_row(uint32_t i, uint32_t lane) {
  return kF32 ? lane : (i >> 3) * 16 + ((i >> 1) & 1) * 8 + (lane >> 2);
}
template <bool kF32>
__device__ __forceinline__ uint32_t chunk_col(uint32_t i, uint32_t lane) {
  return kF32 ? i : ((i >> 2) & 1) * 8 + (lane & 3) * 2 + (i & 1);
}
// What a thread keeps of a chunk: fp32, or pairs of neighbouring tokens in bf16.
template <bool kF32>
struct Chunk {
  uint32_t p[kF32 ? 16 : 8];
  __device__ __forceinline__ void set(uint32_t i, float x, float y) {   // values i and i + 1, i even
    if constexpr (kF32) {
      p[i] = __float_as_uint(x);
      p[i + 1] = __float_as_uint(y);
    } else {
      const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
      p[i / 2] = *reinterpret_cast<const uint32_t *>(&v);
    }
  }
};
// Stores a warp's 16 tokens x 32 columns of the output, by way of its own 2 KB: whole 16-byte pieces of rows leave, where stores of single
// elements took 53 cycles each.
template <bool kF32>
__device__ __forceinline__ void store_chunk(const Chunk<kF32> &f, uint8_t *buf, uint32_t lane, const GroupedArgs &a, uint64_t row, uint32_t rows,
                                            uint32_t col) {
  __syncwarp();   // (the buffer's last contents have been read)
  if constexpr (kF32) {
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) reinterpret_cast<uint32_t *>(buf)[i * 32 + lane] = f.p[i];
  } else {
    // rows of 64 bytes, their four pieces in another order every two rows: neither the pieces of 8 rows nor whole rows collide
    const uint32_t token = (lane >> 4) * 8 + (lane & 7);
#pragma unroll
    for (uint32_t b = 0; b < 2; ++b) {
      const uint32_t piece = (b * 2 + ((lane >> 3) & 1)) ^ ((token >> 1) & 3);
      asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(smem_addr(buf) + token * 64 + piece * 16),
                   "r"(f.p[4 * b]), "r"(f.p[4 * b + 1]), "r"(f.p[4 * b + 2]), "r"(f.p[4 * b + 3])
                   : "memory");
    }
  }
  __syncwarp();
  constexpr uint32_t kPieces = kF32 ? 8 : 4, kSize = kF32 ? 4 : 2, kIn = 16 / kSize;   // 16-byte pieces of a row; elements in one
  if (a.whole && col + 32 <= a.N) {
#pragma unroll
    for (uint32_t j = 0; j < 16 * kPieces / 32; ++j) {
      const uint32_t token = j * (32 / kPieces) + lane / kPieces, piece = lane % kPieces;
      if (token < rows)
        *reinterpret_cast<uint4 *>(a.out + ((row + token) * a.out_pitch + col + piece * kIn) * kSize) =
            *reinterpret_cast<const uint4 *>(buf + token * (32 * kSize) + (kF32 ? piece : piece ^ ((token >> 1) & 3)) * 16);
    }
  } else if (col + lane < a.N) {   // rows that start anywhere: an element per lane
#pragma unroll
    for (uint32_t token = 0; token < 16; ++token) {
      if (token >= rows) break;
      uint8_t *to = a.out + ((row + token) * a.out_pitch + col + lane) * kSize;
      if constexpr (kF32) *reinterpret_cast<uint32_t *>(to) = reinterpret_cast<const uint32_t *>(buf)[token * 32 + lane];
      else *reinterpret_cast<uint16_t *>(to) = *reinterpret_cast<const uint16_t *>(buf + token * 64 + ((lane >> 3) ^ ((token >> 1) & 3)) * 16 + (lane & 7) * 2);
    }
  }
}

// The tiles of all groups, in order: before[e] of them come before group e's.
struct WideLists {
  uint32_t before[kMaxGroups + 1], first[kMaxGroups], n[kMaxGroups];
};
struct WideTile {
  uint32_t e, first, n, cols, block;   // group; its first row and tokens in the tile; operand columns; block of weights.  n = 0: no more
  uint32_t shared;                     // whether other tiles of the group read the same weights
};
constexpr uint32_t kWideTiles = 4;     // tiles that are worked out ahead
// A group's tokens in tiles of at most 256 columns, evenly by whole 32s: the first tiles may have 32 more than the others.
__device__ __forceinline__ uint32_t token_tiles(uint32_t n) { return (n + kWideCols - 1) / kWideCols; }
__device__ __forceinline__ WideTile tile_at(const WideLists &l, uint32_t t, uint32_t E, uint32_t blocks) {
  uint32_t lo = 0, hi = E;   // the last group whose tiles begin at or before t
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (l.before[mid] <= t) lo = mid;
    else hi = mid;
  }
  const uint32_t n = l.n[lo], tiles = token_tiles(n), at = t - l.before[lo];
  const uint32_t band = at / (kWideBand * blocks), in_band = at - band * kWideBand * blocks, width = min(kWideBand, tiles - band * kWideBand);
  WideTile r;
  r.e = lo;
  r.block = in_band / width;
  const uint32_t tile = band * kWideBand + in_band - r.block * width, units = (n + 31) / 32, each = units / tiles, more = units - each * tiles;
  const uint32_t skip = (tile * each + min(tile, more)) * 32;
  r.shared = tiles > 1;
  r.cols = (each + (tile < more ? 1 : 0)) * 32;
  r.first = l.first[lo] + skip;
  r.n = min(r.cols, n - skip);
  return r;
}

// The rows of x that `order` names, one after the other: a tile's rows are then one copy, and of the many tiles that a group's
// blocks of weights make only the first has to look them up.  (Fetched where they lie by the copy engine's gathers of four rows,
// in every tile, they held up the products of 49152 x 2048 x 2816 by 95 us of 440; by 16-byte copies of eight warps by 395.)
// A warp per row, all its loads under way at once up to 4 KB: 49152 rows of 4 KB in 45 us, 4.5 TB/s written (the rows of x come from the
// second-level cache); several rows per warp, other grids and fewer registers took 48 to 55.
constexpr uint32_t kPackRows = 8;
__global__ void __launch_bounds__(32 * kPackRows) pack_rows_kernel(const GroupedArgs a, uint8_t *packed) {
  const uint32_t r = blockIdx.x * kPackRows + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (r >= a.R || (a.offsets && ((int32_t)r < __ldcg(a.offsets) || (int32_t)r >= __ldcg(a.offsets + a.E)))) return;   // (of no group)
  const int32_t src = source_row(a, r);
  if (src < 0 && lane == 0) report(a.status, kStatusBadDescriptor);
  const uint8_t *from = a.x + (src >= 0 ? (uint64_t)src * a.x_pitch : 0);
  uint8_t *to = packed + (uint64_t)r * a.Kb;
  for (uint32_t c0 = lane * 16; c0 < a.Kb; c0 += 8 * 512) {
    uint4 v[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      v[i] = src >= 0 && c0 + i * 512 < a.Kb ? __ldcg(reinterpret_cast<const uint4 *>(from + c0 + i * 512)) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (c0 + i * 512 < a.Kb) *reinterpret_cast<uint4 *>(to + c0 + i * 512) = v[i];
  }
}

template <bool kInt8, bool kPair, bool kF32>
__global__ void __launch_bounds__(kWideThreads, 1) grouped_wide_kernel(const __grid_constant__ WideMaps maps, const GroupedArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * kWideStages + 4 + 2 * kWideTiles];
  __shared__ WideTile todo[kWideTiles];
  __shared__ uint32_t words[3];   // tmem, dead, tiles
  __shared__ WideLists lists;
  __shared__ __align__(16) uint8_t rows_out[kWideReaders][2048];
  __shared__ float token_scale[kInt8 ? kWideReaders : 1][kInt8 ? kWideCols / 2 : 1];
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = cluster_rank();
  uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t ring0 = smem_addr(ring);
  // barriers: a step's operands there (the first block's counts for both) / used; a half's sums there / read (the first block's)
  const uint32_t full = smem_addr(bars), empty = full + 8 * kWideStages, sums_full = empty + 8 * kWideStages, sums_empty = sums_full + 16,
                 tile_full = sums_empty + 16, tile_empty = tile_full + 8 * kWideTiles;
  const uint32_t pairs = gridDim.x / 2, pair = blockIdx.x / 2;
  volatile uint32_t *dead = words + 1;
  const WaitLimit lim = {dead, a.status, a.limit_ns};
  constexpr uint32_t kOut = kPair ? 256 : 512;   // output columns of a tile
  constexpr bool kSplit = splits_registers(kInt8, kPair, kF32);
  const uint32_t blocks = (a.N + kOut - 1) / kOut, steps = (a.Kb + 127) / 128;
  // (the last block of a single matrix's rows may have nothing for the second half)
  auto halves_of = [&](const WideTile &u) { return kPair || u.block * kOut + 256 < a.N ? 2u : 1u; };

  if (tid == 0) {
    for (uint32_t s = 0; s < kWideStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (uint32_t h = 0; h < 2; ++h) {
      mbar_init(sums_full + 8 * h, 1);
      mbar_init(sums_empty + 8 * h, 2 * kWideReaders);
    }
    for (uint32_t i = 0; i < kWideTiles; ++i) {
      mbar_init(tile_full + 8 * i, 1);
      mbar_init(tile_empty + 8 * i, kWideReaders + (rank == 0 ? 2 : 1));
    }
    *dead = 0;
    if (a.even) {
      prefetch_map(&maps.w[0]);
      if constexpr (kPair) prefetch_map(&maps.w[1]);
    }
    prefetch_map(&maps.x128);
    prefetch_map(&maps.x16);
    fence_barrier_init();
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(words)), "r"(2 * kWideCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  if (a.offsets) after_predecessor();   // (only now: nobody who comes after takes the tensor memory first)
  if (warp == 0) {
    // lane l has the groups from per * l on; all loads are asked for before any is looked at
    const uint32_t per = (a.E + 31) / 32, e0 = lane * per;
    int32_t at[9];
    uint32_t n[8], tiles = 0;
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
      tiles += token_tiles(n[i]) * blocks;
    }
    uint32_t before = tiles;
#pragma unroll
    for (uint32_t d = 1; d < 32; d <<= 1) {
      const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, before, d);
      if (lane >= d) before += v;
    }
    if (lane == 31) words[2] = before;
    before -= tiles;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < per && e0 + i < a.E) {
        lists.before[e0 + i] = before;
        lists.first[e0 + i] = (uint32_t)at[i];
        lists.n[e0 + i] = n[i];
        before += token_tiles(n[i]) * blocks;
      }
  }
  __syncthreads();
  cluster_sync();   // both blocks' barriers are set up
  if (!a.offsets) after_predecessor();   // (what is to be done was known without it)
  const uint32_t tmem = words[0], tiles = words[2];
  // the pair's i-th tile; false behind the last, or where a wait has run out
  auto next_tile = [&](uint32_t i, WideTile &u) {
    const uint32_t slot = i % kWideTiles;
    if (!wait_pair(tile_full + 8 * slot, (i / kWideTiles) & 1, lim)) return false;
    u = todo[slot];
    arrive(tile_empty + 8 * slot);
    return u.n > 0;
  };
  if (warp >= 4) {
    // (the readers hold a half's sums: they get the registers that the others do not need)
    if constexpr (kSplit) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kWideRegsMany));
    // ---- sums back; a warp has 32 rows of the weights, and every second 32 tokens ----
    const uint32_t w = warp & 3, side = (warp - 4) >> 2;
    uint32_t uses0 = 0, uses1 = 0;
    uint8_t *buf = rows_out[warp - 4];
    float *my_scale = token_scale[kInt8 ? warp - 4 : 0];
    constexpr uint32_t kScales = kF32 ? 1 : 4;   // rows of the weights that a thread's values of a chunk belong to
    for (uint32_t i = 0;; ++i) {
      // (one lane reads for the warp: every reader would have to be counted)
      WideTile u = {};
      if (lane == 0 && !next_tile(i, u)) u.n = 0;
      u.n = __shfl_sync(0xFFFFFFFFu, u.n, 0);
      if (u.n == 0) break;
      u.e = __shfl_sync(0xFFFFFFFFu, u.e, 0);
      u.first = __shfl_sync(0xFFFFFFFFu, u.first, 0);
      u.block = __shfl_sync(0xFFFFFFFFu, u.block, 0);
      const uint32_t halves = halves_of(u), col = u.block * kOut + rank * 128 + w * 32;
      float scale[2][kScales];
      if constexpr (kInt8) {
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
          for (uint32_t k = 0; k < kScales; ++k) {
            const uint32_t c = (kPair ? col : col + h * 256) + chunk_row<kF32>((k >> 1) * 8 + (k & 1) * 2, lane);
            scale[h][k] = c < a.N ? __ldcg(a.col_scales + (size_t)u.e * a.N + (kPair && h ? (size_t)a.E * a.N : 0) + c) : 0.f;
          }
        __syncwarp();
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) {
          const uint32_t r = (2 * c + side) * 32 + lane;
          const int32_t src = r < u.n ? source_row(a, u.first + r) : -1;
          my_scale[c * 32 + lane] = src >= 0 ? __ldcg(a.row_scales + src) : 0.f;
        }
        __syncwarp();
      }
      // the i-th value of a chunk that begins with the warp's tok0-th token
      auto value = [&](uint32_t v, const float *of, uint32_t tok0, uint32_t i) {
        if constexpr (kInt8)
          return scaled((int32_t)v, my_scale[tok0 + chunk_col<kF32>(i, lane)], of[kF32 ? 0 : (i >> 3) * 2 + ((i >> 1) & 1)]);
        else
          return __uint_as_float(v);
      };
      auto wait_for = [&](uint32_t h, uint32_t &uses) {
        const bool ok = __all_sync(0xFFFFFFFFu, wait_pair(sums_full + 8 * h, uses & 1, lim));
        ++uses;
        tc_after_sync();
        return ok;
      };
      auto release = [&](uint32_t h) {
        tc_before_sync();
        __syncwarp();
        if (lane == 0) arrive_cluster(in_block(sums_empty + 8 * h, 0));
      };
      const uint32_t lanes = tmem + ((32 * w) << 16);
      // Sums leave tensor memory at once and wait in registers for their turn to be stored, which takes five times as long.
      auto first_of = [&](uint32_t c) { return (2 * (c >> 1) + side) * 32 + (c & 1) * 16; };   // first token of the warp's c-th chunk
      auto fetch = [&](uint32_t h, const float *of, Chunk<kF32> *to, const float (*gate)[16]) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c) {
          if (first_of(c) >= u.n) continue;
          uint32_t v[16];
          tmem_load_chunk<kF32>(lanes + h * kWideCols + first_of(c), v);
          tmem_wait();
#pragma unroll
          for (uint32_t i = 0; i < 16; i += 2) {
            const float x = value(v[i], of, c * 16, i), y = value(v[i + 1], of, c * 16, i + 1);
            if constexpr (kPair) to[c].set(i, gate[c][i] * x, gate[c][i + 1] * y);
            else to[c].set(i, x, y);
          }
        }
        release(h);
      };
      auto store = [&](const Chunk<kF32> &f, uint32_t c, uint32_t at) __attribute__((always_inline)) {
        if (first_of(c) < u.n) store_chunk<kF32>(f, buf, lane, a, u.first + first_of(c), u.n - first_of(c), at);
      };
      if constexpr (kPair) {
        float g[8][16];   // W1's values wait here for W3's
        if (!wait_for(0, uses0)) break;
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c) {
          if (first_of(c) >= u.n) continue;
          uint32_t v[16];
          tmem_load_chunk<kF32>(lanes + first_of(c), v);
          tmem_wait();
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) {
            const float x = value(v[i], scale[0], c * 16, i);
            g[c][i] = x / (1.0f + __expf(-x));
          }
        }
        release(0);
        if (!wait_for(1, uses1)) break;
        Chunk<kF32> f[8];
        fetch(1, scale[1], f, g);
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c) store(f[c], c, col);
      } else {
        Chunk<kF32> f[8];
        if (!wait_for(0, uses0)) break;
        fetch(0, scale[0], f, nullptr);
        if constexpr (kF32) {   // (no room for both halves)
#pragma unroll
          for (uint32_t c = 0; c < 8; ++c) store(f[c], c, col);
          if (halves == 2) {
            if (!wait_for(1, uses1)) break;
            fetch(1, scale[1], f, nullptr);
#pragma unroll
            for (uint32_t c = 0; c < 8; ++c) store(f[c], c, col + 256);
          }
        } else {
          Chunk<kF32> f1[8];
          if (halves == 2) {
            if (!wait_for(1, uses1)) break;
            fetch(1, scale[1], f1, nullptr);
          }
#pragma unroll
          for (uint32_t c = 0; c < 8; ++c) store(f[c], c, col);
          if (halves == 2) {
#pragma unroll
            for (uint32_t c = 0; c < 8; ++c) store(f1[c], c, col + 256);
          }
        }
      }
    }
  } else {
    if constexpr (kSplit) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kWideRegsFew));
    if (warp == 0 && lane == 0) {
      // ---- weights and tokens ----
      const uint64_t once = policy_evict_first(), keep = policy_evict_last();
      uint32_t st = 0, round = 0, last_e = 0xFFFFFFFFu;
      bool ok = true;
      WideTile u;
      for (uint32_t i = 0; ok && next_tile(i, u); ++i) {
        const void *m0 = &maps.w[0], *m1 = &maps.w[kPair ? 1 : 0];
        if (!a.even) {
          m0 = a.table + (size_t)u.e * ZIPMOE_GROUPED_ENTRY_BYTES;
          m1 = kPair ? a.table + (size_t)u.e * ZIPMOE_GROUPED_ENTRY_BYTES + 128 : m0;
          if (u.e != last_e) {
            acquire_map(m0);
            if constexpr (kPair) acquire_map(m1);
            last_e = u.e;
          }
        }
        const int32_t z = a.even ? (int32_t)u.e : 0;
        const uint64_t policy = u.shared ? keep : once;
        const uint32_t half = u.cols / 2, halves = halves_of(u), bytes = 2 * (kWidePart * halves + half * 128) + a.extra_tx;
        const int32_t row0 = (int32_t)(u.block * kOut + rank * 128), row1 = row0 + (kPair ? 0 : 256), x_row = (int32_t)(u.first + rank * half);
        for (uint32_t s = 0; s < steps; ++s) {
          ok = round == 0 || wait_pair(empty + 8 * st, (round - 1) & 1, lim);
          if (!ok) break;
          const uint32_t dst = ring0 + st * kWideStage, bar = in_block(full + 8 * st, 0);
          const int32_t x = (int32_t)(s * (kInt8 ? 128 : 64));
          if (rank == 0) mbar_expect_tx(full + 8 * st, bytes);
          pair_load_3d(dst, m0, x, row0, z, bar, policy);
          if (halves == 2) pair_load_3d(dst + kWidePart, m1, x, row1, z, bar, policy);
          if (half == 128) {
            pair_load_3d(dst + 2 * kWidePart, &maps.x128, x, x_row, 0, bar, keep);
          } else {
            for (uint32_t r = 0; r < half; r += 16) pair_load_3d(dst + 2 * kWidePart + r * 128, &maps.x16, x, x_row + (int32_t)r, 0, bar, keep);
          }
          if (++st == kWideStages) {
            st = 0;
            ++round;
          }
        }
      }
    } else if (warp == 1 && lane == 0 && rank == 0) {
      // ---- products, for both blocks ----
      uint32_t seen = 0, used = 0, uses0 = 0, uses1 = 0;   // steps that are known to be there; steps before the present tile
      bool ok = true;
      WideTile u;
      for (uint32_t i = 0; ok && next_tile(i, u); ++i) {
        const uint32_t idesc = (grouped_idesc<kInt8>(u.cols) & 0x00FFFFFFu) | (16u << 24), halves = halves_of(u);
        auto issue = [&](uint32_t h, uint32_t s) {   // step s of a half
          const uint32_t at = used + s, st = at & (kWideStages - 1);
          if (seen == at) {
            ok = ok && wait_pair(full + 8 * st, (at / kWideStages) & 1, lim);
            tc_after_sync();
            ++seen;
          }
          if (!ok) return;
          const uint64_t wd = swizzled_desc(ring0 + st * kWideStage + h * kWidePart), xd = swizzled_desc(ring0 + st * kWideStage + 2 * kWidePart);
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) pair_mma<kInt8>(tmem + h * kWideCols, wd + 2 * j, xd + 2 * j, idesc, s > 0 || j > 0);
          if (h + 1 == halves) pair_commit(empty + 8 * st);
        };
        auto begin = [&](uint32_t h, uint32_t &uses) {   // whatever the half's sums were has been read
          ok = ok && (uses == 0 || wait_pair(sums_empty + 8 * h, (uses - 1) & 1, lim));
          ++uses;
          tc_after_sync();
        };
        static_assert((kWideStages & (kWideStages - 1)) == 0 && kWideAhead < kWideStages, "steps that wait for the second half leave a stage to be filled");
        begin(0, uses0);
        if (halves == 1) {
          for (uint32_t s = 0; s < steps && ok; ++s) issue(0, s);
          if (ok) pair_commit(sums_full);
        } else {
          // the first half's first steps, the second's; both by turns; the first half's last steps, the second's
          const uint32_t head = min(kWideAhead, steps), tail = max(head, steps - head);
          for (uint32_t s = 0; s < head && ok; ++s) issue(0, s);
          if (tail == steps && ok) pair_commit(sums_full);
          begin(1, uses1);
          for (uint32_t s = 0; s < head && ok; ++s) issue(1, s);
          for (uint32_t s = head; s < tail && ok; ++s) {
            issue(0, s);
            issue(1, s);
          }
          if (tail < steps) {
            for (uint32_t s = tail; s < steps && ok; ++s) issue(0, s);
            if (ok) pair_commit(sums_full);
            for (uint32_t s = tail; s < steps && ok; ++s) issue(1, s);
          }
          if (ok) pair_commit(sums_full + 8);
        }
        used += steps;
      }
    } else if (warp == 3 && lane == 0) {
      // ---- which tiles: worked out ahead of the others, who would stop for it ----
      // Every pair takes every pairs-th tile.  Those behind the last whole round are cut by tokens, as far as that makes no further
      // round.  (Given to the pair that would be free first, by costs that go with a tile's tokens, they took as long: a step of
      // fewer tokens waits for its weights all the same.)
      const uint32_t rest = tiles % pairs, whole = tiles - rest;
      uint32_t cuts = 1;
      while (cuts < 4 && rest * cuts * 2 <= pairs) cuts *= 2;
      const uint32_t all = whole + rest * cuts;
      uint32_t given = 0;
      bool ok = true;
      for (uint32_t v = pair; ok; v += pairs) {
        WideTile u = {};
        if (v < whole) {
          u = tile_at(lists, v, a.E, blocks);
        } else if (v < all) {
          u = tile_at(lists, whole + (v - whole) / cuts, a.E, blocks);
          const uint32_t part = (v - whole) % cuts, units = u.cols / 32, each = units / cuts, more = units - each * cuts;
          const uint32_t skip = (part * each + min(part, more)) * 32;
          u.cols = (each + (part < more ? 1 : 0)) * 32;
          u.first += skip;
          u.n = skip < u.n ? min(u.cols, u.n - skip) : 0;
          if (u.n == 0) continue;   // (fewer 32s than parts)
        }
        const uint32_t slot = given % kWideTiles;
        ok = given < kWideTiles || wait_pair(tile_empty + 8 * slot, (given / kWideTiles - 1) & 1, lim);
        if (ok) {
          todo[slot] = u;
          arrive(tile_full + 8 * slot);
          ++given;
        }
        if (u.n == 0) break;
      }
    }
    __syncwarp();
  }
  __syncwarp();
  tc_before_sync();
  cluster_sync();   // neither block's barriers, operands or sums are wanted any more
  tc_after_sync();
  if (*dead)   // let the copies and MMAs that are under way end before the memory goes to somebody else
    for (uint32_t i = 0; i < 200; ++i) __nanosleep(1000);
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kWideCols) : "memory");
}

}  // namespace zipmoe_dev

namespace {

template <bool kInt8, bool kPair, bool kF32>
zipmoe_status launch(int dev, const zipmoe_dev::WideMaps &maps, const zipmoe_dev::GroupedArgs &a, cudaStream_t stream) {
  using namespace zipmoe_dev;
  constexpr uint32_t kSmem = 1024 + kWideStages * kWideStage;
  static bool ready[64];
  if (!ready[dev]) {
    cudaFuncAttributes found;
    if (cudaFuncGetAttributes(&found, grouped_wide_kernel<kInt8, kPair, kF32>) != cudaSuccess || (splits_registers(kInt8, kPair, kF32) && found.numRegs < (int)kWideRegs))
      return ZIPMOE_ERR_CUDA;   // (the split of the registers would not come out)
    if (cudaFuncSetAttribute(grouped_wide_kernel<kInt8, kPair, kF32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess)
      return ZIPMOE_ERR_CUDA;
    ready[dev] = true;
  }
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeClusterDimension;
  attrs[0].val.clusterDim.x = 2;
  attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
  attrs[1] = zipmoe_host::overlapped();
  cudaLaunchConfig_t cfg = {};
  cfg.stream = stream;
  cfg.attrs = attrs;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3(zipmoe_host::current_sms() / 2 * 2);
  cfg.blockDim = dim3(kWideThreads);
  cfg.dynamicSmemBytes = kSmem;
  return cudaLaunchKernelEx(&cfg, grouped_wide_kernel<kInt8, kPair, kF32>, maps, a) == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}

}  // namespace

zipmoe_status zipmoe_host::launch_grouped_wide(int dev, bool int8, bool pair, const zipmoe_dev::GroupedMaps &weights,
                                               const zipmoe_dev::GroupedArgs &a, void *packed, cudaStream_t stream) {
  using namespace zipmoe_dev;
  WideMaps maps;
  maps.w[0] = weights.w[0];
  maps.w[1] = weights.w[1];
  const void *x = a.x;
  uint64_t rows = a.x_rows, pitch = a.x_pitch;
  if (a.order) {
    x = packed;
    rows = a.R;
    pitch = a.Kb;
    pack_rows_kernel<<<(a.R + kPackRows - 1) / kPackRows, 32 * kPackRows, 0, stream>>>(a, static_cast<uint8_t *>(packed));
    if (cudaGetLastError() != cudaSuccess) return ZIPMOE_ERR_CUDA;
  }
  if (!make_byte_map(&maps.x128, x, rows, a.Kb, pitch, 128, 1, pitch, int8) || !make_byte_map(&maps.x16, x, rows, a.Kb, pitch, 16, 1, pitch, int8))
    return ZIPMOE_ERR_CUDA;
  const auto call = [&](auto of_int8, auto of_pair) {
    constexpr bool kInt8 = decltype(of_int8)::value, kPair = decltype(of_pair)::value;
    return a.out_f32 ? launch<kInt8, kPair, true>(dev, maps, a, stream) : launch<kInt8, kPair, false>(dev, maps, a, stream);
  };
  const std::true_type yes;
  const std::false_type no;
  return int8 ? (pair ? call(yes, yes) : call(yes, no)) : (pair ? call(no, yes) : call(no, no));
}
