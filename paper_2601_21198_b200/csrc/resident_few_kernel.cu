// The resident experts for at most 8 tokens, where a call is short enough for every hand-over between blocks to show.
//     g = W1 x,  u = W3 x,  h = SiLU(g) * u,  y = W2 h,  out[t] = bf16(sum_j w[t, j] * y)
// Bound: the active experts' weights, 6 * hidden * inter bytes each, read once; beyond that the latency of a call.
//
// Every block owns a slice of rows - inter / SMs rows of every W1 and W3, hidden / SMs rows of every W2 - and all of their
// columns.  So every sum is finished inside one block: no partial sums cross memory, the experts' combination happens in
// the block that owns the output rows, and blocks wait for one another once, for h.
//   * A chunk is 512 columns of up to 16 rows of W1 and of W3, or of up to 32 rows of W2.  One thread brings it into a ring
//     of stages: a tensor map that sees the matrix as [columns / 64][rows][64] delivers a box of 8 x rows x 64 in one copy,
//     each 64 columns a tile in the 128-byte swizzle.  What is left of a row behind its last whole 64 columns is a chunk of
//     its own, through an ordinary map.  (One bulk copy per row and 1 KB was tried: the copy engine takes 38 ns for each,
//     4 TB/s.  Loads into registers were tried: 12 warps with 16 loads in flight each, 4.8 TB/s.)
//     It runs ahead across experts, and asks the first chunks of W2 into the second-level cache before h is there.
//   * Another warp adds the same columns of the expert's tokens (x, then h, which is the sum of two bf16 numbers).
//   * Eight warps take the chunk's 16-column steps in turn: ldmatrix, mma.sync m16n8k16 (weights the 16 rows, tokens the 8
//     columns; fp32 sums in registers).  The second numbers of h are columns 4 to 7 where an expert has up to 4 tokens (one
//     product for both), and otherwise go through a second product.  With so few tokens these need a tenth of the issue slots
//     of the time that the bytes take; a tcgen05 operand of 128 rows would be nine tenths empty with 10 to 28 rows per block.
//   * At the end of a job (one expert's set of rows) they leave their partial sums in shared memory and go on; four more
//     warps add them and finish the job.
// One token, 2 experts of 4096 x 14336 (705 MB): 108 us, 6.5 TB/s, what a plain copy moves; 6 experts of 2048 x 1408
// (104 MB): 28.0 us, 3.7 TB/s; 8 tokens, 30 of 3008 x 1536 (832 MB): 128 us, 6.5 TB/s; 4 experts of 1024 x 512 (13 MB): 16 us, the
// latencies of a call: routing lists, the first weights, h seen by all, the last sums.
// A chunk takes a block 0.42 us even if it has 4 rows (more stages change nothing), so many experts with narrow slices are
// left to the other kernel.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>

#include "zipmoe.h"
#include "resident.cuh"

namespace zipmoe_dev {

constexpr uint32_t kFewThreads = 64 + 256 + 128;       // weights, activations, eight warps of products, four of sums
constexpr uint32_t kFewCols = 512, kFewRowBytes = kFewCols * 2;
// Bytes between tokens' columns, of x and of h (whose second numbers follow the first): eight tokens' words fall into different
// banks.
constexpr uint32_t kFewPitch = kFewRowBytes + 16, kFewPitchH = 2 * kFewRowBytes + 16;
constexpr uint32_t kFewOneProduct = 4;                 // up to so many tokens both numbers of h are columns of one product
constexpr uint32_t kFewTokenBytes = 9 * 1024;          // eight tokens' x, four tokens' h
constexpr uint32_t kFewAheadBytes = 192 * 1024;        // of W2 that a block asks into the cache before h is there
constexpr uint32_t kFewSumPitch = 20;                  // floats between the columns of a warp's 16 rows of sums: no bank conflicts

struct FewArgs {
  const uint16_t *tokens;
  const int32_t *ids;
  const float *weights;
  const uint8_t *table;
  uint16_t *out;
  ResidentSync *sync;
  uint16_t *h;              // [choices][2 * I]: chunk by chunk the two numbers that h is the sum of (place_of_h)
  uint32_t *status;
  uint64_t limit_ns;
  uint32_t T, k, E, H, I, even;
  uint32_t R1, S1, R2, S2;  // rows of a block, rows of a set: of W1 and W3, of W2
  uint32_t ring_bytes, w_bytes, stages, extra_tx;   // stages: of kFewTokenBytes
};

// shared memory: [ring][sums, two sets][outputs][active experts][masks][ids, weights][barriers, words]
constexpr uint32_t kFewSumBytes = 8 * 2 * 8 * kFewSumPitch * 4;
__host__ __device__ inline uint32_t few_control_bytes(uint32_t E, uint32_t T, uint32_t k) {
  return 2 * kFewSumBytes + T * 32 * 4 + 64 * (uint32_t)sizeof(Active) + pad16(E * 4) + 2 * pad16(T * k * 4) + (2 * kResMaxStages + 4) * 8 + 32;
}

__device__ __forceinline__ void load_a(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma_16816(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t load_b(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
// Column i's first number of h among a row's 2 * I: every chunk has its first numbers, then its second ones (`cols` further).
__device__ __forceinline__ uint32_t place_of_h(uint32_t i, uint32_t I, uint32_t &cols) {
  const uint32_t whole = I & ~63u, c0 = i < whole ? i & ~(kFewCols - 1) : whole;
  cols = i < whole ? min(kFewCols, whole - c0) : I - whole;
  return c0 + i;
}
__device__ __forceinline__ uint32_t nth_bit(uint32_t mask, uint32_t n) {   // place of the n-th set bit (counted from 0)
  for (; n > 0; --n) mask &= mask - 1;
  return __ffs(mask) - 1;
}

__global__ void __launch_bounds__(kFewThreads, 1) resident_few_kernel(const __grid_constant__ EvenMaps even, const __grid_constant__ EvenMaps rests,
                                                                      const FewArgs a) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x, G = gridDim.x, choices = a.T * a.k;
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t *ctl = smem + a.ring_bytes;
  float *sums = reinterpret_cast<float *>(ctl);                       // [2][8 warps][2][8][kFewSumPitch]
  ctl += 2 * kFewSumBytes;
  float *outs = reinterpret_cast<float *>(ctl);                       // [T][32]
  ctl += a.T * 32 * 4;
  Active *act = reinterpret_cast<Active *>(ctl);
  ctl += 64 * sizeof(Active);                                        // at most 8 * 8 choices
  uint32_t *mask = reinterpret_cast<uint32_t *>(ctl);
  ctl += pad16(a.E * 4);
  int32_t *ids = reinterpret_cast<int32_t *>(ctl);
  ctl += pad16(choices * 4);
  float *wts = reinterpret_cast<float *>(ctl);
  ctl += pad16(choices * 4);
  uint64_t *bars = reinterpret_cast<uint64_t *>(ctl);
  uint32_t *words = reinterpret_cast<uint32_t *>(bars + 2 * kResMaxStages + 4);   // unused, dead, active, most
  volatile uint32_t *dead = words + 1;
  const uint32_t ring = smem_addr(smem), full = smem_addr(bars), empty = full + 8 * kResMaxStages, sums_full = empty + 8 * kResMaxStages, sums_empty = sums_full + 16;
  const WaitLimit lim = {dead, a.status, a.limit_ns};

  after_predecessor();
  // ---- everything that has to come from memory first, at once ----
  const uint32_t magic = __ldcg(&a.sync->magic);
  const int32_t my_id = tid < choices ? __ldg(a.ids + tid) : -1;
  const float my_wt = tid < choices && a.weights ? __ldg(a.weights + tid) : 1.0f;
  if (!a.even) prefetch_table(a.table, a.E, cta * kFewThreads + tid, G * kFewThreads);
  else if (tid >= 64 && tid < 67) prefetch_map(&even.w[tid - 64]);
  else if (tid >= 96 && tid < 99 && ((tid < 98 ? a.H : a.I) & 63) != 0) prefetch_map(&rests.w[tid - 96]);
  for (uint32_t i = tid; i < a.E; i += kFewThreads) mask[i] = 0;
  if (tid == 0) {
    for (uint32_t s = 0; s < kResMaxStages; ++s) {
      mbar_init(full + 8 * s, 2);
      mbar_init(empty + 8 * s, 8);
    }
    for (uint32_t b = 0; b < 2; ++b) {
      mbar_init(sums_full + 8 * b, 8);
      mbar_init(sums_empty + 8 * b, 4);
    }
    *dead = 0;
    fence_barrier_init();
  }
  __syncthreads();
  if (tid < choices) {
    ids[tid] = my_id;
    wts[tid] = my_wt;
    if (my_id >= 0 && my_id < (int32_t)a.E) atomicOr(&mask[my_id], 1u << (tid / a.k));
    else if (my_id >= 0) report(a.status, kStatusBadDescriptor);
  }
  __syncthreads();
  if (warp == 0) {   // experts per * lane .. per * lane + per - 1
    const uint32_t per = (a.E + 31) / 32;
    uint32_t cnt[8], sum = 0, most = 0;   // sum: active experts << 16 | choices
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      cnt[i] = i < per && per * lane + i < a.E ? __popc(mask[per * lane + i]) : 0;
      sum += (cnt[i] ? 1u << 16 : 0) + cnt[i];
      most = max(most, cnt[i]);
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    uint32_t at = sum;
#pragma unroll
    for (uint32_t d = 1; d < 32; d <<= 1) {
      const uint32_t p = __shfl_up_sync(0xFFFFFFFFu, at, d);
      if (lane >= d) at += p;
    }
    if (lane == 31) {
      words[2] = at >> 16;
      words[3] = most;
    }
    at -= sum;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (cnt[i]) {
        act[at >> 16] = Active{per * lane + i, cnt[i], 0, at & 0xFFFFu};
        at += (1u << 16) + cnt[i];
      }
  }
  __syncthreads();
  const bool prepared = magic == kResMagic;
  const uint32_t n_active = prepared ? words[2] : 0;
  // a stage has room for 8 tokens' x, which is 4 tokens' h, or for the h of as many tokens as an expert of this call has (with
  // room for one token more stages are in flight, which only delays everybody else: 2 experts of 4096 x 14336 111 us instead of 108)
  const bool wide = words[3] > kFewOneProduct;
  const uint32_t stage_bytes = a.w_bytes + (wide ? (words[3] * kFewPitchH + 1023) / 1024 * 1024 : kFewTokenBytes);
  const uint32_t stages = wide ? min(kResMaxStages, a.ring_bytes / stage_bytes) : a.stages;
  // this block's rows, in sets; a phase's chunks run over experts, sets and columns (gate/up) or sets, experts and columns
  const uint32_t row0[2] = {min(a.I, cta * a.R1), min(a.H, cta * a.R2)}, row1[2] = {min(a.I, (cta + 1) * a.R1), min(a.H, (cta + 1) * a.R2)};
  const uint32_t sets[2] = {(row1[0] - row0[0] + a.S1 - 1) / a.S1, (row1[1] - row0[1] + a.S2 - 1) / a.S2};
  const uint32_t h_blocks = n_active ? (a.I + a.R1 - 1) / a.R1 : 0;   // blocks that have rows of W1

  if (warp == 0) {
    // ---- weights ----
    if (!a.even)
      for (uint32_t i = lane; i < 3 * n_active; i += 32) {   // the experts' maps, W1 and W3 first
        const uint32_t down = i >= 2 * n_active, ai = down ? i - 2 * n_active : i >> 1;
        const uint8_t *m = sliced_map(a.table, act[ai].e, down ? 2 : i & 1);
        acquire_map(m);
        if (((down ? a.I : a.H) & 63) != 0) acquire_map(m + (kRestMap - kSlicedMap));
        if (i < 2) prefetch_map(m);
      }
    __syncwarp();
    if (lane == 0) {
      const uint64_t policy = policy_evict_first();
      auto map_of = [&](uint32_t e, uint32_t j) -> const void * { return a.even ? static_cast<const void *>(&even.w[j]) : sliced_map(a.table, e, j); };
      auto rest_of = [&](uint32_t e, uint32_t j) -> const void * {
        return a.even ? static_cast<const void *>(&rests.w[j]) : sliced_map(a.table, e, j) + (kRestMap - kSlicedMap);
      };
      RingAt at;
      bool ok = true;
      for (uint32_t p = 0; p < 2 && ok; ++p) {
        const uint32_t K = p == 0 ? a.H : a.I, whole = K & ~63u, per_set = p == 0 ? a.S1 : a.S2, jobs = n_active * sets[p];
        for (uint32_t j = 0; j < jobs && ok; ++j) {
          const uint32_t ai = p == 0 ? j / sets[0] : j % n_active, s = p == 0 ? j - ai * sets[0] : j / n_active, e = act[ai].e;
          const int32_t r0 = (int32_t)(row0[p] + s * per_set), z = a.even ? (int32_t)e : 0;
          const void *m0 = map_of(e, p == 0 ? 0 : 2), *m1 = map_of(e, 1);
          if (!a.even && s == 0) {   // the next expert's maps
            const uint32_t next = ai + 1 < n_active ? act[ai + 1].e : act[0].e;
            if (p == 0 && ai + 1 < n_active) {
              prefetch_map(map_of(next, 0));
              prefetch_map(map_of(next, 1));
            } else {
              prefetch_map(map_of(next, 2));
            }
          }
          for (uint32_t c = 0; c < whole; c += kFewCols) {
            if (at.round > 0 && !wait_bar(empty + 8 * at.st, (at.round - 1) & 1, lim)) {
              ok = false;
              break;
            }
            const uint32_t dst = ring + at.st * stage_bytes, bar = full + 8 * at.st;
            mbar_expect_tx(bar, (p == 0 ? 2 : 1) * per_set * kFewRowBytes + a.extra_tx);
            tma_load_4d(dst, m0, 0, r0, (int32_t)(c / 64), z, bar, policy);
            if (p == 0) tma_load_4d(dst + per_set * kFewRowBytes, m1, 0, r0, (int32_t)(c / 64), z, bar, policy);
            at.next(stages);
          }
          if (whole < K && ok) {
            if (at.round > 0 && !wait_bar(empty + 8 * at.st, (at.round - 1) & 1, lim)) {
              ok = false;
              break;
            }
            const uint32_t dst = ring + at.st * stage_bytes, bar = full + 8 * at.st;
            mbar_expect_tx(bar, (p == 0 ? 2 : 1) * per_set * 128 + a.extra_tx);
            tma_load_3d(dst, rest_of(e, p == 0 ? 0 : 2), (int32_t)whole, r0, z, bar, policy);
            if (p == 0) tma_load_3d(dst + per_set * kFewRowBytes, rest_of(e, 1), (int32_t)whole, r0, z, bar, policy);
            at.next(stages);
          }
        }
        if (p == 0 && ok) {   // the beginning of W2, in the order in which it will be wanted
          uint32_t left = kFewAheadBytes / (a.S2 * kFewRowBytes);
          for (uint32_t j = 0; j < n_active * sets[1] && left > 0; ++j) {
            const uint32_t e = act[j % n_active].e;
            for (uint32_t c = 0; c < (a.I & ~63u) && left > 0; c += kFewCols, --left)
              tma_prefetch_4d(map_of(e, 2), 0, (int32_t)(row0[1] + j / n_active * a.S2), (int32_t)(c / 64), a.even ? (int32_t)e : 0);
          }
        }
      }
    }
  } else if (warp == 1) {
    // ---- activations: lane r copies the columns of the expert's r-th token (of h, both numbers at once) ----
    const uint64_t policy = policy_evict_last();
    RingAt at;
    bool ok = true;
    for (uint32_t p = 0; p < 2 && ok; ++p) {
      const uint32_t K = p == 0 ? a.H : a.I, whole = K & ~63u, jobs = n_active * sets[p];
      if (p == 1 && jobs > 0) {
        ok = __all_sync(0xFFFFFFFFu, wait_count(&a.sync->h_done[0], h_blocks, lim));
        fence_async_all();       // what other blocks stored is now read by the copy engine
      }
      for (uint32_t j = 0; j < jobs && ok; ++j) {
        const uint32_t ai = p == 0 ? j / sets[0] : j % n_active;
        const Active ex = act[ai];
        const uint16_t *src = a.tokens;
        if (lane < ex.n) src = p == 0 ? a.tokens + (size_t)nth_bit(mask[ex.e], lane) * K : a.h + (size_t)(ex.slot + lane) * 2 * K;
        for (uint32_t c = 0, cols; c < K; c += cols) {
          cols = c < whole ? min(kFewCols, whole - c) : K - c;
          ok = __all_sync(0xFFFFFFFFu, at.round == 0 || wait_bar(empty + 8 * at.st, (at.round - 1) & 1, lim));
          if (!ok) break;
          const uint32_t numbers = p + 1, bytes = numbers * cols * 2, bar = full + 8 * at.st;
          if (lane == 0) mbar_expect_tx(bar, ex.n * bytes);
          __syncwarp();
          if (lane < ex.n)
            bulk_load(ring + at.st * stage_bytes + a.w_bytes + lane * (p == 0 ? kFewPitch : kFewPitchH), src + numbers * c, bytes, bar, policy);
          at.next(stages);
        }
      }
    }
  } else if (warp < 10) {
    // ---- products ----
    const uint32_t cw = warp - 2;
    const uint32_t a_row = lane & 15, a_half = lane >> 4;   // ldmatrix: this lane's row and half of 16 columns
    RingAt at;
    uint32_t job = 0;
    bool ok = true;
    for (uint32_t p = 0; p < 2 && ok; ++p) {
      const uint32_t K = p == 0 ? a.H : a.I, whole = K & ~63u, per_set = p == 0 ? a.S1 : a.S2, jobs = n_active * sets[p];
      const bool two = p == 0 || per_set > 16;
      for (uint32_t j = 0; j < jobs && ok; ++j, ++job) {
        float d[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        // where this lane's token begins; in down the second numbers are a product of their own, or those of tokens 4 to 7
        // (columns without a token are whatever lies there, and give sums that nobody reads)
        const uint32_t n = p == 1 && a.T > kFewOneProduct ? act[j % n_active].n : 0;
        const bool again = n > kFewOneProduct, halves = p == 1 && !again;
        const uint32_t token = halves ? (lane >> 2) & 3 : again ? min(lane >> 2, n - 1) : lane >> 2, second = halves ? lane >> 4 : 0;
        const uint32_t b_at = a.w_bytes + token * (p == 0 ? kFewPitch : kFewPitchH) + (lane & 3) * 4;
        for (uint32_t c = 0; c < whole; c += kFewCols) {
          ok = __all_sync(0xFFFFFFFFu, wait_bar(full + 8 * at.st, at.round & 1, lim));
          if (!ok) break;
          const uint32_t left = min(kFewCols, whole - c), base = ring + at.st * stage_bytes, b_base = base + b_at + second * left * 2;
#pragma unroll 4
          for (uint32_t q = cw * 16; q < left; q += 128) {
            // 64 columns are per_set lines of 128 bytes; the second 16 rows are W3's box, or the lines after the first
            const uint32_t line = (q >> 6) * per_set + a_row, chunk = ((q & 63) >> 3) + a_half;
            uint32_t w0[4], w1[4];
            load_a(base + line * 128 + ((chunk ^ (line & 7)) << 4), w0);
            if (p == 0) load_a(base + per_set * kFewRowBytes + line * 128 + ((chunk ^ (line & 7)) << 4), w1);
            else if (two) load_a(base + (line + 16) * 128 + ((chunk ^ (line & 7)) << 4), w1);
            const uint32_t b0 = load_b(b_base + q * 2), b1 = load_b(b_base + q * 2 + 16);
            mma_16816(d[0], w0, b0, b1);
            if (two) mma_16816(d[1], w1, b0, b1);
            if (again) {
              const uint32_t c0 = load_b(b_base + (left + q) * 2), c1 = load_b(b_base + (left + q) * 2 + 16);
              mma_16816(d[0], w0, c0, c1);
              if (two) mma_16816(d[1], w1, c0, c1);
            }
          }
          __syncwarp();
          if (lane == 0) arrive(empty + 8 * at.st);
          at.next(stages);
        }
        if (whole < K && ok) {   // up to 64 columns more: a step for each of the first warps
          ok = __all_sync(0xFFFFFFFFu, wait_bar(full + 8 * at.st, at.round & 1, lim));
          if (!ok) break;
          const uint32_t left = K - whole, base = ring + at.st * stage_bytes, q = cw * 16, b_base = base + b_at + second * left * 2;
          if (q < left) {
            const uint32_t place = a_row * 128 + (((q >> 3) + a_half) ^ (a_row & 7)) * 16;
            uint32_t w0[4], w1[4];
            load_a(base + place, w0);
            if (two) load_a(base + place + (p == 0 ? per_set * kFewRowBytes : 16 * 128), w1);
            // (the last 8 of 16 columns may lie behind the row: weights are zero there, tokens have to be)
            const uint32_t b0 = load_b(b_base + q * 2), behind = load_b(b_base + q * 2 + 16), b1 = q + 8 < left ? behind : 0u;
            mma_16816(d[0], w0, b0, b1);
            if (two) mma_16816(d[1], w1, b0, b1);
            if (again) {
              const uint32_t c0 = load_b(b_base + (left + q) * 2), after = load_b(b_base + (left + q) * 2 + 16);
              const uint32_t c1 = q + 8 < left ? after : 0u;
              mma_16816(d[0], w0, c0, c1);
              if (two) mma_16816(d[1], w1, c0, c1);
            }
          }
          __syncwarp();
          if (lane == 0) arrive(empty + 8 * at.st);
          at.next(stages);
        }
        const uint32_t buf = job & 1;
        ok = ok && __all_sync(0xFFFFFFFFu, job < 2 || wait_bar(sums_empty + 8 * buf, ((job >> 1) - 1) & 1, lim));
        if (!ok) break;
        float *own = sums + buf * (kFewSumBytes / 4) + cw * (2 * 8 * kFewSumPitch);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) own[(m * 8 + (lane & 3) * 2 + (i & 1)) * kFewSumPitch + (lane >> 2) + (i >> 1) * 8] = d[m][i];
        __syncwarp();
        if (lane == 0) arrive(sums_full + 8 * buf);
      }
    }
  } else {
    // ---- sums ----
    const uint32_t ct = tid - 320;
    uint32_t job = 0;
    bool ok = true;
    for (uint32_t p = 0; p < 2 && ok; ++p) {
      const uint32_t per_set = p == 0 ? a.S1 : a.S2, jobs = n_active * sets[p];
      for (uint32_t j = 0; j < jobs && ok; ++j, ++job) {
        const uint32_t ai = p == 0 ? j / sets[0] : j % n_active, s = p == 0 ? j - ai * sets[0] : j / n_active;
        const uint32_t r0 = row0[p] + s * per_set, rows = min(per_set, row1[p] - r0);
        const Active ex = act[ai];
        if (p == 1 && ai == 0) {   // a new set of output rows
          for (uint32_t i = ct; i < a.T * 32; i += 128) outs[i] = 0.f;
        }
        const uint32_t buf = job & 1;
        ok = all_agree<128>(wait_bar(sums_full + 8 * buf, (job >> 1) & 1, lim));
        if (!ok) break;
        const float *mine = sums + buf * (kFewSumBytes / 4);
        const uint32_t span = p == 0 ? 16 : 32;
        for (uint32_t i = ct; i < span * ex.n; i += 128) {
          const uint32_t r = i % span, n = i / span;
          if (r >= rows) continue;
          float v[2] = {0.f, 0.f};
#pragma unroll
          for (uint32_t w = 0; w < 8; ++w) {
            const float *from = mine + w * (2 * 8 * kFewSumPitch) + n * kFewSumPitch;
            if (p == 0) {
              v[0] += from[r];
              v[1] += from[8 * kFewSumPitch + r];
            } else {
              const float *column = from + (r >> 4) * 8 * kFewSumPitch + (r & 15);
              v[0] += column[0];
              if (ex.n <= kFewOneProduct) v[1] += column[4 * kFewSumPitch];   // of h's second number
            }
          }
          if (p == 0) {
            uint32_t cols;
            uint16_t *h = a.h + (size_t)(ex.slot + n) * 2 * a.I + place_of_h(r0 + r, a.I, cols);
            split_h(silu_times(v[0], v[1]), h[0], h[cols]);
          } else {
            const uint32_t t = nth_bit(mask[ex.e], n);
            float wt = 0.f;
            for (uint32_t c = 0; c < a.k; ++c)
              if (ids[t * a.k + c] == (int32_t)ex.e) wt += wts[t * a.k + c];
            outs[t * 32 + r] += wt * (v[0] + v[1]);
          }
        }
        __syncwarp();
        if (lane == 0) arrive(sums_empty + 8 * buf);
        if (p == 1 && ai + 1 == n_active) {
          sync_group<128>();
          for (uint32_t i = ct; i < a.T * 32; i += 128) {
            const uint32_t r = i & 31, t = i >> 5;
            if (r < rows) a.out[(size_t)t * a.H + r0 + r] = __bfloat16_as_ushort(__float2bfloat16_rn(outs[i]));
          }
          sync_group<128>();   // (the next set begins by clearing what was just read)
        }
      }
      if (p == 0 && ok && jobs > 0) {   // all of this block's h is out: tell the others
        __threadfence();
        fence_async_all();
        sync_group<128>();
        if (ct == 0) add_release(&a.sync->h_done[0], 1u);
      }
    }
    if (prepared && n_active == 0)      // no token has an expert
      for (uint32_t i = ct; i < a.T * (row1[1] - row0[1]); i += 128) {
        const uint32_t t = i / (row1[1] - row0[1]), r = i - t * (row1[1] - row0[1]);
        a.out[(size_t)t * a.H + row0[1] + r] = 0;
      }
  }
  __syncwarp();
  __syncthreads();
  if (*dead)   // let the copies that this block has under way end before its memory goes to somebody else
    for (uint32_t i = 0; i < 200; ++i) __nanosleep(1000);
  if (tid == 0) {
    if (!prepared) {
      report(a.status, kStatusBadDescriptor);
    } else {
      __threadfence();
      if (atomicAdd(&a.sync->exited, 1u) == G - 1) {   // the last block leaves the counters as it found them
        a.sync->h_done[0] = 0;
        a.sync->exited = 0;
      }
    }
  }
}

}  // namespace zipmoe_dev

namespace zipmoe_host {

zipmoe_status launch_resident_few(const ResidentCall &c, cudaStream_t stream) {
  using namespace zipmoe_dev;
  FewArgs a;
  a.tokens = c.tokens;
  a.ids = c.ids;
  a.weights = c.weights;
  a.table = c.table;
  a.even = c.even_maps != nullptr;
  EvenMaps even = {}, rests = {};
  if (a.even) {
    std::memcpy(&even, c.even_maps, sizeof(even));
    std::memcpy(&rests, c.even_maps + sizeof(even), sizeof(rests));
  }
  a.out = c.out;
  a.sync = c.sync;
  a.h = reinterpret_cast<uint16_t *>(c.h);
  a.status = c.status;
  a.limit_ns = c.limit_ns;
  a.extra_tx = c.extra_tx;
  a.T = c.T;
  a.k = c.k;
  a.E = c.E;
  a.H = c.H;
  a.I = c.I;
  resident_few_rows(c.H, c.I, c.grid, &a.R1, &a.S1, &a.R2, &a.S2);
  a.w_bytes = (2 * a.S1 > a.S2 ? 2 * a.S1 : a.S2) * kFewRowBytes;
  const uint32_t control = few_control_bytes(c.E, c.T, c.k) + 1024;
  a.ring_bytes = (227 * 1024 - control) & ~15u;
  a.stages = std::min(kResMaxStages, a.ring_bytes / (a.w_bytes + kFewTokenBytes));
  static bool ready[64];
  if (!ready[c.device]) {
    if (cudaFuncSetAttribute(resident_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess)
      return ZIPMOE_ERR_CUDA;
    ready[c.device] = true;
  }
  cudaLaunchAttribute together;
  together.id = cudaLaunchAttributeCooperative;
  together.val.cooperative = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = stream;
  cfg.attrs = &together;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(c.grid);
  cfg.blockDim = dim3(kFewThreads);
  cfg.dynamicSmemBytes = control + a.ring_bytes;
  return cudaLaunchKernelEx(&cfg, resident_few_kernel, even, rests, a) == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}

}  // namespace zipmoe_host
