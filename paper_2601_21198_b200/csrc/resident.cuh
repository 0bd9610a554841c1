// What the two kernels behind zipmoe_expert_ffn share: the workspace's head, an entry of the experts' table, rings.
#pragma once
#include <cuda_bf16.h>

#include <cstdint>

#include "zipmoe.h"
#include "resident_choice.h"
#include "tensor_core.cuh"

namespace zipmoe_dev {

constexpr uint32_t kResMaxGrid = 256;
constexpr uint32_t kResMaxStages = 8;
constexpr uint32_t kResMagic = 0x5A464632u;                 // marks a workspace that zipmoe_expert_ffn_workspace_init prepared
// An entry of the table: the map of 128-row boxes, that of a block's slices of rows, that of the columns behind a row's last
// whole 64.
constexpr uint32_t kSlicedMap = 128, kRestMap = 256;

// Maps of all experts' W1, W3 and W2 at once, where they lie at equal distances.
struct EvenMaps {
  CUtensorMap w[3];
};

// The workspace starts with this: zero when no call is running (every call leaves it so).
struct ResidentSync {
  uint32_t magic, pad0[31];
  uint32_t x_done, pad1[31];      // blocks that have packed their part of the tokens
  uint32_t h_done[2], pad2[30];   // per group of experts: blocks that have stored all their h
  uint32_t y_done, pad3[31];      // blocks that have stored all their y, one count per group
  uint32_t exited, pad4[31];
  uint32_t cut[2][kResMaxGrid];   // [g][c]: blocks that have stored their part of the gate/up job cut at the end of block c's share
};

struct Active {
  uint32_t e, n, h_row, slot;   // expert; its tokens; first row of its h block; first of its choices
};

__host__ __device__ inline uint32_t pad16(uint32_t bytes) { return (bytes + 15) & ~15u; }

// The warps that share named barrier 1 give up together or not at all: the barrier counts all of them.
template <int kThreads>
__device__ __forceinline__ bool all_agree(bool ok) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.and.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)ok), "n"(kThreads)
      : "memory");
  return r != 0;
}
template <int kThreads>
__device__ __forceinline__ void sync_group() { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); }

__device__ __forceinline__ float silu_times(float g, float u) { return g / (1.0f + __expf(-g)) * u; }

// h enters W2's product as the sum of two bf16 numbers, 16 significant bits together: rounded to one, outputs were 1.35 to 1.6
// times as far from the values in 64 bits as their own rounding makes them.  The tensor cores take W2 and h in one type, so the
// second number is a second product with the same weights.  The first is the next bf16 number towards zero that is not h
// itself: the second then has h's sign and is not zero, so that an infinite weight still gives an infinite output (and an
// infinite h: the largest finite number and infinity).
__device__ __forceinline__ void split_h(float h, uint16_t &first, uint16_t &second) {
  const uint32_t bits = h != 0.f ? (__float_as_uint(h) - 1) & 0xFFFF0000u : 0u;
  first = (uint16_t)(bits >> 16);
  second = __bfloat16_as_ushort(__float2bfloat16_rn(h - __uint_as_float(bits)));
}

// Expert e's tensor j in its own map of the table.  Which of those a call needs is known only once its ids are there, so
// all are asked into the second-level cache at the start: a map that the copy engine has to fetch from memory holds it up
// for more than 2 us.
__device__ __forceinline__ const uint8_t *wide_map(const uint8_t *table, uint32_t e, uint32_t j) {
  return table + (size_t)(3 * e + j) * ZIPMOE_RESIDENT_ENTRY_BYTES;
}
__device__ __forceinline__ const uint8_t *sliced_map(const uint8_t *table, uint32_t e, uint32_t j) { return wide_map(table, e, j) + kSlicedMap; }
__device__ __forceinline__ void prefetch_table(const uint8_t *table, uint32_t E, uint32_t thread, uint32_t threads) {
  for (uint32_t i = thread; i < 3 * E * (ZIPMOE_RESIDENT_ENTRY_BYTES / 128); i += threads)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(table + (size_t)i * 128));
}

// A place in a ring of stages and how often the ring has gone round.
struct RingAt {
  uint32_t st = 0, round = 0;
  __device__ __forceinline__ void next(uint32_t n) {
    if (++st == n) {
      st = 0;
      ++round;
    }
  }
};

}  // namespace zipmoe_dev

namespace zipmoe_host {

// One checked call of zipmoe_expert_ffn for few tokens.
struct ResidentCall {
  const uint16_t *tokens;
  const int32_t *ids;
  const float *weights;
  const uint8_t *table;
  const uint8_t *even_maps;   // host: the three sliced maps and the three of the rests, or null
  uint16_t *out;
  zipmoe_dev::ResidentSync *sync;
  uint8_t *h;
  uint32_t *status;
  uint64_t limit_ns;
  uint32_t T, k, E, H, I, grid, extra_tx;
  int device;
};
zipmoe_status launch_resident_few(const ResidentCall &c, cudaStream_t stream);

}  // namespace zipmoe_host
