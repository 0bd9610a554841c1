// The routed SwiGLU experts of a few tokens on recovered bf16 weights (pool F of the planner): the counterpart of
// the fused decode + FFN for experts that need no decoding.
//     g = W1 x,  u = W3 x,  h = SiLU(g) * u,  y = W2 h,  out[t] = bf16(sum_j w[t, j] * y)
//
// Bound: the active experts' weights, 6 * hidden * inter bytes each, read once.  At up to 256 tokens the products
// are a fraction of what the tensor cores do in that time, so everything here serves one aim: that the weight stream
// never pauses.  ONE persistent kernel, one block per SM, does the whole call:
//   * A step is 32 KB of weights: 128 rows x 64 columns of W1 and of W3 (gate/up), or 256 rows x 64 columns of W2
//     (down), with the tokens' 64 columns.  A job is all steps of one expert and row block.  The steps of all jobs
//     of a phase form one sequence, cut into equal shares, so every SM streams the same number of bytes whatever the
//     experts and their sizes (steps of experts with very many tokens weigh more).
//   * Phases: gate/up of the first half of the active experts, gate/up of the second half, down of the first, down of
//     the second.  What the third needs was stored before the second began, so nobody waits between them.  Short calls
//     take all experts as one group: fewer jobs are cut.
//   * One thread feeds weights into a ring of shared-memory stages (TMA, 128-byte swizzle) and runs ahead as far as the
//     ring allows, across jobs and phases.
//   * Another warp adds the activations of every step, 64 columns of the expert's own tokens: for gate/up gathered from
//     the token matrix four rows at a time (few tokens), or, once all blocks have packed the tokens in the order the
//     tensor core wants them, one bulk copy; for down the tokens' h rows, which gate/up stores in that order, as the sum of two
//     bf16 numbers: up to 128 tokens both are rows of one operand, whose sums are added when they are read back; more are two
//     stages of activations and two rounds of MMAs for a stage of weights.
//   * One thread issues the MMAs: weights are the M = 128 operand, the expert's tokens the N operand, two accumulators
//     (g and u of the same rows, or two row blocks of y) in tensor memory, double-buffered where no operand of the phase is
//     wider than 128.
//   * Every block works out the same routing lists for itself, and sizes its rings by the most tokens that an expert
//     of this call has: few tokens, more stages.
//   * Eight warps read the accumulators back.  A job inside one share goes straight on.  Of a job that is cut, each
//     block stores its partial sums; for gate/up the block that is done last adds them in share order and goes on, for
//     down the combination of the experts adds them.  No atomics on values: the same bits whatever the timing.
// Blocks wait for one another (tokens packed, h stored, y stored), hence the cooperative launch.
// 64 tokens, 8 experts of 4096 x 14336 (2.8 GB): 427 us, 6.6 TB/s (as fast as a plain copy); 256 tokens: 515 us (85 %); 37
// tokens, 55 experts of 2048 x 1416 (957 MB): 165 us, 5.8 TB/s; 12 tokens, 8 of 2048 x 1408 (138 MB): 44 us, 3.1 TB/s.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include "zipmoe.h"
#include "resident.cuh"

namespace zipmoe_dev {

constexpr uint32_t kResReaders = 8;                         // warps that read accumulators back: two per 32 lanes of tensor memory
constexpr uint32_t kResThreads = 128 + 32 * kResReaders;
constexpr uint32_t kResStageA = 32768;                      // weights of a step
constexpr uint32_t kResInFlight = 4;                        // steps asked for and not there yet (2: 456 us, 3: 429, 4: 430 for 64
                                                            // tokens through 8 large experts); more only delays everybody else
constexpr uint32_t kResFewT = 8;   // up to this many tokens the kernel that gives every block whole rows may run instead
constexpr uint32_t kResGatherRows = 16;   // a gather of four rows takes the copy engine about 130 ns: up to this many tokens
                                          // per expert they are gathered in every step, beyond it packed once

// Bytes of weights from which on the experts are taken in two groups.  One group waits between gate/up and down, two cut
// more jobs.  One against two: 16 experts of 1024 x 512, 32 tokens (50 MB) 37 against 49 us; 8 of 2048 x 1408, 12 tokens
// (138 MB) 45 against 51; 24 of them, 12 tokens (415 MB) 79 against 80; 40 of 2048 x 1000, 16 tokens (490 MB) 93 against 92; 60
// of 2048 x 1408, 32 tokens (1.04 GB) 171 against 168.  Where experts have many tokens a cut costs more: 8 of 4096 x 3584, 256
// tokens (705 MB) 177 against 191; 60 of 2048 x 1408, 256 tokens 231 against 219.
constexpr uint64_t kResTwoGroups = 450000000, kResTwoGroupsMany = 1000000000;

struct ResidentArgs {
  const uint16_t *tokens;
  const int32_t *ids;
  const float *weights;
  const uint8_t *table;
  uint16_t *out;
  ResidentSync *sync;
  uint8_t *x;               // the experts' tokens in the same order as h, [hidden / 64] columns (where tokens are packed)
  uint8_t *h;               // per active expert: [inter / 64][2][rows padded to 8][64] bf16, swizzled as the operand wants it:
                            // the two numbers that h is the sum of
  float *part;              // [group][block][2][2][T][128]: partial sums of a share's two cut jobs (0: begun by others, 1: begun here);
                            // gate/up's have been read when down begins, and down's are stored over them
  float *y;                 // [choices][H]: jobs that lie inside one share
  uint32_t *status;
  uint64_t limit_ns, part_phase;   // part_phase: floats of a group's partial sums
  uint32_t T, k, E, H, I, even, ring_bytes, tmem_cols, extra_tx;
};

// Phases 0, 1: gate/up of the two groups of experts; 2, 3: down.  Jobs of KS steps, RB row blocks per active expert.
// The steps (units) are shared out among P blocks by weight: a unit at position p of W belongs to block floor(p * P / W), so
// block c begins with the first unit at or behind c * W / P.  A step costs what its bytes take: 32 KB from memory at the
// SM's share of its bandwidth, or, with many tokens, 32 KB + 128 bytes per token (twice that in down) into shared memory at 56
// GB/s - the same up to 72 tokens (36).  Weights are in KB of the latter, and all 1 where no expert has more tokens.
struct Phase {
  uint32_t KS, RB, U, P, a0;   // a0: the group's first active expert
  uint32_t W, each, left;      // each, left: W / P, W % P   (W < 2^31: at most 2^17 units per expert, weights of 11008 in all)
  const uint16_t *weight;      // sums of the active experts' weights before each of them; null: all 1
  __device__ __forceinline__ void share(uint32_t total) {
    W = total;
    each = P ? W / P : 0;
    left = P ? W - each * P : 0;
  }
  __device__ __forceinline__ uint32_t position(uint32_t u) const {
    if (!weight) return u;
    const uint32_t per = KS * RB, ja = u / per, a = a0 + ja;
    return per * (weight[a] - weight[a0]) + (u - ja * per) * (weight[a + 1] - weight[a]);
  }
  __device__ __forceinline__ uint32_t begin_position(uint32_t c) const { return c * each + (c * left + P - 1) / P; }   // ceil(c * W / P)
  __device__ __forceinline__ uint32_t owner(uint32_t u) const {   // the last block that begins at or before the unit
    const uint32_t pos = position(u);
    uint32_t c = min(P - 1, (uint32_t)((float)pos * ((float)P / (float)W)));
    while (begin_position(c) > pos) --c;
    while (c + 1 < P && begin_position(c + 1) <= pos) ++c;
    return c;
  }
  // first unit of block c; P gives the end
  __device__ __forceinline__ uint32_t begin(uint32_t c) const {
    const uint32_t x = begin_position(c);
    if (!weight) return x;
    const uint32_t per = KS * RB;
    uint32_t lo = 0, hi = U / per;   // the last expert whose units begin at or before x
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (per * (weight[a0 + mid] - weight[a0]) <= x) lo = mid;
      else hi = mid;
    }
    const uint32_t w = weight[a0 + lo + 1] - weight[a0 + lo];
    return lo * per + (x - per * (weight[a0 + lo] - weight[a0]) + w - 1) / w;
  }
};
__device__ __forceinline__ uint32_t gate_up_weight(uint32_t tokens) { return max(41u, 32 + (tokens + 7) / 8); }
__device__ __forceinline__ uint32_t down_weight(uint32_t tokens) { return max(41u, 32 + (tokens + 3) / 4); }
// Up to this many tokens the two numbers of their h are rows of one operand (256 at most).
constexpr uint32_t kResOneOperand = 128;
__host__ __device__ inline uint32_t down_columns(uint32_t tokens) {
  const uint32_t rows = (tokens + 7) & ~7u;
  return rows <= kResOneOperand ? 2 * rows : (tokens + 15) & ~15u;
}
constexpr uint32_t kResEvenTokens = 72, kResEvenTokensDown = 36;   // up to here all steps weigh the same
struct Piece {
  uint32_t job, a, rb, s0, n;   // steps s0 .. s0 + n of one job: active expert a, row block rb
};
__device__ __forceinline__ bool next_piece(const Phase &p, uint32_t &u, uint32_t end, Piece &q) {
  if (u >= end) return false;
  q.job = u / p.KS;
  const uint32_t ja = q.job / p.RB;
  q.a = p.a0 + ja;
  q.rb = q.job - ja * p.RB;
  q.s0 = u - q.job * p.KS;
  q.n = min(p.KS - q.s0, end - u);
  u += q.n;
  return true;
}

// shared memory after the ring: [token masks of the experts][active experts][expert -> active][sums of weights: gate/up, down][place of
// every choice among its expert's tokens][tokens of the active experts, padded to 8 each][barriers and words]
__host__ __device__ inline uint32_t resident_rows(uint32_t E, uint32_t choices) { return choices + 7 * (E < choices ? E : choices); }
__host__ __device__ inline uint32_t resident_control_bytes(uint32_t E, uint32_t T, uint32_t k) {
  return pad16(E * ((T + 31) / 32) * 4) + E * (uint32_t)sizeof(Active) + pad16(E * 2) + 2 * pad16((E + 1) * 2) +
         pad16(T * k * 2) + pad16(resident_rows(E, T * k) * 2) + (4 * kResMaxStages + 4) * 8 + 32;
}

// the choice's place among its expert's tokens (in token order; a token that lists the expert twice has one place)
__device__ __forceinline__ void place_choice(uint32_t at, int32_t e, const ResidentArgs &a, uint32_t W, const uint32_t *mask,
                                             const Active *act, const uint16_t *active_of, uint16_t *place, uint16_t *token) {
  const uint32_t t = at / a.k;
  uint32_t before = __popc(mask[(uint32_t)e * W + (t >> 5)] & ((1u << (t & 31)) - 1));
  for (uint32_t w = 0; w < (t >> 5); ++w) before += __popc(mask[(uint32_t)e * W + w]);
  place[at] = (uint16_t)before;
  token[act[active_of[e]].h_row + before] = (uint16_t)t;
}

// The accumulators in turn, as the thread that fills them and the warps that read them both count them: two of D columns a
// buffer, one or two buffers.
struct AccRing {
  uint32_t D, bufs, b = 0, uses0 = 0, uses1 = 0;
  __device__ __forceinline__ void start(uint32_t columns) {
    D = columns;
    bufs = D <= 128 ? 2 : 1;
    b = 0;
  }
  __device__ __forceinline__ uint32_t uses() const { return b ? uses1 : uses0; }   // of the present buffer so far
  __device__ __forceinline__ void next() {
    if (b) ++uses1;
    else ++uses0;
    if (bufs == 2) b ^= 1;
  }
};

__global__ void __launch_bounds__(kResThreads, 1) resident_ffn_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ EvenMaps even,
                                                                      const ResidentArgs a) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x, G = gridDim.x;
  const uint32_t W = (a.T + 31) / 32, choices = a.T * a.k, n_rows_max = resident_rows(a.E, choices);
  wait_predecessor();
  // every thread's ids (up to 2048 choices), asked for before anything else
  constexpr uint32_t kIds = (256 * 8 + kResThreads - 1) / kResThreads;
  int32_t my_id[kIds];
#pragma unroll
  for (uint32_t i = 0; i < kIds; ++i) my_id[i] = tid + i * kResThreads < choices ? __ldg(a.ids + tid + i * kResThreads) : -1;
  const uint32_t magic = __ldcg(&a.sync->magic);
  if (!a.even) prefetch_table(a.table, a.E, cta * kResThreads + tid, G * kResThreads);
  else if (tid < 3) prefetch_map(&even.w[tid]);

  uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t *ctl = ring + a.ring_bytes;
  uint32_t *mask = reinterpret_cast<uint32_t *>(ctl);
  ctl += pad16(a.E * W * 4);
  Active *act = reinterpret_cast<Active *>(ctl);
  ctl += a.E * sizeof(Active);
  uint16_t *active_of = reinterpret_cast<uint16_t *>(ctl);
  ctl += pad16(a.E * 2);
  uint16_t *weight_gu = reinterpret_cast<uint16_t *>(ctl);
  ctl += pad16((a.E + 1) * 2);
  uint16_t *weight_dn = reinterpret_cast<uint16_t *>(ctl);
  ctl += pad16((a.E + 1) * 2);
  uint16_t *place = reinterpret_cast<uint16_t *>(ctl);
  ctl += pad16(choices * 2);
  uint16_t *token = reinterpret_cast<uint16_t *>(ctl);
  ctl += pad16(n_rows_max * 2);
  constexpr uint32_t kBars = 4 * kResMaxStages + 4;
  uint64_t *bars = reinterpret_cast<uint64_t *>(ctl);
  uint32_t *words = reinterpret_cast<uint32_t *>(bars + kBars);   // tmem, dead, active, last, most, two for the readers, widest
  volatile uint32_t *dead = words + 1;
  // barriers: weights there / used, activations there / used, accumulators there / read
  const uint32_t w_full = smem_addr(bars), w_empty = w_full + 8 * kResMaxStages, x_full = w_empty + 8 * kResMaxStages,
                 x_empty = x_full + 8 * kResMaxStages, acc_full = x_empty + 8 * kResMaxStages, acc_empty = acc_full + 16;
  const WaitLimit lim = {dead, a.status, a.limit_ns};

  for (uint32_t i = tid; i < a.E * W; i += kResThreads) mask[i] = 0;
  for (uint32_t i = tid; i < n_rows_max; i += kResThreads) token[i] = 0;   // (the rows that fill up to 8 are token 0's)
  if (warp == 3) {
    for (uint32_t b = lane; b < kBars; b += 32) mbar_init(w_full + 8 * b, b >= kBars - 2 ? kResReaders : 1);
    if (lane == 0) {
      *dead = 0;
      prefetch_map(&x_map);
    }
    fence_barrier_init();
  }
  if (warp == 2) tmem_alloc(smem_addr(words), a.tmem_cols);
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  let_successor();
  const uint32_t tmem = words[0];

  // ---- which tokens every expert has: the same in every block ----
#pragma unroll
  for (uint32_t i = 0; i < kIds; ++i) {
    const uint32_t at = tid + i * kResThreads, t = at / a.k;
    if (at >= choices) break;
    if (my_id[i] >= 0 && my_id[i] < (int32_t)a.E) atomicOr(&mask[(uint32_t)my_id[i] * W + (t >> 5)], 1u << (t & 31));
    else if (my_id[i] >= 0) report(a.status, kStatusBadDescriptor);
  }
  __syncthreads();
  if (warp == 0) {   // experts per * lane .. per * lane + per - 1
    const uint32_t per = (a.E + 31) / 32;
    uint32_t cnt[8], n_act = 0, sums = 0, most = 0, widest = 16, heavy = 0;   // sums: padded rows << 16 | choices; heavy: weights
    auto weights_of = [](uint32_t tokens) { return tokens ? gate_up_weight(tokens) | down_weight(tokens) << 16 : 0u; };
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      const uint32_t e = per * lane + i;
      cnt[i] = 0;
      if (i < per && e < a.E)
        for (uint32_t w = 0; w < W; ++w) cnt[i] += __popc(mask[e * W + w]);
      n_act += cnt[i] ? 1 : 0;
      heavy += weights_of(cnt[i]);
      sums += ((cnt[i] + 7) & ~7u) << 16 | cnt[i];
      most = max(most, cnt[i]);
      widest = max(widest, down_columns(cnt[i]));
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    widest = __reduce_max_sync(0xFFFFFFFFu, widest);
    uint32_t at = n_act, sum = sums, before = heavy;   // inclusive sums over the lanes
#pragma unroll
    for (uint32_t d = 1; d < 32; d <<= 1) {
      const uint32_t p = __shfl_up_sync(0xFFFFFFFFu, at, d), q = __shfl_up_sync(0xFFFFFFFFu, sum, d), r = __shfl_up_sync(0xFFFFFFFFu, before, d);
      if (lane >= d) {
        at += p;
        sum += q;
        before += r;
      }
    }
    if (lane == 31) {
      words[2] = at;
      words[4] = most;
      words[7] = widest;
      weight_gu[at] = (uint16_t)before;
      weight_dn[at] = (uint16_t)(before >> 16);
    }
    at -= n_act;
    sum -= sums;
    before -= heavy;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      if (cnt[i]) {
        const uint32_t e = per * lane + i;
        act[at] = Active{e, cnt[i], sum >> 16, sum & 0xFFFFu};
        active_of[e] = (uint16_t)at;
        weight_gu[at] = (uint16_t)before;
        weight_dn[at] = (uint16_t)(before >> 16);
        ++at;
        before += weights_of(cnt[i]);
        sum += ((cnt[i] + 7) & ~7u) << 16 | cnt[i];
      }
    }
  }
  __syncthreads();
  const bool prepared = magic == kResMagic;
  const uint32_t n_active = prepared ? words[2] : 0;
  const bool packed = words[4] > kResGatherRows && n_active > 0;
  const uint32_t N_gu = max(16u, (words[4] + 15) & ~15u), N_dn = words[7];   // the widest operands of this call (N_gu <= N_dn)
  const uint32_t x_stage = N_dn * 128;
  // as many stages of weights as leave two for activations (as many of either kind as fit instead: 256 tokens, 60 experts of
  // 2048 x 1408 238 us, so 234; 128 tokens, 8 of 4096 x 14336 468, so 462; the widest operands of 8 of 4096 x 14336 532, so 534)
  const uint32_t n_w = min(kResMaxStages, (a.ring_bytes - 2 * x_stage) / kResStageA);
  const uint32_t n_x = min(kResMaxStages, (a.ring_bytes - n_w * kResStageA) / x_stage);
  const uint32_t w_ring = smem_addr(ring), x_ring = w_ring + n_w * kResStageA;
  Phase ph[4];
  const bool two_groups = (uint64_t)n_active * a.H * a.I * 6 >= (words[4] > kResEvenTokens ? kResTwoGroupsMany : kResTwoGroups);
  const uint32_t n_first = two_groups ? (n_active + 1) / 2 : n_active;
#pragma unroll
  for (uint32_t p = 0; p < 4; ++p) {
    ph[p].KS = p < 2 ? (a.H + 63) / 64 : (a.I + 63) / 64;
    ph[p].RB = p < 2 ? (a.I + 127) / 128 : (a.H + 255) / 256;
    ph[p].a0 = p & 1 ? n_first : 0;
    ph[p].U = (p & 1 ? n_active - n_first : n_first) * ph[p].RB * ph[p].KS;
    ph[p].P = min(G, ph[p].U);
    ph[p].weight = nullptr;
    ph[p].share(ph[p].U);
    const uint16_t *weight = p < 2 ? weight_gu : weight_dn;
    if (words[4] > (p < 2 ? kResEvenTokens : kResEvenTokensDown) && ph[p].U > 0) {
      const uint32_t total = ph[p].KS * ph[p].RB * (weight[p & 1 ? n_active : n_first] - weight[ph[p].a0]);
      if (total >= (p < 2 ? gate_up_weight(words[4]) : down_weight(words[4])) * ph[p].P) {   // (every block gets a unit)
        ph[p].weight = weight;
        ph[p].share(total);
      }
    }
  }
  // this block's share of a phase
  auto first = [&](const Phase &f) { return cta < f.P ? f.begin(cta) : 0u; };
  auto last = [&](const Phase &f) { return cta < f.P ? f.begin(cta + 1) : 0u; };

  if (warp == 0) {
    // ---- weights ----
    // the tensor maps of the share's experts, eight lanes for each phase: every map is made visible to the copies once
    if (!a.even) {
      const uint32_t p = lane >> 3;
      const Phase f = p == 0 ? ph[0] : p == 1 ? ph[1] : p == 2 ? ph[2] : ph[3];
      const uint32_t u = first(f), end = last(f), per = f.KS * f.RB, kinds = p < 2 ? 2 : 1;
      const uint32_t maps = u < end ? ((end - 1) / per - u / per + 1) * kinds : 0;
      for (uint32_t r = lane & 7; r < maps; r += 8) {
        const uint8_t *m = wide_map(a.table, act[f.a0 + u / per + r / kinds].e, p < 2 ? (r & 1) : 2);
        acquire_map(m);
        prefetch_map(m);
      }
    }
    __syncwarp();
    if (lane == 0) {
      const uint64_t policy = policy_evict_first();
      const uint32_t in_flight = min(kResInFlight, n_w);
      RingAt at, behind;   // behind: the step in_flight before
      uint32_t issued = 0;
      bool ok = true;
#pragma unroll 1
      for (uint32_t p = 0; p < 4 && ok; ++p) {
        const Phase f = p == 0 ? ph[0] : p == 1 ? ph[1] : p == 2 ? ph[2] : ph[3];
        uint32_t u = first(f);
        const uint32_t end = last(f);
        Piece q;
        while (ok && next_piece(f, u, end, q)) {
          const uint32_t e = act[q.a].e;
          const int32_t z = a.even ? (int32_t)e : 0;
          const void *m0 = wide_map(a.table, e, p < 2 ? 0 : 2), *m1 = p < 2 ? wide_map(a.table, e, 1) : m0;
          if (a.even) {
            m0 = &even.w[p < 2 ? 0 : 2];
            m1 = &even.w[p < 2 ? 1 : 2];
          }
          const int32_t y0 = (int32_t)(q.rb * (p < 2 ? 128 : 256)), y1 = p < 2 ? y0 : y0 + 128;
          for (uint32_t s = q.s0; s < q.s0 + q.n; ++s) {
            if (issued++ >= in_flight) {
              ok = wait_bar(w_full + 8 * behind.st, behind.round & 1, lim);
              behind.next(n_w);
            }
            if (!ok || (at.round > 0 && !wait_bar(w_empty + 8 * at.st, (at.round - 1) & 1, lim))) {
              ok = false;
              break;
            }
            const uint32_t dst = w_ring + at.st * kResStageA, bar = w_full + 8 * at.st;
            mbar_expect_tx(bar, kResStageA + a.extra_tx);
            tma_load_3d(dst, m0, (int32_t)(s * 64), y0, z, bar, policy);
            tma_load_3d(dst + 16384, m1, (int32_t)(s * 64), y1, z, bar, policy);
            at.next(n_w);
          }
        }
      }
    }
  } else {
    // ---- where every choice stands among its expert's tokens (the weights are on their way already) ----
#pragma unroll
    for (uint32_t i = 0; i < kIds; ++i) {
      // (warp 0's own ids are looked up again by others: it does not stop for this)
      const uint32_t at = tid + i * kResThreads;
      if (at < choices && my_id[i] >= 0 && my_id[i] < (int32_t)a.E) place_choice(at, my_id[i], a, W, mask, act, active_of, place, token);
    }
    if (warp == 1) {
      for (uint32_t i = 0; i < kIds; ++i) {
        const uint32_t at = lane + i * kResThreads;
        const int32_t e = at < choices ? __ldg(a.ids + at) : -1;
        if (e >= 0 && e < (int32_t)a.E) place_choice(at, e, a, W, mask, act, active_of, place, token);
      }
    }
    asm volatile("bar.sync 2, %0;" ::"n"(kResThreads - 32) : "memory");
  }

  if (warp == 1 && lane < kResGatherRows / 4) {
    // ---- activations; where tokens are not packed, lane r gathers rows 4r .. 4r + 3 of the expert's ----
    constexpr uint32_t kLanes = (1u << (kResGatherRows / 4)) - 1;
    const uint64_t policy = policy_evict_last();
    RingAt at;
    bool ok = true;
#pragma unroll 1
    for (uint32_t p = 0; p < 4 && ok; ++p) {
      const Phase f = p == 0 ? ph[0] : p == 1 ? ph[1] : p == 2 ? ph[2] : ph[3];
      uint32_t u = first(f);
      const uint32_t end = last(f);
      if (u < end && (p >= 2 || packed)) {
        ok = __all_sync(kLanes, p < 2 ? wait_count(&a.sync->x_done, G, lim) : wait_count(&a.sync->h_done[p - 2], p == 2 ? ph[0].P : ph[1].P, lim));
        fence_async_all();       // what other blocks stored is now read by the copy engine
      }
      Piece q;
      while (ok && next_piece(f, u, end, q)) {
        const uint32_t rows = (act[q.a].n + 7) & ~7u, first_row = act[q.a].h_row;
        const uint8_t *src = p < 2 ? a.x + (size_t)first_row * f.KS * 128 : a.h + (size_t)first_row * f.KS * 256;
        int32_t tok[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) tok[i] = 4 * lane < rows ? token[first_row + 4 * lane + i] : 0;
        // a stage per step, or two, one for each number of h
        const uint32_t per_step = p >= 2 && rows > kResOneOperand ? 2 : 1, bytes = p >= 2 && per_step == 1 ? rows * 256 : rows * 128;
        for (uint32_t s = q.s0 * per_step; s < (q.s0 + q.n) * per_step; ++s) {
          ok = __all_sync(kLanes, at.round == 0 || wait_bar(x_empty + 8 * at.st, (at.round - 1) & 1, lim));
          if (!ok) break;
          const uint32_t dst = x_ring + at.st * x_stage, bar = x_full + 8 * at.st;
          if (lane == 0) mbar_expect_tx(bar, bytes);
          __syncwarp(kLanes);
          if (p < 2 && !packed) {
            if (4 * lane < rows)
              tma_gather4(dst + lane * 512, &x_map, (int32_t)(s * 64), tok[0], tok[1], tok[2], tok[3], bar, policy);
          } else if (lane == 0) {
            bulk_load(dst, src + (size_t)s * bytes, bytes, bar, policy);
          }
          at.next(n_x);
        }
      }
    }
  } else if (warp == 2 && lane == 0) {
    // ---- MMAs ----
    RingAt wa, xa;
    AccRing acc;
    bool ok = true;
#pragma unroll 1
    for (uint32_t p = 0; p < 4 && ok; ++p) {
      const Phase f = p == 0 ? ph[0] : p == 1 ? ph[1] : p == 2 ? ph[2] : ph[3];
      if (p == 0) acc.start(N_gu);
      if (p == 2) {   // other columns from here on: whatever was accumulated has to have been read
        ok = (acc.uses0 == 0 || wait_bar(acc_empty, (acc.uses0 - 1) & 1, lim)) &&
             (acc.uses1 == 0 || wait_bar(acc_empty + 8, (acc.uses1 - 1) & 1, lim));
        acc.start(N_dn);
      }
      uint32_t u = first(f);
      const uint32_t end = last(f);
      Piece q;
      while (ok && next_piece(f, u, end, q)) {
        const uint32_t b = acc.b, use = acc.uses();
        if (use > 0 && !wait_bar(acc_empty + 8 * b, (use - 1) & 1, lim)) {
          ok = false;
          break;
        }
        tc_after_sync();
        // columns: the expert's tokens (the rows after them hold what was there before, and give columns that nobody reads)
        const uint32_t n = act[q.a].n, parts = p >= 2 && n > kResOneOperand ? 2 : 1;
        const uint32_t idesc = bf16_idesc(p < 2 ? (n + 15) & ~15u : down_columns(n));
        const uint32_t d0 = tmem + b * 2 * acc.D, d1 = d0 + acc.D;
        for (uint32_t s = 0; s < q.n; ++s) {
          ok = wait_bar(w_full + 8 * wa.st, wa.round & 1, lim);
          const uint32_t at = w_ring + wa.st * kResStageA;
          const uint64_t a0 = swizzled_desc(at), a1 = swizzled_desc(at + 16384);
          for (uint32_t part = 0; ok && part < parts; ++part) {
            ok = wait_bar(x_full + 8 * xa.st, xa.round & 1, lim);
            if (!ok) break;
            tc_after_sync();
            const uint64_t bd = swizzled_desc(x_ring + xa.st * x_stage);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
              tc_mma(d0, a0 + 2 * j, bd + 2 * j, idesc, s > 0 || part > 0 || j > 0);
              tc_mma(d1, a1 + 2 * j, bd + 2 * j, idesc, s > 0 || part > 0 || j > 0);
            }
            tc_commit(x_empty + 8 * xa.st);
            xa.next(n_x);
          }
          if (!ok) break;
          tc_commit(w_empty + 8 * wa.st);
          wa.next(n_w);
        }
        if (ok) tc_commit(acc_full + 8 * b);
        acc.next();
      }
    }
  } else if (warp >= 4) {
    // ---- accumulators back; a thread has one row of the job's 128 (twice), and every second group of 8 tokens ----
    const uint32_t w = warp & 3, half = (warp - 4) >> 2, row = 32 * w + lane, rtid = tid - 128;
    AccRing acc;
    uint32_t piece = 0;
    bool ok = true;
    if (packed) {
      // a warp per choice: the token's row, 16 bytes per lane at a time, to where the tensor core's operand has them
      const uint32_t chunks = ph[0].KS * 8;
      for (uint32_t i = cta * kResReaders + (warp - 4); i < choices; i += G * kResReaders) {
        const int32_t e = __ldg(a.ids + i);
        if (e < 0 || e >= (int32_t)a.E) continue;
        const Active ex = act[active_of[e]];
        const uint32_t r = place[i], rows = (ex.n + 7) & ~7u;
        const uint16_t *src = a.tokens + (size_t)(i / a.k) * a.H;
        uint8_t *dst = a.x + ((size_t)ex.h_row * ph[0].KS + r) * 128;
        for (uint32_t c0 = lane; c0 < chunks; c0 += 256) {
          uint4 x[8];
#pragma unroll
          for (uint32_t v = 0; v < 8; ++v) {
            const uint32_t c = c0 + 32 * v;
            x[v] = c * 8 < a.H ? __ldg(reinterpret_cast<const uint4 *>(src + c * 8)) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
          for (uint32_t v = 0; v < 8; ++v) {
            const uint32_t c = c0 + 32 * v;
            if (c < chunks) *reinterpret_cast<uint4 *>(dst + (size_t)(c >> 3) * rows * 128 + (((c & 7) ^ (r & 7)) << 4)) = x[v];
          }
        }
      }
      __threadfence();
      fence_async_all();
      sync_group<32 * kResReaders>();
      if (rtid == 0) add_release(&a.sync->x_done, 1u);
    }
#pragma unroll 1
    for (uint32_t p = 0; p < 4 && ok; ++p) {
      const Phase f = p == 0 ? ph[0] : p == 1 ? ph[1] : p == 2 ? ph[2] : ph[3];
      uint32_t u = first(f);
      const uint32_t end = last(f);
      if (p == 0 || p == 2) acc.start(p == 0 ? N_gu : N_dn);
      float *part = a.part + (p & 1) * a.part_phase;
      Piece q;
      while (ok && next_piece(f, u, end, q)) {
        const uint32_t b = acc.b, use = acc.uses();
        acc.next();
        ++piece;
        const Active ex = act[q.a];
        const bool whole = q.n == f.KS;
        float *mine = part + ((size_t)cta * 2 + (q.s0 > 0 ? 0 : 1)) * (2 * a.T * 128) + row;
        // a finished pair of sums of the expert's i-th token
        const uint32_t rows = (ex.n + 7) & ~7u, ir = q.rb * 128 + row;
        uint8_t *h = a.h + ((size_t)ex.h_row * ph[2].KS + (size_t)(ir >> 6) * rows) * 256 + (ir & 7) * 2;
        const uint32_t chunk = (ir & 63) >> 3;
        auto finish = [&](uint32_t i, float v0, float v1) {
          if (p < 2) {
            if (ir < ph[2].KS * 64) {   // (rows between inter and the next multiple of 64 are zeros: W2 has no columns there)
              uint16_t first, second;
              split_h(ir < a.I ? silu_times(v0, v1) : 0.f, first, second);
              uint8_t *to = h + i * 128 + ((chunk ^ (i & 7)) << 4);
              *reinterpret_cast<uint16_t *>(to) = first;
              *reinterpret_cast<uint16_t *>(to + rows * 128) = second;
            }
          } else {
            float *y = a.y + (size_t)(ex.slot + i) * a.H;
            const uint32_t c = q.rb * 256 + row;
            if (c < a.H) y[c] = v0;
            if (c + 128 < a.H) y[c + 128] = v1;
          }
        };
        // finished sums of gate/up, 8 tokens of which the first is a multiple of 8: neighbouring lanes, which have neighbouring rows,
        // swap every second token, so that each stores two rows of a token at once
        uint8_t *h2 = h - (ir & 1) * 2;
        auto store_h = [&](uint32_t t0, const float (&g)[8], const float (&u)[8]) {
#pragma unroll
          for (uint32_t m = 0; m < 8; m += 2) {
            if (t0 + m >= ex.n) break;
            uint32_t own[2];
#pragma unroll
            for (uint32_t e = 0; e < 2; ++e) {
              uint16_t first, second;
              split_h(ir < a.I ? silu_times(g[m + e], u[m + e]) : 0.f, first, second);
              own[e] = first | (uint32_t)second << 16;
            }
            const bool odd = lane & 1;
            const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, odd ? own[0] : own[1], 1), t = t0 + m + odd;
            const uint32_t even_row = odd ? got : own[0], odd_row = odd ? own[1] : got;
            if (t < ex.n && ir < ph[2].KS * 64) {
              uint8_t *to = h2 + t * 128 + ((chunk ^ (t & 7)) << 4);
              *reinterpret_cast<uint32_t *>(to) = __byte_perm(even_row, odd_row, 0x5410);
              *reinterpret_cast<uint32_t *>(to + rows * 128) = __byte_perm(even_row, odd_row, 0x7632);
            }
          }
        };
        auto emit = [&](uint32_t i, float v0, float v1) {
          if (whole) {
            finish(i, v0, v1);
          } else {
            mine[(size_t)i * 128] = v0;
            mine[(size_t)(a.T + i) * 128] = v1;
          }
        };
        // a gate/up job that is cut: the block that is done with its part last adds all parts, in share order.  That is
        // mostly the one that began the job, at the end of its share, and finds the others' parts there: its own never leave
        // the tensor memory.
        const bool join = !whole && p < 2;
        const uint32_t c0 = join ? f.owner(q.job * f.KS) : 0, c1 = join ? f.owner(q.job * f.KS + f.KS - 1) : 0;
        volatile uint32_t *others_there = words + 5 + (piece & 1);
        ok = wait_bar(acc_full + 8 * b, use & 1, lim);
        if (rtid == 0) *others_there = join && q.s0 == 0 && load_acquire(&a.sync->cut[p][c0]) == c1 - c0;
        ok = all_agree<32 * kResReaders>(ok);
        if (!ok) break;
        tc_after_sync();
        const uint32_t d0 = tmem + ((32 * w) << 16) + b * 2 * acc.D, d1 = d0 + acc.D;
        if (*others_there) {
          const size_t next_block = 2 * (2 * a.T * 128);
          const float *from = part + (c0 + 1) * next_block + row;
          for (uint32_t c = 8 * half; c < ex.n; c += 32) {
            float g[2][8], v[2][8];   // the next block's part: of 16 tokens at a time
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) {
              const uint32_t t = min(c + 16 * (i >> 3) + (i & 7), ex.n - 1);
              g[i >> 3][i & 7] = __ldcg(from + (size_t)t * 128);
              v[i >> 3][i & 7] = __ldcg(from + (size_t)(a.T + t) * 128);
            }
#pragma unroll
            for (uint32_t m = 0; m < 2; ++m) {
              const uint32_t t0 = c + 16 * m;
              if (t0 >= ex.n) continue;
              uint32_t v0[8], v1[8];
              tmem_load8(d0 + t0, v0);
              tmem_load8(d1 + t0, v1);
              tmem_wait();
#pragma unroll
              for (uint32_t n = 0; n < 8; ++n) {   // (from zero, as below: the same bits for either way)
                g[m][n] = 0.f + __uint_as_float(v0[n]) + g[m][n];
                v[m][n] = 0.f + __uint_as_float(v1[n]) + v[m][n];
              }
              for (uint32_t o = 1; o < c1 - c0; ++o)
#pragma unroll
                for (uint32_t n = 0; n < 8; ++n) {
                  const uint32_t t = min(t0 + n, ex.n - 1);
                  g[m][n] += __ldcg(from + o * next_block + (size_t)t * 128);
                  v[m][n] += __ldcg(from + o * next_block + (size_t)(a.T + t) * 128);
                }
              store_h(t0, g[m], v[m]);
            }
          }
          tc_before_sync();
          __syncwarp();
          if (lane == 0) arrive(acc_empty + 8 * b);
          continue;
        }
        for (uint32_t c = 8 * half; c < ex.n; c += 16) {
          uint32_t v0[8], v1[8];
          tmem_load8(d0 + c, v0);
          tmem_load8(d1 + c, v1);
          if (p >= 2 && rows <= kResOneOperand) {   // the sums over h's second number are `rows` columns further
            uint32_t w0[8], w1[8];
            tmem_load8(d0 + rows + c, w0);
            tmem_load8(d1 + rows + c, w1);
            tmem_wait();
#pragma unroll
            for (uint32_t n = 0; n < 8; ++n) {
              v0[n] = __float_as_uint(__uint_as_float(v0[n]) + __uint_as_float(w0[n]));
              v1[n] = __float_as_uint(__uint_as_float(v1[n]) + __uint_as_float(w1[n]));
            }
          } else {
            tmem_wait();
          }
          if (whole && p < 2) {
            float g[8], u[8];
#pragma unroll
            for (uint32_t n = 0; n < 8; ++n) {
              g[n] = __uint_as_float(v0[n]);
              u[n] = __uint_as_float(v1[n]);
            }
            store_h(c, g, u);
            continue;
          }
#pragma unroll
          for (uint32_t n = 0; n < 8; ++n)
            if (c + n < ex.n) emit(c + n, __uint_as_float(v0[n]), __uint_as_float(v1[n]));
        }
        tc_before_sync();
        __syncwarp();
        if (lane == 0) arrive(acc_empty + 8 * b);
        if (!join) continue;
        __threadfence();
        sync_group<32 * kResReaders>();
        if (rtid == 0) {
          words[3] = atomicAdd(&a.sync->cut[p][c0], 1u) == c1 - c0;
          __threadfence();
        }
        sync_group<32 * kResReaders>();
        if (words[3]) {
          if (ex.n <= 16) {
            for (uint32_t n0 = 4 * half; n0 < ex.n; n0 += 8) {
              float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
              for (uint32_t c = c0; c <= c1; ++c) {
                const float *from = part + ((size_t)c * 2 + (c == c0 ? 1 : 0)) * (2 * a.T * 128) + row;
#pragma unroll
                for (uint32_t n = 0; n < 4; ++n)
                  if (n0 + n < ex.n) {
                    s0[n] += __ldcg(from + (size_t)(n0 + n) * 128);
                    s1[n] += __ldcg(from + (size_t)(a.T + n0 + n) * 128);
                  }
              }
#pragma unroll
              for (uint32_t n = 0; n < 4; ++n)
                if (n0 + n < ex.n) finish(n0 + n, s0[n], s1[n]);
            }
            continue;
          }
          // many tokens: a warp per token, four rows per lane; four tokens' parts are asked for at a time (10 us less for 231
          // tokens of one expert, 3 us more for one)
          const uint32_t row4 = 4 * lane, ir4 = q.rb * 128 + row4, h_rows = ph[2].KS * 64;
          uint8_t *to = a.h + ((size_t)ex.h_row * ph[2].KS + (size_t)(ir4 >> 6) * rows) * 256 + (ir4 & 7) * 2;
          const uint32_t chunk4 = (ir4 & 63) >> 3;
          for (uint32_t n0 = warp - 4; n0 < ex.n; n0 += 4 * kResReaders) {
            float4 g[4], v[4];
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) g[n] = v[n] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (uint32_t c = c0; c <= c1; ++c) {
              const float *from = part + ((size_t)c * 2 + (c == c0 ? 1 : 0)) * (2 * a.T * 128) + row4;
              float4 x[4], y[4];
#pragma unroll
              for (uint32_t n = 0; n < 4; ++n) {
                const uint32_t i = min(n0 + n * kResReaders, ex.n - 1);
                x[n] = __ldcg(reinterpret_cast<const float4 *>(from + (size_t)i * 128));
                y[n] = __ldcg(reinterpret_cast<const float4 *>(from + (size_t)(a.T + i) * 128));
              }
#pragma unroll
              for (uint32_t n = 0; n < 4; ++n) {
                g[n] = make_float4(g[n].x + x[n].x, g[n].y + x[n].y, g[n].z + x[n].z, g[n].w + x[n].w);
                v[n] = make_float4(v[n].x + y[n].x, v[n].y + y[n].y, v[n].z + y[n].z, v[n].w + y[n].w);
              }
            }
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) {
              const uint32_t i = n0 + n * kResReaders;
              if (i >= ex.n || ir4 >= h_rows) continue;
              // (inter is a multiple of 8: four rows are all inside it or all behind it)
              ushort4 first = make_ushort4(0, 0, 0, 0), second = first;
              if (ir4 < a.I) {
                split_h(silu_times(g[n].x, v[n].x), first.x, second.x);
                split_h(silu_times(g[n].y, v[n].y), first.y, second.y);
                split_h(silu_times(g[n].z, v[n].z), first.z, second.z);
                split_h(silu_times(g[n].w, v[n].w), first.w, second.w);
              }
              uint8_t *at = to + i * 128 + ((chunk4 ^ (i & 7)) << 4);
              *reinterpret_cast<ushort4 *>(at) = first;
              *reinterpret_cast<ushort4 *>(at + rows * 128) = second;
            }
          }
        }
      }
      // everything this block stores in the phase is out: tell the others
      if (ok && cta < f.P) {
        __threadfence();
        if (p < 2) fence_async_all();
        sync_group<32 * kResReaders>();
        if (rtid == 0) add_release(p < 2 ? &a.sync->h_done[p] : &a.sync->y_done, 1u);
      }
    }
  }
  __syncwarp();
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  if (*dead)   // let the copies and MMAs that this block has under way end before its memory goes to somebody else
    for (uint32_t i = 0; i < 200; ++i) __nanosleep(1000);
  if (warp == 2) tmem_free(tmem, a.tmem_cols);
  if (tid == 0 && !*dead) wait_count(&a.sync->y_done, ph[2].P + ph[3].P, lim);
  __syncthreads();

  // ---- out[t] = sum over the token's choices ----
  const uint32_t vecs = a.H / 4, items = a.T * vecs;   // four columns of a token each
  if (!*dead && prepared && items * 8 <= 2 * G * kResThreads) {
    // few outputs: up to 8 lanes share the choices of an item (64 threads per token and all its choices in each: 5 to 10 us
    // longer for one token)
    uint32_t lanes = 8;
    while (lanes > 1 && (items * lanes > G * kResThreads || lanes >= 2 * a.k)) lanes >>= 1;
    const uint32_t per_block = kResThreads / lanes, l = tid % lanes;
    for (uint32_t it0 = cta * per_block; it0 < items; it0 += G * per_block) {
      const uint32_t it = it0 + tid / lanes;
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      const uint32_t t = it / vecs, c = (it - t * vecs) * 4;
      if (it < items) {
#pragma unroll 2
        for (uint32_t j = l; j < a.k; j += lanes) {
          const int32_t e = __ldg(a.ids + t * a.k + j);
          if (e < 0 || e >= (int32_t)a.E) continue;
          const uint32_t ai = active_of[e], i = place[t * a.k + j];
          const uint32_t p = ai < n_first ? 2 : 3;
          const Phase f = p == 2 ? ph[2] : ph[3];
          const uint32_t u0 = ((ai - f.a0) * f.RB + c / 256) * f.KS;
          const uint32_t c0 = f.owner(u0), c1 = f.owner(u0 + f.KS - 1);
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
          if (c0 == c1) {
            v = __ldcg(reinterpret_cast<const float4 *>(a.y + (size_t)(act[ai].slot + i) * a.H + c));
          } else {
            const float *from = a.part + (p & 1) * a.part_phase + (size_t)(((c >> 7) & 1) * a.T + i) * 128 + (c & 127);
            for (uint32_t b = c0; b <= c1; b += 4) {
              float4 r[4];
#pragma unroll
              for (uint32_t n = 0; n < 4; ++n)
                r[n] = b + n <= c1 ? __ldcg(reinterpret_cast<const float4 *>(from + ((size_t)(b + n) * 2 + (b + n == c0 ? 1 : 0)) * (2 * a.T * 128)))
                                   : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
              for (uint32_t n = 0; n < 4; ++n) {
                v.x += r[n].x;
                v.y += r[n].y;
                v.z += r[n].z;
                v.w += r[n].w;
              }
            }
          }
          const float wt = a.weights ? __ldg(a.weights + t * a.k + j) : 1.0f;
          s.x += wt * v.x;
          s.y += wt * v.y;
          s.z += wt * v.z;
          s.w += wt * v.w;
        }
      }
      for (uint32_t d = lanes >> 1; d > 0; d >>= 1) {
        s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, d);
        s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, d);
        s.z += __shfl_xor_sync(0xFFFFFFFFu, s.z, d);
        s.w += __shfl_xor_sync(0xFFFFFFFFu, s.w, d);
      }
      if (it < items && l == 0) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(s.x, s.y), hi = __floats2bfloat162_rn(s.z, s.w);
        *reinterpret_cast<uint2 *>(a.out + (size_t)t * a.H + c) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
      }
    }
  } else if (!*dead && prepared) {
    // many: a turn is 256 columns (a row block of down) of six tokens, or twelve with up to four choices each; 64 threads have
    // a token's columns, four each.  Which blocks have parts of an expert's job is worked out once per row block.  (As above:
    // 9 us longer for 256 tokens.)
    uint32_t *owners = reinterpret_cast<uint32_t *>(ring);   // [active experts]: first and last block (the ring is done with)
    auto combine = [&](auto most_choices) {
      constexpr uint32_t kK = decltype(most_choices)::value, kN = 8 / kK, kTokens = kResThreads / 64 * kN;
      const uint32_t RB = ph[2].RB, groups = (a.T + kTokens - 1) / kTokens, turns = RB * groups;
      uint32_t rb_now = 0xFFFFFFFFu;
      for (uint32_t turn = cta * turns / G; turn < (cta + 1) * turns / G; ++turn) {
        const uint32_t rb = turn / groups, t0 = (turn - rb * groups) * kTokens + (tid >> 6), v4 = tid & 63, c = rb * 256 + v4 * 4;
        if (rb != rb_now) {
          __syncthreads();
          for (uint32_t ai = tid; ai < n_active; ai += kResThreads) {
            const Phase f = ai < n_first ? ph[2] : ph[3];
            const uint32_t u0 = ((ai - f.a0) * RB + rb) * f.KS;
            owners[ai] = f.owner(u0) | f.owner(u0 + f.KS - 1) << 16;
          }
          __syncthreads();
          rb_now = rb;
        }
        if (c >= a.H) continue;
        // every choice's sum, or the first two parts of it, are asked for before the first is used
        const uint32_t in_part = ((v4 >> 5) * a.T) * 128 + (v4 & 31) * 4;
        const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
        const size_t next_block = 2 * (2 * a.T * 128);
        float4 y[8], z[8];
        const float *from[8];
        uint32_t more[8];
        float wt[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          const uint32_t t = t0 + i / kK * (kResThreads / 64), j = i % kK, at = t * a.k + j;
          y[i] = z[i] = zero;
          more[i] = 0;
          wt[i] = 0.f;
          if (t >= a.T || j >= a.k) continue;
          const int32_t e = __ldg(a.ids + at);
          if (e < 0 || e >= (int32_t)a.E) continue;   // (adds nothing, whatever its weight is)
          wt[i] = a.weights ? __ldg(a.weights + at) : 1.0f;
          const uint32_t ai = active_of[e], r = place[at], c0 = owners[ai] & 0xFFFFu, c1 = owners[ai] >> 16;
          if (c0 == c1) {
            y[i] = __ldcg(reinterpret_cast<const float4 *>(a.y + (size_t)(act[ai].slot + r) * a.H + c));
          } else {
            from[i] = a.part + (ai < n_first ? 0 : 1) * a.part_phase + c0 * next_block + in_part + (size_t)r * 128;
            more[i] = c1 - c0;
            y[i] = __ldcg(reinterpret_cast<const float4 *>(from[i] + next_block / 2));
            z[i] = __ldcg(reinterpret_cast<const float4 *>(from[i] + next_block));
          }
        }
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
          y[i] = make_float4(y[i].x + z[i].x, y[i].y + z[i].y, y[i].z + z[i].z, y[i].w + z[i].w);
          for (uint32_t b = 2; b <= more[i]; b += 4) {
            float4 r[4];
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n)
              r[n] = b + n <= more[i] ? __ldcg(reinterpret_cast<const float4 *>(from[i] + (b + n) * next_block)) : zero;
#pragma unroll
            for (uint32_t n = 0; n < 4; ++n) y[i] = make_float4(y[i].x + r[n].x, y[i].y + r[n].y, y[i].z + r[n].z, y[i].w + r[n].w);
          }
        }
#pragma unroll
        for (uint32_t n = 0; n < kN; ++n) {
          const uint32_t t = t0 + n * (kResThreads / 64);
          if (t >= a.T) continue;
          float4 s = zero;
#pragma unroll
          for (uint32_t i = n * kK; i < (n + 1) * kK; ++i)
            s = make_float4(s.x + wt[i] * y[i].x, s.y + wt[i] * y[i].y, s.z + wt[i] * y[i].z, s.w + wt[i] * y[i].w);
          const __nv_bfloat162 lo = __floats2bfloat162_rn(s.x, s.y), hi = __floats2bfloat162_rn(s.z, s.w);
          *reinterpret_cast<uint2 *>(a.out + (size_t)t * a.H + c) =
              make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
        }
      }
    };
    if (a.k <= 4) combine(std::integral_constant<uint32_t, 4>());
    else combine(std::integral_constant<uint32_t, 8>());
  }
  __syncthreads();
  if (tid == 0) {
    if (!prepared) report(a.status, kStatusBadDescriptor);
    if (prepared) {
      __threadfence();
      if (atomicAdd(&a.sync->exited, 1u) == G - 1) {   // the last block leaves the counters as it found them
        for (uint32_t c = 0; c < kResMaxGrid; ++c) a.sync->cut[0][c] = a.sync->cut[1][c] = 0;
        a.sync->x_done = 0;
        a.sync->h_done[0] = a.sync->h_done[1] = 0;
        a.sync->y_done = 0;
        a.sync->exited = 0;
      }
    }
  }
}

__global__ void resident_init_kernel(ResidentSync *s) {
  uint32_t *w = reinterpret_cast<uint32_t *>(s);
  for (uint32_t i = threadIdx.x; i < sizeof(ResidentSync) / 4; i += blockDim.x) w[i] = i == 0 ? kResMagic : 0u;
}

}  // namespace zipmoe_dev

namespace {

constexpr uint32_t kResidentMaxT = 256, kResidentMaxK = 8, kResidentMaxExperts = 256, kResidentMaxDim = 32768;
bool dims_ok(uint32_t E, uint32_t H, uint32_t I) {
  return E > 0 && E <= kResidentMaxExperts && H > 0 && I > 0 && H % 8 == 0 && I % 8 == 0 && H <= kResidentMaxDim &&
         I <= kResidentMaxDim;
}

bool g_resident_ready[64];

uint32_t resident_grid() { return std::min(zipmoe_host::current_sms(), zipmoe_dev::kResMaxGrid); }

struct ResidentPlan {
  uint32_t grid, tmem_cols, ring, smem;
  uint64_t part_phase, off_x, off_h, off_part, off_y, total;
};

zipmoe_status resident_plan(uint32_t T, uint32_t k, const zipmoe_resident_experts *ex, ResidentPlan *p) {
  if (T > kResidentMaxT || k == 0 || k > kResidentMaxK || !dims_ok(ex->n_experts, ex->hidden, ex->inter))
    return ZIPMOE_ERR_UNSUPPORTED;
  const uint64_t H = ex->hidden, I = ex->inter;
  p->grid = resident_grid();
  // two accumulators for both numbers of as many tokens as an expert can have, twice if they fit (the kernel goes by the
  // call's own most)
  const uint32_t N = std::max(16u, (T + 15) / 16 * 16);
  p->tmem_cols = 32;
  while (p->tmem_cols < std::min(512u, 8 * N)) p->tmem_cols <<= 1;
  const uint32_t control = zipmoe_dev::resident_control_bytes(ex->n_experts, T, k) + 1024;
  p->ring = (227u * 1024u - control) & ~15u;
  p->smem = control + p->ring;
  auto up = [](uint64_t v) { return (v + 255) / 256 * 256; };
  const uint64_t choices = (uint64_t)T * k, rows = zipmoe_dev::resident_rows(ex->n_experts, T * k);
  uint64_t at = up(sizeof(zipmoe_dev::ResidentSync));
  p->off_x = at; at = up(at + rows * ((H + 63) / 64) * 128);
  p->off_h = at; at = up(at + rows * ((I + 63) / 64) * 256);
  p->part_phase = (uint64_t)T * p->grid * 2 * 2 * 128;
  p->off_part = at; at = up(at + 2 * p->part_phase * 4);
  p->off_y = at; at = up(at + choices * H * 4);
  p->total = at;
  return ZIPMOE_OK;
}

}  // namespace

extern "C" zipmoe_status zipmoe_resident_experts_plan(const uint16_t *const *tensors, uint32_t n_experts, uint32_t hidden,
                                                      uint32_t inter, void *table, zipmoe_resident_experts *experts) {
  using zipmoe_dev::kRestMap;
  using zipmoe_dev::kSlicedMap;
  if (!dims_ok(n_experts, hidden, inter)) return ZIPMOE_ERR_UNSUPPORTED;
  if (!tensors || !table || !experts) return ZIPMOE_ERR_INVALID_ARG;
  for (uint32_t i = 0; i < 3 * n_experts; ++i)
    if (!tensors[i] || (reinterpret_cast<uintptr_t>(tensors[i]) & 15)) return ZIPMOE_ERR_INVALID_ARG;
  static_assert(sizeof(CUtensorMap) == kSlicedMap && 3 * sizeof(CUtensorMap) == ZIPMOE_RESIDENT_ENTRY_BYTES, "an entry is three tensor maps");
  const uint64_t bytes = 2ull * hidden * inter;
  uint32_t R1, S1, R2, S2;
  const uint32_t grid = resident_grid();
  zipmoe_host::resident_few_rows(hidden, inter, grid, &R1, &S1, &R2, &S2);
  // both maps of n tensors of kind j (0 w1, 1 w3, 2 w2), `distance` bytes apart
  auto describe = [&](uint8_t *to, const uint16_t *base, uint32_t j, uint64_t n, uint64_t distance) {
    const uint32_t rows = j < 2 ? inter : hidden, cols = j < 2 ? hidden : inter;
    CUtensorMap map;
    if (!zipmoe_host::make_wide_map(&map, base, rows, cols, 128, n, distance)) return false;
    std::memset(to, 0, ZIPMOE_RESIDENT_ENTRY_BYTES);
    std::memcpy(to, &map, sizeof(map));
    const uint32_t box_rows = j < 2 ? S1 : S2;
    if (cols >= 64 && !zipmoe_host::make_sliced_map(&map, base, rows, cols, box_rows, n, distance)) return false;
    std::memcpy(to + kSlicedMap, &map, sizeof(map));   // (fewer columns: nothing is loaded through it)
    if (cols % 64) {
      if (!zipmoe_host::make_wide_map(&map, base, rows, cols, box_rows, n, distance)) return false;
      std::memcpy(to + kRestMap, &map, sizeof(map));
    }
    return true;
  };
  for (uint32_t i = 0; i < 3 * n_experts; ++i)
    if (!describe(static_cast<uint8_t *>(table) + (size_t)i * ZIPMOE_RESIDENT_ENTRY_BYTES, tensors[i], i % 3, 1, bytes)) return ZIPMOE_ERR_CUDA;
  std::memset(experts, 0, sizeof(*experts));
  experts->n_experts = n_experts;
  experts->hidden = hidden;
  experts->inter = inter;
  experts->grid = grid;
  // evenly spaced experts: one map per kind of tensor serves them all (distances that a map can hold)
  uint64_t distance[3];
  bool even = true;
  for (uint32_t j = 0; j < 3; ++j) {
    const uintptr_t first = reinterpret_cast<uintptr_t>(tensors[j]);
    const uintptr_t second = n_experts > 1 ? reinterpret_cast<uintptr_t>(tensors[3 + j]) : first + bytes;
    distance[j] = second - first;
    even = even && second > first && distance[j] >= bytes && distance[j] < (1ull << 40);
    for (uint32_t e = 2; e < n_experts && even; ++e)
      even = reinterpret_cast<uintptr_t>(tensors[3 * e + j]) == first + e * distance[j];
  }
  for (uint32_t j = 0; j < 3 && even; ++j) {
    uint8_t all[ZIPMOE_RESIDENT_ENTRY_BYTES];
    if (!describe(all, tensors[j], j, n_experts, distance[j])) return ZIPMOE_ERR_CUDA;
    std::memcpy(experts->maps + 128 * j, all, 128);
    std::memcpy(experts->maps + 128 * (3 + j), all + kSlicedMap, 128);
    std::memcpy(experts->maps + 128 * (6 + j), all + kRestMap, 128);
  }
  experts->even = even;
  return ZIPMOE_OK;
}

extern "C" zipmoe_status zipmoe_expert_ffn_workspace_bytes(uint32_t T, uint32_t k, const zipmoe_resident_experts *ex,
                                                           uint64_t *workspace_bytes) {
  if (!ex || !workspace_bytes) return ZIPMOE_ERR_INVALID_ARG;
  ResidentPlan p;
  const zipmoe_status rc = resident_plan(T, k, ex, &p);
  if (rc != ZIPMOE_OK) return rc;
  *workspace_bytes = p.total;
  return ZIPMOE_OK;
}

extern "C" zipmoe_status zipmoe_expert_ffn_workspace_init(void *workspace, uint64_t workspace_bytes, zipmoe_stream stream) {
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return ZIPMOE_ERR_INVALID_ARG;
  if (workspace_bytes < sizeof(zipmoe_dev::ResidentSync)) return ZIPMOE_ERR_BUFFER_TOO_SMALL;
  zipmoe_dev::resident_init_kernel<<<1, 256, 0, reinterpret_cast<cudaStream_t>(stream)>>>(
      static_cast<zipmoe_dev::ResidentSync *>(workspace));
  return cudaGetLastError() == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}

extern "C" zipmoe_status zipmoe_stream_capture_id(zipmoe_stream stream, uint64_t *capture_id) {
  if (!capture_id) return ZIPMOE_ERR_INVALID_ARG;
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  unsigned long long id = 0;
  if (cudaStreamGetCaptureInfo(reinterpret_cast<cudaStream_t>(stream), &capture, &id) != cudaSuccess ||
      capture == cudaStreamCaptureStatusInvalidated) {
    (void)cudaGetLastError();
    return ZIPMOE_ERR_CUDA;
  }
  *capture_id = capture == cudaStreamCaptureStatusActive ? id : 0;
  return ZIPMOE_OK;
}

extern "C" zipmoe_status zipmoe_expert_ffn(const uint16_t *tokens, uint32_t T, const int32_t *topk_ids,
                                           const float *topk_weights, uint32_t k, const zipmoe_resident_experts *ex,
                                           uint16_t *out, void *workspace, uint64_t workspace_bytes,
                                           uint32_t *status_word, zipmoe_stream stream_) {
  using namespace zipmoe_dev;
  zipmoe_host::TraceRange trace("zipmoe_expert_ffn");
  if (!ex) return ZIPMOE_ERR_INVALID_ARG;
  ResidentPlan p;
  const zipmoe_status rc = resident_plan(T, k, ex, &p);
  if (rc != ZIPMOE_OK) return rc;
  if (T == 0) return ZIPMOE_OK;
  if (!tokens || !topk_ids || !out || !workspace || !ex->table || ex->even > 1) return ZIPMOE_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(workspace)) & 15) ||
      (reinterpret_cast<uintptr_t>(ex->table) & 63) ||
      ((reinterpret_cast<uintptr_t>(topk_ids) | reinterpret_cast<uintptr_t>(topk_weights) | reinterpret_cast<uintptr_t>(status_word)) & 3))
    return ZIPMOE_ERR_INVALID_ARG;
  if (workspace_bytes < p.total) return ZIPMOE_ERR_BUFFER_TOO_SMALL;
  // (other boxes than those of the plan's maps: the barriers would wait for bytes that never come)
  if (ex->grid != p.grid || ex->reserved) return ZIPMOE_ERR_INVALID_ARG;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return ZIPMOE_ERR_CUDA;
  if (!g_resident_ready[dev]) {
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return ZIPMOE_ERR_CUDA;
    if (major != 10) return ZIPMOE_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(resident_ffn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) != cudaSuccess)
      return ZIPMOE_ERR_CUDA;
    g_resident_ready[dev] = true;
  }
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  uint32_t tries = 0, extra_tx = 0;
  zipmoe_host::wait_fault_setting(&extra_tx, &tries);
  const uint64_t limit_ns = tries < zipmoe_host::kWaitTries ? 1000000ull : 1000000000ull;   // (1 ms in the tests of the limit)
  if (T <= kResFewT && zipmoe_host::whole_rows_pay(T * k, ex->n_experts, ex->hidden, ex->inter, p.grid)) {
    zipmoe_host::ResidentCall c;
    c.tokens = tokens;
    c.ids = topk_ids;
    c.weights = topk_weights;
    c.table = static_cast<const uint8_t *>(ex->table);
    c.even_maps = ex->even ? ex->maps + 3 * 128 : nullptr;
    c.out = out;
    c.sync = reinterpret_cast<ResidentSync *>(ws);
    c.h = ws + p.off_h;
    c.status = status_word;
    c.limit_ns = limit_ns;
    c.T = T;
    c.k = k;
    c.E = ex->n_experts;
    c.H = ex->hidden;
    c.I = ex->inter;
    c.grid = p.grid;
    c.extra_tx = extra_tx;
    c.device = dev;
    return zipmoe_host::launch_resident_few(c, reinterpret_cast<cudaStream_t>(stream_));
  }
  CUtensorMap x_map;
  if (!zipmoe_host::make_bf16_map(&x_map, tokens, T, ex->hidden, ex->hidden, 1, false)) return ZIPMOE_ERR_CUDA;
  ResidentArgs a;
  a.ids = topk_ids;
  a.weights = topk_weights;
  a.table = static_cast<const uint8_t *>(ex->table);
  a.even = ex->even;
  EvenMaps even = {};
  if (ex->even) std::memcpy(&even, ex->maps, sizeof(even));
  a.out = out;
  a.sync = reinterpret_cast<ResidentSync *>(ws);
  a.tokens = tokens;
  a.x = ws + p.off_x;
  a.h = ws + p.off_h;
  a.part = reinterpret_cast<float *>(ws + p.off_part);
  a.y = reinterpret_cast<float *>(ws + p.off_y);
  a.status = status_word;
  a.extra_tx = extra_tx;
  a.limit_ns = limit_ns;
  a.T = T;
  a.k = k;
  a.E = ex->n_experts;
  a.H = ex->hidden;
  a.I = ex->inter;
  a.part_phase = p.part_phase;
  a.ring_bytes = p.ring;
  a.tmem_cols = p.tmem_cols;
  cudaLaunchAttribute together;
  together.id = cudaLaunchAttributeCooperative;
  together.val.cooperative = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = reinterpret_cast<cudaStream_t>(stream_);
  cfg.attrs = &together;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(p.grid);
  cfg.blockDim = dim3(kResThreads);
  cfg.dynamicSmemBytes = p.smem;
  return cudaLaunchKernelEx(&cfg, resident_ffn_kernel, x_map, even, a) == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}
