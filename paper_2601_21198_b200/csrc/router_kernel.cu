// The router: logits = tokens x gate^T + bias, the k largest per token, and their softmax weights, in one launch.
// Bound: the tokens' bytes for a long prompt (the gate stays in the second-level cache), latency for a few tokens.
//   * A cluster of 1 to 8 blocks takes 128 tokens (the M operand of a tcgen05 MMA; N = all experts, padded to 16) and
//     splits the hidden dimension among its blocks.  Each block streams its columns of tokens and gate through a ring of
//     TMA stages and accumulates [128 x N] in tensor memory.  Rows and columns past the matrices come in as zeros, so no
//     size needs a path of its own; a single token reads one row.
//   * Every block leaves its partial logits in its shared memory; after a cluster barrier the block of rank r adds, in
//     rank order, the parts of tokens r, r + S, ... straight from its neighbours' shared memory.  (Sent there by their
//     owners instead they need a second barrier, before the rings may be written over: 2 us slower for 8192 tokens.)
//   * Eight lanes pick a token's k experts, four tokens to a warp: a logit becomes a 32-bit key that orders as the number
//     does (NaN on top), every lane holds an eighth of them, and each choice is the lanes' own best and three exchanges.
//     (A whole warp per token spends most of its instructions on two experts per lane: 450 per token, 6 of 16 us for 8192.)
// 8192 tokens, 64 experts, 2048 columns: 14.1 us, 2.6 TB/s (of which 4 us are the exchange and the choice, behind the last
// product); 777 tokens, 60 experts: 7.0 us; one token: 5.5 us.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "zipmoe.h"
#include "tensor_core.cuh"

namespace zipmoe_dev {

constexpr uint32_t kMaxExperts = 256, kMaxTopK = 8;
constexpr uint32_t kRouterRows = 128, kRouterThreads = 256, kRouterMaxStages = 8;

struct RouterArgs {
  const float *bias;
  int32_t *ids;
  float *weights, *logits;
  uint32_t *status;
  uint64_t limit_ns;
  uint32_t T, E, H, k, flags, N, stages, tmem_cols, extra_tx;
};

// A key that orders as the logit does: NaN above all, then +infinity down to -infinity; 0 for -infinity, so that it
// can also stand for "no expert".
__device__ __forceinline__ uint32_t logit_key(float l) {
  const uint32_t b = __float_as_uint(l);
  if (l != l) return 0xFFFFFFFFu;
  if (b == 0xFF800000u) return 0u;
  if (b == 0x80000000u) return 0x80000000u;                  // -0 equals +0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t key) {   // (NaN's key gives a NaN)
  return __uint_as_float((key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key);
}

// The expert of a lane's i-th value: eight lanes hold four neighbouring ones each, then the next 32.
__device__ __forceinline__ uint32_t expert_of(uint32_t q, uint32_t i) { return (i >> 2) * 32 + q * 4 + (i & 3); }

// Eight lanes (q = 0..7) pick the k largest of their token's logits (l[i] is expert_of(q, i); -infinity past the last) and
// write ids and weights, unless `there` is false.  The four groups of a warp work in step.
template <int kPer>
__device__ __forceinline__ void pick_experts(const float (&l)[kPer], uint32_t k, uint32_t flags, uint32_t q, bool there, int32_t *ids,
                                             float *weights) {
  uint32_t key[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) key[i] = logit_key(l[i]);
  int32_t my_id = -1;       // lane j keeps choice j
  uint32_t my_key = 0, top_key = 0;
#pragma unroll 1
  for (uint32_t j = 0; j < k; ++j) {
    // the lane's best, pair by pair (equal keys: the first, which is the lowest expert)
    uint32_t top_of[kPer], place[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      top_of[i] = key[i];
      place[i] = i;
    }
#pragma unroll
    for (int d = 1; d < kPer; d *= 2)
#pragma unroll
      for (int i = 0; i < kPer; i += 2 * d)
        if (top_of[i + d] > top_of[i]) {
          top_of[i] = top_of[i + d];
          place[i] = place[i + d];
        }
    uint32_t best = top_of[0];
    const uint32_t at = place[0];
    uint32_t e = expert_of(q, at);
    const uint32_t own = e;
#pragma unroll
    for (uint32_t d = 1; d < 8; d <<= 1) {
      const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, best, d), other_e = __shfl_xor_sync(0xFFFFFFFFu, e, d);
      if (other > best || (other == best && other_e < e)) {
        best = other;
        e = other_e;
      }
    }
    if (j == 0) top_key = best;
    if (q == j && best != 0) {
      my_id = (int32_t)e;
      my_key = best;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (own == e && at == (uint32_t)i) key[i] = 0;
  }
  const float top = key_logit(top_key);
  const float p = my_id >= 0 ? __expf(key_logit(my_key) - top) : 0.f;
  float sum = p;
  if (flags & ZIPMOE_ROUTE_SOFTMAX_ALL) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += l[i] == -INFINITY ? 0.f : __expf(l[i] - top);
  }
#pragma unroll
  for (uint32_t d = 1; d < 8; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
  if (there && q < k) {
    ids[q] = my_id;
    weights[q] = my_id >= 0 ? __fdiv_rn(p, sum) : 0.f;
  }
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {   // the same place in another block's shared memory
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// four neighbouring floats of another block's shared memory.  Volatile: it stays behind the cluster's barrier.
__device__ __forceinline__ float4 load_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

// kPer: experts per lane, E <= 8 * kPer
template <int kPer>
__global__ void __launch_bounds__(kRouterThreads) router_kernel(const __grid_constant__ CUtensorMap x_map,
                                                               const __grid_constant__ CUtensorMap gate_map, const RouterArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * kRouterMaxStages + 1];
  __shared__ uint32_t words[2];   // tmem, dead
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = cluster_rank(), S = cluster_size();
  uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t ring0 = smem_addr(ring), stage_bytes = (kRouterRows + a.N) * 128;
  const uint32_t pitch = a.N + 4;   // floats between tokens: the 16-byte pieces of eight of them fall into different banks
  const uint32_t full = smem_addr(bars), empty = full + 8 * kRouterMaxStages, done = empty + 8 * kRouterMaxStages;
  volatile uint32_t *dead = words + 1;
  const WaitLimit lim = {dead, a.status, a.limit_ns};
  const uint32_t t0 = (blockIdx.x / S) * kRouterRows, rows = min(kRouterRows, a.T - t0);
  const uint32_t steps = (a.H + 63) / 64, s0 = rank * steps / S, s1 = (rank + 1) * steps / S;   // at least one: S <= steps

  if (tid == 0) {
    for (uint32_t s = 0; s < a.stages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    mbar_init(done, 1);
    *dead = 0;
    prefetch_map(&x_map);
    prefetch_map(&gate_map);
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(smem_addr(words), a.tmem_cols);
  after_predecessor();
  tc_before_sync();
  __syncthreads();
  tc_after_sync();
  const uint32_t tmem = words[0];

  if (warp == 0 && lane == 0) {
    const uint64_t once = policy_evict_first(), keep = policy_evict_last();
    uint32_t st = 0, round = 0;
    for (uint32_t s = s0; s < s1; ++s) {
      if (round > 0 && !wait_bar(empty + 8 * st, (round - 1) & 1, lim)) break;
      const uint32_t dst = ring0 + st * stage_bytes, bar = full + 8 * st;
      mbar_expect_tx(bar, stage_bytes + a.extra_tx);
      tma_load_2d(dst, &x_map, (int32_t)(s * 64), (int32_t)t0, bar, once);
      tma_load_2d(dst + kRouterRows * 128, &gate_map, (int32_t)(s * 64), 0, bar, keep);
      if (++st == a.stages) {
        st = 0;
        ++round;
      }
    }
  } else if (warp == 1 && lane == 0) {
    const uint32_t idesc = bf16_idesc(a.N);
    uint32_t st = 0, round = 0;
    bool ok = true;
    for (uint32_t s = s0; s < s1; ++s) {
      ok = wait_bar(full + 8 * st, round & 1, lim);
      if (!ok) break;
      tc_after_sync();
      const uint64_t xd = swizzled_desc(ring0 + st * stage_bytes), gd = swizzled_desc(ring0 + st * stage_bytes + kRouterRows * 128);
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) tc_mma(tmem, xd + 2 * j, gd + 2 * j, idesc, s > s0 || j > 0);
      tc_commit(empty + 8 * st);
      if (++st == a.stages) {
        st = 0;
        ++round;
      }
    }
    if (ok) tc_commit(done);
  }
  __syncwarp();

  // (wanted at the end, asked for now)
  const uint32_t q = lane & 7;
  float bias[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) bias[i] = a.bias && expert_of(q, i) < a.E ? __ldg(a.bias + expert_of(q, i)) : 0.f;

  // ---- partial logits into shared memory, over the ring (every MMA has read it); row = token ----
  float *part = reinterpret_cast<float *>(ring);
  const bool ok = __all_sync(0xFFFFFFFFu, wait_bar(done, 0, lim));
  tc_after_sync();
  const uint32_t row = 32 * (warp & 3) + lane;
  if (ok && 32 * (warp & 3) < rows) {
    for (uint32_t c = 8 * (warp >> 2); c < a.N; c += 16) {
      uint32_t v[8];
      tmem_load8(tmem + ((32 * (warp & 3)) << 16) + c, v);
      tmem_wait();
      float4 *to = reinterpret_cast<float4 *>(part + row * pitch + c);
      to[0] = make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]));
      to[1] = make_float4(__uint_as_float(v[4]), __uint_as_float(v[5]), __uint_as_float(v[6]), __uint_as_float(v[7]));
    }
  }
  __syncwarp();
  tc_before_sync();
  cluster_sync();
  tc_after_sync();
  if (*dead)   // let the copies and MMAs that this block has under way end before its memory goes to somebody else
    for (uint32_t i = 0; i < 200; ++i) __nanosleep(1000);
  if (warp == 1) tmem_free(tmem, a.tmem_cols);

  // ---- the tokens of this rank ----
  if (!*dead) {
    uint32_t base[8];
#pragma unroll
    for (uint32_t r = 0; r < 8; ++r) base[r] = in_block(ring0, r < S ? r : 0);
    const bool wide_logits = a.logits && a.E % 4 == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0;
    // token rank + S * n for n = warp * 4 + lane / 8, then the next 32
    for (uint32_t n0 = warp * 4; rank + S * n0 < rows; n0 += kRouterThreads / 8) {
      const uint32_t m = rank + S * (n0 + (lane >> 3));
      const bool there = m < rows;
      const uint64_t t = t0 + m;
      float l[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) l[i] = 0.f;
      const uint32_t at = ((there ? m : rank) * pitch + q * 4) * 4;
#pragma unroll
      for (uint32_t i = 0; i < kPer; i += 4) {
        if (i * 8 >= a.N) break;
        const bool in = i * 8 + q * 4 < a.N;   // (the operand's columns up to N are there, zeros past the experts)
        float4 v[8];
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r)
          if (r < S) v[r] = load_cluster(base[r] + (in ? at + i * 32 : 0));
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r)
          if (r < S) {
            l[i] += v[r].x;
            l[i + 1] += v[r].y;
            l[i + 2] += v[r].z;
            l[i + 3] += v[r].w;
          }
      }
#pragma unroll
      for (uint32_t i = 0; i < kPer; i += 4) {
        const uint32_t e = expert_of(q, i);
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) l[i + c] = e + c < a.E ? l[i + c] + bias[i + c] : -INFINITY;
        if (there && wide_logits) {
          if (e < a.E) *reinterpret_cast<float4 *>(a.logits + t * a.E + e) = make_float4(l[i], l[i + 1], l[i + 2], l[i + 3]);
        } else if (there && a.logits) {
#pragma unroll
          for (uint32_t c = 0; c < 4; ++c)
            if (e + c < a.E) a.logits[t * a.E + e + c] = l[i + c];
        }
      }
      pick_experts<kPer>(l, a.k, a.flags, q, there, a.ids + t * a.k, a.weights + t * a.k);
    }
  }
  __syncwarp();
  cluster_sync();   // nobody leaves while a neighbour may still read its shared memory
}

}  // namespace zipmoe_dev

namespace {

bool g_router_ready[64];

template <int kPer>
zipmoe_status launch_router(int dev, const CUtensorMap &x_map, const CUtensorMap &gate_map, const zipmoe_dev::RouterArgs &a, uint32_t S,
                            uint32_t smem, cudaStream_t stream) {
  using namespace zipmoe_dev;
  static bool ready[64];
  if (!ready[dev]) {
    if (cudaFuncSetAttribute(router_kernel<kPer>, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024) != cudaSuccess)
      return ZIPMOE_ERR_CUDA;
    ready[dev] = true;
  }
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeClusterDimension;
  attrs[0].val.clusterDim.x = S;
  attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
  attrs[1] = zipmoe_host::overlapped();
  cudaLaunchConfig_t cfg = {};
  cfg.stream = stream;
  cfg.attrs = attrs;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3((a.T + kRouterRows - 1) / kRouterRows * S);
  cfg.blockDim = dim3(kRouterThreads);
  cfg.dynamicSmemBytes = smem;
  return cudaLaunchKernelEx(&cfg, router_kernel<kPer>, x_map, gate_map, a) == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}

}  // namespace

extern "C" zipmoe_status zipmoe_route(const zipmoe_route_args *r, zipmoe_stream stream) {
  using namespace zipmoe_dev;
  zipmoe_host::TraceRange trace("zipmoe_route");
  if (!r) return ZIPMOE_ERR_INVALID_ARG;
  const uint32_t T = r->T, n_experts = r->n_experts, hidden = r->hidden;
  if (n_experts == 0 || n_experts > kMaxExperts || r->k == 0 || r->k > kMaxTopK || r->k > n_experts || hidden == 0 || hidden > 32768 ||
      hidden % 8 || r->token_pitch % 8)
    return ZIPMOE_ERR_UNSUPPORTED;
  if ((r->flags & ~ZIPMOE_ROUTE_SOFTMAX_ALL) || r->reserved) return ZIPMOE_ERR_INVALID_ARG;
  if (T == 0) return ZIPMOE_OK;
  if (!r->tokens || !r->gate || !r->topk_ids || !r->topk_weights || r->token_pitch < hidden) return ZIPMOE_ERR_INVALID_ARG;
  auto bits = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
  if (((bits(r->tokens) | bits(r->gate)) & 15) ||
      ((bits(r->bias) | bits(r->topk_ids) | bits(r->topk_weights) | bits(r->logits) | bits(r->status_word)) & 3))
    return ZIPMOE_ERR_INVALID_ARG;
  if (r->token_pitch >= 1ull << 39 || T > 1u << 30) return ZIPMOE_ERR_UNSUPPORTED;   // (what a tensor map and a grid can hold)
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return ZIPMOE_ERR_CUDA;
  if (!g_router_ready[dev]) {
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return ZIPMOE_ERR_CUDA;
    if (major != 10) return ZIPMOE_ERR_UNSUPPORTED;
    g_router_ready[dev] = true;
  }
  RouterArgs a;
  a.bias = r->bias;
  a.ids = r->topk_ids;
  a.weights = r->topk_weights;
  a.logits = r->logits;
  a.status = r->status_word;
  uint32_t tries = 0;
  zipmoe_host::wait_fault_setting(&a.extra_tx, &tries);
  a.limit_ns = tries < zipmoe_host::kWaitTries ? 1000000ull : 1000000000ull;   // (1 ms in the tests of the limit)
  a.T = T;
  a.E = n_experts;
  a.H = hidden;
  a.k = r->k;
  a.flags = r->flags;
  a.N = (n_experts + 15) / 16 * 16;
  a.tmem_cols = 32;
  while (a.tmem_cols < a.N) a.tmem_cols <<= 1;
  // two blocks per SM up to 128 experts, so that one streams while the other picks; then as many blocks per 128 tokens as
  // the device runs at once
  const uint32_t tiles = (T + kRouterRows - 1) / kRouterRows, steps = (hidden + 63) / 64, stage = (kRouterRows + a.N) * 128;
  const uint32_t per_sm = a.N <= 128 ? 2 : 1, at_once = zipmoe_host::current_sms() * per_sm;
  a.stages = std::min(kRouterMaxStages, (per_sm == 2 ? 108u : 216u) * 1024 / stage);
  uint32_t S = 8;
  while (S > 1 && (S > steps || tiles * S > at_once)) S >>= 1;
  const uint32_t smem = 1024 + std::max(a.stages * stage, kRouterRows * (a.N + 4) * 4);
  CUtensorMap x_map, gate_map;
  if (!zipmoe_host::make_bf16_map(&x_map, r->tokens, T, hidden, r->token_pitch, kRouterRows, true) ||
      !zipmoe_host::make_bf16_map(&gate_map, r->gate, n_experts, hidden, hidden, a.N, true))
    return ZIPMOE_ERR_CUDA;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (n_experts <= 32) return launch_router<4>(dev, x_map, gate_map, a, S, smem, s);
  if (n_experts <= 64) return launch_router<8>(dev, x_map, gate_map, a, S, smem, s);
  if (n_experts <= 128) return launch_router<16>(dev, x_map, gate_map, a, S, smem, s);
  return launch_router<32>(dev, x_map, gate_map, a, S, smem, s);
}
