// The router: logits = tokens x gate^T + bias, the k largest per token, and their softmax weights.
// One block per token: every warp takes experts in turn (each lane sums 8 columns of every 256), then the first warp
// picks the k largest.  A logit is compared through a 32-bit key that orders as the number does, with NaN on top.
#include <cuda_runtime.h>

#include <cstdint>

#include "zipmoe.h"
#include "decode_device.cuh"

namespace zipmoe_dev {

constexpr uint32_t kMaxExperts = 256, kMaxTopK = 8;

struct RouterArgs {
  const uint16_t *tokens, *gate;
  const float *bias;
  int32_t *ids;
  float *weights, *logits;
  uint64_t token_pitch;
  uint32_t T, E, H, k, flags;
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

// One warp picks the k largest of the logits l[0..E) (shared memory) of token t and writes ids and weights.
__device__ __forceinline__ void pick_experts(const float *l, uint32_t E, uint32_t k, uint32_t flags, uint32_t lane,
                                             int32_t *ids, float *weights) {
  uint32_t key[kMaxExperts / 32];
#pragma unroll
  for (uint32_t i = 0; i < kMaxExperts / 32; ++i) {
    const uint32_t e = lane + 32 * i;
    key[i] = e < E ? logit_key(l[e]) : 0u;
  }
  int32_t my_id = -1;       // lane j keeps choice j
  float my_logit = -INFINITY, top = -INFINITY;
  for (uint32_t j = 0; j < k; ++j) {
    uint32_t best = 0, at = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMaxExperts / 32; ++i)
      if (key[i] > best) {
        best = key[i];
        at = lane + 32 * i;
      }
    const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, best);
    if (most == 0) break;
    const uint32_t e = __reduce_min_sync(0xFFFFFFFFu, best == most ? at : 0xFFFFFFFFu);
    const float v = l[e];
    if (j == 0) top = v;
    if (lane == j) {
      my_id = (int32_t)e;
      my_logit = v;
    }
#pragma unroll
    for (uint32_t i = 0; i < kMaxExperts / 32; ++i)
      if (e == lane + 32 * i) key[i] = 0;
  }
  float p = my_id >= 0 ? __expf(my_logit - top) : 0.f, sum = p;
  if (flags & ZIPMOE_ROUTE_SOFTMAX_ALL) {
    sum = 0.f;
    for (uint32_t e = lane; e < E; e += 32) sum += l[e] == -INFINITY ? 0.f : __expf(l[e] - top);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
  if (lane < k) {
    ids[lane] = my_id;
    weights[lane] = my_id >= 0 ? __fdiv_rn(p, sum) : 0.f;
  }
}

__global__ void __launch_bounds__(256) router_kernel(const RouterArgs a) {
  __shared__ float s_logit[kMaxExperts];
  const uint32_t t = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint16_t *x = a.tokens + t * a.token_pitch;
  for (uint32_t e = warp; e < a.E; e += 8) {
    const uint16_t *g = a.gate + (uint64_t)e * a.H;
    float sum = 0.f;
    for (uint32_t c = lane * 8; c < a.H; c += 256) {
      const uint4 xv = __ldg(reinterpret_cast<const uint4 *>(x + c)), gv = __ldg(reinterpret_cast<const uint4 *>(g + c));
      const uint32_t xw[4] = {xv.x, xv.y, xv.z, xv.w}, gw[4] = {gv.x, gv.y, gv.z, gv.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum = fmaf(__uint_as_float(xw[i] << 16), __uint_as_float(gw[i] << 16), sum);
        sum = fmaf(__uint_as_float(xw[i] & 0xFFFF0000u), __uint_as_float(gw[i] & 0xFFFF0000u), sum);
      }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (lane == 0) {
      if (a.bias) sum += a.bias[e];
      s_logit[e] = sum;
      if (a.logits) a.logits[(uint64_t)t * a.E + e] = sum;
    }
  }
  __syncthreads();
  if (warp == 0) pick_experts(s_logit, a.E, a.k, a.flags, lane, a.ids + (uint64_t)t * a.k, a.weights + (uint64_t)t * a.k);
}

}  // namespace zipmoe_dev

extern "C" zipmoe_status zipmoe_route(const uint16_t *tokens, uint32_t T, uint64_t token_pitch, const uint16_t *gate,
                                      uint32_t n_experts, uint32_t hidden, const float *bias, uint32_t k, uint32_t flags,
                                      int32_t *topk_ids, float *topk_weights, float *logits, uint32_t *status_word,
                                      zipmoe_stream stream) {
  zipmoe_host::TraceRange trace("zipmoe_route");
  (void)status_word;
  if (n_experts == 0 || n_experts > zipmoe_dev::kMaxExperts || k == 0 || k > zipmoe_dev::kMaxTopK || k > n_experts ||
      hidden == 0 || hidden > 32768 || hidden % 8 || token_pitch % 8)
    return ZIPMOE_ERR_UNSUPPORTED;
  if (flags & ~ZIPMOE_ROUTE_SOFTMAX_ALL) return ZIPMOE_ERR_INVALID_ARG;
  if (T == 0) return ZIPMOE_OK;
  if (!tokens || !gate || !topk_ids || !topk_weights || token_pitch < hidden) return ZIPMOE_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(gate)) & 15) ||
      ((reinterpret_cast<uintptr_t>(bias) | reinterpret_cast<uintptr_t>(topk_ids) | reinterpret_cast<uintptr_t>(topk_weights) |
        reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(status_word)) & 3))
    return ZIPMOE_ERR_INVALID_ARG;
  zipmoe_dev::RouterArgs a;
  a.tokens = tokens;
  a.gate = gate;
  a.bias = bias;
  a.ids = topk_ids;
  a.weights = topk_weights;
  a.logits = logits;
  a.token_pitch = token_pitch;
  a.T = T;
  a.E = n_experts;
  a.H = hidden;
  a.k = k;
  a.flags = flags;
  zipmoe_dev::router_kernel<<<T, 256, 0, reinterpret_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}
