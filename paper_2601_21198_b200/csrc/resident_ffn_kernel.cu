// The routed SwiGLU experts of a few tokens on recovered bf16 weights (pool F of the planner): the counterpart of
// the fused decode + FFN for experts that need no decoding.
//     g = W1 x,  u = W3 x,  h = bf16(SiLU(g) * u),  y = W2 h,  out[t] = bf16(sum_j w[t, j] * y)
// Bound: the active experts' weights, 6 * hidden * inter bytes each, read once.
// One warp per (choice, row): dot products in fp32.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

#include "zipmoe.h"
#include "decode_device.cuh"

namespace zipmoe_dev {

struct ResidentArgs {
  const uint16_t *tokens;
  const int32_t *ids;
  const float *weights;
  const uint8_t *table;
  uint16_t *out;
  uint16_t *h;         // [T * k][I]
  uint32_t *status;
  uint32_t T, k, E, H, I;
};

__device__ __forceinline__ const uint16_t *resident_tensor(const ResidentArgs &a, uint32_t tensor) {
  return *reinterpret_cast<const uint16_t *const *>(a.table + (size_t)tensor * ZIPMOE_RESIDENT_ENTRY_BYTES);
}
__device__ __forceinline__ float dot_row(const uint16_t *p, const uint16_t *q, uint32_t n, uint32_t lane) {
  float sum = 0.f;
  for (uint32_t c = lane * 8; c < n; c += 256) {
    const uint4 a = *reinterpret_cast<const uint4 *>(p + c), b = *reinterpret_cast<const uint4 *>(q + c);
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), sum);
      sum = fmaf(__uint_as_float(x[i] & 0xFFFF0000u), __uint_as_float(y[i] & 0xFFFF0000u), sum);
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
  return sum;
}

// grid (ceil(I / 8), T * k)
__global__ void __launch_bounds__(256) resident_gate_up_kernel(const ResidentArgs a) {
  const uint32_t lane = threadIdx.x & 31, row = blockIdx.x * 8 + (threadIdx.x >> 5), slot = blockIdx.y;
  const int32_t e = a.ids[slot];
  if (e >= (int32_t)a.E) report(a.status, kStatusBadDescriptor);
  if (e < 0 || e >= (int32_t)a.E || row >= a.I) return;
  const uint16_t *x = a.tokens + (size_t)(slot / a.k) * a.H;
  const float g = dot_row(resident_tensor(a, 3 * e) + (size_t)row * a.H, x, a.H, lane);
  const float u = dot_row(resident_tensor(a, 3 * e + 1) + (size_t)row * a.H, x, a.H, lane);
  if (lane == 0) a.h[(size_t)slot * a.I + row] = __bfloat16_as_ushort(__float2bfloat16_rn(g / (1.0f + __expf(-g)) * u));
}

// grid (ceil(H / 8), T)
__global__ void __launch_bounds__(256) resident_down_kernel(const ResidentArgs a) {
  const uint32_t lane = threadIdx.x & 31, row = blockIdx.x * 8 + (threadIdx.x >> 5), t = blockIdx.y;
  if (row >= a.H) return;
  float sum = 0.f;
  for (uint32_t j = 0; j < a.k; ++j) {
    const uint32_t slot = t * a.k + j;
    const int32_t e = a.ids[slot];
    if (e < 0 || e >= (int32_t)a.E) continue;
    const float y = dot_row(resident_tensor(a, 3 * e + 2) + (size_t)row * a.I, a.h + (size_t)slot * a.I, a.I, lane);
    sum += (a.weights ? a.weights[slot] : 1.0f) * y;
  }
  if (lane == 0) a.out[(size_t)t * a.H + row] = __bfloat16_as_ushort(__float2bfloat16_rn(sum));
}

}  // namespace zipmoe_dev

namespace {
constexpr uint32_t kResidentMaxT = 256, kResidentMaxK = 8, kResidentMaxExperts = 256, kResidentMaxDim = 32768;
bool dims_ok(uint32_t E, uint32_t H, uint32_t I) {
  return E > 0 && E <= kResidentMaxExperts && H > 0 && I > 0 && H % 8 == 0 && I % 8 == 0 && H <= kResidentMaxDim &&
         I <= kResidentMaxDim;
}
}  // namespace

extern "C" zipmoe_status zipmoe_resident_experts_plan(const uint16_t *const *tensors, uint32_t n_experts, uint32_t hidden,
                                                      uint32_t inter, void *table) {
  if (!dims_ok(n_experts, hidden, inter)) return ZIPMOE_ERR_UNSUPPORTED;
  if (!tensors || !table) return ZIPMOE_ERR_INVALID_ARG;
  for (uint32_t i = 0; i < 3 * n_experts; ++i)
    if (!tensors[i] || (reinterpret_cast<uintptr_t>(tensors[i]) & 15)) return ZIPMOE_ERR_INVALID_ARG;
  std::memset(table, 0, (size_t)3 * n_experts * ZIPMOE_RESIDENT_ENTRY_BYTES);
  for (uint32_t i = 0; i < 3 * n_experts; ++i)
    std::memcpy(static_cast<uint8_t *>(table) + (size_t)i * ZIPMOE_RESIDENT_ENTRY_BYTES, &tensors[i], sizeof(tensors[i]));
  return ZIPMOE_OK;
}

extern "C" zipmoe_status zipmoe_expert_ffn_workspace_bytes(uint32_t T, uint32_t k, const zipmoe_resident_experts *ex,
                                                           uint64_t *workspace_bytes) {
  if (!ex || !workspace_bytes) return ZIPMOE_ERR_INVALID_ARG;
  if (T > kResidentMaxT || k == 0 || k > kResidentMaxK || !dims_ok(ex->n_experts, ex->hidden, ex->inter))
    return ZIPMOE_ERR_UNSUPPORTED;
  *workspace_bytes = (uint64_t)T * k * ex->inter * 2;
  return ZIPMOE_OK;
}

extern "C" zipmoe_status zipmoe_expert_ffn(const uint16_t *tokens, uint32_t T, const int32_t *topk_ids,
                                           const float *topk_weights, uint32_t k, const zipmoe_resident_experts *ex,
                                           uint16_t *out, void *workspace, uint64_t workspace_bytes,
                                           uint32_t *status_word, zipmoe_stream stream_) {
  using namespace zipmoe_dev;
  zipmoe_host::TraceRange trace("zipmoe_expert_ffn");
  uint64_t need = 0;
  const zipmoe_status rc = zipmoe_expert_ffn_workspace_bytes(T, k, ex, &need);
  if (rc != ZIPMOE_OK) return rc;
  if (T == 0) return ZIPMOE_OK;
  if (!tokens || !topk_ids || !out || !workspace || !ex->table) return ZIPMOE_ERR_INVALID_ARG;
  if (workspace_bytes < need) return ZIPMOE_ERR_BUFFER_TOO_SMALL;
  if (((reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(workspace)) & 15) ||
      (reinterpret_cast<uintptr_t>(ex->table) & 63) ||
      ((reinterpret_cast<uintptr_t>(topk_ids) | reinterpret_cast<uintptr_t>(topk_weights) | reinterpret_cast<uintptr_t>(status_word)) & 3))
    return ZIPMOE_ERR_INVALID_ARG;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  ResidentArgs a;
  a.tokens = tokens;
  a.ids = topk_ids;
  a.weights = topk_weights;
  a.table = static_cast<const uint8_t *>(ex->table);
  a.out = out;
  a.h = static_cast<uint16_t *>(workspace);
  a.status = status_word;
  a.T = T;
  a.k = k;
  a.E = ex->n_experts;
  a.H = ex->hidden;
  a.I = ex->inter;
  resident_gate_up_kernel<<<dim3((a.I + 7) / 8, T * k), 256, 0, stream>>>(a);
  resident_down_kernel<<<dim3((a.H + 7) / 8, T), 256, 0, stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}
