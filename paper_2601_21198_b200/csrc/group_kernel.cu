// The lists that group the router's choices by expert, and the weighted sum that takes grouped rows back to their tokens.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "zipmoe.h"
#include "tensor_core.cuh"

namespace zipmoe_dev {

// ---- grouping: a stable counting sort of the choices by expert -----------------
// Bound: latency (12 bytes per choice are nothing).  One cluster of 1 to 16 blocks; every warp owns a run of consecutive choices
// and counts its experts in a row of its own in shared memory, 32 choices at a time.  Lanes with the same expert find one another
// with a ballot per bit of its number (the match instruction takes longer, the more experts differ: 8.8 us for 777 x 4 choices of
// 60, so 6.4, both in one block), so that nothing is added atomically and the order is the choices' own.  The blocks' sums meet
// through distributed shared memory; then every warp knows where its first choice of each expert goes.
constexpr uint32_t kGroupMaxExperts = 256;

struct GroupArgs {
  const int32_t *ids;
  int32_t *offsets, *order, *place;
  uint32_t *status;
  uint32_t n, E;
};

constexpr uint32_t kGroupHeld = 8;   // choices per lane that stay in registers, with their places among the warp's

__global__ void __launch_bounds__(1024) group_kernel(const GroupArgs a) {
  extern __shared__ uint32_t count[];                    // [warps][E]: choices of the warp's run; then where its next one goes
  __shared__ uint32_t total[kGroupMaxExperts], sums[8];  // the block's choices of every expert
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5, rank = cluster_rank(), S = cluster_size();
  uint32_t *mine = count + warp * a.E;
  const uint32_t bits = 32 - __clz(a.E - 1 | 1);
  for (uint32_t i = lane; i < a.E; i += 32) mine[i] = 0;
  after_predecessor();
  // the warp's run of whole 32s
  const uint32_t pieces = (a.n + 31) / 32, w = rank * warps + warp, W = S * warps;
  const uint32_t p0 = (uint32_t)((uint64_t)pieces * w / W), p1 = (uint32_t)((uint64_t)pieces * (w + 1) / W);
  int32_t held[kGroupHeld];
  uint32_t place[kGroupHeld];
  auto load = [&](uint32_t p) {
    const uint32_t at = p * 32 + lane;
    return at < a.n ? __ldcg(a.ids + at) : -1;
  };
#pragma unroll
  for (uint32_t i = 0; i < kGroupHeld; ++i) held[i] = p0 + i < p1 ? load(p0 + i) : -1;
  __syncwarp();
  // takes 32 choices: what the counter of this lane's expert shows for it, and the counters moved on
  auto take = [&](int32_t id) {
    const bool there = id >= 0 && id < (int32_t)a.E;
    uint32_t same = __ballot_sync(0xFFFFFFFFu, there);
    for (uint32_t b = 0; b < bits; ++b) {
      const uint32_t set = __ballot_sync(0xFFFFFFFFu, (id >> b) & 1);
      same &= (id >> b) & 1 ? set : ~set;
    }
    const uint32_t before = same & ((1u << lane) - 1);
    const uint32_t base = there ? mine[id] : 0;
    __syncwarp();
    if (there && before == 0) mine[id] = base + __popc(same);
    __syncwarp();
    return base + __popc(before);
  };
#pragma unroll
  for (uint32_t i = 0; i < kGroupHeld; ++i)
    if (p0 + i < p1) {
      place[i] = take(held[i]);
      if (held[i] >= (int32_t)a.E) report(a.status, kStatusBadDescriptor);
    }
  for (uint32_t p = p0 + kGroupHeld; p < p1; ++p) {
    const int32_t id = load(p);
    take(id);
    if (id >= (int32_t)a.E) report(a.status, kStatusBadDescriptor);
  }
  __syncthreads();
  // exclusive sums over the block's warps, expert by expert
  for (uint32_t e = tid; e < a.E; e += blockDim.x) {
    uint32_t sum = 0;
    for (uint32_t i = 0; i < warps; ++i) {
      const uint32_t c = count[i * a.E + e];
      count[i * a.E + e] = sum;
      sum += c;
    }
    total[e] = sum;
  }
  cluster_sync();
  // over the blocks, then over the experts
  uint32_t all = 0, before = 0;
  if (tid < a.E) {
    const uint32_t at = smem_addr(total + tid);
    for (uint32_t r = 0; r < S; ++r) {
      uint32_t c;
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(in_block(at, r)));
      if (r < rank) before += c;
      all += c;
    }
  }
  uint32_t upto = all;   // inclusive over the warp's experts
#pragma unroll
  for (uint32_t d = 1; d < 32; d <<= 1) {
    const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
    if (lane >= d) upto += v;
  }
  if (warp < 8 && lane == 31) sums[warp] = upto;
  cluster_sync();        // (also: nobody overwrites its totals, or leaves, while a neighbour reads them)
  if (tid < a.E) {
    uint32_t begin = upto - all;
    for (uint32_t i = 0; i < warp; ++i) begin += sums[i];
    if (rank == 0) {
      a.offsets[tid] = (int32_t)begin;
      if (tid == a.E - 1) a.offsets[a.E] = (int32_t)(begin + all);
    }
    total[tid] = begin + before;
  }
  __syncthreads();
  for (uint32_t i = lane; i < a.E; i += 32) mine[i] += total[i];
  __syncwarp();
  auto write = [&](uint32_t p, int32_t id, uint32_t to) {
    const uint32_t at = p * 32 + lane;
    const bool there = id >= 0 && id < (int32_t)a.E;
    if (there) a.order[to] = (int32_t)at;
    if (a.place && at < a.n) a.place[at] = there ? (int32_t)to : -1;
  };
#pragma unroll
  for (uint32_t i = 0; i < kGroupHeld; ++i)
    if (p0 + i < p1) write(p0 + i, held[i], held[i] >= 0 && held[i] < (int32_t)a.E ? mine[held[i]] + place[i] : 0);
  if (p0 + kGroupHeld < p1) {   // the others are counted again, behind those
    __syncwarp();
#pragma unroll
    for (uint32_t i = 0; i < kGroupHeld; ++i) take(held[i]);
    for (uint32_t p = p0 + kGroupHeld; p < p1; ++p) {
      const int32_t id = load(p);
      write(p, id, take(id));
    }
  }
}

// ---- combination: out[t] = sum over j of weights[t, j] * y[place[t, j]] --------
// Bound: the bytes of y.  A thread has four neighbouring columns and walks over tokens: all its choices' columns are asked for at
// once, and the next token's places and weights with them.  They are added in the order of the choices, in fp32.  8192 tokens of six
// choices of 2048 columns of fp32: 67 us, 6.5 TB/s, as fast as a copy.  (A block per token: 138 us; the places came before anything
// else could be asked for.)
struct CombineArgs {
  const void *y;
  const int32_t *place;
  const float *weights;
  __nv_bfloat16 *out;
  uint64_t y_pitch, out_pitch;
  uint32_t *status;
  uint32_t T, k, cols, rows;
};

// Blocks of an SM at once.  8192 tokens of six choices of 2048 columns: 70.6 us with three, 66.7 with four, 78.4 with five (which spill);
// 4096 tokens of two of 4096: 35.9 with four, 28.5 with six.  Seven and eight choices share an instance that spills with four (96 bytes
// of fp32): 104 and 111 us for 8192 tokens, 4.8 and 5.2 TB/s, where two, four and six choices reach 5.0, 5.8 and 6.3.
__host__ __device__ constexpr uint32_t combine_blocks(uint32_t k) { return k <= 2 ? 6 : k <= 4 ? 5 : 4; }

template <bool kF32, bool kWide, uint32_t kK>
__global__ void __launch_bounds__(256, combine_blocks(kK)) combine_rows_kernel(const CombineArgs a) {
  constexpr uint32_t kV = kWide ? 4 : 1;
  after_predecessor();
  const uint32_t units = a.cols / kV, stride = gridDim.y * blockDim.y;
  int32_t at[kK], next_at[kK];   // rows of the token's choices; -1: none
  float w[kK], next_w[kK];
  auto ask = [&](uint32_t t) {
#pragma unroll
    for (uint32_t j = 0; j < kK; ++j) {
      next_at[j] = j < a.k ? __ldcg(a.place + (uint64_t)t * a.k + j) : -1;
      next_w[j] = j < a.k && a.weights ? __ldcg(a.weights + (uint64_t)t * a.k + j) : 1.f;
    }
  };
  uint32_t t = blockIdx.y * blockDim.y + threadIdx.y;
  if (t < a.T) ask(t);
  for (; t < a.T; t += stride) {
#pragma unroll
    for (uint32_t j = 0; j < kK; ++j) {
      const bool there = next_at[j] >= 0 && (uint32_t)next_at[j] < a.rows;
      if (!there && next_at[j] >= 0) report(a.status, kStatusBadDescriptor);
      at[j] = there ? next_at[j] : -1;
      w[j] = there ? next_w[j] : 0.f;   // (a choice that is none adds nothing, whatever its weight)
    }
    bool asked = t + stride >= a.T;
    for (uint32_t c = blockIdx.x * blockDim.x + threadIdx.x; c < units; c += gridDim.x * blockDim.x) {
      float v[kK][kV];
#pragma unroll
      for (uint32_t j = 0; j < kK; ++j) {
        const uint64_t from = (at[j] >= 0 ? (uint64_t)at[j] : 0) * a.y_pitch + (uint64_t)c * kV;
        if constexpr (kWide && kF32) {
          const float4 x = at[j] >= 0 ? __ldcs(reinterpret_cast<const float4 *>(static_cast<const float *>(a.y) + from)) : make_float4(0.f, 0.f, 0.f, 0.f);
          v[j][0] = x.x;
          v[j][1] = x.y;
          v[j][2] = x.z;
          v[j][3] = x.w;
        } else if constexpr (kWide) {
          const uint2 x = at[j] >= 0 ? __ldcs(reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(a.y) + from)) : make_uint2(0, 0);
          v[j][0] = __uint_as_float(x.x << 16);
          v[j][1] = __uint_as_float(x.x & 0xFFFF0000u);
          v[j][2] = __uint_as_float(x.y << 16);
          v[j][3] = __uint_as_float(x.y & 0xFFFF0000u);
        } else if constexpr (kF32) {
          v[j][0] = at[j] >= 0 ? __ldcs(static_cast<const float *>(a.y) + from) : 0.f;
        } else {
          v[j][0] = at[j] >= 0 ? __uint_as_float((uint32_t)__ldcs(static_cast<const uint16_t *>(a.y) + from) << 16) : 0.f;
        }
      }
      if (!asked) {
        ask(t + stride);
        asked = true;
      }
      float sum[kV];
#pragma unroll
      for (uint32_t i = 0; i < kV; ++i) {
        sum[i] = 0.f;
#pragma unroll
        for (uint32_t j = 0; j < kK; ++j) sum[i] = fmaf(w[j], v[j][i], sum[i]);
      }
      __nv_bfloat16 *to = a.out + (uint64_t)t * a.out_pitch + (uint64_t)c * kV;
      if constexpr (kWide) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(sum[0], sum[1]), hi = __floats2bfloat162_rn(sum[2], sum[3]);
        *reinterpret_cast<uint2 *>(to) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
      } else {
        *to = __float2bfloat16_rn(sum[0]);
      }
    }
    if (!asked) ask(t + stride);   // (a thread without a column)
  }
}

}  // namespace zipmoe_dev

namespace {

uintptr_t bits(const void *p) { return reinterpret_cast<uintptr_t>(p); }

zipmoe_status current_device(int *dev) {
  static bool ready[64];
  if (cudaGetDevice(dev) != cudaSuccess || *dev < 0 || *dev >= 64) return ZIPMOE_ERR_CUDA;
  if (!ready[*dev]) {
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev) != cudaSuccess) return ZIPMOE_ERR_CUDA;
    if (major != 10) return ZIPMOE_ERR_UNSUPPORTED;
    ready[*dev] = true;
  }
  return ZIPMOE_OK;
}

// Blocks that a cluster of group_kernel may have on the device: 8 everywhere, 16 where it says that such clusters fit.
uint32_t largest_cluster(int dev) {
  static std::atomic<uint32_t> known[64];
  if (const uint32_t n = known[dev].load(std::memory_order_relaxed)) return n;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 16;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(16);
  cfg.blockDim = dim3(1024);
  cfg.dynamicSmemBytes = 32 * zipmoe_dev::kGroupMaxExperts * 4;
  int clusters = 0;
  const bool fits = cudaFuncSetAttribute(zipmoe_dev::group_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                    cudaOccupancyMaxActiveClusters(&clusters, zipmoe_dev::group_kernel, &cfg) == cudaSuccess && clusters > 0;
  if (!fits) cudaGetLastError();   // (nobody else is to find it)
  known[dev].store(fits ? 16 : 8, std::memory_order_relaxed);
  return fits ? 16 : 8;
}

}  // namespace

extern "C" zipmoe_status zipmoe_group_tokens(const zipmoe_group_args *g, zipmoe_stream stream) {
  using namespace zipmoe_dev;
  zipmoe_host::TraceRange trace("zipmoe_group_tokens");
  if (!g) return ZIPMOE_ERR_INVALID_ARG;
  if (g->n_experts == 0 || g->n_experts > kGroupMaxExperts || g->k == 0 || g->k > 8 || (uint64_t)g->T * g->k > 1u << 30) return ZIPMOE_ERR_UNSUPPORTED;
  if (g->reserved || !g->offsets || (g->T && (!g->topk_ids || !g->order))) return ZIPMOE_ERR_INVALID_ARG;
  if ((bits(g->topk_ids) | bits(g->offsets) | bits(g->order) | bits(g->place) | bits(g->status_word)) & 3) return ZIPMOE_ERR_INVALID_ARG;
  int dev = 0;
  const zipmoe_status rc = current_device(&dev);
  if (rc != ZIPMOE_OK) return rc;
  const GroupArgs a = {g->topk_ids, g->offsets, g->order, g->place, g->status_word, g->T * g->k, g->n_experts};
  // As many blocks as leave a warp 32 choices: 2000 x 4 choices of 64 take 7.4 us in two blocks and 4.7 in eight, 8192 x 6 take 9.8 in
  // eight and 7.3 in sixteen.
  const uint32_t pieces = (a.n + 31) / 32, threads = std::max(256u, std::min(1024u, pieces * 32)), most = largest_cluster(dev);
  uint32_t S = 1;
  while (S < most && pieces > S * 32) S <<= 1;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeClusterDimension;
  attrs[0].val.clusterDim.x = S;
  attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
  attrs[1] = zipmoe_host::overlapped();
  cudaLaunchConfig_t cfg = {};
  cfg.stream = reinterpret_cast<cudaStream_t>(stream);
  cfg.attrs = attrs;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3(S);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = threads / 32 * a.E * 4;   // at most 32 KB
  return cudaLaunchKernelEx(&cfg, group_kernel, a) == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}

extern "C" zipmoe_status zipmoe_combine_rows(const zipmoe_combine_args *c, zipmoe_stream stream) {
  using namespace zipmoe_dev;
  zipmoe_host::TraceRange trace("zipmoe_combine_rows");
  if (!c) return ZIPMOE_ERR_INVALID_ARG;
  if (c->k == 0 || c->k > 8 || c->cols == 0 || c->cols > 1u << 20 || (uint64_t)c->T * c->k > 1u << 30) return ZIPMOE_ERR_UNSUPPORTED;
  if ((c->flags & ~ZIPMOE_GROUPED_F32) || c->reserved) return ZIPMOE_ERR_INVALID_ARG;
  if (c->T == 0) return ZIPMOE_OK;
  if (!c->y || !c->place || !c->out || c->y_pitch < c->cols || c->out_pitch < c->cols) return ZIPMOE_ERR_INVALID_ARG;
  const bool f32 = c->flags & ZIPMOE_GROUPED_F32;
  if ((bits(c->y) & (f32 ? 3 : 1)) || (bits(c->out) & 1) || ((bits(c->place) | bits(c->weights) | bits(c->status_word)) & 3))
    return ZIPMOE_ERR_INVALID_ARG;
  int dev = 0;
  const zipmoe_status rc = current_device(&dev);
  if (rc != ZIPMOE_OK) return rc;
  const CombineArgs a = {c->y, c->place, c->weights, reinterpret_cast<__nv_bfloat16 *>(c->out), c->y_pitch, c->out_pitch, c->status_word,
                         c->T, c->k, c->cols, c->rows};
  const bool wide = c->cols % 4 == 0 && c->y_pitch % 4 == 0 && c->out_pitch % 4 == 0 && (bits(c->y) & (f32 ? 15 : 7)) == 0 && (bits(c->out) & 7) == 0;
  const uint32_t units = wide ? c->cols / 4 : c->cols;
  uint32_t x = 32;
  while (x < 256 && x < units) x <<= 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = reinterpret_cast<cudaStream_t>(stream);
  cfg.blockDim = dim3(x, 256 / x);
  // blocks that stay: as many as the device runs at once
  const uint32_t most = c->k <= 2 ? 2 : c->k <= 4 ? 4 : c->k <= 6 ? 6 : 8;
  const uint32_t across = (units + x - 1) / x, at_once = zipmoe_host::current_sms() * combine_blocks(most);
  cfg.gridDim = dim3(std::min(across, at_once), std::min(std::max(1u, at_once / across), (c->T + 256 / x - 1) / (256 / x)));
  cudaLaunchAttribute attr = zipmoe_host::overlapped();
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const auto call = [&](auto of_f32, auto of_wide, auto of_k) {
    return cudaLaunchKernelEx(&cfg, combine_rows_kernel<decltype(of_f32)::value, decltype(of_wide)::value, decltype(of_k)::value>, a);
  };
  const auto by_type = [&](auto of_k) {
    const std::true_type yes;
    const std::false_type no;
    return f32 ? (wide ? call(yes, yes, of_k) : call(yes, no, of_k)) : (wide ? call(no, yes, of_k) : call(no, no, of_k));
  };
  using std::integral_constant;
  const cudaError_t err = most == 2   ? by_type(integral_constant<uint32_t, 2>())
                          : most == 4 ? by_type(integral_constant<uint32_t, 4>())
                          : most == 6 ? by_type(integral_constant<uint32_t, 6>())
                                      : by_type(integral_constant<uint32_t, 8>());
  return err == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}
