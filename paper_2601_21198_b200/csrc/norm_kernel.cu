// Residual addition and root-mean-square norm, with bf16 rows or 8-bit rows and scales as the result.
//     h = x + r,  y = h * rsqrt(mean(h^2) + eps) * w,  s = max |y| / 448,  q = e4m3(y / s)
// One pass: a row stays in registers between the two sums and the stores.  The scale needs no second reduction over
// y: max |y| = rsqrt(...) * max |h * w|, so the sum of squares and the maximum are reduced together.
// Bound: bytes.  Per element 2 read for x, 2 (bf16) or 4 (fp32) read and written for the residual stream, 2 or 1
// written.  One block per row, 8 consecutive elements per thread and vector.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "zipmoe.h"
#include "decode_device.cuh"

namespace zipmoe_dev {

struct NormArgs {
  const uint16_t *x;
  const void *residual;
  void *residual_out;
  const uint16_t *weight;
  uint16_t *out;
  uint8_t *out_q;
  float *scales;
  uint64_t x_pitch, residual_pitch, residual_out_pitch, out_pitch;
  uint32_t rows, cols, group, groups;   // group 0: the whole row (groups = 1)
  float eps;
};

// the larger of two values, NaN if either is (fmaxf would drop it and the scale would hide it)
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// 8 consecutive bf16 of a row, the ones past its end as zeros.  kAligned: the row is made of whole 16-byte vectors.
template <bool kAligned>
__device__ __forceinline__ void load8(const uint16_t *p, uint32_t left, float *v) {
  if (kAligned) {
    const uint4 w = *reinterpret_cast<const uint4 *>(p);
    v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
    v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) v[i] = i < left ? __uint_as_float((uint32_t)p[i] << 16) : 0.f;
  }
}
template <bool kAligned>
__device__ __forceinline__ void load8(const float *p, uint32_t left, float *v) {
  if (kAligned) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
  }
}
template <bool kAligned>
__device__ __forceinline__ void store8(uint16_t *p, uint32_t left, const float *v) {
  if (kAligned) {
    *reinterpret_cast<uint4 *>(p) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < left) p[i] = __bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
  }
}
template <bool kAligned>
__device__ __forceinline__ void store8(float *p, uint32_t left, const float *v) {
  if (kAligned) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < left) p[i] = v[i];
  }
}
template <bool kAligned>
__device__ __forceinline__ void store8_e4m3(uint8_t *p, uint32_t left, const float *v, float inv_scale) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i] * inv_scale, v[4 * i + 1] * inv_scale), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2] * inv_scale, v[4 * i + 3] * inv_scale), __NV_SATFINITE, __NV_E4M3);
    w[i] = lo | (hi << 16);
  }
  if (kAligned) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
      if (i < left) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}

// kVecs: 8-element vectors per thread (cols <= blockDim.x * 8 * kVecs).  Res: void (none), uint16_t (bf16) or float.
template <typename Res, int kVecs, bool kAligned>
__global__ void __launch_bounds__(1024) add_rmsnorm_kernel(const NormArgs a) {
  __shared__ float s_sum[32], s_max[32];
  const uint32_t row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  const uint16_t *x = a.x + row * a.x_pitch;
  float h[kVecs][8], w[kVecs][8];
  float sum = 0.f, big = 0.f;
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const uint32_t c = (threadIdx.x + i * blockDim.x) * 8;
    if (c >= a.cols) {
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] = w[i][j] = 0.f;
      continue;
    }
    load8<kAligned>(x + c, a.cols - c, h[i]);
    load8<kAligned>(a.weight + c, a.cols - c, w[i]);
    if constexpr (!std::is_void<Res>::value) {
      float r[8];
      load8<kAligned>(static_cast<const Res *>(a.residual) + row * a.residual_pitch + c, a.cols - c, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] += r[j];
      if (a.residual_out) store8<kAligned>(static_cast<Res *>(a.residual_out) + row * a.residual_out_pitch + c, a.cols - c, h[i]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum += h[i][j] * h[i][j];
      big = max_nan(big, fabsf(h[i][j] * w[i][j]));
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    big = max_nan(big, __shfl_xor_sync(0xFFFFFFFFu, big, d));
  }
  if (lane == 0) {
    s_sum[warp] = sum;
    s_max[warp] = big;
  }
  __syncthreads();
  sum = 0.f;
  big = 0.f;
  for (uint32_t i = 0; i < n_warps; ++i) {
    sum += s_sum[i];
    big = max_nan(big, s_max[i]);
  }
  const float inv = rsqrtf(sum / (float)a.cols + a.eps);
  const float row_scale = big * inv * (1.f / 448.f);
  if (a.out_q && a.group == 0 && threadIdx.x == 0) a.scales[row] = row_scale;
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const uint32_t c = (threadIdx.x + i * blockDim.x) * 8;
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = h[i][j] * inv * w[i][j];
    if (a.out && c < a.cols) store8<kAligned>(a.out + row * a.out_pitch + c, a.cols - c, y);
    if (a.out_q) {
      float scale = row_scale;
      if (a.group) {   // the group's columns are those of group / 8 neighbouring lanes
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max_nan(m, fabsf(y[j]));
        for (uint32_t d = a.group / 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
        scale = m * (1.f / 448.f);
        if (c < a.cols && c % a.group == 0) a.scales[(uint64_t)row * a.groups + c / a.group] = scale;
      }
      if (c < a.cols) store8_e4m3<kAligned>(a.out_q + row * a.out_pitch + c, a.cols - c, y, scale > 0.f ? 1.f / scale : 1.f);
    }
  }
}

}  // namespace zipmoe_dev

namespace {

template <typename Res, bool kAligned>
void launch_norm(const zipmoe_dev::NormArgs &a, cudaStream_t stream) {
  using namespace zipmoe_dev;
  const uint32_t vecs = (a.cols + 7) / 8;
  auto threads = [&](uint32_t per) { return ((vecs + per - 1) / per + 31) / 32 * 32; };
  if (vecs <= 512) add_rmsnorm_kernel<Res, 1, kAligned><<<a.rows, threads(1), 0, stream>>>(a);
  else if (vecs <= 2048) add_rmsnorm_kernel<Res, 2, kAligned><<<a.rows, threads(2), 0, stream>>>(a);
  else add_rmsnorm_kernel<Res, 4, kAligned><<<a.rows, threads(4), 0, stream>>>(a);
}

}  // namespace

extern "C" zipmoe_status zipmoe_add_rmsnorm(const zipmoe_norm_args *n, zipmoe_stream stream_) {
  zipmoe_host::TraceRange trace("zipmoe_add_rmsnorm");
  if (!n || n->cols == 0 || (n->flags & ~ZIPMOE_NORM_RESIDUAL_F32) || !(n->eps >= 0.f) || n->reserved) return ZIPMOE_ERR_INVALID_ARG;
  if (n->cols > 32768) return ZIPMOE_ERR_UNSUPPORTED;
  if (n->rows == 0) return ZIPMOE_OK;
  if (!n->x || !n->weight || (!n->out && !n->out_q) || (n->out_q != nullptr) != (n->scales != nullptr) || (n->residual_out && !n->residual))
    return ZIPMOE_ERR_INVALID_ARG;
  if (n->x_pitch < n->cols || n->out_pitch < n->cols || (n->residual && n->residual_pitch < n->cols) ||
      (n->residual_out && n->residual_out_pitch < n->cols))
    return ZIPMOE_ERR_INVALID_ARG;
  const uint32_t group = n->group >= n->cols ? 0 : n->group;
  if (group && group != 32 && group != 64 && group != 128 && group != 256) return ZIPMOE_ERR_UNSUPPORTED;
  const bool f32 = n->flags & ZIPMOE_NORM_RESIDUAL_F32;
  auto bits = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
  const uintptr_t bf16_bits = bits(n->x) | bits(n->weight) | bits(n->out), residual_bits = bits(n->residual) | bits(n->residual_out);
  if ((bf16_bits & 1) || (residual_bits & (f32 ? 3 : 1)) || (bits(n->scales) & 3)) return ZIPMOE_ERR_INVALID_ARG;
  zipmoe_dev::NormArgs a;
  a.x = n->x;
  a.residual = n->residual;
  a.residual_out = n->residual_out;
  a.weight = n->weight;
  a.out = n->out;
  a.out_q = n->out_q;
  a.scales = n->scales;
  a.x_pitch = n->x_pitch;
  a.residual_pitch = n->residual_pitch;
  a.residual_out_pitch = n->residual_out_pitch;
  a.out_pitch = n->out_pitch;
  a.rows = n->rows;
  a.cols = n->cols;
  a.group = group;
  a.groups = group ? (n->cols + group - 1) / group : 1;
  a.eps = n->eps;
  const bool aligned = (n->cols | n->x_pitch | n->out_pitch | (n->residual ? n->residual_pitch : 0) |
                        (n->residual_out ? n->residual_out_pitch : 0)) % 8 == 0 &&
                       ((bf16_bits | residual_bits) & 15) == 0 && (bits(n->out_q) & 7) == 0;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!n->residual) aligned ? launch_norm<void, true>(a, stream) : launch_norm<void, false>(a, stream);
  else if (f32) aligned ? launch_norm<float, true>(a, stream) : launch_norm<float, false>(a, stream);
  else aligned ? launch_norm<uint16_t, true>(a, stream) : launch_norm<uint16_t, false>(a, stream);
  return cudaGetLastError() == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}
