// Rows of bf16 to 8-bit integers with a scale per row:  a = max |x|,  q = rint(127 x / a),  scale = a / 127.
// Bound: 3 bytes per element.  A row stays in registers between its maximum and its stores.  8192 rows of 4096: 18.3 us, 5.5 TB/s.
// With x = X 2^i and a = A 2^j, X and A whole numbers below 256, the quotient t = 127 X 2^(i-j) / A is either half way between two
// integers, or |254 X - (2m + 1) A 2^(j-i)| / (2A 2^(j-i)) >= t / (254 X) > t 2^-16 away from there.  x * (127 / a) with two roundings
// is off by t 2^-23 at most: rounded to 19 significant bits (t 2^-19 at most from there) it is the half where t is one, and on
// the right side of it where t is not.  So the integers are those that the real numbers give, without a division per element.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "zipmoe.h"
#include "tensor_core.cuh"

namespace zipmoe_dev {

struct QuantizeArgs {
  const uint16_t *x;
  int8_t *q;
  float *scales;
  uint64_t x_pitch, q_pitch;
  uint32_t rows, cols;
};

// The quotient, correctly rounded, as times() rounds the product.
__device__ __forceinline__ float divided(float x, float y) {
  float r;
  asm("div.rn.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
// x * by, rounded to 19 bits, rounded to an integer.  Where a row has a NaN or an infinity its scale is NaN and its integers are 0,
// so that whatever is computed from it is NaN.
__device__ __forceinline__ uint32_t quantized(float x, float by) {
  const float t = __fmul_rn(x, by), c = __fmul_rn(t, 33.f);
  return (uint32_t)__float2int_rn(__fsub_rn(c, __fsub_rn(c, t))) & 0xFFu;
}

// kThreads threads per row, kVectors vectors of 8 columns each (kWide) or as many single columns; blocks of 128 threads at least.
template <uint32_t kThreads, uint32_t kVectors, bool kWide>
__global__ void __launch_bounds__(kThreads < 128 ? 128 : kThreads) quantize_kernel(const QuantizeArgs a) {
  constexpr uint32_t kRows = kThreads < 128 ? 128 / kThreads : 1, kV = kWide ? kVectors : 8 * kVectors;
  __shared__ uint32_t tops[32];
  after_predecessor();
  const uint32_t t = threadIdx.x % kThreads, row = blockIdx.x * kRows + threadIdx.x / kThreads;
  const bool there = row < a.rows;
  const uint16_t *x = a.x + (there ? (uint64_t)row * a.x_pitch : 0);
  uint32_t top = 0;    // magnitudes order as their bits do, infinity and NaN above all numbers
  uint4 v[kWide ? kV : 1];
  uint16_t s[kWide ? 1 : kV];
  if constexpr (kWide) {
#pragma unroll
    for (uint32_t i = 0; i < kV; ++i) {
      const uint32_t c = (i * kThreads + t) * 8;
      v[i] = there && c < a.cols ? __ldcs(reinterpret_cast<const uint4 *>(x + c)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (uint32_t i = 0; i < kV; ++i) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) top = max(top, max((w[j] << 16) & 0x7FFF0000u, w[j] & 0x7FFF0000u));
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kV; ++i) {
      const uint32_t c = i * kThreads + t;
      s[i] = there && c < a.cols ? x[c] : 0;
      top = max(top, (uint32_t)(s[i] & 0x7FFF) << 16);
    }
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if constexpr (kThreads > 32) {
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    constexpr uint32_t kWarps = kThreads / 32;
    const uint32_t first = threadIdx.x / kThreads * kWarps;
#pragma unroll
    for (uint32_t i = 0; i < kWarps; ++i) top = max(top, tops[first + i]);
  }
  if (!there) return;
  const bool finite = top < 0x7F800000u;
  const float m = __uint_as_float(top);
  if (t == 0) a.scales[row] = finite ? divided(m, 127.f) : __uint_as_float(0x7FC00000u);
  const bool zeros = top == 0 || !finite;
  // 127 / a is a number, and x * (127 / a) loses nothing, while a is neither very small nor very large; others are moved by 2^96
  const float move = m >= 0x1p100f ? 0x1p-96f : m < 0x1p-90f ? 0x1p96f : 1.f, by = zeros ? 0.f : divided(127.f, times(m, move));
  int8_t *q = a.q + (uint64_t)row * a.q_pitch;
  if constexpr (kWide) {
#pragma unroll
    for (uint32_t i = 0; i < kV; ++i) {
      const uint32_t c = (i * kThreads + t) * 8;
      if (c >= a.cols) break;
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      uint32_t o[2] = {0, 0};
      if (!zeros)
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          float x0 = __uint_as_float(w[j] << 16), x1 = __uint_as_float(w[j] & 0xFFFF0000u);
          if (move != 1.f) {
            x0 = times(x0, move);
            x1 = times(x1, move);
          }
          const uint32_t lo = quantized(x0, by), hi = quantized(x1, by);
          o[j >> 1] |= (lo | hi << 8) << (16 * (j & 1));
        }
      *reinterpret_cast<uint2 *>(q + c) = make_uint2(o[0], o[1]);
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kV; ++i) {
      const uint32_t c = i * kThreads + t;
      if (c < a.cols) q[c] = zeros ? 0 : (int8_t)quantized(times(__uint_as_float((uint32_t)s[i] << 16), move), by);
    }
  }
}

}  // namespace zipmoe_dev

namespace {

template <uint32_t kThreads, uint32_t kVectors>
cudaError_t launch(const zipmoe_dev::QuantizeArgs &a, bool wide, cudaStream_t stream) {
  constexpr uint32_t kRows = kThreads < 128 ? 128 / kThreads : 1;
  cudaLaunchAttribute attr = zipmoe_host::overlapped_if_whole((a.rows + kRows - 1) / kRows, zipmoe_host::current_sms());
  cudaLaunchConfig_t cfg = {};
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((a.rows + kRows - 1) / kRows);
  cfg.blockDim = dim3(kThreads < 128 ? 128 : kThreads);
  return wide ? cudaLaunchKernelEx(&cfg, zipmoe_dev::quantize_kernel<kThreads, kVectors, true>, a)
              : cudaLaunchKernelEx(&cfg, zipmoe_dev::quantize_kernel<kThreads, kVectors, false>, a);
}

}  // namespace

extern "C" zipmoe_status zipmoe_quantize_rows(const uint16_t *x, uint64_t x_pitch, uint32_t rows, uint32_t cols, int8_t *q, uint64_t q_pitch,
                                              float *scales, zipmoe_stream stream) {
  using namespace zipmoe_dev;
  zipmoe_host::TraceRange trace("zipmoe_quantize_rows");
  if (cols == 0 || cols > 65536 || rows > 1u << 30) return ZIPMOE_ERR_UNSUPPORTED;
  if (rows == 0) return ZIPMOE_OK;
  auto bits = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
  if (!x || !q || !scales || x_pitch < cols || q_pitch < cols || (bits(x) & 1) || (bits(scales) & 3)) return ZIPMOE_ERR_INVALID_ARG;
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return ZIPMOE_ERR_CUDA;
  static bool ready[64];
  if (!ready[dev]) {
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return ZIPMOE_ERR_CUDA;
    if (major != 10) return ZIPMOE_ERR_UNSUPPORTED;
    ready[dev] = true;
  }
  const QuantizeArgs a = {x, q, scales, x_pitch, q_pitch, rows, cols};
  const bool wide = cols % 8 == 0 && x_pitch % 8 == 0 && q_pitch % 8 == 0 && (bits(x) & 15) == 0 && (bits(q) & 7) == 0;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t err;
  // few registers, so that many rows are under way on an SM
  if (cols <= 1024) err = launch<32, 4>(a, wide, s);
  else if (cols <= 2048) err = launch<64, 4>(a, wide, s);
  else if (cols <= 4096) err = launch<128, 4>(a, wide, s);
  else if (cols <= 8192) err = launch<256, 4>(a, wide, s);
  else if (cols <= 16384) err = launch<512, 4>(a, wide, s);
  else if (cols <= 32768) err = launch<1024, 4>(a, wide, s);
  else err = launch<1024, 8>(a, wide, s);
  return err == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}
