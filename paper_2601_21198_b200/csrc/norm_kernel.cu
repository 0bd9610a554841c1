// Residual addition and root-mean-square norm, with bf16 rows or 8-bit rows and scales as the result.
//     h = x + r,  y = h * rsqrt(mean(h^2) + eps) * w,  s = max |y| / 448,  q = e4m3(y / s)
// The scale of a whole row needs no second reduction over y: max |y| = rsqrt(...) * max |h * w|, so the sum of squares
// and the maximum are reduced together.
// Bound: bytes.  Per element 2 read for x, 2 (bf16) or 4 (fp32) read and written for the residual stream, 2 or 1
// written.  Up to 16384 columns (8192 unaligned) a row stays in registers (8 or 16 elements per thread) between the sums
// and the stores, and blocks stay on their SM and walk over the rows: the next row is asked for before the present one is
// reduced, so that loads are under way during the barrier and the stores, and the weight is read once per block.  Wider
// rows are read twice, the second time from the cache.
// 8192 rows of 4096, bf16 throughout: 45 us, 5.9 TB/s (92 % of a plain copy); 1531 rows of 1408 with an fp32 residual and
// scales of 128 columns: 6.1 us, 3.9 TB/s; 64 rows of 4096 to 8 bits: 1.9 us; one row of 2048: 1.5 us, which is the launch.
// A warp owns segments of 256 columns.  Where everything is made of whole 16-byte vectors a lane has 8 consecutive
// columns of a segment; otherwise columns lane, lane + 32, ... of it, so that loads of single elements still cover
// whole lines.  Either way a group of 32 to 256 columns lies within one warp.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "zipmoe.h"
#include "tensor_core.cuh"

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
  uint32_t rows, cols, group_log2, groups;   // groups of 2^group_log2 columns; group_log2 0: the whole row (groups = 1)
  float eps;
};

// The larger magnitude of two, NaN if either is (fmaxf would drop it and the scale would hide it).  It is never negative,
// so across lanes it is compared as the integer its bits are: that orders as the number does, NaN above infinity, and a
// warp's maximum is one instruction.
__device__ __forceinline__ float max_magnitude(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
  return r;
}
__device__ __forceinline__ float warp_max(float v) { return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v))); }

// Two fp32 operations per instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// A lane's 8 elements of a segment as they are loaded: 16 or 32 bytes in one piece, or one by one (zeros past the row).
template <typename T, bool kAligned>
struct Loaded;
template <>
struct Loaded<uint16_t, true> {
  uint4 w;
  __device__ __forceinline__ void load(const uint16_t *p, uint32_t, uint32_t lane) { w = __ldcs(reinterpret_cast<const uint4 *>(p) + lane); }
  __device__ __forceinline__ void get(float2 *v) const {
    v[0] = make_float2(bf16_lo(w.x), bf16_hi(w.x));
    v[1] = make_float2(bf16_lo(w.y), bf16_hi(w.y));
    v[2] = make_float2(bf16_lo(w.z), bf16_hi(w.z));
    v[3] = make_float2(bf16_lo(w.w), bf16_hi(w.w));
  }
};
template <>
struct Loaded<float, true> {
  float4 a, b;
  __device__ __forceinline__ void load(const float *p, uint32_t, uint32_t lane) {
    a = __ldcs(reinterpret_cast<const float4 *>(p) + 2 * lane);
    b = __ldcs(reinterpret_cast<const float4 *>(p) + 2 * lane + 1);
  }
  __device__ __forceinline__ void get(float2 *v) const {
    v[0] = make_float2(a.x, a.y);
    v[1] = make_float2(a.z, a.w);
    v[2] = make_float2(b.x, b.y);
    v[3] = make_float2(b.z, b.w);
  }
};
__device__ __forceinline__ float as_float(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float as_float(float f) { return f; }
template <typename T>
struct Loaded<T, false> {
  T e[8];
  __device__ __forceinline__ void load(const T *p, uint32_t left, uint32_t lane) {
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) e[j] = 32 * j + lane < left ? p[32 * j + lane] : T(0);
  }
  __device__ __forceinline__ void get(float2 *v) const {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) v[j] = make_float2(as_float(e[2 * j]), as_float(e[2 * j + 1]));
  }
};

__device__ __forceinline__ float element(const float2 *v, uint32_t j) { return j & 1 ? v[j >> 1].y : v[j >> 1].x; }

template <bool kAligned>
__device__ __forceinline__ void store8(uint16_t *p, uint32_t left, uint32_t lane, const float2 *v) {
  if (kAligned) {
    reinterpret_cast<uint4 *>(p)[lane] =
        make_uint4(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y), pack_bf16(v[3].x, v[3].y));
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j)
      if (32 * j + lane < left) p[32 * j + lane] = __bfloat16_as_ushort(__float2bfloat16_rn(element(v, j)));
  }
}
template <bool kAligned>
__device__ __forceinline__ void store8(float *p, uint32_t left, uint32_t lane, const float2 *v) {
  if (kAligned) {
    reinterpret_cast<float4 *>(p)[2 * lane] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    reinterpret_cast<float4 *>(p)[2 * lane + 1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j)
      if (32 * j + lane < left) p[32 * j + lane] = element(v, j);
  }
}
// e4m3 of v * inv
template <bool kAligned>
__device__ __forceinline__ void store8_e4m3(uint8_t *p, uint32_t left, uint32_t lane, const float2 *v, const float2 *inv) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(mul2(v[2 * i], inv[2 * i]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(mul2(v[2 * i + 1], inv[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
    w[i] = __byte_perm(lo, hi, 0x5410);
  }
  if (kAligned) {
    reinterpret_cast<uint2 *>(p)[lane] = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j)
      if (32 * j + lane < left) p[32 * j + lane] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
}

enum NormScales { kNoScales = 0, kRowScales = 1, kGroupScales = 2 };

// What the two kernels below do with a segment's y: bf16 and / or e4m3 and scales.
template <bool kAligned, int kScales>
__device__ __forceinline__ void store_y(const NormArgs &a, uint64_t row, uint32_t column, uint32_t lane, bool mine, const float2 *y,
                                        float to_q) {
  const uint32_t left = a.cols - column;
  if ((kScales == kNoScales || a.out) && mine) store8<kAligned>(a.out + row * a.out_pitch + column, left, lane, y);
  if constexpr (kScales == kNoScales) return;
  float2 inv[4];
  if constexpr (kScales == kRowScales) {
#pragma unroll
    for (int j = 0; j < 4; ++j) inv[j] = make_float2(to_q, to_q);
  } else if constexpr (kAligned) {   // the group's columns are those of group / 8 neighbouring lanes
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max_magnitude(max_magnitude(m, y[j].x), y[j].y);
    uint32_t bits = __float_as_uint(m);
    const uint32_t lanes = 1u << (a.group_log2 - 3);
    for (uint32_t d = lanes >> 1; d > 0; d >>= 1) bits = max(bits, __shfl_xor_sync(0xFFFFFFFFu, bits, d));
    const float scale = __uint_as_float(bits) * (1.f / 448.f), per = scale > 0.f ? 1.f / scale : 1.f;
    if (mine && (lane & (lanes - 1)) == 0) a.scales[row * a.groups + ((column + lane * 8) >> a.group_log2)] = scale;
#pragma unroll
    for (int j = 0; j < 4; ++j) inv[j] = make_float2(per, per);
  } else {                           // the group's columns are group / 32 elements of every lane
    float m[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) m[j] = warp_max(32 * j + lane < left ? max_magnitude(0.f, element(y, j)) : 0.f);
#pragma unroll
    for (uint32_t per = 1; per < 8; per *= 2)   // 64, 128, 256 columns: pairs of halves
      if (a.group_log2 >= (per == 1 ? 6u : per == 2 ? 7u : 8u)) {
#pragma unroll
        for (uint32_t j = 0; j < 8; j += 2 * per) {
          const float both = max_magnitude(m[j], m[j + per]);
#pragma unroll
          for (uint32_t q = j; q < j + 2 * per; ++q) m[q] = both;
        }
      }
    float per[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      const float scale = m[j] * (1.f / 448.f);
      const uint32_t c = column + 32 * j;
      if (lane == 0 && c < a.cols && (c & ((1u << a.group_log2) - 1)) == 0) a.scales[row * a.groups + (c >> a.group_log2)] = scale;
      per[j] = scale > 0.f ? 1.f / scale : 1.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) inv[j] = make_float2(per[2 * j], per[2 * j + 1]);
  }
  if (mine) store8_e4m3<kAligned>(a.out_q + row * a.out_pitch + column, left, lane, y, inv);
}

// The block's sum and largest magnitude, given to all of its threads; the two shared arrays alternate between calls, so
// that one barrier is enough.
template <int kScales>
__device__ __forceinline__ void reduce_block(float &sum, float &big, uint32_t lane, uint32_t warp, uint32_t n_warps,
                                             float (&s_sum)[32], float (&s_max)[32]) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
  if (kScales == kRowScales) big = warp_max(big);
  if (n_warps == 1) return;
  if (lane == 0) {
    s_sum[warp] = sum;
    if (kScales == kRowScales) s_max[warp] = big;
  }
  __syncthreads();
  sum = lane < n_warps ? s_sum[lane] : 0.f;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
  if (kScales == kRowScales) big = warp_max(lane < n_warps ? s_max[lane] : 0.f);
}

// What the sums give: y = value * to_y, and for a whole row's scale q = e4m3(y * to_q).
template <int kScales>
__device__ __forceinline__ void row_factors(const NormArgs &a, uint64_t row, float sum, float big, float &to_y, float &to_q) {
  to_y = rsqrtf(sum / (float)a.cols + a.eps);
  to_q = 1.f;
  if (kScales == kRowScales) {
    const float scale = big * to_y * (1.f / 448.f);
    if (threadIdx.x == 0) a.scales[row] = scale;
    to_q = scale > 0.f ? 1.f / scale : 1.f;
  }
}

// Rows that stay in registers, kVecs segments per warp.  Res: void (none), uint16_t (bf16) or float.
template <typename Res, int kVecs, bool kAligned, int kScales>
__global__ void __launch_bounds__(1024) add_rmsnorm_kernel(const NormArgs a) {
  constexpr bool kHasRes = !std::is_void<Res>::value;
  using R = typename std::conditional<kHasRes, Res, uint16_t>::type;
  __shared__ float s_sum[2][32], s_max[2][32];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  auto column = [&](int i) { return (warp + i * n_warps) * 256; };
  auto there = [&](int i) { return i == 0 || column(i) < a.cols; };   // (no warp lies wholly past the row)
  auto mine = [&](int i) { return there(i) && (!kAligned || column(i) + lane * 8 < a.cols); };
  Loaded<uint16_t, kAligned> w[kVecs] = {}, x[kVecs] = {};
  Loaded<R, kAligned> r[kVecs] = {};
  auto fetch = [&](uint64_t row) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (mine(i)) {
        x[i].load(a.x + row * a.x_pitch + column(i), a.cols - column(i), lane);
        if (kHasRes) r[i].load(static_cast<const R *>(a.residual) + row * a.residual_pitch + column(i), a.cols - column(i), lane);
      }
  };
  after_predecessor();
  uint64_t row = blockIdx.x;
  fetch(row);
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
    if (mine(i)) w[i].load(a.weight + column(i), a.cols - column(i), lane);
  for (uint32_t turn = 0; row < a.rows; ++turn) {
    float2 h[kVecs][4], sums = make_float2(0.f, 0.f);
    float big = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      x[i].get(h[i]);
      if constexpr (kHasRes) {
        float2 rf[4];
        r[i].get(rf);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[i][j] = add2(h[i][j], rf[j]);
      }
    }
    const uint64_t now = row;
    row += gridDim.x;
    if (kHasRes && a.residual_out) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
        if (mine(i)) store8<kAligned>(static_cast<R *>(a.residual_out) + now * a.residual_out_pitch + column(i), a.cols - column(i), lane, h[i]);
    }
    if (row < a.rows) fetch(row);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sums = fma2(h[i][j], h[i][j], sums);
      if (kScales == kRowScales) {   // from here on h * w: its largest magnitude is needed, and nothing but its multiples
        float2 wf[4];
        w[i].get(wf);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          h[i][j] = mul2(h[i][j], wf[j]);
          big = max_magnitude(max_magnitude(big, h[i][j].x), h[i][j].y);
        }
      }
    }
    float sum = sums.x + sums.y, to_y, to_q;
    reduce_block<kScales>(sum, big, lane, warp, n_warps, s_sum[turn & 1], s_max[turn & 1]);
    row_factors<kScales>(a, now, sum, big, to_y, to_q);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      if (!there(i)) continue;
      float2 wf[4];
      if (kScales != kRowScales) w[i].get(wf);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        h[i][j] = mul2(h[i][j], make_float2(to_y, to_y));
        if (kScales != kRowScales) h[i][j] = mul2(h[i][j], wf[j]);
      }
      store_y<kAligned, kScales>(a, now, column(i), lane, mine(i), h[i], to_q);
    }
  }
}

// Wider rows: a warp goes over its segments twice.  (The residual is written in the second pass, since it may lie over
// the input.)
template <typename Res, bool kAligned, int kScales>
__global__ void __launch_bounds__(512, 2) add_rmsnorm_wide_kernel(const NormArgs a) {
  constexpr bool kHasRes = !std::is_void<Res>::value;
  using R = typename std::conditional<kHasRes, Res, uint16_t>::type;
  __shared__ float s_sum[2][32], s_max[2][32];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  auto load = [&](uint64_t row, uint32_t column, bool mine, float2 *h, float2 *wf) {
    const uint32_t left = a.cols - column;
    Loaded<uint16_t, kAligned> w = {}, x = {};
    Loaded<R, kAligned> r = {};
    if (mine) {
      x.load(a.x + row * a.x_pitch + column, left, lane);
      if (kHasRes) r.load(static_cast<const R *>(a.residual) + row * a.residual_pitch + column, left, lane);
      w.load(a.weight + column, left, lane);
    }
    x.get(h);
    w.get(wf);
    if constexpr (kHasRes) {
      float2 rf[4];
      r.get(rf);
#pragma unroll
      for (int j = 0; j < 4; ++j) h[j] = add2(h[j], rf[j]);
    }
  };
  after_predecessor();
  uint32_t turn = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, ++turn) {
    float2 sums = make_float2(0.f, 0.f);
    float big = 0.f;
#pragma unroll 2
    for (uint32_t column = warp * 256; column < a.cols; column += n_warps * 256) {
      float2 h[4], wf[4];
      load(row, column, !kAligned || column + lane * 8 < a.cols, h, wf);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sums = fma2(h[j], h[j], sums);
        if (kScales == kRowScales) {
          const float2 v = mul2(h[j], wf[j]);
          big = max_magnitude(max_magnitude(big, v.x), v.y);
        }
      }
    }
    float sum = sums.x + sums.y, to_y, to_q;
    reduce_block<kScales>(sum, big, lane, warp, n_warps, s_sum[turn & 1], s_max[turn & 1]);
    row_factors<kScales>(a, row, sum, big, to_y, to_q);
#pragma unroll 2
    for (uint32_t column = warp * 256; column < a.cols; column += n_warps * 256) {
      float2 h[4], wf[4];
      const bool mine = !kAligned || column + lane * 8 < a.cols;
      load(row, column, mine, h, wf);
      if (kHasRes && a.residual_out && mine)
        store8<kAligned>(static_cast<R *>(a.residual_out) + row * a.residual_out_pitch + column, a.cols - column, lane, h);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        h[j] = kScales == kRowScales ? mul2(mul2(h[j], wf[j]), make_float2(to_y, to_y)) : mul2(mul2(h[j], make_float2(to_y, to_y)), wf[j]);
      store_y<kAligned, kScales>(a, row, column, lane, mine, h, to_q);
    }
  }
}

}  // namespace zipmoe_dev

namespace {

cudaError_t launch(void (*kernel)(zipmoe_dev::NormArgs), uint32_t blocks, uint32_t warps, const zipmoe_dev::NormArgs &a, cudaStream_t stream) {
  const cudaLaunchAttribute overlapped = zipmoe_host::overlapped();
  cudaLaunchConfig_t cfg = {};
  cfg.stream = stream;
  cfg.attrs = const_cast<cudaLaunchAttribute *>(&overlapped);
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(32 * warps);
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

// A row to a block of as many warps as it has segments of 256 columns, up to 32.  Where that is not
// enough, or there are many rows for every SM, a warp takes two segments: half the instructions of the reductions.
template <typename Res, bool kAligned, int kScales>
cudaError_t launch_sizes(const zipmoe_dev::NormArgs &a, cudaStream_t stream) {
  using namespace zipmoe_dev;
  const uint32_t segments = (a.cols + 255) / 256, sms = zipmoe_host::current_sms();
  auto grid = [&](uint32_t warps) { return (uint32_t)std::min<uint64_t>(a.rows, (uint64_t)sms * std::min(32u, 32 / warps)); };
  if (segments > (kAligned ? 64 : 32)) {
    const uint32_t per_warp = (segments + 15) / 16, warps = (segments + per_warp - 1) / per_warp;
    return launch(add_rmsnorm_wide_kernel<Res, kAligned, kScales>, grid(warps), warps, a, stream);
  }
  if constexpr (kAligned) {
    if (segments > 32 || (segments >= 2 && a.rows >= 16 * sms)) {
      const uint32_t warps = (segments + 1) / 2;
      return launch(add_rmsnorm_kernel<Res, 2, kAligned, kScales>, grid(warps), warps, a, stream);
    }
  }
  return launch(add_rmsnorm_kernel<Res, 1, kAligned, kScales>, grid(segments), segments, a, stream);
}
template <typename Res, bool kAligned>
cudaError_t launch_norm(const zipmoe_dev::NormArgs &a, cudaStream_t stream) {
  if (!a.out_q) return launch_sizes<Res, kAligned, zipmoe_dev::kNoScales>(a, stream);
  if (a.group_log2 == 0) return launch_sizes<Res, kAligned, zipmoe_dev::kRowScales>(a, stream);
  return launch_sizes<Res, kAligned, zipmoe_dev::kGroupScales>(a, stream);
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
  a.group_log2 = group == 32 ? 5 : group == 64 ? 6 : group == 128 ? 7 : group == 256 ? 8 : 0;
  a.groups = group ? (n->cols + group - 1) / group : 1;
  a.eps = n->eps;
  const bool aligned = (n->cols | n->x_pitch | n->out_pitch | (n->residual ? n->residual_pitch : 0) |
                        (n->residual_out ? n->residual_out_pitch : 0)) % 8 == 0 &&
                       ((bf16_bits | residual_bits) & 15) == 0 && (bits(n->out_q) & 7) == 0;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  const cudaError_t rc = !n->residual ? (aligned ? launch_norm<void, true>(a, stream) : launch_norm<void, false>(a, stream))
                         : f32        ? (aligned ? launch_norm<float, true>(a, stream) : launch_norm<float, false>(a, stream))
                                      : (aligned ? launch_norm<uint16_t, true>(a, stream) : launch_norm<uint16_t, false>(a, stream));
  return rc == cudaSuccess ? ZIPMOE_OK : ZIPMOE_ERR_CUDA;
}
