// What the grouped products share: the weights' tensor maps, the calls' arguments, and the tensor core's two operand types.
#pragma once
#include <cuda.h>

#include <cstdint>

#include "zipmoe.h"
#include "tensor_core.cuh"

namespace zipmoe_dev {

constexpr uint32_t kMaxGroups = 256;
constexpr uint32_t kPairRows = 64;   // rows of W1, then as many of W3, make the 128 of an operand

// The maps of all groups' weights at once, where they lie at equal distances, in the order of a table's entry: boxes of 128 rows of
// W1 (or the one matrix) and W3, and for pairs boxes of 64.
struct GroupedMaps {
  CUtensorMap w[4];
};
constexpr uint32_t kPairMap = 2 * sizeof(CUtensorMap);   // where an entry's boxes of 64 rows begin

struct GroupedArgs {
  const uint8_t *x;         // rows of Kb bytes, x_pitch bytes apart
  const int32_t *offsets;   // [E + 1], or null: all rows are group 0's
  const int32_t *order;     // row r of the product is row order[r] / k of x; null: row r
  const float *row_scales;  // int8: of the rows of x
  const float *col_scales;  // int8: [E][N], of the second of a pair behind those of the first
  const uint8_t *table;     // the groups' maps, where they are not evenly spaced
  uint8_t *out;             // rows of N elements, out_pitch elements apart
  uint32_t *status;
  uint64_t x_pitch, out_pitch, limit_ns;
  uint32_t x_rows, k, R, E, N, Kb, even, out_f32, wide, whole, extra_tx;   // wide: rows of out may be stored four elements, whole: 16 bytes at a time
};

// One product of a step: 32 bytes of K.  kInt8: s8 x s8 -> s32, else bf16 x bf16 -> fp32; a is the weights' operand.
template <bool kInt8>
__device__ __forceinline__ void grouped_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate) {
  if constexpr (kInt8)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
  else
    tc_mma(d_tmem, a_desc, b_desc, idesc, accumulate);
}
// The instruction's descriptor: N columns (tokens), M = 128 rows (weights).
template <bool kInt8>
__device__ __forceinline__ uint32_t grouped_idesc(uint32_t n) {
  return kInt8 ? (2u << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (8u << 24) : bf16_idesc(n);
}

// The rows of a group between two offsets (without offsets there is one group, of all rows); false where they do not lie in order
// inside the product's R rows.
__device__ __forceinline__ uint32_t rows_between(const GroupedArgs &a, int32_t begin, int32_t end, bool &fine) {
  if (!a.offsets) return a.R;
  const bool here = begin >= 0 && end >= begin && end <= (int32_t)a.R;
  fine &= here;
  return here ? (uint32_t)(end - begin) : 0;
}

// The row of x that row r of the product reads; -1 where `order` points outside.
__device__ __forceinline__ int32_t source_row(const GroupedArgs &a, uint32_t r) {
  if (!a.order) return r < a.x_rows ? (int32_t)r : -1;
  const int32_t c = __ldcg(a.order + r);
  const uint32_t t = (uint32_t)c / a.k;
  return c >= 0 && t < a.x_rows ? (int32_t)t : -1;
}

// What an exact sum of 8-bit integers stands for.  Scales may be subnormal (a row of tiny numbers), their products need not be.
__device__ __forceinline__ float scaled(int32_t sum, float row_scale, float col_scale) {
  return times(times(__int2float_rn(sum), row_scale), col_scale);
}

__device__ __forceinline__ float silu_product(float g, float u) { return g / (1.0f + __expf(-g)) * u; }

// 16 bytes into shared memory, or 16 zero bytes
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

}  // namespace zipmoe_dev

namespace zipmoe_host {

// n dense row-major matrices of rows x row_bytes, `distance` bytes apart: boxes of 128 bytes x box_rows rows of one of them, in the
// 128-byte swizzle, zeros outside.
inline bool make_byte_map(CUtensorMap *map, const void *base, uint64_t rows, uint64_t row_bytes, uint64_t pitch_bytes, uint32_t box_rows,
                          uint64_t n, uint64_t distance, bool int8) {
  const EncodeTiled encode = encode_tiled();
  const uint32_t size = int8 ? 1 : 2;
  const cuuint64_t dims[3] = {row_bytes / size, rows, n}, strides[2] = {pitch_bytes, distance};
  const cuuint32_t box[3] = {128 / size, box_rows, 1}, step[3] = {1, 1, 1};
  return encode && encode(map, int8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims,
                          strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}}  // namespace zipmoe_host
