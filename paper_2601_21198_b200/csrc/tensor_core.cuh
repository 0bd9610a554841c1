// What the kernels that stream bf16 matrices through tensor memory share: tensor-map copies, tcgen05 wrappers for
// K-major operands in the 128-byte swizzle, bounded waits, and the host's way to a tensor map.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "decode_device.cuh"

namespace zipmoe_dev {

__device__ __forceinline__ uint64_t global_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}

// Every wait below ends: the block's `dead` word (shared memory) is set when one has lasted longer than limit_ns, and
// makes all others return at once.  The caller then leaves its loop; nothing is left unsynchronised.
struct WaitLimit {
  volatile uint32_t *dead;
  uint32_t *status;
  uint64_t limit_ns;
};
static __device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, const WaitLimit &w) {
  const uint64_t t0 = global_ns();
  for (;;) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*w.dead) return false;
    if (global_ns() - t0 > w.limit_ns) {
      *w.dead = 1;
      report(w.status, kStatusWaitTimeout);
      return false;
    }
  }
}
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, const WaitLimit &w) {
  return mbar_try_wait(bar, parity) || wait_slow(bar, parity, w);
}
__device__ __forceinline__ uint32_t load_acquire(const uint32_t *p) {
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add_release(uint32_t *p, uint32_t v) {
  asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// waits until *p has reached `want`
__device__ __forceinline__ bool wait_count(const uint32_t *p, uint32_t want, const WaitLimit &w) {
  if (load_acquire(p) >= want) return true;
  const uint64_t t0 = global_ns();
  for (;;) {
    if (load_acquire(p) >= want) return true;
    if (*w.dead) return false;
    if (global_ns() - t0 > w.limit_ns) {
      *w.dead = 1;
      report(w.status, kStatusWaitTimeout);
      return false;
    }
    __nanosleep(20);
  }
}

// A kernel launched with programmatic stream serialization is set up while its predecessor drains: it waits here before it
// reads or writes anything, and lets its own successor do the same.  (Launched the ordinary way, the wait returns at once.)
__device__ __forceinline__ void wait_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// One thread's signal counts for its block.  A kernel that takes tensor memory gives it behind a barrier of the block behind the
// allocation: a successor may take its own before it waits, and the two would then wait for each other.
__device__ __forceinline__ void let_successor() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void after_predecessor() {
  wait_predecessor();
  let_successor();
}

// The product, correctly rounded, subnormal numbers included (which this library's compilation flushes otherwise).
__device__ __forceinline__ float times(float x, float y) {
  float r;
  asm("mul.rn.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}

__device__ __forceinline__ uint64_t policy_evict_first() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t policy_evict_last() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}
// one box of a tensor map into shared memory; x in elements, x * element size a multiple of 16 bytes
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void *map, int32_t x, int32_t y, uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], "
      "[%4], %5;" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void *map, int32_t x, int32_t y, int32_t z, uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], "
      "[%5], %6;" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *map, int32_t x, int32_t y, int32_t z, int32_t w, uint32_t bar,
                                            uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], "
      "[%6], %7;" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_prefetch_4d(const void *map, int32_t x, int32_t y, int32_t z, int32_t w) {
  asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}
// four rows of a 2-D tensor map whose box is 64 columns x 1 row: the rows land one after the other
__device__ __forceinline__ void tma_gather4(uint32_t dst, const void *map, int32_t x, int32_t r0, int32_t r1, int32_t r2, int32_t r3,
                                            uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes.L2::cache_hint [%0], "
      "[%1, {%2, %3, %4, %5, %6}], [%7], %8;" ::"r"(dst),
      "l"(map), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t policy) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar), "l"(policy)
               : "memory");
}
__device__ __forceinline__ void prefetch_map(const void *map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// a tensor map that lies in global memory: whatever wrote it there before the launch is visible to the copies
__device__ __forceinline__ void acquire_map(const void *map) {
  asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(map) : "memory");
}
__device__ __forceinline__ void fence_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// K-major operand, rows of 128 bytes (64 bf16) in the 128-byte swizzle, 8-row groups 1024 bytes apart.  The slice of
// 16 columns j starts 32 j bytes further: add 2 j to the descriptor.
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// bf16 x bf16 -> fp32, M = 128
__device__ __forceinline__ uint32_t bf16_idesc(uint32_t n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (8u << 24);
}
__device__ __forceinline__ void tc_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
// one arrival on the barrier once every MMA this thread has issued so far has completed
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t cols) {   // a whole warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t cols) {    // the warp that allocated
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}
// 8 columns of the warp's 32 lanes; the values are there after tmem_wait()
__device__ __forceinline__ void tmem_load8(uint32_t addr, uint32_t *v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

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

// ---- blocks of a cluster ----
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

}  // namespace zipmoe_dev

namespace zipmoe_host {

// SMs of the current device; 148 where there is none (a host-only size query)
inline uint32_t current_sms() {
  static int known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < 64) {
    int sms = 0;
    if (known[dev] == 0 && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) known[dev] = sms;
    if (known[dev] > 0) return (uint32_t)known[dev];
  }
  (void)cudaGetLastError();
  return 148;
}

inline cudaLaunchAttribute overlapped() {
  cudaLaunchAttribute a;
  a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  a.val.programmaticStreamSerializationAllowed = 1;
  return a;
}

// The same for a grid of `blocks`, of which `at_once` fit the device.  One that does not fit as a whole is not set up ahead: it
// would gain next to nothing, since most of its blocks start late anyway, and its first ones would hold registers and slots of the
// SMs while they wait.  (Its predecessor's blocks have all started by then, so it takes nothing from them.)
inline cudaLaunchAttribute overlapped_if_whole(uint64_t blocks, uint64_t at_once) {
  cudaLaunchAttribute a = overlapped();
  a.val.programmaticStreamSerializationAllowed = blocks <= at_once;
  return a;
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
// The driver's call that writes tensor maps; null if it does not offer one.
inline EncodeTiled encode_tiled() {
  static const EncodeTiled encode = [] {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      fn = nullptr;
    (void)cudaGetLastError();
    return reinterpret_cast<EncodeTiled>(fn);
  }();
  return encode;
}

// What the maps below have in common: bf16, boxes whose rows are 64 columns in the 128-byte swizzle, zeros outside.
inline bool encode_bf16(CUtensorMap *map, uint32_t rank, const void *base, const cuuint64_t *dims, const cuuint64_t *strides,
                        const cuuint32_t *box, bool wide_fetch) {
  const EncodeTiled encode = encode_tiled();
  const cuuint32_t step[4] = {1, 1, 1, 1};
  return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(base), dims, strides, box, step,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          wide_fetch ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// A row-major matrix: boxes of 64 columns x box_rows rows.  False if the driver does not offer the call or refuses it.
inline bool make_bf16_map(CUtensorMap *map, const void *base, uint64_t rows, uint64_t cols, uint64_t pitch_elems, uint32_t box_rows,
                          bool wide_fetch) {
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch_elems * 2};
  const cuuint32_t box[2] = {64, box_rows};
  return encode_bf16(map, 2, base, dims, strides, box, wide_fetch);
}
// n dense row-major matrices `distance` bytes apart: boxes of 64 columns x box_rows rows of one of them.
inline bool make_wide_map(CUtensorMap *map, const void *base, uint64_t rows, uint64_t cols, uint32_t box_rows, uint64_t n,
                          uint64_t distance) {
  const cuuint64_t dims[3] = {cols, rows, n}, strides[2] = {cols * 2, distance};
  const cuuint32_t box[3] = {64, box_rows, 1};
  return encode_bf16(map, 3, base, dims, strides, box, true);
}
// The same without the columns behind the last whole 64, seen as [n][cols / 64][rows][64]: a box of 8 x box_rows x 64 is
// 512 columns of box_rows rows.
inline bool make_sliced_map(CUtensorMap *map, const void *base, uint64_t rows, uint64_t cols, uint32_t box_rows, uint64_t n,
                            uint64_t distance) {
  const cuuint64_t dims[4] = {64, rows, cols / 64, n}, strides[3] = {cols * 2, 128, distance};
  const cuuint32_t box[4] = {64, box_rows, 8, 1};
  return encode_bf16(map, 4, base, dims, strides, box, true);
}

}  // namespace zipmoe_host
