// The entry points of the grouped products: how a layer's weights are described once, and the checks of a call.
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstring>

#include "zipmoe.h"
#include "grouped_choice.h"
#include "grouped_launch.h"

namespace {

constexpr uint32_t kFlags = ZIPMOE_GROUPED_PAIR | ZIPMOE_GROUPED_INT8;
uintptr_t bits(const void *p) { return reinterpret_cast<uintptr_t>(p); }

bool sizes_ok(uint32_t n_groups, uint32_t rows, uint32_t cols, uint32_t flags) {
  return n_groups > 0 && n_groups <= zipmoe_dev::kMaxGroups && rows > 0 && rows <= 1u << 20 && cols > 0 && cols <= 65536 &&
         cols % (flags & ZIPMOE_GROUPED_INT8 ? 16 : 8) == 0;
}

std::atomic<uint32_t> g_test_kernel{0};   // 1: the kernel for few tokens, 2: the other

bool wide_pays(const zipmoe_grouped_weights *w, uint32_t rows, bool gathered) {
  if (const uint32_t forced = g_test_kernel.load()) return forced == 2;
  return zipmoe_host::grouped_wide_pays({w->n_groups, rows, w->rows, w->cols * (w->flags & ZIPMOE_GROUPED_INT8 ? 1 : 2),
                                         (w->flags & ZIPMOE_GROUPED_INT8) != 0, (w->flags & ZIPMOE_GROUPED_PAIR) != 0, gathered},
                                        zipmoe_host::current_sms());
}

uint64_t workspace_need(const zipmoe_grouped_weights *w, uint32_t rows, bool gathered) {
  return gathered && wide_pays(w, rows, true) ? (uint64_t)rows * w->cols * (w->flags & ZIPMOE_GROUPED_INT8 ? 1 : 2) : 0;
}

}  // namespace

extern "C" zipmoe_status zipmoe_grouped_workspace_bytes(const zipmoe_grouped_weights *w, uint32_t rows, uint32_t gathered,
                                                        uint64_t *workspace_bytes) {
  if (!w || !workspace_bytes || (w->flags & ~kFlags)) return ZIPMOE_ERR_INVALID_ARG;
  if (!sizes_ok(w->n_groups, w->rows, w->cols, w->flags) || rows > 1u << 30) return ZIPMOE_ERR_UNSUPPORTED;
  *workspace_bytes = workspace_need(w, rows, gathered != 0);
  return ZIPMOE_OK;
}

extern "C" zipmoe_status zipmoe_grouped_weights_plan(const void *const *tensors, uint32_t n_groups, uint32_t rows, uint32_t cols, uint32_t flags,
                                                     void *table, zipmoe_grouped_weights *weights) {
  if (flags & ~kFlags) return ZIPMOE_ERR_INVALID_ARG;
  if (!sizes_ok(n_groups, rows, cols, flags)) return ZIPMOE_ERR_UNSUPPORTED;
  if (!tensors || !table || !weights) return ZIPMOE_ERR_INVALID_ARG;
  static_assert(4 * sizeof(CUtensorMap) == ZIPMOE_GROUPED_ENTRY_BYTES, "an entry is four tensor maps");
  const uint32_t each = flags & ZIPMOE_GROUPED_PAIR ? 2 : 1;
  const bool int8 = flags & ZIPMOE_GROUPED_INT8;
  for (uint32_t i = 0; i < each * n_groups; ++i)
    if (!tensors[i] || (bits(tensors[i]) & 15)) return ZIPMOE_ERR_INVALID_ARG;
  const uint64_t row_bytes = (uint64_t)cols * (int8 ? 1 : 2), bytes = rows * row_bytes;
  std::memset(weights, 0, sizeof(*weights));
  std::memset(table, 0, (size_t)n_groups * ZIPMOE_GROUPED_ENTRY_BYTES);
  // the maps of matrix j of an entry (0 the one matrix or W1, 1 W3), of n groups
  auto describe = [&](uint8_t *entry, uint32_t j, const void *base, uint64_t n, uint64_t distance) {
    CUtensorMap map;
    if (!zipmoe_host::make_byte_map(&map, base, rows, row_bytes, row_bytes, 128, n, distance, int8)) return false;
    std::memcpy(entry + 128 * j, &map, sizeof(map));
    if (each == 1) return true;
    if (!zipmoe_host::make_byte_map(&map, base, rows, row_bytes, row_bytes, zipmoe_dev::kPairRows, n, distance, int8)) return false;
    std::memcpy(entry + zipmoe_dev::kPairMap + 128 * j, &map, sizeof(map));
    return true;
  };
  // evenly spaced groups: one map serves them all
  bool even = true;
  for (uint32_t j = 0; j < each && even; ++j) {
    const uintptr_t first = bits(tensors[j]), second = n_groups > 1 ? bits(tensors[each + j]) : first + bytes;
    const uint64_t distance = second - first;
    even = second > first && distance >= bytes && distance < 1ull << 40;
    for (uint32_t e = 2; e < n_groups && even; ++e) even = bits(tensors[each * e + j]) == first + e * distance;
    if (even && !describe(weights->maps, j, tensors[j], n_groups, distance)) return ZIPMOE_ERR_CUDA;
  }
  for (uint32_t i = 0; i < each * n_groups && !even; ++i)
    if (!describe(static_cast<uint8_t *>(table) + (size_t)(i / each) * ZIPMOE_GROUPED_ENTRY_BYTES, i % each, tensors[i], 1, bytes))
      return ZIPMOE_ERR_CUDA;
  weights->n_groups = n_groups;
  weights->rows = rows;
  weights->cols = cols;
  weights->flags = flags;
  weights->even = even;
  return ZIPMOE_OK;
}

extern "C" zipmoe_status zipmoe_grouped_matmul(const zipmoe_grouped_weights *w, const zipmoe_grouped_args *g, zipmoe_stream stream) {
  using namespace zipmoe_dev;
  zipmoe_host::TraceRange trace("zipmoe_grouped_matmul");
  if (!w || !g || (w->flags & ~kFlags) || w->even > 1 || w->reserved || (g->flags & ~ZIPMOE_GROUPED_F32) || g->reserved[0] || g->reserved[1])
    return ZIPMOE_ERR_INVALID_ARG;
  if (!sizes_ok(w->n_groups, w->rows, w->cols, w->flags)) return ZIPMOE_ERR_UNSUPPORTED;
  const bool int8 = w->flags & ZIPMOE_GROUPED_INT8, pair = w->flags & ZIPMOE_GROUPED_PAIR, f32 = g->flags & ZIPMOE_GROUPED_F32;
  const uint32_t size = int8 ? 1 : 2;
  if (g->rows > 1u << 30 || g->x_rows > 1u << 30 || g->x_pitch > 1ull << 39 || g->k > 8 || g->x_pitch * size % 16) return ZIPMOE_ERR_UNSUPPORTED;
  if (g->rows == 0) return ZIPMOE_OK;
  if (!g->x || !g->out || g->x_rows == 0 || g->x_pitch < w->cols || g->out_pitch < w->rows || (!w->even && !w->table)) return ZIPMOE_ERR_INVALID_ARG;
  if ((!g->offsets && w->n_groups != 1) || (g->order && g->k == 0) || (!g->order && g->x_rows < g->rows)) return ZIPMOE_ERR_INVALID_ARG;
  if (int8 != (g->row_scales != nullptr) || int8 != (g->col_scales != nullptr)) return ZIPMOE_ERR_INVALID_ARG;
  if ((bits(g->x) & 15) || (bits(w->table) & 63) || (bits(g->out) & (f32 ? 3 : 1)) ||
      ((bits(g->offsets) | bits(g->order) | bits(g->row_scales) | bits(g->col_scales) | bits(g->status_word)) & 3))
    return ZIPMOE_ERR_INVALID_ARG;
  const uint64_t need = workspace_need(w, g->rows, g->order != nullptr);
  if (need && (!g->workspace || (bits(g->workspace) & 15))) return ZIPMOE_ERR_INVALID_ARG;
  if (g->workspace_bytes < need) return ZIPMOE_ERR_BUFFER_TOO_SMALL;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return ZIPMOE_ERR_CUDA;
  static bool ready[64];
  if (!ready[dev]) {
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return ZIPMOE_ERR_CUDA;
    if (major != 10) return ZIPMOE_ERR_UNSUPPORTED;
    ready[dev] = true;
  }
  GroupedArgs a;
  a.x = static_cast<const uint8_t *>(g->x);
  a.offsets = g->offsets;
  a.order = g->order;
  a.row_scales = g->row_scales;
  a.col_scales = g->col_scales;
  a.table = static_cast<const uint8_t *>(w->table);
  a.out = static_cast<uint8_t *>(g->out);
  a.status = g->status_word;
  a.x_pitch = g->x_pitch * size;
  a.out_pitch = g->out_pitch;
  uint32_t tries = 0;
  zipmoe_host::wait_fault_setting(&a.extra_tx, &tries);
  a.limit_ns = tries < zipmoe_host::kWaitTries ? 1000000ull : 1000000000ull;   // (1 ms in the tests of the limit)
  a.x_rows = g->x_rows;
  a.k = g->k;
  a.R = g->rows;
  a.E = w->n_groups;
  a.N = w->rows;
  a.Kb = w->cols * size;
  a.even = w->even;
  a.out_f32 = f32;
  a.wide = g->out_pitch % 4 == 0 && (bits(g->out) & (f32 ? 15 : 7)) == 0;
  a.whole = g->out_pitch % (f32 ? 4 : 8) == 0 && (bits(g->out) & 15) == 0;
  GroupedMaps maps;
  std::memcpy(&maps, w->maps, sizeof(maps));
  if (wide_pays(w, g->rows, g->order != nullptr)) return zipmoe_host::launch_grouped_wide(dev, int8, pair, maps, a, g->workspace, reinterpret_cast<cudaStream_t>(stream));
  return zipmoe_host::launch_grouped_few(dev, int8, pair, maps, a, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" zipmoe_status zipmoe_linear_int8_workspace_bytes(const zipmoe_grouped_weights *w, uint32_t rows, uint64_t *workspace_bytes) {
  if (!w || !workspace_bytes || w->flags != ZIPMOE_GROUPED_INT8 || w->n_groups != 1) return ZIPMOE_ERR_INVALID_ARG;
  if (!sizes_ok(1, w->rows, w->cols, w->flags) || rows > 1u << 30) return ZIPMOE_ERR_UNSUPPORTED;
  *workspace_bytes = (uint64_t)rows * w->cols + 4ull * rows;
  return ZIPMOE_OK;
}

extern "C" zipmoe_status zipmoe_linear_int8(const zipmoe_grouped_weights *w, const zipmoe_linear_args *l, zipmoe_stream stream) {
  zipmoe_host::TraceRange trace("zipmoe_linear_int8");
  if (!l || l->reserved) return ZIPMOE_ERR_INVALID_ARG;
  uint64_t need = 0;
  zipmoe_status rc = zipmoe_linear_int8_workspace_bytes(w, l->rows, &need);
  if (rc != ZIPMOE_OK || l->rows == 0) return rc;
  if (!l->workspace || (bits(l->workspace) & 15)) return ZIPMOE_ERR_INVALID_ARG;
  if (l->workspace_bytes < need) return ZIPMOE_ERR_BUFFER_TOO_SMALL;
  int8_t *q = static_cast<int8_t *>(l->workspace);
  float *scales = reinterpret_cast<float *>(q + (uint64_t)l->rows * w->cols);   // (cols are whole 16s)
  zipmoe_grouped_args g = {};
  g.x = q;
  g.x_pitch = w->cols;
  g.row_scales = scales;
  g.col_scales = l->col_scales;
  g.out = l->out;
  g.out_pitch = l->out_pitch;
  g.status_word = l->status_word;
  g.x_rows = g.rows = l->rows;
  g.flags = l->flags;
  // (what the product would refuse is refused before anything is launched)
  if ((l->flags & ~ZIPMOE_GROUPED_F32) || !l->out || !l->col_scales || l->out_pitch < w->rows || w->even != 1 || w->reserved ||
      (bits(l->out) & (l->flags & ZIPMOE_GROUPED_F32 ? 3 : 1)) || ((bits(l->col_scales) | bits(l->status_word)) & 3))
    return ZIPMOE_ERR_INVALID_ARG;
  rc = zipmoe_quantize_rows(l->x, l->x_pitch, l->rows, w->cols, q, w->cols, scales, stream);
  return rc == ZIPMOE_OK ? zipmoe_grouped_matmul(w, &g, stream) : rc;
}

extern "C" void zipmoe_test_grouped_kernel(uint32_t which) { g_test_kernel.store(which); }
