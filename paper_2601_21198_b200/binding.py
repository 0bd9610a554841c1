"""Thin ctypes binding over the C ABI in include/zipmoe.h.

Every function here has the name of the C entry point it forwards to and does
argument marshalling only (numpy arrays / torch tensors -> pointers and sizes).
`DecodePlan` holds what zipmoe_launch_plan wrote for several blobs (buffers,
descriptors, tables); it computes nothing of the codec or of the layout.

There is no fallback: if the CUDA library has not been built, importing this
module raises.
"""
import ctypes
import os
import struct
import threading
import weakref

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libzipmoe.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "CUDA library %s not found: build it with `python -m paper_2601_21198_b200.build` "
        "(there is no CPU fallback)" % LIB_PATH)

_lib = ctypes.CDLL(LIB_PATH)

DECODE_SHORT_CODES = 1      # zipmoe_decode flag: no code above 8 bits, max_record_bytes exact and <= NARROW_RECORD_BYTES
NARROW_RECORD_BYTES = 2080  # a tile record of 16 rows
OK = 0
ERR_INVALID_ARG, ERR_BAD_FORMAT, ERR_BUFFER_TOO_SMALL, ERR_CUDA, ERR_DECODE_CORRUPT, ERR_UNSUPPORTED = -1, -2, -3, -4, -5, -6
LAYOUT_LINEAR, LAYOUT_BLOCKED = 0, 1
DEVICE_PAD_BYTES = 256

_u64, _u32, _vp, _int = ctypes.c_uint64, ctypes.c_uint32, ctypes.c_void_p, ctypes.c_int


class EncodeOpts(ctypes.Structure):
    _fields_ = [("chunk_elems", _u32), ("max_code_len", _u32), ("layout", _u32), ("n_threads", _u32)]


class BlobInfo(ctypes.Structure):
    _fields_ = [("n_elems", _u64), ("rows", _u32), ("cols", _u32), ("layout", _u32), ("chunk_elems", _u32),
                ("tile_elems", _u32), ("max_code_len", _u32), ("n_chunks", _u32), ("n_tiles", _u32),
                ("table_off", _u64), ("chunk_off_off", _u64), ("payload_off", _u64), ("payload_bytes", _u64),
                ("sm_off", _u64), ("sm_bytes", _u64), ("total_bytes", _u64)]


CHUNK_DESC_DTYPE = np.dtype([
    ("payload_off", "<u8"), ("sm_off", "<u8"), ("out_off", "<u8"), ("row_pitch", "<u4"), ("tiles_per_rowblk", "<u4"),
    ("tile0", "<u4"), ("n_tiles", "<u4"), ("tile_elems", "<u4"), ("last_tile_elems", "<u4"), ("table_id", "<u4"),
    ("tile_prefix", "<u4"), ("run_first_chunk", "<u4"), ("run_first_tile", "<u4"), ("run_end_tile", "<u4"),
    ("tiles_per_chunk", "<u4"), ("max_record_bytes", "<u4"), ("reserved", "<u4")], align=True)
assert CHUNK_DESC_DTYPE.itemsize == 80
TABLE_BYTES = 256

class CompressedExperts(ctypes.Structure):
    _fields_ = [("n_experts", _u32), ("hidden", _u32), ("inter", _u32), ("n_chunks", _u32), ("chunks", _vp),
                ("tensor_first_chunk", _vp), ("tables", _vp), ("n_tables", _u32), ("reserved", _u32),
                ("payload", _vp), ("payload_bytes", _u64), ("sm", _vp), ("sm_bytes", _u64)]


_lib.zipmoe_version.restype = _u32
_lib.zipmoe_status_string.restype = ctypes.c_char_p
_lib.zipmoe_status_string.argtypes = [_int]
_lib.zipmoe_encode_bound.argtypes = [_u64, _u64, ctypes.POINTER(EncodeOpts), ctypes.POINTER(_u64)]
_lib.zipmoe_encode.argtypes = [_vp, _u64, _u64, ctypes.POINTER(EncodeOpts), _vp, _u64, ctypes.POINTER(_u64)]
_lib.zipmoe_blob_info_get.argtypes = [_vp, _u64, ctypes.POINTER(BlobInfo)]
_lib.zipmoe_blob_validate.argtypes = [_vp, _u64]
_lib.zipmoe_blob_plan.argtypes = [_vp, _u64, _u64, _u64, _u64, _u32, _u32, _u32, _vp, _vp]
_lib.zipmoe_decode.argtypes = [_vp, _u32, _u32, _vp, _u32, _vp, _u64, _vp, _u64, _vp, _u64, _vp, _vp, _u32, _u32]
_lib.zipmoe_recover.argtypes = [_vp, _vp, _u64, _vp, _vp]
_lib.zipmoe_recover.restype = _int
_lib.zipmoe_ffn_workspace_bytes.argtypes = [_u32, _u32, ctypes.POINTER(CompressedExperts), ctypes.POINTER(_u64)]
_lib.zipmoe_decode_expert_ffn.argtypes = [_vp, _u32, _vp, _vp, _u32, ctypes.POINTER(CompressedExperts), _vp, _vp, _u64,
                                          _vp, _vp]
_lib.zipmoe_decode_expert_ffn_noalloc.argtypes = [_vp, _u32, _vp, _vp, _u32, ctypes.POINTER(CompressedExperts), _vp, _vp,
                                                  _vp]
_lib.zipmoe_decode_expert_ffn_noalloc.restype = _int
NOALLOC_SCRATCH_BYTES = 8 << 20
for _f in ("zipmoe_ffn_workspace_bytes", "zipmoe_decode_expert_ffn", "zipmoe_encode_bound", "zipmoe_encode", "zipmoe_blob_info_get", "zipmoe_blob_validate",
           "zipmoe_blob_plan", "zipmoe_decode"):
    getattr(_lib, _f).restype = _int


class ZipMoEError(RuntimeError):
    def __init__(self, where, status):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, zipmoe_status_string(status), status))


def _check(where, status):
    if status != OK:
        raise ZipMoEError(where, status)


def _ptr(a):
    """Address of a numpy array, a torch tensor, an int, or None."""
    if a is None:
        return None
    if isinstance(a, int):
        return a
    if isinstance(a, np.ndarray):
        return a.ctypes.data
    return a.data_ptr()


_lib.zipmoe_test_wait_fault.argtypes = [_u32, _u32]
_lib.zipmoe_test_wait_fault.restype = None


def zipmoe_test_wait_fault(extra_tx_bytes, tries):
    """Test switch: record barriers armed for extra_tx_bytes too many, waits limited to `tries`; (0, 0) = normal."""
    _lib.zipmoe_test_wait_fault(int(extra_tx_bytes), int(tries))


_lib.zipmoe_test_foreign_counter.argtypes = [_u32]
_lib.zipmoe_test_foreign_counter.restype = None


def zipmoe_test_foreign_counter(on):
    """Test switch: dynamically distributed launches find another launch's tag in their work counter; 0 = normal."""
    _lib.zipmoe_test_foreign_counter(int(on))


def zipmoe_version():
    return int(_lib.zipmoe_version())


def zipmoe_status_string(status):
    return _lib.zipmoe_status_string(int(status)).decode()


def _opts(chunk_elems, max_code_len, layout, n_threads):
    return EncodeOpts(int(chunk_elems), int(max_code_len), int(layout), int(n_threads))


def zipmoe_encode_bound(rows, cols, chunk_elems=0, max_code_len=0, layout=LAYOUT_LINEAR, n_threads=0):
    out = _u64(0)
    o = _opts(chunk_elems, max_code_len, layout, n_threads)
    _check("zipmoe_encode_bound", _lib.zipmoe_encode_bound(rows, cols, ctypes.byref(o), ctypes.byref(out)))
    return out.value


def zipmoe_encode(bf16, rows=None, cols=None, chunk_elems=0, max_code_len=0, layout=LAYOUT_LINEAR, n_threads=0):
    """bf16 bit patterns (numpy uint16, row-major) -> blob (numpy uint8)."""
    x = np.ascontiguousarray(bf16, dtype=np.uint16)
    if rows is None:
        rows, cols = (x.shape if x.ndim == 2 else (1, x.size))
    if rows * cols != x.size:
        raise ValueError("rows * cols != number of elements")
    cap = zipmoe_encode_bound(rows, cols, chunk_elems, max_code_len, layout, n_threads)
    blob = np.empty(cap, np.uint8)
    n = _u64(0)
    o = _opts(chunk_elems, max_code_len, layout, n_threads)
    _check("zipmoe_encode", _lib.zipmoe_encode(_ptr(x), rows, cols, ctypes.byref(o), _ptr(blob), cap, ctypes.byref(n)))
    return blob[: n.value].copy()


def zipmoe_blob_info_get(blob):
    blob = np.ascontiguousarray(blob, dtype=np.uint8)
    info = BlobInfo()
    _check("zipmoe_blob_info_get", _lib.zipmoe_blob_info_get(_ptr(blob), blob.size, ctypes.byref(info)))
    return info


def zipmoe_blob_validate(blob):
    blob = np.ascontiguousarray(blob, dtype=np.uint8)
    return int(_lib.zipmoe_blob_validate(_ptr(blob), blob.size))


def zipmoe_blob_plan(blob, payload_base, sm_base, out_base, table_id, chunk_base, tile_base):
    """Returns (descs: numpy structured array [n_chunks], table: numpy uint8 [256])."""
    blob = np.ascontiguousarray(blob, dtype=np.uint8)
    info = zipmoe_blob_info_get(blob)
    descs = np.zeros(info.n_chunks, CHUNK_DESC_DTYPE)
    table = np.zeros(TABLE_BYTES, np.uint8)
    _check("zipmoe_blob_plan", _lib.zipmoe_blob_plan(_ptr(blob), blob.size, payload_base, sm_base, out_base, table_id,
                                                     chunk_base, tile_base, _ptr(descs), _ptr(table)))
    return descs, table


def zipmoe_decode(chunks, n_chunks, n_tiles, tables, n_tables, payload, payload_bytes, sm, sm_bytes, out_bf16,
                  out_elems, status_word=None, stream=None, max_record_bytes=0, flags=0):
    """All pointer arguments are device tensors (or raw device addresses)."""
    _check("zipmoe_decode", _lib.zipmoe_decode(_ptr(chunks), n_chunks, n_tiles, _ptr(tables), n_tables, _ptr(payload),
                                                payload_bytes, _ptr(sm), sm_bytes, _ptr(out_bf16), out_elems,
                                                _ptr(status_word), _ptr(stream), int(max_record_bytes), int(flags)))


def zipmoe_recover(exp, sm, n_elems, out_bf16, stream=None):
    """Merge decompressed exponent bytes and sign+mantissa bytes (device tensors) into bf16."""
    _check("zipmoe_recover", _lib.zipmoe_recover(_ptr(exp), _ptr(sm), n_elems, _ptr(out_bf16), _ptr(stream)))


# ---- cache-pool planning (host only) ------------------------------------------------------------
class PlanCosts(ctypes.Structure):
    """zipmoe_plan_costs: delays c (decompress one E-chunk), v (read one E-chunk), u (read one SM-chunk),
    L decompression workers, K E-chunks per tensor, n_tensors per expert."""
    _fields_ = [("c", ctypes.c_double), ("v", ctypes.c_double), ("u", ctypes.c_double), ("L", _u32), ("K", _u32),
                ("n_tensors", _u32)]


_dp = ctypes.POINTER(ctypes.c_double)
_lib.zipmoe_plan_hit_distribution.argtypes = [_dp, _u32, _dp]
_lib.zipmoe_plan_selection_probs.argtypes = [_dp, _u32, _u32, _u32, ctypes.c_double, _dp, ctypes.POINTER(_u32)]
_lib.zipmoe_plan_makespan.argtypes = [_u32, ctypes.POINTER(_u32), ctypes.POINTER(PlanCosts), _dp]
_lib.zipmoe_plan_expected_makespan.argtypes = [_dp, _u32, _u32, ctypes.POINTER(_u32), ctypes.POINTER(PlanCosts), _dp]
_lib.zipmoe_plan_cache_pools.argtypes = [_dp, _u32, _u32, _u32, ctypes.c_double, _dp, ctypes.POINTER(PlanCosts),
                                         ctypes.c_double, _dp, ctypes.POINTER(_u32), _dp]
for _f in ("zipmoe_plan_hit_distribution", "zipmoe_plan_selection_probs", "zipmoe_plan_makespan",
           "zipmoe_plan_expected_makespan", "zipmoe_plan_cache_pools"):
    getattr(_lib, _f).restype = _int


def _dbl(a):
    a = np.ascontiguousarray(a, dtype=np.float64)
    return a, a.ctypes.data_as(_dp)


def _u32x4(v):
    return (_u32 * 4)(*[int(x) for x in v])


def zipmoe_plan_hit_distribution(q):
    q, qp = _dbl(q)
    phi = np.zeros(q.size + 1)
    _check("zipmoe_plan_hit_distribution", _lib.zipmoe_plan_hit_distribution(qp, q.size, phi.ctypes.data_as(_dp)))
    return phi


def zipmoe_plan_selection_probs(f, k, max_iters=1000, tol=1e-12):
    f, fp = _dbl(f)
    q = np.zeros(f.size)
    it = _u32(0)
    _check("zipmoe_plan_selection_probs",
           _lib.zipmoe_plan_selection_probs(fp, f.size, k, max_iters, tol, q.ctypes.data_as(_dp), ctypes.byref(it)))
    return q, int(it.value)


def zipmoe_plan_makespan(k, hits, costs):
    out = ctypes.c_double(0)
    _check("zipmoe_plan_makespan", _lib.zipmoe_plan_makespan(k, _u32x4(hits), ctypes.byref(costs), ctypes.byref(out)))
    return out.value


def zipmoe_plan_expected_makespan(q, k, capacity, costs):
    q, qp = _dbl(q)
    out = ctypes.c_double(0)
    _check("zipmoe_plan_expected_makespan",
           _lib.zipmoe_plan_expected_makespan(qp, q.size, k, _u32x4(capacity), ctypes.byref(costs), ctypes.byref(out)))
    return out.value


def zipmoe_plan_cache_pools(f, k, pool_mask, budget, expert_size, costs, step):
    """Returns (ratios[4], capacity[4], expected makespan)."""
    f, fp = _dbl(f)
    size, sp = _dbl(expert_size)
    ratios = np.zeros(4)
    cap = (_u32 * 4)()
    out = ctypes.c_double(0)
    _check("zipmoe_plan_cache_pools",
           _lib.zipmoe_plan_cache_pools(fp, f.size, k, pool_mask, budget, sp, ctypes.byref(costs), step,
                                        ratios.ctypes.data_as(_dp), cap, ctypes.byref(out)))
    return ratios, [int(c) for c in cap], out.value


# ---- cache-affinity scheduling (host only) --------------------------------------------------------
class SchedTask(ctypes.Structure):
    _fields_ = [("expert", _u32), ("state", _u32)]


class SchedCosts(ctypes.Structure):
    _fields_ = [("c", ctypes.c_double), ("u", ctypes.c_double), ("rho", ctypes.c_double), ("K", _u32), ("L", _u32)]


SCHED_STATES = {"M": 0, "C": 1, "S": 2, "E": 3}
_lib.zipmoe_plan_simulate.argtypes = [ctypes.POINTER(SchedTask), _u32, _dp, _u32, ctypes.POINTER(SchedCosts),
                                      ctypes.POINTER(_u32), ctypes.POINTER(_u32), _dp, _dp]
_lib.zipmoe_plan_schedule.argtypes = [ctypes.POINTER(SchedTask), _u32, _dp, _u32, ctypes.POINTER(SchedCosts),
                                      ctypes.POINTER(_u32), ctypes.POINTER(_u32), ctypes.POINTER(_u32), _dp]
_lib.zipmoe_plan_simulate.restype = _int
_lib.zipmoe_plan_schedule.restype = _int


def _sched_args(tasks, p, costs):
    arr = (SchedTask * len(tasks))(*[SchedTask(int(n), SCHED_STATES[s] if isinstance(s, str) else int(s)) for n, s in tasks])
    pv, pp = _dbl(p)
    return arr, pv, pp, SchedCosts(*costs)


def zipmoe_plan_simulate(tasks, p, costs, blocks):
    """tasks: [(expert, state)], p: expert times, costs: (c, u, rho, K, L), blocks: lists of task indices.
    Returns (makespan, charge)."""
    arr, pv, pp, cs = _sched_args(tasks, p, costs)
    order = [j for B in blocks for j in B]
    block_of = [b for b, B in enumerate(blocks) for _ in B]
    n = len(tasks)
    mk, ch = ctypes.c_double(0), ctypes.c_double(0)
    _check("zipmoe_plan_simulate",
           _lib.zipmoe_plan_simulate(arr, n, pp, pv.size, ctypes.byref(cs), (_u32 * n)(*order), (_u32 * n)(*block_of),
                                     ctypes.byref(mk), ctypes.byref(ch)))
    return mk.value, ch.value


def zipmoe_plan_schedule(tasks, p, costs):
    """Returns (blocks: lists of task indices in priority order, makespan)."""
    arr, pv, pp, cs = _sched_args(tasks, p, costs)
    n = len(tasks)
    order, block_of, nb, mk = (_u32 * n)(), (_u32 * n)(), _u32(0), ctypes.c_double(0)
    _check("zipmoe_plan_schedule",
           _lib.zipmoe_plan_schedule(arr, n, pp, pv.size, ctypes.byref(cs), order, block_of, ctypes.byref(nb),
                                     ctypes.byref(mk)))
    blocks = [[] for _ in range(nb.value)]
    for j, b in zip(order, block_of):
        blocks[b].append(int(j))
    return blocks, mk.value


def zipmoe_ffn_workspace_bytes(T, k, experts):
    out = _u64(0)
    _check("zipmoe_ffn_workspace_bytes", _lib.zipmoe_ffn_workspace_bytes(T, k, ctypes.byref(experts), ctypes.byref(out)))
    return out.value


def zipmoe_decode_expert_ffn(tokens, T, topk_ids, topk_weights, k, experts, out, workspace, workspace_bytes,
                             status_word=None, stream=None):
    """Pointer arguments are device tensors (or raw device addresses); `experts` is a CompressedExperts."""
    _check("zipmoe_decode_expert_ffn",
           _lib.zipmoe_decode_expert_ffn(_ptr(tokens), T, _ptr(topk_ids), _ptr(topk_weights), k, ctypes.byref(experts),
                                         _ptr(out), _ptr(workspace), workspace_bytes, _ptr(status_word), _ptr(stream)))


def zipmoe_decode_expert_ffn_noalloc(tokens, T, topk_ids, topk_weights, k, experts, out, status_word=None, stream=None):
    """zipmoe_decode_expert_ffn without a workspace argument: the library's built-in scratch is used, so the
    caller (and this binding) allocates nothing.  Raises ZipMoEError(ERR_BUFFER_TOO_SMALL) when the call needs
    more than NOALLOC_SCRATCH_BYTES of scratch."""
    _check("zipmoe_decode_expert_ffn_noalloc",
           _lib.zipmoe_decode_expert_ffn_noalloc(_ptr(tokens), T, _ptr(topk_ids), _ptr(topk_weights), k,
                                                 ctypes.byref(experts), _ptr(out), _ptr(status_word), _ptr(stream)))


# ---- the rest of the expert sublayer: norm, router, experts that are already recovered --------------------
NORM_RESIDUAL_F32 = 1       # zipmoe_add_rmsnorm flag: residual and residual_out are fp32
ROUTE_SOFTMAX_ALL = 1       # zipmoe_route flag: weights are not renormalised over the chosen experts
RESIDENT_ENTRY_BYTES = 384


class ResidentExpertsStruct(ctypes.Structure):
    """zipmoe_resident_experts."""
    _fields_ = [("n_experts", _u32), ("hidden", _u32), ("inter", _u32), ("even", _u32), ("table", _vp), ("maps", ctypes.c_uint8 * 1152),
                ("grid", _u32), ("reserved", _u32)]


# zipmoe_norm_args and zipmoe_route_args, packed in one go (a call with one pointer costs a sixth of one with 17 arguments)
_NORM_ARGS = struct.Struct("<11Q4IfI")
_ROUTE_ARGS = struct.Struct("<8Q6I")
assert _NORM_ARGS.size == 112 and _ROUTE_ARGS.size == 88
_lib.zipmoe_add_rmsnorm.argtypes = [ctypes.c_char_p, _vp]
_lib.zipmoe_route.argtypes = [ctypes.c_char_p, _vp]
_lib.zipmoe_resident_experts_plan.argtypes = [ctypes.POINTER(_vp), _u32, _u32, _u32, _vp, ctypes.POINTER(ResidentExpertsStruct)]
_lib.zipmoe_expert_ffn_workspace_bytes.argtypes = [_u32, _u32, ctypes.POINTER(ResidentExpertsStruct), ctypes.POINTER(_u64)]
_lib.zipmoe_expert_ffn_workspace_init.argtypes = [_vp, _u64, _vp]
_lib.zipmoe_expert_ffn_workspace_init.restype = _int
_lib.zipmoe_stream_capture_id.argtypes = [_vp, ctypes.POINTER(_u64)]
_lib.zipmoe_stream_capture_id.restype = _int
_lib.zipmoe_expert_ffn.argtypes = [_vp, _u32, _vp, _vp, _u32, ctypes.POINTER(ResidentExpertsStruct), _vp, _vp, _u64, _vp, _vp]
for _f in ("zipmoe_add_rmsnorm", "zipmoe_route", "zipmoe_resident_experts_plan", "zipmoe_expert_ffn_workspace_bytes",
           "zipmoe_expert_ffn"):
    getattr(_lib, _f).restype = _int


def zipmoe_add_rmsnorm(x, x_pitch, residual, residual_pitch, residual_out, residual_out_pitch, weight, rows, cols, eps, out,
                       out_q, out_pitch, scales=None, group=0, flags=0, stream=None):
    """Pointer arguments are device tensors (or raw device addresses, or None); pitches in elements."""
    args = _NORM_ARGS.pack(_ptr(x) or 0, x_pitch, _ptr(residual) or 0, residual_pitch, _ptr(residual_out) or 0,
                           residual_out_pitch, _ptr(weight) or 0, _ptr(out) or 0, _ptr(out_q) or 0, out_pitch,
                           _ptr(scales) or 0, rows, cols, group, flags, eps, 0)
    _check("zipmoe_add_rmsnorm", _lib.zipmoe_add_rmsnorm(args, _ptr(stream)))


def zipmoe_route(tokens, T, token_pitch, gate, n_experts, hidden, bias, k, flags, topk_ids, topk_weights, logits=None,
                 status_word=None, stream=None):
    """Pointer arguments are device tensors (or raw device addresses, or None)."""
    args = _ROUTE_ARGS.pack(_ptr(tokens) or 0, token_pitch, _ptr(gate) or 0, _ptr(bias) or 0, _ptr(topk_ids) or 0,
                            _ptr(topk_weights) or 0, _ptr(logits) or 0, _ptr(status_word) or 0, T, n_experts, hidden, k, flags, 0)
    _check("zipmoe_route", _lib.zipmoe_route(args, _ptr(stream)))


def zipmoe_resident_experts_plan(tensors, n_experts, hidden, inter):
    """tensors: 3 * n_experts device tensors (or addresses).  Returns (table: numpy uint8, to be copied to the device;
    ResidentExpertsStruct, whose `table` is then to be set to that copy's address)."""
    if len(tensors) != 3 * n_experts:
        raise ValueError("three tensors per expert are wanted")
    ptrs = (_vp * max(len(tensors), 1))(*[_ptr(t) for t in tensors])
    table = np.zeros(3 * n_experts * RESIDENT_ENTRY_BYTES, np.uint8)
    experts = ResidentExpertsStruct()
    _check("zipmoe_resident_experts_plan",
           _lib.zipmoe_resident_experts_plan(ptrs, n_experts, hidden, inter, _ptr(table), ctypes.byref(experts)))
    return table, experts


def zipmoe_expert_ffn_workspace_bytes(T, k, experts):
    out = _u64(0)
    _check("zipmoe_expert_ffn_workspace_bytes",
           _lib.zipmoe_expert_ffn_workspace_bytes(T, k, ctypes.byref(experts), ctypes.byref(out)))
    return out.value


def zipmoe_expert_ffn_workspace_init(workspace, workspace_bytes, stream=None):
    """Prepares a new device workspace; once, before its first zipmoe_expert_ffn."""
    _check("zipmoe_expert_ffn_workspace_init",
           _lib.zipmoe_expert_ffn_workspace_init(_ptr(workspace), workspace_bytes, _ptr(stream)))


def zipmoe_stream_capture_id(stream):
    """0, or the number of the capture that `stream` (a raw handle) takes part in."""
    out = _u64(0)
    _check("zipmoe_stream_capture_id", _lib.zipmoe_stream_capture_id(_ptr(stream), ctypes.byref(out)))
    return out.value


def zipmoe_expert_ffn(tokens, T, topk_ids, topk_weights, k, experts, out, workspace, workspace_bytes, status_word=None,
                      stream=None):
    """Pointer arguments are device tensors (or raw device addresses); `experts` is a ResidentExpertsStruct."""
    _check("zipmoe_expert_ffn",
           _lib.zipmoe_expert_ffn(_ptr(tokens), T, _ptr(topk_ids), _ptr(topk_weights), k, ctypes.byref(experts), _ptr(out),
                                  _ptr(workspace), workspace_bytes, _ptr(status_word), _ptr(stream)))


# ---- the experts' products for prompts, and products in 8-bit integers -----------------------------------
GROUPED_PAIR, GROUPED_INT8, GROUPED_F32 = 1, 2, 4
GROUPED_ENTRY_BYTES = 512


class GroupedWeightsStruct(ctypes.Structure):
    """zipmoe_grouped_weights."""
    _fields_ = [("n_groups", _u32), ("rows", _u32), ("cols", _u32), ("flags", _u32), ("even", _u32), ("reserved", _u32),
                ("table", _vp), ("maps", ctypes.c_uint8 * 512)]


# zipmoe_group_args, zipmoe_grouped_args, zipmoe_combine_args and zipmoe_linear_args
_GROUP_ARGS = struct.Struct("<5Q4I")
_GROUPED_ARGS = struct.Struct("<11Q6I")
_COMBINE_ARGS = struct.Struct("<7Q6I")
_LINEAR_ARGS = struct.Struct("<8Q2IQ")
assert _GROUP_ARGS.size == 56 and _GROUPED_ARGS.size == 112 and _COMBINE_ARGS.size == 80 and _LINEAR_ARGS.size == 80
_lib.zipmoe_group_tokens.argtypes = [ctypes.c_char_p, _vp]
_lib.zipmoe_grouped_weights_plan.argtypes = [ctypes.POINTER(_vp), _u32, _u32, _u32, _u32, _vp, ctypes.POINTER(GroupedWeightsStruct)]
_lib.zipmoe_grouped_matmul.argtypes = [ctypes.POINTER(GroupedWeightsStruct), ctypes.c_char_p, _vp]
_lib.zipmoe_grouped_workspace_bytes.argtypes = [ctypes.POINTER(GroupedWeightsStruct), _u32, _u32, ctypes.POINTER(_u64)]
_lib.zipmoe_grouped_workspace_bytes.restype = _int
_lib.zipmoe_combine_rows.argtypes = [ctypes.c_char_p, _vp]
_lib.zipmoe_linear_int8_workspace_bytes.argtypes = [ctypes.POINTER(GroupedWeightsStruct), _u32, ctypes.POINTER(_u64)]
_lib.zipmoe_linear_int8.argtypes = [ctypes.POINTER(GroupedWeightsStruct), ctypes.c_char_p, _vp]
_lib.zipmoe_linear_int8_workspace_bytes.restype = _lib.zipmoe_linear_int8.restype = _int
_lib.zipmoe_quantize_rows.argtypes = [_vp, _u64, _u32, _u32, _vp, _u64, _vp, _vp]
for _f in ("zipmoe_group_tokens", "zipmoe_grouped_weights_plan", "zipmoe_grouped_matmul", "zipmoe_combine_rows", "zipmoe_quantize_rows"):
    getattr(_lib, _f).restype = _int


_lib.zipmoe_test_grouped_kernel.argtypes = [_u32]
_lib.zipmoe_test_grouped_kernel.restype = None


def zipmoe_test_grouped_kernel(which):
    """Test switch: 1 zipmoe_grouped_matmul's kernel for few tokens, 2 the one for many, 0 normal."""
    _lib.zipmoe_test_grouped_kernel(int(which))


def zipmoe_group_tokens(topk_ids, T, k, n_experts, offsets, order, place=None, status_word=None, stream=None):
    """Pointer arguments are device tensors (or raw device addresses, or None)."""
    args = _GROUP_ARGS.pack(_ptr(topk_ids) or 0, _ptr(offsets) or 0, _ptr(order) or 0, _ptr(place) or 0, _ptr(status_word) or 0, T, k,
                            n_experts, 0)
    _check("zipmoe_group_tokens", _lib.zipmoe_group_tokens(args, _ptr(stream)))


def zipmoe_grouped_weights_plan(tensors, n_groups, rows, cols, flags=0):
    """tensors: n_groups device tensors (or addresses), 2 * n_groups with GROUPED_PAIR.  Returns (table: numpy uint8, to be
    copied to the device unless the struct's `even` is 1; GroupedWeightsStruct, whose `table` is then to be set to that copy's
    address)."""
    if len(tensors) != (2 if flags & GROUPED_PAIR else 1) * n_groups:
        raise ValueError("a tensor per group, or two of a pair, are wanted")
    ptrs = (_vp * max(len(tensors), 1))(*[_ptr(t) for t in tensors])
    table = np.zeros(n_groups * GROUPED_ENTRY_BYTES, np.uint8)
    weights = GroupedWeightsStruct()
    _check("zipmoe_grouped_weights_plan",
           _lib.zipmoe_grouped_weights_plan(ptrs, n_groups, rows, cols, flags, _ptr(table), ctypes.byref(weights)))
    return table, weights


def zipmoe_grouped_workspace_bytes(weights, rows, gathered):
    out = _u64(0)
    _check("zipmoe_grouped_workspace_bytes",
           _lib.zipmoe_grouped_workspace_bytes(ctypes.byref(weights), rows, int(gathered), ctypes.byref(out)))
    return out.value


def zipmoe_grouped_matmul(weights, x, x_pitch, x_rows, out, out_pitch, rows, offsets=None, order=None, k=0, row_scales=None,
                          col_scales=None, flags=0, workspace=None, workspace_bytes=0, status_word=None, stream=None):
    """Pointer arguments are device tensors (or raw device addresses, or None); `weights` is a GroupedWeightsStruct."""
    args = _GROUPED_ARGS.pack(_ptr(x) or 0, x_pitch, _ptr(offsets) or 0, _ptr(order) or 0, _ptr(row_scales) or 0, _ptr(col_scales) or 0,
                              _ptr(out) or 0, out_pitch, _ptr(status_word) or 0, _ptr(workspace) or 0, workspace_bytes, x_rows, rows, k,
                              flags, 0, 0)
    _check("zipmoe_grouped_matmul", _lib.zipmoe_grouped_matmul(ctypes.byref(weights), args, _ptr(stream)))


def zipmoe_combine_rows(y, y_pitch, rows, place, weights, T, k, cols, out, out_pitch, flags=0, status_word=None, stream=None):
    """Pointer arguments are device tensors (or raw device addresses, or None)."""
    args = _COMBINE_ARGS.pack(_ptr(y) or 0, y_pitch, _ptr(place) or 0, _ptr(weights) or 0, _ptr(out) or 0, out_pitch,
                              _ptr(status_word) or 0, T, k, cols, rows, flags, 0)
    _check("zipmoe_combine_rows", _lib.zipmoe_combine_rows(args, _ptr(stream)))


def zipmoe_quantize_rows(x, x_pitch, rows, cols, q, q_pitch, scales, stream=None):
    """Pointer arguments are device tensors (or raw device addresses); pitches in elements."""
    _check("zipmoe_quantize_rows",
           _lib.zipmoe_quantize_rows(_ptr(x), x_pitch, rows, cols, _ptr(q), q_pitch, _ptr(scales), _ptr(stream)))


def zipmoe_linear_int8_workspace_bytes(weights, rows):
    out = _u64(0)
    _check("zipmoe_linear_int8_workspace_bytes", _lib.zipmoe_linear_int8_workspace_bytes(ctypes.byref(weights), rows, ctypes.byref(out)))
    return out.value


def zipmoe_linear_int8(weights, x, x_pitch, rows, col_scales, out, out_pitch, workspace, workspace_bytes, flags=0, status_word=None,
                       stream=None):
    """Pointer arguments are device tensors (or raw device addresses, or None); `weights` is a GroupedWeightsStruct."""
    args = _LINEAR_ARGS.pack(_ptr(x) or 0, x_pitch, _ptr(col_scales) or 0, _ptr(out) or 0, out_pitch, _ptr(workspace) or 0,
                             workspace_bytes, _ptr(status_word) or 0, rows, flags, 0)
    _check("zipmoe_linear_int8", _lib.zipmoe_linear_int8(ctypes.byref(weights), args, _ptr(stream)))


class LaunchInfo(ctypes.Structure):
    _fields_ = [("payload_bytes", _u64), ("sm_bytes", _u64), ("out_elems", _u64), ("n_chunks", _u32), ("n_tiles", _u32),
                ("n_tables", _u32), ("max_record_bytes", _u32), ("max_code_len", _u32), ("flags", _u32)]


_lib.zipmoe_launch_plan_size.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_u64), _u32, ctypes.POINTER(LaunchInfo)]
_lib.zipmoe_launch_plan.argtypes = [ctypes.POINTER(_vp), ctypes.POINTER(_u64), _u32, _vp, _vp, _vp, _vp, _vp, _vp,
                                    ctypes.POINTER(LaunchInfo)]
_lib.zipmoe_launch_plan_size.restype = _int
_lib.zipmoe_launch_plan.restype = _int


class DecodePlan:
    """One decode launch over several blobs, as zipmoe_launch_plan lays it out: the three contiguous host
    buffers, the chunk descriptors and the tables.  Marshalling only: the layout is the library's."""

    def __init__(self, blobs):
        blobs = [np.ascontiguousarray(b, dtype=np.uint8) for b in blobs]
        n = len(blobs)
        ptrs = (_vp * max(n, 1))(*[b.ctypes.data for b in blobs])
        sizes = (_u64 * max(n, 1))(*[b.size for b in blobs])
        info = LaunchInfo()
        _check("zipmoe_launch_plan_size", _lib.zipmoe_launch_plan_size(ptrs, sizes, n, ctypes.byref(info)))
        self.payload = np.empty(info.payload_bytes + DEVICE_PAD_BYTES, np.uint8)
        self.sm = np.empty(info.sm_bytes + DEVICE_PAD_BYTES, np.uint8)
        self.descs = np.zeros(info.n_chunks, CHUNK_DESC_DTYPE)
        self.tables = np.zeros(n * TABLE_BYTES, np.uint8)
        self.tensor_first_chunk = np.zeros(n, np.uint32)
        out_base = np.zeros(n, np.uint64)
        _check("zipmoe_launch_plan",
               _lib.zipmoe_launch_plan(ptrs, sizes, n, _ptr(self.payload), _ptr(self.sm), _ptr(self.descs),
                                       _ptr(self.tables), _ptr(self.tensor_first_chunk), _ptr(out_base), ctypes.byref(info)))
        self.infos = [zipmoe_blob_info_get(b) for b in blobs]
        self.out_base = [int(v) for v in out_base]
        self.payload_base = [int(self.descs["payload_off"][int(c)]) if inf.n_chunks else 0
                             for c, inf in zip(self.tensor_first_chunk, self.infos)]
        self.sm_base = [int(self.descs["sm_off"][int(c)]) if inf.n_chunks else 0
                        for c, inf in zip(self.tensor_first_chunk, self.infos)]
        self.payload_bytes, self.sm_bytes, self.out_elems = info.payload_bytes, info.sm_bytes, info.out_elems
        self.n_chunks, self.n_tiles, self.n_tables = info.n_chunks, info.n_tiles, info.n_tables
        self.max_record_bytes, self.max_code_len, self.flags = info.max_record_bytes, info.max_code_len, info.flags

    def algorithmic_bytes(self):
        """Bytes one decode must move: E-chunk section + SM bytes read, bf16 written."""
        n = sum(inf.n_elems for inf in self.infos)
        return self.payload_bytes + n + 2 * n

    def to_device(self, device="cuda"):
        import torch
        return DevicePlan(self, torch.device(device))

    def tensor_slice(self, out, i):
        inf = self.infos[i]
        return out[self.out_base[i]: self.out_base[i] + inf.n_elems]


class DevicePlan:
    """Device copies of a DecodePlan's buffers (torch owns the memory)."""

    def __init__(self, plan, device):
        import torch
        self.plan = plan
        self.device = device
        self.descs = torch.from_numpy(plan.descs.view(np.uint8).copy()).to(device)
        self.tables = torch.from_numpy(plan.tables).to(device)
        self.payload = torch.from_numpy(plan.payload).to(device)
        self.sm = torch.from_numpy(plan.sm).to(device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def new_output(self):
        import torch
        return torch.zeros(self.plan.out_elems, dtype=torch.int16, device=self.device)

    def decode(self, out, stream=None):
        """One zipmoe_decode launch on `stream` (a torch stream or None = current)."""
        import torch
        p = self.plan
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        zipmoe_decode(self.descs, p.n_chunks, p.n_tiles, self.tables, p.n_tables, self.payload, p.payload_bytes,
                      self.sm, p.sm_bytes, out, p.out_elems, self.status, s.cuda_stream, p.max_record_bytes, p.flags)


def pad_expert_inter(w1, w3, w2, multiple=256):
    """The fused expert FFN takes experts whose hidden and intermediate sizes are multiples of 256.  An expert with
    another intermediate size (w1, w3 [inter, hidden]; w2 [hidden, inter], uint16 bf16 patterns) is padded with zero
    rows (w1, w3) and zero columns (w2) up to the next multiple: the added units compute SiLU(0) * 0 = 0 and feed
    zero weights, so the FFN's result is unchanged.  Returns (w1, w3, w2, padded inter)."""
    inter, hidden = w1.shape
    assert w3.shape == (inter, hidden) and w2.shape == (hidden, inter)
    padded = -(-inter // multiple) * multiple
    if padded == inter:
        return w1, w3, w2, inter
    a = np.zeros((padded, hidden), np.uint16)
    b = np.zeros((padded, hidden), np.uint16)
    c = np.zeros((hidden, padded), np.uint16)
    a[:inter], b[:inter], c[:, :inter] = w1, w3, w2
    return a, b, c, padded


class DeviceExperts:
    """The compressed experts of one layer on the device: blobs[3*e + j] (j: 0 w1, 1 w3, 2 w2, blocked
    layout) laid out by DecodePlan, plus the CompressedExperts struct the fused call takes."""

    def __init__(self, blobs, hidden, inter, device="cuda"):
        import torch
        assert len(blobs) % 3 == 0
        self.plan = DecodePlan(blobs)
        self.dev = self.plan.to_device(device)
        self.tensor_first_chunk = torch.from_numpy(self.plan.tensor_first_chunk.view(np.int32).copy()).to(self.dev.device)
        p, d = self.plan, self.dev
        self.struct = CompressedExperts(len(blobs) // 3, hidden, inter, p.n_chunks, d.descs.data_ptr(),
                                        self.tensor_first_chunk.data_ptr(), d.tables.data_ptr(), p.n_tables, 0,
                                        d.payload.data_ptr(), p.payload_bytes, d.sm.data_ptr(), p.sm_bytes)
        self.hidden, self.inter = hidden, inter
        self._ws = {}

    def ffn(self, tokens, topk_ids, topk_weights, out=None, stream=None):
        """tokens [T, hidden] int16 (bf16 patterns), topk_ids [T, k] int32, topk_weights [T, k] float32 or None:
        device tensors.  Returns out [T, hidden] int16."""
        import torch
        T, k = topk_ids.shape
        key = (T, k)
        if key not in self._ws:
            n = zipmoe_ffn_workspace_bytes(T, k, self.struct)
            self._ws[key] = torch.empty(n, dtype=torch.uint8, device=self.dev.device)
        ws = self._ws[key]
        if out is None:
            out = torch.empty(T, self.hidden, dtype=torch.int16, device=self.dev.device)
        s = torch.cuda.current_stream(self.dev.device) if stream is None else stream
        zipmoe_decode_expert_ffn(tokens, T, topk_ids, topk_weights, k, self.struct, out, ws, ws.numel(),
                                 self.dev.status, s.cuda_stream)
        return out


class _Kinds:
    """The torch types that hold a kind of element: bf16 values may come as int16 bit patterns, e4m3 as bytes."""

    def __init__(self):
        import torch
        self.bf16 = (torch.bfloat16, torch.int16, torch.uint16)
        self.e4m3 = (torch.float8_e4m3fn, torch.uint8)
        self.fp32 = (torch.float32,)
        self.int32 = (torch.int32,)
        self.int8 = (torch.int8,)
        self.current_stream = torch._C._cuda_getCurrentRawStream   # handle of a device's current stream
        self.capturing = torch._C._cuda_isCurrentStreamCapturing
        self.current_device = torch._C._cuda_getDevice


_kinds = None


def _get_kinds():
    global _kinds
    if _kinds is None:
        _kinds = _Kinds()
    return _kinds


def _empty(shape, dtype, device, stream):
    """New device memory for work on `stream` (None: the current one): it must come from that stream's own pool, or
    what was queued on another stream for its last user could still be running."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _refuse(name, t, shape, kinds, index, what):
    raise ValueError("%s: a %s tensor %s of %s on CUDA device %d is wanted, not %s of %s on %s (strides %s)" %
                     (name, what, shape, kinds[0], index, tuple(t.shape), t.dtype, t.device, t.stride()))


def _rows(name, t, shape, kinds, index):
    """Address and row pitch, in elements, of a tensor of this shape on device `index` whose rows are dense."""
    stride = t.stride()
    if t.shape != shape or t.dtype not in kinds or t.get_device() != index or (stride[1] != 1 and shape[1] > 1):
        _refuse(name, t, shape, kinds, index, "row by row dense")
    return t.data_ptr(), (stride[0] if shape[0] > 1 else shape[1])


def _dense(name, t, shape, kinds, index):
    """Address of a contiguous tensor of this shape on device `index`."""
    if t.shape != shape or t.dtype not in kinds or t.get_device() != index or not t.is_contiguous():
        _refuse(name, t, shape, kinds, index, "contiguous")
    return t.data_ptr()


def _device_of(name, t):
    index = t.get_device()
    if index < 0:
        raise ValueError("%s: a tensor on a CUDA device is wanted, not on %s" % (name, t.device))
    return index


def _on_device(index):
    """Context in which the tensors' device is the current one: the library launches on the current device, and the
    default stream has the same handle on all of them."""
    import torch
    return torch.cuda.device(index)


def _handle(kinds, index, stream):
    """Raw handle of a torch stream of device `index` (None: its current one)."""
    if stream is None:
        return kinds.current_stream(index)
    if stream.device_index != index:
        raise ValueError("a stream of CUDA device %d is wanted, not of device %d" % (index, stream.device_index))
    return stream.cuda_stream


class RmsNorm:
    """Residual addition and root-mean-square norm with one weight vector (bf16, or int16 bf16 patterns).  x and out are
    bf16 tensors or int16 patterns [rows, cols] whose rows may lie apart; the residual stream is of that kind or fp32."""

    def __init__(self, weight, eps=1e-6):
        self.kinds = _get_kinds()
        self.index = _device_of("weight", weight)
        self.weight, self.eps, self.cols = weight, float(eps), weight.numel()
        self.weight_at = _dense("weight", weight, (self.cols,), self.kinds.bf16, self.index)

    def n_groups(self, group):
        return 1 if group <= 0 or group >= self.cols else -(-self.cols // group)

    def _call(self, x, residual, residual_out, out, out_q, scales, group, stream):
        kinds, index, rows, cols = self.kinds, self.index, x.shape[0], self.cols
        if kinds.current_device() != index:
            with _on_device(index):
                return self._call(x, residual, residual_out, out, out_q, scales, group, stream)
        shape, bf16 = (rows, cols), kinds.bf16
        x_at, x_pitch = _rows("x", x, shape, bf16, index)
        res = res_out = res_pitch = res_out_pitch = flags = 0
        if residual is not None:
            of = bf16
            if residual.dtype not in bf16:
                of, flags = kinds.fp32, NORM_RESIDUAL_F32
            res, res_pitch = _rows("residual", residual, shape, of, index)
            if residual_out is not None:
                res_out, res_out_pitch = _rows("residual_out", residual_out, shape, of, index)
        elif residual_out is not None:
            raise ValueError("residual_out without a residual")
        out_at = q_at = scales_at = 0
        if out is not None:
            out_at, out_pitch = _rows("out", out, shape, bf16, index)
        if out_q is not None:
            q_at, q_pitch = _rows("out_q", out_q, shape, kinds.e4m3, index)
            if out is not None and out_pitch != q_pitch:
                raise ValueError("out and out_q have rows %d and %d apart" % (out_pitch, q_pitch))
            out_pitch = q_pitch
            scales_at = _dense("scales", scales, (rows, self.n_groups(group)), kinds.fp32, index)
        args = _NORM_ARGS.pack(x_at, x_pitch, res, res_pitch, res_out, res_out_pitch, self.weight_at, out_at, q_at, out_pitch, scales_at,
                               rows, cols, group if group > 0 else 0, flags, self.eps, 0)
        status = _lib.zipmoe_add_rmsnorm(args, _handle(kinds, index, stream))
        if status:
            raise ZipMoEError("zipmoe_add_rmsnorm", status)

    def add_norm(self, x, residual=None, residual_out=None, out=None, stream=None):
        """Returns out [rows, cols] (bf16); residual_out (may be `residual` itself) gets x + residual."""
        if out is None:
            out = _empty(x.shape, x.dtype, x.device, stream)
        self._call(x, residual, residual_out, out, None, None, 0, stream)
        return out

    def add_norm_8bit(self, x, residual=None, residual_out=None, out_q=None, scales=None, group=0, out=None, stream=None):
        """Returns (out_q [rows, cols] e4m3, scales [rows, groups] fp32); `out`, if given, gets the bf16 rows as well."""
        if out_q is None:
            out_q = _empty(x.shape, self.kinds.e4m3[0], x.device, stream)
        if scales is None:
            scales = _empty((x.shape[0], self.n_groups(group)), self.kinds.fp32[0], x.device, stream)
        self._call(x, residual, residual_out, out, out_q, scales, group, stream)
        return out_q, scales


class Router:
    """The router of one layer: gate [n_experts, hidden] (bf16, or int16 patterns), bias [n_experts] fp32 or None."""

    def __init__(self, gate, k, bias=None, renormalise=True):
        import torch
        self.kinds = _get_kinds()
        self.index = _device_of("gate", gate)
        self.n_experts, self.hidden = gate.shape
        self.gate, self.bias, self.k = gate, bias, int(k)
        self.gate_at = _dense("gate", gate, (self.n_experts, self.hidden), self.kinds.bf16, self.index)
        self.bias_at = 0 if bias is None else _dense("bias", bias, (self.n_experts,), self.kinds.fp32, self.index)
        self.flags = 0 if renormalise else ROUTE_SOFTMAX_ALL
        self.status = torch.zeros(1, dtype=torch.int32, device=gate.device)
        self.status_at = self.status.data_ptr()

    def route(self, tokens, ids=None, weights=None, logits=None, stream=None):
        """tokens [T, hidden] -> ids [T, k] int32, weights [T, k] fp32; logits, if given, gets [T, n_experts] fp32."""
        kinds, index, T = self.kinds, self.index, tokens.shape[0]
        if kinds.current_device() != index:
            with _on_device(index):
                return self.route(tokens, ids, weights, logits, stream)
        chosen = (T, self.k)
        tokens_at, pitch = _rows("tokens", tokens, (T, self.hidden), kinds.bf16, index)
        if ids is None:
            ids = _empty(chosen, kinds.int32[0], tokens.device, stream)
        if weights is None:
            weights = _empty(chosen, kinds.fp32[0], tokens.device, stream)
        ids_at = _dense("ids", ids, chosen, kinds.int32, index)
        weights_at = _dense("weights", weights, chosen, kinds.fp32, index)
        logits_at = 0 if logits is None else _dense("logits", logits, (T, self.n_experts), kinds.fp32, index)
        args = _ROUTE_ARGS.pack(tokens_at, pitch, self.gate_at, self.bias_at, ids_at, weights_at, logits_at, self.status_at, T,
                                self.n_experts, self.hidden, self.k, self.flags, 0)
        status = _lib.zipmoe_route(args, _handle(kinds, index, stream))
        if status:
            raise ZipMoEError("zipmoe_route", status)
        return ids, weights


class _Scratch:
    """The workspaces of zipmoe_expert_ffn on one device, shared by all layers there: one per stream, as large as the
    largest call so far (a call leaves its workspace ready for the next one, whatever the sizes of either), and, while a
    stream is being captured, one for that capture alone, which only the graph's replays prepare."""

    def __init__(self, device):
        self.kinds, self.device, self.lock = _get_kinds(), device, threading.Lock()
        self.own, self.captured = {}, {}      # stream handle -> workspace; stream handle -> (capture, workspace)

    def get(self, need, handle, stream):
        if (stream is not None or self.kinds.capturing()) and (capture := zipmoe_stream_capture_id(handle)):
            # its memory comes from the graph's pool, which lives as long as the graph: it is kept here for the rest of
            # the capture only
            with self.lock:
                of, ws = self.captured.get(handle, (0, None))
                if of != capture or ws.numel() < need:
                    ws = self._prepared(need, handle, stream)
                    self.captured[handle] = capture, ws
                return ws
        ws = self.own.get(handle)
        if ws is None or ws.numel() < need:
            with self.lock:
                ws = self.own.get(handle)
                if ws is None or ws.numel() < need:
                    self.own.pop(handle, None)      # back to the stream's pool: what is queued there comes before its next use
                    del ws
                    ws = self.own[handle] = self._prepared(need, handle, stream)
        return ws

    def _prepared(self, need, handle, stream):
        ws = _empty(need, self.kinds.e4m3[1], self.device, stream)
        zipmoe_expert_ffn_workspace_init(ws, need, handle)
        return ws


_scratch, _scratch_lock = weakref.WeakValueDictionary(), threading.Lock()


def _scratch_of(device, index):
    """The device's workspaces; they go with the last layer that holds them."""
    with _scratch_lock:
        found = _scratch.get(index)
        if found is None:
            found = _scratch[index] = _Scratch(device)
        return found


class ResidentExperts:
    """Recovered experts of one layer: tensors[3*e + j] (j: 0 w1 [inter, hidden], 1 w3, 2 w2 [hidden, inter]) are dense
    bf16 (or int16 pattern) device tensors of these shapes or flat, for example the slices of a DevicePlan.decode output."""

    def __init__(self, tensors, hidden, inter):
        import torch
        if len(tensors) % 3 or not tensors:
            raise ValueError("three tensors per expert are wanted")
        self.kinds = _get_kinds()
        self.index = _device_of("tensor 0", tensors[0])
        addresses = []
        for i, t in enumerate(tensors):
            shape = (hidden * inter,) if len(t.shape) == 1 else (hidden, inter) if i % 3 == 2 else (inter, hidden)
            addresses.append(_dense("tensor %d" % i, t, shape, self.kinds.bf16, self.index))
        self.tensors = list(tensors)      # the experts' memory is theirs: keep it while the table points at it
        self.device = tensors[0].device
        self.hidden, self.inter = hidden, inter
        with _on_device(self.index):
            table, self.struct = zipmoe_resident_experts_plan(addresses, len(tensors) // 3, hidden, inter)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.status_at = self.status.data_ptr()
        # calls may come on any stream: this copy from the host returns when it has arrived, and so have the zeros before it
        self.table = torch.from_numpy(table).to(self.device)
        self.struct.table = self.table.data_ptr()
        self._struct_at = ctypes.byref(self.struct)
        self._scratch, self._need = _scratch_of(self.device, self.index), {}
        self._prompt, self._prompt_lock = None, threading.Lock()

    @classmethod
    def from_decode(cls, plan, out, hidden, inter):
        """The experts that one decode launch recovered: `plan` a DecodePlan over 3 * n_experts blobs, `out` its output."""
        return cls([plan.tensor_slice(out, i) for i in range(len(plan.infos))], hidden, inter)

    def _workspace(self, T, k, handle, stream):
        """A workspace large enough for T tokens with k experts each."""
        need = self._need.get((T, k))
        if need is None:
            # some more tokens than asked for, in few steps: a workspace seldom grows
            fits = T if T > 256 else 256 if T > 128 else 1 << max(T - 1, 15).bit_length()
            need = self._need[(T, k)] = zipmoe_expert_ffn_workspace_bytes(fits, k, self.struct)
        return self._scratch.get(need, handle, stream)

    def ffn(self, tokens, topk_ids, topk_weights, out=None, stream=None):
        """tokens [T, hidden] bf16 (or int16 patterns), topk_ids [T, k] int32, topk_weights [T, k] float32 or None: device
        tensors.  Returns out [T, hidden].  Every stream has a workspace of its own, and so has every capture of a stream by
        torch.cuda.graph: calls on different streams, replays of different graphs and both may overlap, and no call has to
        come before a capture."""
        kinds, index = self.kinds, self.index
        if kinds.current_device() != index:
            with _on_device(index):
                return self.ffn(tokens, topk_ids, topk_weights, out, stream)
        T, k = chosen = topk_ids.shape
        shape = (T, self.hidden)
        tokens_at = _dense("tokens", tokens, shape, kinds.bf16, index)
        ids_at = _dense("topk_ids", topk_ids, chosen, kinds.int32, index)
        weights_at = None if topk_weights is None else _dense("topk_weights", topk_weights, chosen, kinds.fp32, index)
        if out is None:
            out = _empty(shape, tokens.dtype, self.device, stream)
        out_at = _dense("out", out, shape, kinds.bf16, index)
        handle = _handle(kinds, index, stream)
        ws = self._workspace(T, k, handle, stream)
        status = _lib.zipmoe_expert_ffn(tokens_at, T, ids_at, weights_at, k, self._struct_at, out_at, ws.data_ptr(), ws.numel(),
                                        self.status_at, handle)
        if status:
            raise ZipMoEError("zipmoe_expert_ffn", status)
        return out

    def ffn_prompt(self, tokens, topk_ids, topk_weights, out=None, stream=None):
        """What ffn computes, for any number of tokens: the choices are grouped by expert, every expert's tokens go through W1
        and W3 and then W2 as grouped products, and each token's rows are added.  The gated activations between the products are
        rounded to bf16, where ffn keeps 16 bits of them: outputs are 0.0023 to 0.0024 of their norm from the values in 64 bits,
        ffn's 0.0017.  tokens' rows may lie apart.  The lists, activations and rows between the calls are new memory of the
        stream's pool: calls on different streams and captures are independent of one another.  They come to T * k * (4 * hidden + 2 *
        inter) bytes (131072 tokens with eight experts each of 4096 x 1408: 20 GB): very long prompts are better given in pieces.
        An id of n_experts or more sets `status` to 1."""
        kinds, index = self.kinds, self.index
        if kinds.current_device() != index:
            with _on_device(index):
                return self.ffn_prompt(tokens, topk_ids, topk_weights, out, stream)
        gate_up, down = self._products()
        _rows("tokens", tokens, (topk_ids.shape[0], self.hidden), kinds.bf16, index)
        if topk_weights is not None:
            _dense("topk_weights", topk_weights, topk_ids.shape, kinds.fp32, index)
        groups = group_tokens(topk_ids, len(self.tensors) // 3, status=self.status, stream=stream)
        h = gate_up.product(tokens, groups, gather=True, stream=stream)
        y = down.product(h, groups, out=_empty((h.shape[0], self.hidden), kinds.fp32[0], self.device, stream), stream=stream)
        if out is None:
            out = _empty((topk_ids.shape[0], self.hidden), tokens.dtype, self.device, stream)
        return combine_rows(y, groups, topk_weights, out=out, stream=stream)

    def _products(self):
        """The two grouped products of ffn_prompt, described at its first call."""
        if self._prompt is None:
            with self._prompt_lock:      # one description for all threads: kernels read its tables as long as it is kept
                if self._prompt is None:
                    shaped = [t.view(self.hidden, self.inter) if i % 3 == 2 else t.view(self.inter, self.hidden) for i, t in enumerate(self.tensors)]
                    self._prompt = (GroupedMatrix(shaped[0::3], up=shaped[1::3], status=self.status),
                                    GroupedMatrix(shaped[2::3], status=self.status))
        return self._prompt


class TokenGroups:
    """The choices of `topk_ids` [T, k] grouped by expert, as zipmoe_group_tokens lists them: offsets [n_experts + 1], order
    [T * k] (the choice that each row is), place [T, k] (the row of each choice, -1 for none), int32 device tensors.  Made by
    hand, for example of part of another's offsets, they are checked like any tensor: for type, device, shape and density."""

    def __init__(self, offsets, order, place, n_experts):
        int32, index = _get_kinds().int32, _device_of("place", place)
        if len(place.shape) != 2:
            raise ValueError("place: a row per token is wanted, not a tensor %s" % (tuple(place.shape),))
        T, k = place.shape
        _dense("place", place, (T, k), int32, index)
        _dense("offsets", offsets, (n_experts + 1,), int32, index)
        _dense("order", order, (T * k,), int32, index)
        self._set(offsets, order, place, n_experts, index)

    def _set(self, offsets, order, place, n_experts, index):
        self.offsets, self.order, self.place, self.n_experts, self.index = offsets, order, place, n_experts, index
        self.tokens, self.k = place.shape
        self.rows = order.shape[0]
        return self


def group_tokens(topk_ids, n_experts, offsets=None, order=None, place=None, status=None, stream=None):
    """topk_ids [T, k] int32 -> TokenGroups.  offsets, order and place, if given, are the tensors to be filled (entries of order
    behind the last group are left as they were); status [1] int32, if given, gets code 1 for an id of n_experts or more."""
    kinds, index = _get_kinds(), _device_of("topk_ids", topk_ids)
    if kinds.current_device() != index:
        with _on_device(index):
            return group_tokens(topk_ids, n_experts, offsets, order, place, status, stream)
    T, k = shape = topk_ids.shape
    int32 = kinds.int32
    ids_at = _dense("topk_ids", topk_ids, shape, int32, index)
    if offsets is None:
        offsets = _empty((n_experts + 1,), int32[0], topk_ids.device, stream)
    if order is None:
        order = _empty((T * k,), int32[0], topk_ids.device, stream)
    if place is None:
        place = _empty(shape, int32[0], topk_ids.device, stream)
    args = _GROUP_ARGS.pack(ids_at, _dense("offsets", offsets, (n_experts + 1,), int32, index), _dense("order", order, (T * k,), int32, index),
                            _dense("place", place, shape, int32, index), 0 if status is None else _dense("status", status, (1,), int32, index),
                            T, k, n_experts, 0)
    status_code = _lib.zipmoe_group_tokens(args, _handle(kinds, index, stream))
    if status_code:
        raise ZipMoEError("zipmoe_group_tokens", status_code)
    return TokenGroups.__new__(TokenGroups)._set(offsets, order, place, n_experts, index)      # (checked above)


class GroupedMatrix:
    """The weights of one grouped product: matrices[e] [rows, cols] of group e, all bf16 (or int16 patterns) or all int8, dense;
    `up`, if given, holds the second matrices of pairs: the product is then SiLU(first) * second.  int8 matrices have scales
    [rows] or [n_groups, rows] fp32 (up_scales for the second ones).  What this puts on the device is there on return, after
    the current stream's work so far: products may be called on any stream.  With a `status` of the caller's, evenly spaced
    bf16 or single int8 matrices need nothing there, and nothing is waited for."""

    def __init__(self, matrices, up=None, scales=None, up_scales=None, status=None):
        import torch
        kinds = self.kinds = _get_kinds()
        if not matrices or (up is not None and len(up) != len(matrices)):
            raise ValueError("a matrix per group, and as many second ones, are wanted")
        index = self.index = _device_of("matrix 0", matrices[0])
        self.device = matrices[0].device
        self.n_groups, (self.rows, self.cols) = len(matrices), matrices[0].shape
        self.int8, self.pair = matrices[0].dtype in kinds.int8, up is not None
        self.kind = kinds.int8 if self.int8 else kinds.bf16
        self.tensors = list(matrices) if up is None else [m for both in zip(matrices, up) for m in both]
        addresses = [_dense("matrix %d" % i, t, (self.rows, self.cols), self.kind, index) for i, t in enumerate(self.tensors)]
        self.scales, self.scales_at = None, 0
        if self.int8:
            if scales is None or self.pair != (up_scales is not None):
                raise ValueError("int8 matrices have scales, and second ones theirs")
            shape = (self.n_groups, self.rows)
            both = [s.view(shape) if s.dim() == 1 and self.n_groups == 1 else s for s in ((scales, up_scales) if self.pair else (scales,))]
            for name, s in zip(("scales", "up_scales"), both):
                _dense(name, s, shape, kinds.fp32, index)
            self.scales = torch.cat(both) if self.pair else both[0]
            self.scales_at = self.scales.data_ptr()
        elif scales is not None or up_scales is not None:
            raise ValueError("scales go with int8 matrices")
        flags = (GROUPED_PAIR if self.pair else 0) | (GROUPED_INT8 if self.int8 else 0)
        with _on_device(index):
            table, self.struct = zipmoe_grouped_weights_plan(addresses, self.n_groups, self.rows, self.cols, flags)
            capturing = kinds.capturing()
        self.table = None
        prepared = status is None or not self.struct.even or (self.int8 and self.pair)      # something is put on the device here
        if prepared and capturing:
            raise ValueError("weights are described before a capture, not within it")
        if not self.struct.even:      # (evenly spaced weights need no table)
            self.table = torch.from_numpy(table).to(self.device)
            self.struct.table = self.table.data_ptr()
        self._struct_at = ctypes.byref(self.struct)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device) if status is None else status
        self.status_at = _dense("status", self.status, (1,), kinds.int32, index)
        if prepared:      # calls may come on any stream
            torch.cuda.current_stream(self.device).synchronize()

    def product(self, x, groups=None, gather=False, row_scales=None, out=None, stream=None):
        """x [x_rows, cols] of the weights' kind -> out [rows, rows of the matrices], bf16 (x's dtype; torch.bfloat16 for int8)
        unless `out` is given, which may be fp32.  groups None: one group, all rows of x.  gather: row r of the product is the
        token that choice groups.order[r] belongs to (x is [groups.tokens, cols]); else row r of x (x is [groups.rows, cols]).
        row_scales [x_rows] fp32 goes with int8.  Rows of no group are left as they were."""
        kinds, index = self.kinds, self.index
        if kinds.current_device() != index:
            with _on_device(index):
                return self.product(x, groups, gather, row_scales, out, stream)
        offsets_at = order_at = k = 0
        if groups is None:
            if self.n_groups != 1 or gather:
                raise ValueError("the groups' lists are wanted")
            x_rows = rows = x.shape[0]
        else:
            if groups.n_experts != self.n_groups or groups.index != index:
                raise ValueError("lists of %d groups on CUDA device %d are wanted, not of %d on device %d" %
                                 (self.n_groups, index, groups.n_experts, groups.index))
            rows, x_rows, offsets_at = groups.rows, groups.rows, groups.offsets.data_ptr()
            if gather:
                x_rows, order_at, k = groups.tokens, groups.order.data_ptr(), groups.k
        x_at, x_pitch = _rows("x", x, (x_rows, self.cols), self.kind, index)
        scales_at = 0
        if self.int8:
            if row_scales is None:
                raise ValueError("int8 rows have scales")
            scales_at = _dense("row_scales", row_scales, (x_rows,), kinds.fp32, index)
        elif row_scales is not None:
            raise ValueError("scales go with int8 rows")
        if out is None:
            out = _empty((rows, self.rows), kinds.bf16[0] if self.int8 else x.dtype, self.device, stream)
        f32 = out.dtype in kinds.fp32
        out_at, out_pitch = _rows("out", out, (rows, self.rows), kinds.fp32 if f32 else kinds.bf16, index)
        need, scratch_at = 0, 0
        if gather:
            need = zipmoe_grouped_workspace_bytes(self.struct, rows, True)
            if need:      # (given back to the stream's pool on return: what is queued there comes before its next use)
                scratch = _empty((need,), kinds.e4m3[1], self.device, stream)
                scratch_at = scratch.data_ptr()
        args = _GROUPED_ARGS.pack(x_at, x_pitch, offsets_at, order_at, scales_at, self.scales_at, out_at, out_pitch, self.status_at,
                                  scratch_at, need, x_rows, rows, k, GROUPED_F32 if f32 else 0, 0, 0)
        status = _lib.zipmoe_grouped_matmul(self._struct_at, args, _handle(kinds, index, stream))
        if status:
            raise ZipMoEError("zipmoe_grouped_matmul", status)
        return out


def combine_rows(y, groups, weights, out=None, stream=None):
    """y [groups.rows, cols] bf16 (or int16 patterns) or fp32, weights [T, k] fp32 or None -> out [T, cols] bf16: every token's rows,
    added with their weights."""
    kinds, index = _get_kinds(), _device_of("y", y)
    if kinds.current_device() != index:
        with _on_device(index):
            return combine_rows(y, groups, weights, out, stream)
    if groups.index != index:
        raise ValueError("lists on CUDA device %d are wanted, not on device %d" % (index, groups.index))
    T, k, cols = groups.tokens, groups.k, y.shape[1]
    f32 = y.dtype in kinds.fp32
    y_at, y_pitch = _rows("y", y, (groups.rows, cols), kinds.fp32 if f32 else kinds.bf16, index)
    weights_at = 0 if weights is None else _dense("weights", weights, (T, k), kinds.fp32, index)
    if out is None:
        out = _empty((T, cols), kinds.bf16[0] if f32 else y.dtype, y.device, stream)
    out_at, out_pitch = _rows("out", out, (T, cols), kinds.bf16, index)
    args = _COMBINE_ARGS.pack(y_at, y_pitch, groups.place.data_ptr(), weights_at, out_at, out_pitch, 0, T, k, cols, groups.rows,
                              GROUPED_F32 if f32 else 0, 0)
    status = _lib.zipmoe_combine_rows(args, _handle(kinds, index, stream))
    if status:
        raise ZipMoEError("zipmoe_combine_rows", status)
    return out


def quantize_rows(x, q=None, scales=None, stream=None):
    """x [rows, cols] bf16 (or int16 patterns) whose rows may lie apart -> q [rows, cols] int8, scales [rows] fp32."""
    kinds, index = _get_kinds(), _device_of("x", x)
    if kinds.current_device() != index:
        with _on_device(index):
            return quantize_rows(x, q, scales, stream)
    rows, cols = shape = x.shape
    x_at, x_pitch = _rows("x", x, shape, kinds.bf16, index)
    if q is None:
        q = _empty(shape, kinds.int8[0], x.device, stream)
    if scales is None:
        scales = _empty((rows,), kinds.fp32[0], x.device, stream)
    q_at, q_pitch = _rows("q", q, shape, kinds.int8, index)
    status = _lib.zipmoe_quantize_rows(x_at, x_pitch, rows, cols, q_at, q_pitch, _dense("scales", scales, (rows,), kinds.fp32, index),
                                       _handle(kinds, index, stream))
    if status:
        raise ZipMoEError("zipmoe_quantize_rows", status)
    return q, scales


class Int8Linear:
    """A dense projection in 8-bit integers: weight [rows, cols] int8 and scales [rows] fp32, or from_bf16's of a bf16 weight."""

    def __init__(self, weight, scales):
        self.matrix = GroupedMatrix([weight], scales=scales)
        self.rows, self.cols, self.status = self.matrix.rows, self.matrix.cols, self.matrix.status

    @classmethod
    def from_bf16(cls, weight):
        """weight [rows, cols] bf16 (or int16 patterns), for example a tensor that was decoded: each output channel with a scale
        of its own.  It is rounded on the current stream, and the rounding has ended on return."""
        return cls(*quantize_rows(weight))

    def product(self, x, out=None, stream=None):
        """x [tokens, cols] bf16 (or int16 patterns) -> out [tokens, rows], bf16 (x's dtype) unless `out` is given, which may be
        fp32: every token is rounded to 8 bits with a scale of its own, the sums are exact."""
        m = self.matrix
        kinds, index = m.kinds, m.index
        if kinds.current_device() != index:
            with _on_device(index):
                return self.product(x, out, stream)
        rows = x.shape[0]
        x_at, x_pitch = _rows("x", x, (rows, self.cols), kinds.bf16, index)
        if out is None:
            out = _empty((rows, self.rows), x.dtype, x.device, stream)
        f32 = out.dtype in kinds.fp32
        out_at, out_pitch = _rows("out", out, (rows, self.rows), kinds.fp32 if f32 else kinds.bf16, index)
        # the integers and their scales; given back to the stream's pool on return: what is queued there comes before its next use
        need = rows * (self.cols + 4)
        scratch = _empty((need,), kinds.e4m3[1], x.device, stream)
        args = _LINEAR_ARGS.pack(x_at, x_pitch, m.scales_at, out_at, out_pitch, scratch.data_ptr(), need, m.status_at, rows,
                                 GROUPED_F32 if f32 else 0, 0)
        status = _lib.zipmoe_linear_int8(m._struct_at, args, _handle(kinds, index, stream))
        if status:
            raise ZipMoEError("zipmoe_linear_int8", status)
        return out
