"""Thin ctypes binding of libiris_b200.so: same names as include/iris_b200.h, argument marshalling, and for the operators on
logits checks of the tensors that they are given.

PyTorch appears here only to obtain device pointers and the current stream.  There is no fallback:
if the shared library is missing or cannot be loaded, importing a symbol raises.
"""
from __future__ import annotations

import ctypes as C
import importlib
import os
import struct

IRIS_OK = 0
IRIS_ERR_ARG, IRIS_ERR_RANGE, IRIS_ERR_NOMEM, IRIS_ERR_CUDA = -1, -2, -3, -4
IRIS_ERR_UNSUPPORTED, IRIS_ERR_TIMEOUT, IRIS_ERR_STATE = -5, -6, -7
IRIS_F16, IRIS_BF16 = 0, 1
DTYPES = {"fp16": IRIS_F16, "bf16": IRIS_BF16}
IRIS_F32 = 2
LOGIT_DTYPES = {"fp16": IRIS_F16, "bf16": IRIS_BF16, "fp32": IRIS_F32}   # operators on logits
IRIS_DISTILL_RENORM, IRIS_DISTILL_TAIL = 0, 1
IRIS_MODE_BULK_SYNCHRONOUS, IRIS_MODE_FUSED_SEQUENTIAL, IRIS_MODE_WORKGROUP_SPECIALIZED = 0, 1, 2
MODES = {"bulk_synchronous": 0, "fused_sequential": 1, "workgroup_specialized": 2}
IRIS_SEM_RELAXED, IRIS_SEM_ACQUIRE, IRIS_SEM_RELEASE, IRIS_SEM_ACQ_REL = 0, 1, 2, 3
IRIS_SCOPE_BLOCK, IRIS_SCOPE_GPU, IRIS_SCOPE_SYS = 0, 1, 2
IRIS_OP_ADD, IRIS_OP_XCHG, IRIS_OP_AND, IRIS_OP_OR, IRIS_OP_XOR, IRIS_OP_MIN, IRIS_OP_MAX = range(7)
ATOMIC_OPS = {"add": 0, "xchg": 1, "and": 2, "or": 3, "xor": 4, "min": 5, "max": 6}
IRIS_B_N_BY_K, IRIS_B_K_BY_N = 0, 1
IRIS_MAX_WORLD = 8
IRIS_TILE = 128

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libiris_b200.so")

# Every symbol include/iris_b200.h declares.
EXPORTS = [
    "iris_last_error", "iris_version", "iris_heap_create", "iris_heap_create_ex", "iris_heap_destroy", "iris_heap_world",
    "iris_heap_bytes_per_rank", "iris_heap_base", "iris_heap_bases", "iris_malloc", "iris_heap_reset", "iris_translate",
    "iris_status_check", "iris_put_tile", "iris_get_tile", "iris_atomic_add", "iris_atomic_cas",
    "iris_atomic_add_contended", "iris_atomic_cas_contended", "iris_flags_fill", "iris_all_store_bench",
    "iris_gemm_all_scatter_ex", "iris_gemm_all_scatter_unfused", "gemm_all_scatter", "iris_gemm_heap_bytes", "iris_heap_epoch", "iris_num_tiles",
    "iris_consume_bias", "iris_consume_bias_ranks", "iris_gemm_all_scatter_host", "iris_gemm_out_offset", "iris_gemm_takeover_stats",
    "iris_gemm_all_scatter_noalloc", "iris_heap_create_from_bases", "iris_heap_local_rank", "iris_ipc_alloc", "iris_ipc_free", "iris_ipc_export",
    "iris_ipc_open", "iris_ipc_close", "iris_atomic_add_u64", "iris_atomic_cas_u64", "iris_copy_tile", "iris_load_tile", "iris_store_tile", "iris_atomic_rmw",
    "iris_token_logprobs", "iris_token_logprobs_backward", "iris_distill_topk", "iris_distill_topk_backward",
]


class IrisError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"iris error {code}: {msg}")
        self.code = code


class GemmArgs(C.Structure):
    _fields_ = [
        ("A", C.c_void_p), ("B_shards", C.POINTER(C.c_void_p)), ("heap", C.c_void_p),
        ("M", C.c_int), ("N", C.c_int), ("K", C.c_int), ("world", C.c_int), ("mode", C.c_int), ("dtype", C.c_int),
        ("c_off", C.c_uint64), ("flag_off", C.c_uint64), ("lock_off", C.c_uint64),
        ("epoch", C.c_int32), ("comm_ctas", C.c_int), ("max_ctas", C.c_int), ("raster_group", C.c_int),
        ("block_n", C.c_int), ("spin_timeout_ns", C.c_uint64), ("cta_pair", C.c_int), ("static_schedule", C.c_int), ("stream_k", C.c_int), ("wg_tail", C.c_int), ("rank_first", C.c_int), ("rank_count", C.c_int), ("pace_stores", C.c_int),
        ("consumer_bias", C.c_void_p), ("consumer_out_off", C.c_uint64), ("b_layout", C.c_int), ("fuse_tail", C.c_int), ("stage_k", C.c_int),
    ]


# The argument blocks of the operators on logits, in the header's order (P pointer, q int64, i int, f float, natural alignment).  They are called
# once a decoded token, where filling a ctypes.Structure would take longer than the kernel: packing one is a tenth of that.
_LOGPROB_ARGS = struct.Struct("@PqqqifPiiPPPPP")
_LOGPROB_GRAD_ARGS = struct.Struct("@PqqqifPiPPPPPq")
_DISTILL_ARGS = struct.Struct("@PqqqifPPiifPPPPq")


_lib = None


def lib() -> C.CDLL:
    """Load the library (no CUDA call is made by loading it)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2511_12500_b200.build` (needs nvcc); there is no fallback")
    L = C.CDLL(LIB_PATH)
    vp, u64, sz, i32, ci = C.c_void_p, C.c_uint64, C.c_size_t, C.c_int32, C.c_int
    L.iris_last_error.restype = C.c_char_p
    L.iris_version.restype = C.c_char_p
    L.iris_heap_create.restype = vp
    L.iris_heap_create.argtypes = [ci, sz]
    L.iris_heap_create_ex.argtypes = [ci, sz, vp, C.POINTER(vp)]
    L.iris_heap_create_from_bases.argtypes = [ci, sz, C.POINTER(u64), ci, C.POINTER(vp)]
    L.iris_heap_local_rank.argtypes = [vp]
    L.iris_ipc_alloc.argtypes = [sz, C.POINTER(vp)]
    L.iris_ipc_free.argtypes = [vp]
    L.iris_ipc_export.argtypes = [vp, C.c_char_p]
    L.iris_ipc_open.argtypes = [C.c_char_p, C.POINTER(vp)]
    L.iris_ipc_close.argtypes = [vp]
    L.iris_heap_destroy.argtypes = [vp]
    L.iris_heap_world.argtypes = [vp]
    L.iris_heap_bytes_per_rank.restype = sz
    L.iris_heap_bytes_per_rank.argtypes = [vp]
    L.iris_heap_base.restype = vp
    L.iris_heap_base.argtypes = [vp, ci]
    L.iris_heap_bases.argtypes = [vp, C.POINTER(u64)]
    L.iris_malloc.argtypes = [vp, sz, sz, C.POINTER(u64)]
    L.iris_heap_reset.argtypes = [vp]
    L.iris_translate.argtypes = [vp, vp, ci, ci, C.POINTER(vp)]
    L.iris_status_check.argtypes = [vp, vp, C.POINTER(i32)]
    for f in (L.iris_put_tile, L.iris_get_tile):
        f.argtypes = [vp, vp, vp, sz, sz, sz, sz, ci, ci, vp]
    L.iris_copy_tile.argtypes = [vp, vp, vp, sz, sz, sz, sz, ci, ci, ci, vp]
    for f in (L.iris_load_tile, L.iris_store_tile):
        f.argtypes = [vp, vp, vp, sz, sz, sz, sz, ci, ci, vp]
    L.iris_atomic_rmw.argtypes = [vp, ci, vp, sz, sz, ci, ci, i32, ci, ci, vp, vp]
    L.iris_atomic_add.argtypes = [vp, vp, sz, sz, ci, ci, i32, ci, ci, vp, vp]
    L.iris_atomic_cas.argtypes = [vp, vp, sz, sz, ci, ci, i32, i32, ci, ci, vp, vp]
    L.iris_atomic_add_u64.argtypes = [vp, vp, sz, sz, ci, ci, u64, ci, ci, vp, vp]
    L.iris_atomic_cas_u64.argtypes = [vp, vp, sz, sz, ci, ci, u64, u64, ci, ci, vp, vp]
    L.iris_atomic_add_contended.argtypes = [vp, vp, sz, ci, ci, i32, ci, ci, vp, vp]
    L.iris_atomic_cas_contended.argtypes = [vp, vp, sz, ci, ci, i32, i32, ci, ci, vp, vp]
    L.iris_flags_fill.argtypes = [vp, u64, sz, i32, vp]
    L.iris_all_store_bench.argtypes = [vp, u64, u64, u64, sz, sz, i32, ci, ci, vp]
    L.iris_gemm_all_scatter_ex.argtypes = [C.POINTER(GemmArgs), vp]
    L.iris_gemm_all_scatter_unfused.argtypes = [C.POINTER(GemmArgs), vp, vp]
    L.gemm_all_scatter.argtypes = [vp, C.POINTER(vp), vp, ci, ci, ci, ci, ci]
    L.iris_gemm_heap_bytes.restype = sz
    L.iris_gemm_heap_bytes.argtypes = [ci, ci, ci]
    L.iris_heap_epoch.restype = i32
    L.iris_heap_epoch.argtypes = [vp]
    L.iris_num_tiles.restype = C.c_int64
    L.iris_num_tiles.argtypes = [ci, ci, ci]
    L.iris_consume_bias.argtypes = [vp, u64, u64, u64, vp, ci, ci, ci, ci, i32, ci, u64, vp]
    L.iris_consume_bias_ranks.argtypes = [vp, u64, u64, u64, vp, ci, ci, ci, ci, ci, ci, i32, ci, u64, vp]
    L.iris_gemm_all_scatter_host.argtypes = [vp, C.POINTER(vp), vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci]
    L.iris_gemm_takeover_stats.argtypes = [vp, C.POINTER(C.c_int32)]
    L.iris_gemm_out_offset.restype = u64
    L.iris_gemm_out_offset.argtypes = [ci, ci, ci]
    L.iris_gemm_all_scatter_noalloc.argtypes = [vp, C.POINTER(vp), C.POINTER(u64), sz, ci, ci, ci, ci, ci, u64, u64, i32, vp]
    for f in (L.iris_token_logprobs, L.iris_token_logprobs_backward, L.iris_distill_topk, L.iris_distill_topk_backward):
        f.argtypes = [C.c_char_p, vp]   # a packed argument block
    _lib = L
    return L


def iris_last_error() -> str:
    return lib().iris_last_error().decode()


def _ck(rc: int) -> int:
    if rc != IRIS_OK:
        raise IrisError(rc, iris_last_error())
    return rc


def _ptr(x) -> int | None:
    """Device/host address of a torch tensor, numpy array, int or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(type(x))


def _stream(stream) -> int | None:
    if stream is None:
        import torch
        # the handle alone: making a torch.cuda.Stream of it takes 3 us, half of a small call
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream


# ---------------------------------------------------------------------------------------------- heap
def iris_heap_create(world: int, bytes_per_rank: int, external_base=None) -> int:
    h = C.c_void_p()
    _ck(lib().iris_heap_create_ex(world, bytes_per_rank, _ptr(external_base), C.byref(h)))
    return h.value


def iris_heap_create_from_bases(world: int, bytes_per_rank: int, bases, local_rank: int) -> int:
    """Heap over several processes: bases[r] = this process's device address of rank r's slot."""
    if len(bases) != world:
        raise ValueError("one base per rank")
    arr = (C.c_uint64 * world)(*[int(b) for b in bases])
    h = C.c_void_p()
    _ck(lib().iris_heap_create_from_bases(world, bytes_per_rank, arr, local_rank, C.byref(h)))
    return h.value


def iris_heap_local_rank(heap: int) -> int:
    return lib().iris_heap_local_rank(heap)


IRIS_IPC_HANDLE_BYTES = 64


def iris_ipc_alloc(nbytes: int) -> int:
    p = C.c_void_p()
    _ck(lib().iris_ipc_alloc(nbytes, C.byref(p)))
    return p.value


def iris_ipc_free(ptr: int):
    _ck(lib().iris_ipc_free(ptr))


def iris_ipc_export(ptr: int) -> bytes:
    buf = C.create_string_buffer(IRIS_IPC_HANDLE_BYTES)
    _ck(lib().iris_ipc_export(ptr, buf))
    return buf.raw


def iris_ipc_open(handle: bytes) -> int:
    if len(handle) != IRIS_IPC_HANDLE_BYTES:
        raise ValueError("an exported handle has IRIS_IPC_HANDLE_BYTES bytes")
    p = C.c_void_p()
    _ck(lib().iris_ipc_open(handle, C.byref(p)))
    return p.value


def iris_ipc_close(ptr: int):
    _ck(lib().iris_ipc_close(ptr))


def iris_heap_destroy(heap: int):
    _ck(lib().iris_heap_destroy(heap))


def iris_heap_world(heap: int) -> int:
    return lib().iris_heap_world(heap)


def iris_heap_bytes_per_rank(heap: int) -> int:
    return lib().iris_heap_bytes_per_rank(heap)


def iris_heap_base(heap: int, rank: int) -> int:
    p = lib().iris_heap_base(heap, rank)
    if not p:
        raise IrisError(IRIS_ERR_ARG, iris_last_error())
    return p


def iris_heap_bases(heap: int) -> list[int]:
    out = (C.c_uint64 * IRIS_MAX_WORLD)()
    _ck(lib().iris_heap_bases(heap, out))
    return list(out[: iris_heap_world(heap)])


def iris_malloc(heap: int, nbytes: int, align: int = 0) -> int:
    off = C.c_uint64()
    _ck(lib().iris_malloc(heap, nbytes, align, C.byref(off)))
    return off.value


def iris_heap_reset(heap: int):
    _ck(lib().iris_heap_reset(heap))


def iris_translate(heap: int, ptr: int, from_rank: int, to_rank: int) -> int:
    out = C.c_void_p()
    _ck(lib().iris_translate(heap, ptr, from_rank, to_rank, C.byref(out)))
    return out.value


def iris_status_check(heap: int, stream=None):
    """Synchronise and raise IrisError(IRIS_ERR_TIMEOUT) if a device-side wait expired."""
    detail = (C.c_int32 * 8)()
    rc = lib().iris_status_check(heap, _stream(stream), detail)
    if rc != IRIS_OK:
        e = IrisError(rc, iris_last_error())
        e.detail = list(detail)
        raise e


# ---------------------------------------------------------------------------------------- tile ops
def iris_put_tile(heap, src, dst, rows, row_bytes, src_pitch, dst_pitch, from_rank, to_rank, stream=None):
    _ck(lib().iris_put_tile(heap, src, dst, rows, row_bytes, src_pitch, dst_pitch, from_rank, to_rank, _stream(stream)))


def iris_get_tile(heap, src, dst, rows, row_bytes, src_pitch, dst_pitch, from_rank, to_rank, stream=None):
    _ck(lib().iris_get_tile(heap, src, dst, rows, row_bytes, src_pitch, dst_pitch, from_rank, to_rank, _stream(stream)))


def iris_copy_tile(heap, src, dst, rows, row_bytes, src_pitch, dst_pitch, cur_rank, from_rank, to_rank, stream=None):
    _ck(lib().iris_copy_tile(heap, src, dst, rows, row_bytes, src_pitch, dst_pitch, cur_rank, from_rank, to_rank, _stream(stream)))


def iris_load_tile(heap, src, out, rows, row_bytes, src_pitch, out_pitch, from_rank, to_rank, stream=None):
    _ck(lib().iris_load_tile(heap, src, _ptr(out), rows, row_bytes, src_pitch, out_pitch, from_rank, to_rank, _stream(stream)))


def iris_store_tile(heap, values, dst, rows, row_bytes, values_pitch, dst_pitch, from_rank, to_rank, stream=None):
    _ck(lib().iris_store_tile(heap, _ptr(values), dst, rows, row_bytes, values_pitch, dst_pitch, from_rank, to_rank, _stream(stream)))


def iris_atomic_rmw(heap, op, ptr, count, stride_bytes, from_rank, to_rank, value, sem=IRIS_SEM_RELAXED, scope=IRIS_SCOPE_GPU,
                    old_out=None, stream=None):
    _ck(lib().iris_atomic_rmw(heap, op, ptr, count, stride_bytes, from_rank, to_rank, value, sem, scope, _ptr(old_out), _stream(stream)))


def iris_atomic_add(heap, ptr, count, stride_bytes, from_rank, to_rank, value, sem=IRIS_SEM_RELAXED,
                    scope=IRIS_SCOPE_GPU, old_out=None, stream=None):
    _ck(lib().iris_atomic_add(heap, ptr, count, stride_bytes, from_rank, to_rank, value, sem, scope, _ptr(old_out), _stream(stream)))


def iris_atomic_cas(heap, ptr, count, stride_bytes, from_rank, to_rank, compare, value, sem=IRIS_SEM_RELAXED,
                    scope=IRIS_SCOPE_GPU, old_out=None, stream=None):
    _ck(lib().iris_atomic_cas(heap, ptr, count, stride_bytes, from_rank, to_rank, compare, value, sem, scope, _ptr(old_out), _stream(stream)))


def iris_atomic_add_u64(heap, ptr, count, stride_bytes, from_rank, to_rank, value, sem=IRIS_SEM_RELAXED,
                        scope=IRIS_SCOPE_GPU, old_out=None, stream=None):
    _ck(lib().iris_atomic_add_u64(heap, ptr, count, stride_bytes, from_rank, to_rank, value, sem, scope, _ptr(old_out), _stream(stream)))


def iris_atomic_cas_u64(heap, ptr, count, stride_bytes, from_rank, to_rank, compare, value, sem=IRIS_SEM_RELAXED,
                        scope=IRIS_SCOPE_GPU, old_out=None, stream=None):
    _ck(lib().iris_atomic_cas_u64(heap, ptr, count, stride_bytes, from_rank, to_rank, compare, value, sem, scope, _ptr(old_out), _stream(stream)))


def iris_atomic_add_contended(heap, ptr, threads, from_rank, to_rank, value, sem=IRIS_SEM_RELAXED, scope=IRIS_SCOPE_GPU,
                              old_out=None, stream=None):
    _ck(lib().iris_atomic_add_contended(heap, ptr, threads, from_rank, to_rank, value, sem, scope, _ptr(old_out), _stream(stream)))


def iris_atomic_cas_contended(heap, ptr, threads, from_rank, to_rank, compare, value_base, sem=IRIS_SEM_RELAXED,
                              scope=IRIS_SCOPE_GPU, old_out=None, stream=None):
    _ck(lib().iris_atomic_cas_contended(heap, ptr, threads, from_rank, to_rank, compare, value_base, sem, scope, _ptr(old_out), _stream(stream)))


def iris_flags_fill(heap, off, count, value, stream=None):
    _ck(lib().iris_flags_fill(heap, off, count, value, _stream(stream)))


def iris_all_store_bench(heap, payload_off, recv_off, flag_off, S, tile_bytes, epoch, ctas=0, pull=0, stream=None):
    _ck(lib().iris_all_store_bench(heap, payload_off, recv_off, flag_off, S, tile_bytes, epoch, ctas, pull, _stream(stream)))


# ------------------------------------------------------------------------------- GEMM + all-scatter
def iris_num_tiles(M: int, N: int, world: int) -> int:
    n = lib().iris_num_tiles(M, N, world)
    if n < 0:
        raise IrisError(int(n), iris_last_error())
    return int(n)


def iris_gemm_heap_bytes(M: int, N: int, world: int) -> int:
    return lib().iris_gemm_heap_bytes(M, N, world)


def iris_heap_epoch(heap: int) -> int:
    return lib().iris_heap_epoch(heap)


def _shards(B_shards):
    arr = (C.c_void_p * len(B_shards))(*[_ptr(b) for b in B_shards])
    return arr


def iris_gemm_all_scatter_ex(heap, A, B_shards, M, N, K, world, mode, dtype, c_off, flag_off, lock_off=0, epoch=1,
                             comm_ctas=0, max_ctas=0, raster_group=0, block_n=0, spin_timeout_ns=0, cta_pair=0, static_schedule=0, stream_k=0, wg_tail=0, rank_first=0, rank_count=0, pace_stores=0, consumer_bias=None, consumer_out_off=0, b_layout=0, fuse_tail=0, stage_k=0, stream=None, comm_stream=None):
    arr = _shards(B_shards)
    a = GemmArgs(_ptr(A), C.cast(arr, C.POINTER(C.c_void_p)), heap, M, N, K, world, mode, dtype, c_off, flag_off, lock_off,
                 epoch, comm_ctas, max_ctas, raster_group, block_n, spin_timeout_ns, cta_pair, static_schedule, stream_k, wg_tail, rank_first, rank_count, pace_stores, _ptr(consumer_bias), consumer_out_off, b_layout, fuse_tail, stage_k)
    if comm_stream is not None:     # the two-kernel, two-stream form (producers on `stream`, communication kernel on `comm_stream`)
        _ck(lib().iris_gemm_all_scatter_unfused(C.byref(a), _stream(stream), _stream(comm_stream)))
    else:
        _ck(lib().iris_gemm_all_scatter_ex(C.byref(a), _stream(stream)))


def iris_gemm_all_scatter_unfused(heap, A, B_shards, M, N, K, world, dtype, c_off, flag_off, lock_off, epoch, producer_stream, comm_stream, **kw):
    """Workgroup-specialised schedule as two kernels on two streams (see the header)."""
    iris_gemm_all_scatter_ex(heap, A, B_shards, M, N, K, world, IRIS_MODE_WORKGROUP_SPECIALIZED, dtype, c_off, flag_off, lock_off, epoch,
                             stream=producer_stream, comm_stream=comm_stream, **kw)


def gemm_all_scatter(A, B_shards, heap, M, N, K, world, mode):
    """The short form: bf16, C at offset 0, default stream (see the header)."""
    arr = _shards(B_shards)
    _ck(lib().gemm_all_scatter(_ptr(A), C.cast(arr, C.POINTER(C.c_void_p)), heap, M, N, K, world, mode))


def iris_consume_bias(heap, c_off, out_off, flag_off, bias, M, N, world, dtype, epoch, ctas=0, timeout_ns=0, stream=None):
    _ck(lib().iris_consume_bias(heap, c_off, out_off, flag_off, _ptr(bias), M, N, world, dtype, epoch, ctas, timeout_ns, _stream(stream)))


def iris_consume_bias_ranks(heap, c_off, out_off, flag_off, bias, M, N, world, rank_first, rank_count, dtype, epoch, ctas=0, timeout_ns=0, stream=None):
    _ck(lib().iris_consume_bias_ranks(heap, c_off, out_off, flag_off, _ptr(bias), M, N, world, rank_first, rank_count, dtype, epoch, ctas, timeout_ns,
                                      _stream(stream)))


def iris_gemm_takeover_stats(heap):
    """(half tiles kept by their producers, publication tiles still queued) of the last workgroup-specialised pair launch."""
    out = (C.c_int32 * 2)()
    _ck(lib().iris_gemm_takeover_stats(heap, out))
    return int(out[0]), int(out[1])


def iris_gemm_out_offset(M: int, N: int, world: int) -> int:
    return lib().iris_gemm_out_offset(M, N, world)


def iris_gemm_all_scatter_host(A_host, B_shards_host, C_host, flags_host, bias_host, OUT_host, heap, M, N, K, world, mode, dtype,
                               out_slot=0):
    arr = _shards(B_shards_host)
    _ck(lib().iris_gemm_all_scatter_host(_ptr(A_host), C.cast(arr, C.POINTER(C.c_void_p)), _ptr(C_host), _ptr(flags_host),
                                         _ptr(bias_host), _ptr(OUT_host), heap, M, N, K, world, mode, dtype, out_slot))


def iris_gemm_all_scatter_noalloc(A, B_shards, slot_bases, bytes_per_rank, M, N, K, world, dtype, c_off, flag_off, epoch, stream=None):
    """Workgroup-specialised gemm_all_scatter for callers that must not allocate device memory: no heap handle, the
    locks and the status block sit in a fixed array inside the library (at most 16384 publication tiles).  Blocks
    until the work on `stream` has finished.  Calls that overlap on the GPU race on that array."""
    arr = _shards(B_shards)
    bases = (C.c_uint64 * len(slot_bases))(*slot_bases)
    _ck(lib().iris_gemm_all_scatter_noalloc(_ptr(A), C.cast(arr, C.POINTER(C.c_void_p)), bases, bytes_per_rank, M, N, K, world, dtype,
                                            c_off, flag_off, epoch, _stream(stream)))


# ------------------------------------------------------------------------------------- operators on logits
# Shapes, types and rules are the header's.  Tensors other than logits and dlogits are contiguous, ids are int64, the
# rest fp32; row_stride and grad_stride are in elements (0 = vocab).  What is given as a tensor is checked against the
# sizes of the call: its type, its layout, that it is long enough and that the GPU can read it (IRIS_ERR_ARG).  Addresses are
# taken as they are.  _accept (csrc/py_tensors.c) passes what is right in the usual way, in half a microsecond; anything else, and everything
# where that extension is not built or the tensors have no C interface, is looked at by _look.
_accept = None
_LOGITS = {}   # dtype -> torch type


def _first_call():
    global _accept
    import torch
    _LOGITS.update({IRIS_F16: torch.float16, IRIS_BF16: torch.bfloat16, IRIS_F32: torch.float32})
    interface = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)
    _accept = _none
    importlib.invalidate_caches()   # it may have been built since this process began
    try:
        from . import _tensors
    except ImportError:
        return
    if interface is not None and _tensors.setup(interface, torch.Tensor):
        _accept = _tensors.addresses


def _none(*args):
    return None


def _refuse(what, why):
    raise IrisError(IRIS_ERR_ARG, f"{what} {why}")


def _look_at_type(x, dtype, what):
    if not hasattr(x, "data_ptr"):
        _refuse(what, f"is a {type(x).__name__}, neither a tensor nor an address")
    if x.dtype is not dtype:
        _refuse(what, f"is {x.dtype}, not {dtype}")


def _look_at_place(x, what):
    if not x.is_cuda and not x.is_pinned():
        _refuse(what, "is not on the GPU")


def _look_at_buffer(x, size, count, what):
    import torch
    if x is None or isinstance(x, int) or count <= 0:   # nothing is read or written of 0 elements
        return
    _look_at_type(x, torch.int64 if size == 8 else torch.float32, what)
    if not x.is_contiguous():
        _refuse(what, "is not contiguous")
    if x.numel() < count:
        _refuse(what, f"has {x.numel()} elements, the call needs {count}")
    _look_at_place(x, what)


def _look_at_rows(x, rows, vocab, dtype, stride, what):
    if x is None or isinstance(x, int) or rows <= 0 or vocab <= 0 or dtype not in _LOGITS:   # nothing to read, or refused by the library
        return
    _look_at_type(x, _LOGITS[dtype], what)
    shape, strides = tuple(x.shape), x.stride()
    if not x.is_contiguous() and vocab > 1 and strides[-1] != 1:
        _refuse(what, f"has a row's elements {strides[-1]} elements apart")
    if stride == 0 and rows > 1 and not (x.is_contiguous() and (len(shape) == 1 or shape and shape[-1] == vocab)):
        _refuse(what, f"of shape {shape}, strides {strides}, has other rows than {rows} of {vocab} one after the other, and the row stride is not given")
    last = sum((n - 1) * s for n, s in zip(shape, strides)) if x.numel() else -1
    if (rows - 1) * (stride or vocab) + vocab - 1 > last:
        _refuse(what, f"of shape {shape}, strides {strides}, does not hold {rows} rows of {vocab}, {stride or vocab} elements apart")
    _look_at_place(x, what)


def _look(names, rows, vocab, dtype, logits, row_stride, dlogits, grad_stride, *buffers):
    """What _accept does, a question at a time."""
    _look_at_rows(logits, rows, vocab, dtype, row_stride, "logits")
    _look_at_rows(dlogits, rows, vocab, dtype, grad_stride, "dlogits")
    for what, x, size, each in zip(names, buffers[::3], buffers[1::3], buffers[2::3]):
        _look_at_buffer(x, size, rows * each, what)
    return [_ptr(x) or 0 for x in (logits, dlogits, *buffers[::3])]


def iris_token_logprobs(logits, rows, vocab, dtype, targets=None, n_targets=0, logprob=None, entropy=None, stats=None, top_k=0, top_ids=None,
                        top_logprob=None, scale=1.0, row_stride=0, stream=None):
    if _accept is None:
        _first_call()
    args = (rows, vocab, dtype, logits, row_stride, None, 0, targets, 8, n_targets, logprob, 4, n_targets, entropy, 4, 1, stats, 4, 2, top_ids, 8, top_k,
            top_logprob, 4, top_k)
    z, _, t, lp, en, st, ti, tl = _accept(*args) or _look(("targets", "logprob", "entropy", "stats", "top_ids", "top_logprob"), *args)
    rc = lib().iris_token_logprobs(_LOGPROB_ARGS.pack(z, rows, vocab, row_stride, dtype, scale, t, n_targets, top_k, lp, en, st, ti, tl), _stream(stream))
    if rc:
        _ck(rc)


def iris_token_logprobs_backward(logits, rows, vocab, dtype, targets, n_targets, stats, grad_logprob, dlogits, entropy=None, grad_entropy=None,
                                 scale=1.0, row_stride=0, grad_stride=0, stream=None):
    if _accept is None:
        _first_call()
    args = (rows, vocab, dtype, logits, row_stride, dlogits, grad_stride, targets, 8, n_targets, stats, 4, 2, grad_logprob, 4, n_targets, entropy, 4, 1,
            grad_entropy, 4, 1)
    z, dz, t, st, g, en, gh = _accept(*args) or _look(("targets", "stats", "grad_logprob", "entropy", "grad_entropy"), *args)
    rc = lib().iris_token_logprobs_backward(_LOGPROB_GRAD_ARGS.pack(z, rows, vocab, row_stride, dtype, scale, t, n_targets, st, g, en, gh, dz, grad_stride),
                                            _stream(stream))
    if rc:
        _ck(rc)


def _distill(fn, weight_name, logits, rows, vocab, dtype, teacher, teacher_ids, list_k, mode, weight, loss, stats, dlogits, scale, teacher_scale, row_stride,
             grad_stride, stream):
    if _accept is None:
        _first_call()
    args = (rows, vocab, dtype, logits, row_stride, dlogits, grad_stride, teacher, 4, list_k, teacher_ids, 8, list_k, weight, 4, 1, loss, 4, 1, stats, 4, 3)
    z, dz, v, ids, w, lo, st = _accept(*args) or _look(("teacher", "teacher_ids", weight_name, "loss", "stats"), *args)
    rc = fn(_DISTILL_ARGS.pack(z, rows, vocab, row_stride, dtype, scale, v, ids, list_k, mode, teacher_scale, w, lo, st, dz, grad_stride), _stream(stream))
    if rc:
        _ck(rc)


def iris_distill_topk(logits, rows, vocab, dtype, teacher, teacher_ids, list_k, loss, mode=IRIS_DISTILL_RENORM, stats=None, weight=None, dlogits=None,
                      scale=1.0, teacher_scale=1.0, row_stride=0, grad_stride=0, stream=None):
    """Loss per row and, with `dlogits`, weight * its gradient, in one pass over the logits."""
    _distill(lib().iris_distill_topk, "weight", logits, rows, vocab, dtype, teacher, teacher_ids, list_k, mode, weight, loss, stats, dlogits, scale,
             teacher_scale, row_stride, grad_stride, stream)


def iris_distill_topk_backward(logits, rows, vocab, dtype, teacher, teacher_ids, list_k, stats, grad_loss, dlogits, mode=IRIS_DISTILL_RENORM,
                               scale=1.0, teacher_scale=1.0, row_stride=0, grad_stride=0, stream=None):
    """grad_loss * the gradient, from the statistics that iris_distill_topk left."""
    _distill(lib().iris_distill_topk_backward, "grad_loss", logits, rows, vocab, dtype, teacher, teacher_ids, list_k, mode, grad_loss, None, stats, dlogits,
             scale, teacher_scale, row_stride, grad_stride, stream)
