"""ctypes binding of libsymph.so: same names as the C entry points, torch tensors in, status checked."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
# SYMPH_LIBRARY_PATH: development override to load an experimental build of the same library
_LIB_PATH = os.environ.get("SYMPH_LIBRARY_PATH") or os.path.join(_HERE, "libsymph.so")
_lib = None

SYMPH_BF16, SYMPH_FP32 = 0, 1

EXPORTED_SYMBOLS = (
    "symph_kv_buffer_bytes", "symph_kv_pack", "symph_kv_unpack", "symph_kv_pack_layers", "symph_kv_unpack_layers",
    "symph_kv_pack_batch_layers", "symph_kv_unpack_batch_layers", "symph_stage_batch_layers_to_host",
    "symph_stage_batch_layers_to_device", "symph_kv_pack_tail", "symph_kv_unpack_tail", "symph_kv_pack_units", "symph_kv_unpack_units", "symph_kv_append",
    "symph_prefix_prefill_attn", "symph_prefix_prefill_attn_workspace_bytes", "symph_prefix_prefill_attn_tuned",
    "symph_prefix_prefill_attn_workspace_bytes_tuned", "symph_prefix_prefill_attn_static", "symph_debug_attn_flags", "symph_stage_to_host",
    "symph_stage_to_device", "symph_stage_layer_to_host", "symph_stage_layer_to_device", "symph_device_copy",
    "symph_build_tables", "symph_tree_mask", "symph_tree_attn", "symph_tree_attn_workspace_bytes", "symph_tree_accept",
    "symph_kv_commit", "symph_beam_select", "symph_beam_select_workspace_bytes", "symph_kv_fork", "symph_kv_copy_blocks",
    "symph_kv_free", "symph_kv_free_workspace_bytes", "symph_kv_compact", "symph_kv_compact_workspace_bytes",
    "symph_mfma_reference", "symph_debug_check_tables",
    "symph_status_string",
    # symph_pool.h (host code only)
    "symph_pool_create", "symph_pool_destroy", "symph_pool_advise", "symph_pool_drop", "symph_pool_claim",
    "symph_pool_framework_take", "symph_pool_framework_give", "symph_pool_settle", "symph_pool_resident_layers",
    "symph_pool_unit_slots", "symph_pool_table", "symph_pool_counts",
)


class SymphError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class _CacheStruct(C.Structure):
    _fields_ = [("k_base", C.c_void_p), ("v_base", C.c_void_p), ("layer_stride", C.c_int64),
                ("block_stride", C.c_int64), ("n_layers", C.c_int32), ("n_blocks", C.c_int32),
                ("block_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class AttnTuning(C.Structure):
    """symph_attn_tuning: a field left 0 keeps the library's default."""
    _fields_ = [("slots", C.c_int32), ("c_min", C.c_int32), ("coarse", C.c_int32), ("decode", C.c_int32),
                ("decode_wgs", C.c_int32), ("reserved", C.c_int32 * 3)]


class _PoolChange(C.Structure):
    _fields_ = [("session", C.c_int64), ("layer", C.c_int32), ("kind", C.c_int32), ("n_slots", C.c_int32),
                ("slot_begin", C.c_int32)]


PoolChange = _PoolChange


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libsymph.so (built in-tree by ``paper_2412_16434_amd/build.py``). Raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2412_16434_amd.build` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(_LIB_PATH)
    i32, i64, vp, f32 = C.c_int32, C.c_int64, C.c_void_p, C.c_float
    cp = C.POINTER(_CacheStruct)
    lib.symph_kv_buffer_bytes.restype = i64
    lib.symph_kv_buffer_bytes.argtypes = [cp, i64]
    for fn in (lib.symph_kv_pack, lib.symph_kv_unpack):
        fn.restype = i32
        fn.argtypes = [cp, vp, i32, vp, vp, i32, i64, vp, i64, vp]
    for fn in (lib.symph_kv_pack_layers, lib.symph_kv_unpack_layers, lib.symph_kv_pack_batch_layers,
               lib.symph_kv_unpack_batch_layers):
        fn.restype = i32
        fn.argtypes = [cp, i32, i32, vp, i32, vp, vp, i32, i64, vp, i64, vp]
    for fn in (lib.symph_stage_batch_layers_to_host, lib.symph_stage_batch_layers_to_device):
        fn.restype = i32
        fn.argtypes = [vp, vp, cp, i32, i32, i64, vp, vp, vp]
    for fn in (lib.symph_kv_pack_tail, lib.symph_kv_unpack_tail):
        fn.restype = i32
        fn.argtypes = [cp, vp, i32, vp, vp, vp, i32, i64, vp, i64, vp]
    for fn in (lib.symph_kv_pack_units, lib.symph_kv_unpack_units):
        fn.restype = i32
        fn.argtypes = [cp, vp, i32, vp, vp, vp, i32, i64, vp, i64, vp]
    for fn in (lib.symph_stage_layer_to_host, lib.symph_stage_layer_to_device):
        fn.restype = i32
        fn.argtypes = [vp, vp, cp, i32, vp, vp, i32, vp, vp, vp]
    lib.symph_kv_append.restype = i32
    lib.symph_kv_append.argtypes = [cp, i32, vp, vp, vp, vp, vp, i32, i32, i32, vp]
    lib.symph_prefix_prefill_attn.restype = i32
    lib.symph_prefix_prefill_attn.argtypes = [cp, i32, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, f32,
                                              vp, i64, vp]
    lib.symph_prefix_prefill_attn_workspace_bytes.restype = i64
    lib.symph_prefix_prefill_attn_workspace_bytes.argtypes = [cp, i32, i32, i32, i32, i32]
    tp = C.POINTER(AttnTuning)
    lib.symph_prefix_prefill_attn_tuned.restype = i32
    lib.symph_prefix_prefill_attn_tuned.argtypes = lib.symph_prefix_prefill_attn.argtypes + [tp]
    lib.symph_prefix_prefill_attn_workspace_bytes_tuned.restype = i64
    lib.symph_prefix_prefill_attn_workspace_bytes_tuned.argtypes = [cp, i32, i32, i32, i32, i32, tp]
    lib.symph_prefix_prefill_attn_static.restype = i32
    lib.symph_prefix_prefill_attn_static.argtypes = lib.symph_prefix_prefill_attn.argtypes[:16] + [vp]
    lib.symph_debug_attn_flags.restype = i32
    lib.symph_debug_attn_flags.argtypes = [vp, vp, C.POINTER(i32)]
    lib.symph_build_tables.restype = i32
    lib.symph_build_tables.argtypes = [vp, vp, vp, i32, vp, i32, vp, i32, vp, i32, i32, i64, vp, vp, vp, vp, vp, vp, vp]
    lib.symph_tree_mask.restype = i32
    lib.symph_tree_mask.argtypes = [vp, vp, vp, i32, i32, i32, vp, i32, vp, vp]
    lib.symph_tree_attn.restype = i32
    lib.symph_tree_attn.argtypes = [cp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, i32, i32, i32, i32, i32, f32, vp, i64, vp]
    lib.symph_tree_attn_workspace_bytes.restype = i64
    lib.symph_tree_attn_workspace_bytes.argtypes = [cp, i32, i32, i32, i32, i32]
    lib.symph_tree_accept.restype = i32
    lib.symph_tree_accept.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
    lib.symph_kv_commit.restype = i32
    lib.symph_kv_commit.argtypes = [cp, vp, vp, i32, vp, vp, i32, vp]
    lib.symph_beam_select.restype = i32
    lib.symph_beam_select.argtypes = [vp, i64, i32, i32, i32, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, i64, vp]
    lib.symph_beam_select_workspace_bytes.restype = i64
    lib.symph_beam_select_workspace_bytes.argtypes = [i32, i32, i32]
    lib.symph_kv_fork.restype = i32
    lib.symph_kv_fork.argtypes = [vp, i32, vp, vp, i32, vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.symph_kv_copy_blocks.restype = i32
    lib.symph_kv_copy_blocks.argtypes = [cp, vp, vp, vp, i32, vp]
    lib.symph_kv_free.restype = i32
    lib.symph_kv_free.argtypes = [vp, vp, vp, i32, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, i64, vp]
    lib.symph_kv_compact.restype = i32
    lib.symph_kv_compact.argtypes = [vp, i32, i32, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, i64, vp]
    for fn in (lib.symph_kv_free_workspace_bytes, lib.symph_kv_compact_workspace_bytes):
        fn.restype = i64
        fn.argtypes = [i32]
    for fn in (lib.symph_stage_to_host, lib.symph_stage_to_device):
        fn.restype = i32
        fn.argtypes = [vp, vp, i64, vp, vp, vp]
    lib.symph_device_copy.restype = i32
    lib.symph_device_copy.argtypes = [vp, vp, i64, vp]
    lib.symph_mfma_reference.restype = i32
    lib.symph_mfma_reference.argtypes = [i32, C.POINTER(C.c_int64), vp, vp]
    lib.symph_debug_check_tables.restype = i32
    lib.symph_debug_check_tables.argtypes = [cp, vp, i32, vp, i32, i32, vp, C.POINTER(i32)]
    lib.symph_status_string.restype = C.c_char_p
    lib.symph_status_string.argtypes = [i32]
    ip = C.POINTER(i32)
    lib.symph_pool_create.restype = i32
    lib.symph_pool_create.argtypes = [i32, i32, i32, C.POINTER(vp)]
    lib.symph_pool_destroy.restype = None
    lib.symph_pool_destroy.argtypes = [vp]
    lib.symph_pool_advise.restype = i32
    lib.symph_pool_advise.argtypes = [vp, i64, i32]
    lib.symph_pool_drop.restype = i32
    lib.symph_pool_drop.argtypes = [vp, i64]
    lib.symph_pool_claim.restype = i32
    lib.symph_pool_claim.argtypes = [vp, i64, ip, i32, ip]
    lib.symph_pool_framework_take.restype = i32
    lib.symph_pool_framework_take.argtypes = [vp, i32, ip]
    lib.symph_pool_framework_give.restype = i32
    lib.symph_pool_framework_give.argtypes = [vp, i32, ip]
    lib.symph_pool_settle.restype = i32
    lib.symph_pool_settle.argtypes = [vp, C.POINTER(_PoolChange), i32, ip, i32, ip, ip]
    lib.symph_pool_resident_layers.restype = i32
    lib.symph_pool_resident_layers.argtypes = [vp, i64]
    lib.symph_pool_unit_slots.restype = i32
    lib.symph_pool_unit_slots.argtypes = [vp, i64]
    lib.symph_pool_table.restype = i32
    lib.symph_pool_table.argtypes = [vp, i64, i32, ip, i32]
    lib.symph_pool_counts.restype = i32
    lib.symph_pool_counts.argtypes = [vp, ip, ip, ip]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().symph_status_string(int(status)).decode()


@dataclass
class KVCache:
    """A paged K,V cache in device memory: two torch tensors ``[L][n_blocks][bs][H_kv][d]`` (bf16 or fp32)."""
    k_pool: "object"
    v_pool: "object"

    def __post_init__(self):
        import torch
        k, v = self.k_pool, self.v_pool
        if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("pools must be two [L][n_blocks][bs][H_kv][d] tensors of one dtype")
        if k.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("cache dtype must be bfloat16 or float32")
        if k.stride()[2:] != (k.shape[3] * k.shape[4], k.shape[4], 1) or v.stride() != k.stride():
            raise ValueError("token, head and dim axes must be dense")

    @property
    def dtype_code(self) -> int:
        return SYMPH_BF16 if self.k_pool.dtype == _torch().bfloat16 else SYMPH_FP32

    def struct(self) -> _CacheStruct:
        k = self.k_pool
        layer_stride, block_stride = k.stride()[:2]
        return _CacheStruct(k.data_ptr(), self.v_pool.data_ptr(), layer_stride, block_stride, *k.shape, self.dtype_code)


_torch_module = None


def _torch():
    """The torch module: imported on the first call that needs it, not with the package."""
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dev(t, name: str, dtype=None, allow_none: bool = False, pinned_ok: bool = False):
    """Check what the C side cannot see: the tensor is on the GPU (or, for buffers, pinned host memory), contiguous and
    of the element type the entry point reads it as.  Returns its data pointer."""
    if t is None:
        if allow_none:
            return None
        raise ValueError(f"{name} is required")
    if not (t.is_cuda or (pinned_ok and t.is_pinned())):
        raise ValueError(f"{name} must be a device tensor" + (" or pinned host memory" if pinned_ok else ""))
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, not {t.dtype}")
    return t.data_ptr()


def _table(t, name: str = "block_table"):
    """(pointer, row stride in entries) of an int32 [n_sessions][stride] block table on the device; (None, 0) if absent."""
    if t is None:
        return None, 0
    if t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D int32 tensor [n_sessions][max_blocks]")
    return _dev(t, name, _torch().int32), t.shape[1]


def _lens(t, name: str):
    return _dev(t, name, _torch().int32)


def _offsets(t, name: str):
    return _dev(t, name, _torch().int64)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        # The handle of the current stream without the Stream object around it (2.7 us of an 11.5 us call).
        torch = _torch()
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None and torch.cuda.is_initialized():
            return raw(torch.cuda.current_device()) or None
        return torch.cuda.current_stream().cuda_stream or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _event_ptr(event) -> int:
    """hipEvent_t of a torch.cuda.Event (torch creates the handle on the first record)."""
    if isinstance(event, int):
        return event
    if not event.cuda_event:
        event.record()
    return event.cuda_event


def _check(status: int, where: str) -> None:
    if status != 0:
        raise SymphError(status, where)


def kv_buffer_bytes(cache: KVCache, total_tokens: int) -> int:
    st = cache.struct()
    n = load_library().symph_kv_buffer_bytes(C.byref(st), int(total_tokens))
    if n < 0:
        raise SymphError(-1, "symph_kv_buffer_bytes")
    return int(n)


def _migrate(fn_name: str, cache: KVCache, head_args, block_table, prefix_lens, mid, offsets, total_tokens, buf, stream):
    """Shared marshalling of the pack / unpack family: (cache, [layer range], table, stride, lens, [extra], offsets, n,
    total, buf, bytes, stream)."""
    st = cache.struct()
    tp, stride = _table(block_table)
    _check(getattr(load_library(), fn_name)(
        C.byref(st), *head_args, tp, stride, _lens(prefix_lens, "prefix_lens"), *mid, _offsets(offsets, "offsets"),
        prefix_lens.shape[0], int(total_tokens), _dev(buf, "buf", pinned_ok=True), buf.numel() * buf.element_size(),
        _stream_ptr(stream)), fn_name)


def kv_pack(cache: KVCache, block_table, prefix_lens, buf_token_offsets, total_tokens: int, buf, stream=None) -> None:
    """Gather into ``buf`` (any dtype, 1-D device tensor of at least kv_buffer_bytes bytes)."""
    _migrate("symph_kv_pack", cache, (), block_table, prefix_lens, (), buf_token_offsets, total_tokens, buf, stream)


def kv_unpack(cache: KVCache, dst_block_table, prefix_lens, buf_token_offsets, total_tokens: int, buf,
              stream=None) -> None:
    _migrate("symph_kv_unpack", cache, (), dst_block_table, prefix_lens, (), buf_token_offsets, total_tokens, buf,
             stream)


def kv_pack_layers(cache: KVCache, layer_begin: int, layer_end: int, block_table, prefix_lens, buf_token_offsets,
                   total_tokens: int, buf, stream=None) -> None:
    """Gather layers ``layer_begin .. layer_end-1`` only into ``buf`` (whole-cache layout)."""
    _migrate("symph_kv_pack_layers", cache, (int(layer_begin), int(layer_end)), block_table, prefix_lens, (),
             buf_token_offsets, total_tokens, buf, stream)


def kv_unpack_layers(cache: KVCache, layer_begin: int, layer_end: int, dst_block_table, prefix_lens,
                     buf_token_offsets, total_tokens: int, buf, stream=None) -> None:
    _migrate("symph_kv_unpack_layers", cache, (int(layer_begin), int(layer_end)), dst_block_table, prefix_lens, (),
             buf_token_offsets, total_tokens, buf, stream)


def kv_pack_batch_layers(cache: KVCache, layer_begin: int, layer_end: int, block_table, prefix_lens, buf_token_offsets,
                         total_tokens: int, buf, stream=None) -> None:
    """Gather layers ``layer_begin .. layer_end-1`` into ``buf`` laid out layer -> session -> K|V -> token."""
    _migrate("symph_kv_pack_batch_layers", cache, (int(layer_begin), int(layer_end)), block_table, prefix_lens, (),
             buf_token_offsets, total_tokens, buf, stream)


def kv_unpack_batch_layers(cache: KVCache, layer_begin: int, layer_end: int, dst_block_table, prefix_lens,
                           buf_token_offsets, total_tokens: int, buf, stream=None) -> None:
    _migrate("symph_kv_unpack_batch_layers", cache, (int(layer_begin), int(layer_end)), dst_block_table, prefix_lens, (),
             buf_token_offsets, total_tokens, buf, stream)


def stage_batch_layers_to_host(h_pinned, d_buf, cache: KVCache, layer_begin: int, layer_end: int, total_tokens: int,
                               producer_stream, side_stream, event) -> None:
    """One copy of the layers' contiguous piece of a layer-major buffer, device -> pinned host, on ``side_stream``."""
    st = cache.struct()
    _check(load_library().symph_stage_batch_layers_to_host(
        _ptr(h_pinned), _ptr(d_buf), C.byref(st), int(layer_begin), int(layer_end), int(total_tokens),
        _stream_ptr(producer_stream), _stream_ptr(side_stream), _event_ptr(event)), "symph_stage_batch_layers_to_host")


def stage_batch_layers_to_device(d_buf, h_pinned, cache: KVCache, layer_begin: int, layer_end: int, total_tokens: int,
                                 consumer_stream, side_stream, event) -> None:
    st = cache.struct()
    _check(load_library().symph_stage_batch_layers_to_device(
        _ptr(d_buf), _ptr(h_pinned), C.byref(st), int(layer_begin), int(layer_end), int(total_tokens),
        _stream_ptr(consumer_stream), _stream_ptr(side_stream), _event_ptr(event)), "symph_stage_batch_layers_to_device")


def _units(fn_name, slots: KVCache, unit_table, unit_lens, unit_token_offsets, unit_chunk_rows, total_unit_tokens, buf,
           stream):
    st = slots.struct()
    tp, stride = _table(unit_table, "unit_table")
    _check(getattr(load_library(), fn_name)(
        C.byref(st), tp, stride, _lens(unit_lens, "unit_lens"), _offsets(unit_token_offsets, "unit_token_offsets"),
        _offsets(unit_chunk_rows, "unit_chunk_rows"), unit_lens.shape[0], int(total_unit_tokens),
        _dev(buf, "buf", pinned_ok=True), buf.numel() * buf.element_size(), _stream_ptr(stream)), fn_name)


def kv_pack_units(slots: KVCache, unit_table, unit_lens, unit_token_offsets, unit_chunk_rows, total_unit_tokens: int,
                  buf, stream=None) -> None:
    """Gather single layers of sessions from one pool of slots (a one-layer KVCache) into their chunks of ``buf``."""
    _units("symph_kv_pack_units", slots, unit_table, unit_lens, unit_token_offsets, unit_chunk_rows, total_unit_tokens,
           buf, stream)


def kv_unpack_units(slots: KVCache, unit_table, unit_lens, unit_token_offsets, unit_chunk_rows, total_unit_tokens: int,
                    buf, stream=None) -> None:
    _units("symph_kv_unpack_units", slots, unit_table, unit_lens, unit_token_offsets, unit_chunk_rows,
           total_unit_tokens, buf, stream)


def debug_check_tables(cache: KVCache, block_table, lens, is_destination: bool, stream=None) -> int:
    """-1 if the table and lengths keep the contract the kernels rely on, else the first offending session."""
    st = cache.struct()
    bad = C.c_int32(-1)
    tp, stride = _table(block_table)
    rc = load_library().symph_debug_check_tables(
        C.byref(st), tp, stride, _lens(lens, "lens"), lens.shape[0], 1 if is_destination else 0, _stream_ptr(stream),
        C.byref(bad))
    if rc != 0 and bad.value < 0:
        _check(rc, "symph_debug_check_tables")
    return bad.value


def kv_pack_tail(cache: KVCache, block_table, prefix_lens, tail_begin, tail_offsets, total_tail_tokens: int, buf,
                 stream=None) -> None:
    """Gather tokens ``tail_begin[s] .. prefix_lens[s]-1`` of every session (all layers) into ``buf``."""
    _migrate("symph_kv_pack_tail", cache, (), block_table, prefix_lens, (_lens(tail_begin, "tail_begin"),),
             tail_offsets, total_tail_tokens, buf, stream)


def kv_unpack_tail(cache: KVCache, dst_block_table, prefix_lens, tail_begin, tail_offsets, total_tail_tokens: int, buf,
                   stream=None) -> None:
    """Scatter a tail buffer (see ``kv_pack_tail``) into the cache through ``dst_block_table``."""
    _migrate("symph_kv_unpack_tail", cache, (), dst_block_table, prefix_lens, (_lens(tail_begin, "tail_begin"),),
             tail_offsets, total_tail_tokens, buf, stream)


def kv_append(cache: KVCache, layer: int, k_new, v_new, cu_new_lens, prefix_lens, block_table, stream=None) -> None:
    """Write the new turn's K,V rows of ``layer`` into the paged cache behind each session's prefix."""
    st = cache.struct()
    dt = cache.k_pool.dtype
    tp, stride = _table(block_table)
    _check(load_library().symph_kv_append(
        C.byref(st), int(layer), _dev(k_new, "k_new", dt), _dev(v_new, "v_new", dt), _lens(cu_new_lens, "cu_new_lens"),
        _lens(prefix_lens, "prefix_lens"), tp, stride, prefix_lens.shape[0], k_new.shape[0], _stream_ptr(stream)),
        "symph_kv_append")


def _tuning_ref(tuning):
    return None if tuning is None else C.byref(tuning)


def prefix_prefill_attn_workspace_bytes(cache: KVCache, n_sessions: int, n_q_heads: int, total_new_tokens: int,
                                        max_new_len: int, max_prefix_len: int, tuning: Optional[AttnTuning] = None) -> int:
    st = cache.struct()
    lib = load_library()
    if tuning is None:
        n = lib.symph_prefix_prefill_attn_workspace_bytes(C.byref(st), n_sessions, n_q_heads, total_new_tokens,
                                                          max_new_len, max_prefix_len)
    else:
        n = lib.symph_prefix_prefill_attn_workspace_bytes_tuned(C.byref(st), n_sessions, n_q_heads, total_new_tokens,
                                                                max_new_len, max_prefix_len, C.byref(tuning))
    if n < 0:
        raise SymphError(-1, "symph_prefix_prefill_attn_workspace_bytes")
    return int(n)


def _attn_args(cache: KVCache, layer, q, k_new, v_new, out, cu_new_lens, prefix_lens, block_table, max_new_len,
               max_prefix_len, scale):
    """The argument list the attention entry points share, up to and including ``scale``."""
    dt = cache.k_pool.dtype
    if q.dim() != 3 or out.shape != q.shape or k_new.dim() != 3 or v_new.shape != k_new.shape:
        raise ValueError("q / out must be [T][H_q][d] and k_new / v_new [T][H_kv][d]")
    tp, stride = _table(block_table)
    i32 = _torch().int32
    if (q.is_cuda and k_new.is_cuda and v_new.is_cuda and out.is_cuda and cu_new_lens.is_cuda and prefix_lens.is_cuda
            and q.dtype == dt and k_new.dtype == dt and v_new.dtype == dt and out.dtype == dt and cu_new_lens.dtype == i32
            and prefix_lens.dtype == i32 and q.is_contiguous() and k_new.is_contiguous() and v_new.is_contiguous()
            and out.is_contiguous() and cu_new_lens.is_contiguous() and prefix_lens.is_contiguous()):
        ptrs = [q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), out.data_ptr(), cu_new_lens.data_ptr(),
                prefix_lens.data_ptr()]
    else:  # (one of these says what is wrong)
        ptrs = [_dev(q, "q", dt), _dev(k_new, "k_new", dt), _dev(v_new, "v_new", dt), _dev(out, "out", dt),
                _lens(cu_new_lens, "cu_new_lens"), _lens(prefix_lens, "prefix_lens")]
    n_tokens, n_q_heads, _ = q.shape
    return [int(layer), *ptrs, tp, stride, prefix_lens.shape[0], n_q_heads, n_tokens, int(max_new_len),
            int(max_prefix_len), float(scale)]


_attn_call = None
_draft_calls = None  # the compiled marshalling's module, or False: the general path makes the drafted step's calls


def _load_draft_calls():
    """The same for the operators of a drafted step (they share the module: what it needs of torch is bound once)."""
    global _draft_calls
    compiled = _attn_call or _load_attn_call()
    if compiled is not _attn_call:  # (no library)
        return False
    _draft_calls = False
    module = getattr(compiled, "__self__", None)
    if hasattr(module, "bind_draft"):
        lib = load_library()
        module.bind_draft(*(C.cast(f, C.c_void_p).value for f in (
            lib.symph_build_tables, lib.symph_tree_mask, lib.symph_tree_attn, lib.symph_tree_accept, lib.symph_kv_commit)),
            _torch().int64)
        _draft_calls = module
    return _draft_calls


_beam_calls = None  # the same for beam search


def _load_beam_calls():
    global _beam_calls
    compiled = _attn_call or _load_attn_call()
    if compiled is not _attn_call:  # (no library)
        return False
    _beam_calls = False
    module = getattr(compiled, "__self__", None)
    if hasattr(module, "bind_beam"):
        if _draft_calls is None:
            _load_draft_calls()
        lib, tensor = load_library(), _torch().Tensor
        module.bind_beam(*(C.cast(f, C.c_void_p).value for f in (
            lib.symph_beam_select, lib.symph_kv_fork, lib.symph_kv_copy_blocks, lib.symph_kv_free, lib.symph_kv_compact)),
            tensor, getattr(tensor, "__dlpack_c_exchange_api__", None))
        _beam_calls = module
    return _beam_calls


def _beam_call(stream):
    return stream is None and (_load_beam_calls() if _beam_calls is None else _beam_calls)


def _on_this_device(stream, **tensors) -> None:
    """Without a stream the call goes to the current device's: the tensors have to be there."""
    if stream is None:
        torch = _torch()
        for name, t in tensors.items():
            if t is not None and t.is_cuda and t.get_device() != torch.cuda.current_device():
                raise ValueError(f"{name} is on cuda:{t.get_device()}, the current device is cuda:{torch.cuda.current_device()}")


def _load_attn_call():
    """The compiled marshalling of the ordinary attention call (``csrc/attn_call.c``), bound to the library's entry point; where
    it is not built (or not for this interpreter), or torch lacks what it needs, what leaves every call to the general path."""
    global _attn_call
    try:
        lib = load_library()
    except ImportError:  # (the general path says so, behind its checks)
        return lambda *args: None
    torch = _torch()
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    try:
        from . import _attn_call as module
    except ImportError:
        module = None
    if module is None or raw is None or device is None:
        _attn_call = lambda *args: None
    else:
        module.bind(C.cast(lib.symph_prefix_prefill_attn, C.c_void_p).value, torch.bfloat16, torch.float32, torch.int32, raw,
                    device)
        _attn_call = module.attn
    return _attn_call


def prefix_prefill_attn(cache: KVCache, layer: int, q, k_new, v_new, out, cu_new_lens, prefix_lens, block_table,
                        max_new_len: int, max_prefix_len: int, scale: float, workspace=None, stream=None,
                        tuning: Optional[AttnTuning] = None) -> None:
    """out[T][H_q][d] <- attention of the new turn over [cached prefix ; causal new tokens] for one layer."""
    if stream is None and tuning is None and type(cache) is KVCache:  # (a subclass may have a struct() of its own)
        status = (_attn_call or _load_attn_call())(cache.k_pool, cache.v_pool, layer, q, k_new, v_new, out, cu_new_lens,
                                                   prefix_lens, block_table, max_new_len, max_prefix_len, scale, workspace)
        if status is not None:
            return _check(status, "symph_prefix_prefill_attn")
    st = cache.struct()
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    args = _attn_args(cache, layer, q, k_new, v_new, out, cu_new_lens, prefix_lens, block_table, max_new_len,
                      max_prefix_len, scale)
    args += [_dev(workspace, "workspace", allow_none=True), ws_bytes, _stream_ptr(stream)]
    lib = load_library()
    if tuning is None:
        _check(lib.symph_prefix_prefill_attn(C.byref(st), *args), "symph_prefix_prefill_attn")
    else:
        _check(lib.symph_prefix_prefill_attn_tuned(C.byref(st), *args, C.byref(tuning)),
               "symph_prefix_prefill_attn_tuned")


def prefix_prefill_attn_static(cache: KVCache, layer: int, q, k_new, v_new, out, cu_new_lens, prefix_lens, block_table,
                               max_new_len: int, max_prefix_len: int, scale: float, stream=None) -> None:
    """The same attention without a workspace argument: the library's fixed scratch array is used (nothing allocated)."""
    st = cache.struct()
    args = _attn_args(cache, layer, q, k_new, v_new, out, cu_new_lens, prefix_lens, block_table, max_new_len,
                      max_prefix_len, scale)
    _check(load_library().symph_prefix_prefill_attn_static(C.byref(st), *args, _stream_ptr(stream)),
           "symph_prefix_prefill_attn_static")


def _vector(t, name: str, dtype, length: Optional[int] = None, allow_none: bool = False):
    """Pointer of a 1-D device tensor of ``dtype`` with at least ``length`` entries."""
    if t is None and allow_none:
        return None
    ptr = _dev(t, name, dtype)
    if t.dim() != 1:
        raise ValueError(f"{name} must be 1-D")
    if length is not None and t.shape[0] < length:
        raise ValueError(f"{name} must have {length} entries, not {t.shape[0]}")
    return ptr


def build_tables(prefix_lens, new_lens, block_table, free_blocks, block_size: int, n_blocks: int, total_new_tokens: int,
                 cu_new_lens=None, token_offsets=None, slot_map=None, positions=None, blocks_taken=None, held_blocks=None,
                 held_after=None, free_begin=None, stream=None) -> None:
    """Block table entries for ``new_lens`` more tokens of every session, taken from ``free_blocks`` in session order, and
    what is asked for of: prefix sums (``cu_new_lens`` int32, ``token_offsets`` int64), the slot of every new token in a
    layer's pool (``slot_map`` int64, -1: none), ``positions`` and the entries of the free list used up so far."""
    calls = stream is None and (_load_draft_calls() if _draft_calls is None else _draft_calls)
    if calls:
        status = calls.tables(prefix_lens, new_lens, block_table, free_blocks, block_size, n_blocks, total_new_tokens,
                              cu_new_lens, token_offsets, slot_map, positions, blocks_taken, held_blocks, held_after,
                              free_begin)
        if status is not None:
            return _check(status, "symph_build_tables")
    torch = _torch()
    i32, i64 = torch.int32, torch.int64
    n, t = prefix_lens.shape[0], int(total_new_tokens)
    tp, stride = _table(block_table)
    if tp is not None and block_table.shape[0] < n:
        raise ValueError(f"block_table must have {n} rows, not {block_table.shape[0]}")
    _check(load_library().symph_build_tables(
        _vector(prefix_lens, "prefix_lens", i32), _vector(new_lens, "new_lens", i32, n),
        _vector(held_blocks, "held_blocks", i32, n, True), n, tp, stride, _vector(free_blocks, "free_blocks", i32),
        free_blocks.shape[0], _vector(free_begin, "free_begin", i32, 1, True), int(block_size), int(n_blocks), t,
        _vector(cu_new_lens, "cu_new_lens", i32, n + 1, True), _vector(token_offsets, "token_offsets", i64, n + 1, True),
        _vector(slot_map, "slot_map", i64, t, True), _vector(positions, "positions", i32, t, True),
        _vector(blocks_taken, "blocks_taken", i32, 1, True), _vector(held_after, "held_after", i32, n, True),
        _stream_ptr(stream)), "symph_build_tables")


def _mask_words(mask, rows: int, name: str):
    """(pointer, words of a row) of an int64 [rows][words] mask."""
    if mask is None or mask.dim() != 2 or mask.shape[0] < rows:
        raise ValueError(f"{name} must be an int64 tensor [{rows}][words]")
    return _dev(mask, name, _torch().int64), mask.shape[1]


def tree_mask(parents, cu_new_lens, max_new_len: int, mask, prefix_lens=None, positions=None, stream=None) -> None:
    """mask[T][words] (int64, 64 bits a word) <- bit j of row i: node j is node i or an ancestor of it.  ``parents`` holds
    indices within the session (anything outside 0 .. i-1: a root); ``positions`` <- prefix length + number of ancestors."""
    calls = stream is None and (_load_draft_calls() if _draft_calls is None else _draft_calls)
    if calls:
        status = calls.mask(parents, cu_new_lens, max_new_len, mask, prefix_lens, positions)
        if status is not None:
            return _check(status, "symph_tree_mask")
    i32 = _torch().int32
    n, t = cu_new_lens.shape[0] - 1, parents.shape[0]
    mp, words = _mask_words(mask, t, "mask")
    _check(load_library().symph_tree_mask(
        _vector(parents, "parents", i32), _vector(cu_new_lens, "cu_new_lens", i32),
        _vector(prefix_lens, "prefix_lens", i32, n, True), n, t, int(max_new_len), mp, words,
        _vector(positions, "positions", i32, t, True), _stream_ptr(stream)), "symph_tree_mask")


def tree_attn_workspace_bytes(cache: KVCache, n_sessions: int, n_q_heads: int, total_new_tokens: int, max_new_len: int,
                              max_prefix_len: int) -> int:
    st = cache.struct()
    n = load_library().symph_tree_attn_workspace_bytes(C.byref(st), n_sessions, n_q_heads, total_new_tokens, max_new_len,
                                                       max_prefix_len)
    if n < 0:
        raise SymphError(-1, "symph_tree_attn_workspace_bytes")
    return int(n)


def tree_attn(cache: KVCache, layer: int, q, k_new, v_new, out, tree_mask, cu_new_lens, prefix_lens, block_table,
              max_new_len: int, max_prefix_len: int, scale: float, workspace=None, stream=None) -> None:
    """out[T][H_q][d] <- attention of drafted tokens over [cached prefix ; the drafted tokens whose bit is set in
    ``tree_mask`` (int64 [T][words])] for one layer.  A row that sees nothing is zero."""
    calls = stream is None and type(cache) is KVCache and (_load_draft_calls() if _draft_calls is None else _draft_calls)
    if calls:
        status = calls.tree(cache.k_pool, cache.v_pool, layer, q, k_new, v_new, out, cu_new_lens, prefix_lens, block_table,
                            max_new_len, max_prefix_len, scale, workspace, tree_mask)
        if status is not None:
            return _check(status, "symph_tree_attn")
    st = cache.struct()
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    args = _attn_args(cache, layer, q, k_new, v_new, out, cu_new_lens, prefix_lens, block_table, max_new_len,
                      max_prefix_len, scale)
    n, (hkv, d) = prefix_lens.shape[0], cache.k_pool.shape[3:]
    if q.shape[2] != d or k_new.shape != (q.shape[0], hkv, d):
        raise ValueError(f"q must be [T][H_q][{d}] and k_new / v_new [T][{hkv}][{d}]")
    if cu_new_lens.shape[0] < n + 1 or (block_table is not None and block_table.shape[0] < n):
        raise ValueError(f"cu_new_lens must have {n + 1} entries and block_table {n} rows")
    mp, words = _mask_words(tree_mask, q.shape[0], "tree_mask")
    _check(load_library().symph_tree_attn(C.byref(st), *args[:5], mp, words, *args[5:],
                                          _dev(workspace, "workspace", allow_none=True), ws_bytes, _stream_ptr(stream)),
           "symph_tree_attn")


def tree_accept(draft_tokens, parents, target_tokens, cu_new_lens, prefix_lens, rows, n_accepted, next_tokens,
                new_prefix_lens=None, stream=None) -> None:
    """The path of every session's tree that agrees with ``target_tokens`` (the model's token behind each node): ``rows`` <-
    rows of the accepted nodes from entry cu[s] on, then -1; ``n_accepted``, ``next_tokens`` and the new lengths per session."""
    calls = stream is None and (_load_draft_calls() if _draft_calls is None else _draft_calls)
    if calls:
        status = calls.accept(draft_tokens, parents, target_tokens, cu_new_lens, prefix_lens, rows, n_accepted, next_tokens,
                              new_prefix_lens)
        if status is not None:
            return _check(status, "symph_tree_accept")
    i32 = _torch().int32
    n, t = cu_new_lens.shape[0] - 1, draft_tokens.shape[0]
    _check(load_library().symph_tree_accept(
        _vector(draft_tokens, "draft_tokens", i32), _vector(parents, "parents", i32, t),
        _vector(target_tokens, "target_tokens", i32, t), _vector(cu_new_lens, "cu_new_lens", i32),
        _vector(prefix_lens, "prefix_lens", i32, n, True), n, t, _vector(rows, "rows", i32, t),
        _vector(n_accepted, "n_accepted", i32, n), _vector(next_tokens, "next_tokens", i32, n),
        _vector(new_prefix_lens, "new_prefix_lens", i32, n, True), _stream_ptr(stream)), "symph_tree_accept")


def kv_commit(cache: KVCache, k_new, v_new, rows, slot_map, stream=None) -> None:
    """Row ``rows[t]`` of ``k_new`` / ``v_new`` [L][n_rows][H_kv][d] into slot ``slot_map[t]`` of every layer, for every t where
    both are valid (>= 0 and in range)."""
    calls = stream is None and type(cache) is KVCache and (_load_draft_calls() if _draft_calls is None else _draft_calls)
    if calls:
        status = calls.commit(cache.k_pool, cache.v_pool, k_new, v_new, rows, slot_map)
        if status is not None:
            return _check(status, "symph_kv_commit")
    st = cache.struct()
    k = cache.k_pool
    if k_new.dim() != 4 or v_new.shape != k_new.shape or (k_new.shape[0], *k_new.shape[2:]) != (k.shape[0], *k.shape[3:]):
        raise ValueError("k_new / v_new must be [L][n_rows][H_kv][d]")
    torch = _torch()
    n = rows.shape[0]
    _check(load_library().symph_kv_commit(
        C.byref(st), _dev(k_new, "k_new", k.dtype), _dev(v_new, "v_new", k.dtype), k_new.shape[1],
        _vector(rows, "rows", torch.int32), _vector(slot_map, "slot_map", torch.int64, n), n, _stream_ptr(stream)),
        "symph_kv_commit")


def beam_select_workspace_bytes(n_rows: int, vocab: int, max_next: int) -> int:
    n = load_library().symph_beam_select_workspace_bytes(int(n_rows), int(vocab), int(max_next))
    if n < 0:
        raise SymphError(-1, "symph_beam_select_workspace_bytes")
    return int(n)


def _scratch(workspace):
    """(pointer, bytes) of a workspace, which may be None."""
    if workspace is None:
        return None, 0
    return _dev(workspace, "workspace"), workspace.numel() * workspace.element_size()


def beam_select(logits, scores, cu_rows, cu_next, max_next: int, parents, tokens, next_scores, end_token: int = -1,
                end_scores=None, workspace=None, stream=None) -> None:
    """The best ``cu_next[s+1] - cu_next[s]`` continuations of every session over its beams (rows ``cu_rows[s]`` .. of ``logits``
    [n_rows][vocab], bf16 or fp32, dense along the vocabulary) by score = ``scores`` + log-probability: ``parents`` (the beam's
    row), ``tokens`` and ``next_scores``, best first; -1, -1 and -inf where there are fewer.  ``end_token`` never continues a beam;
    its score goes to ``end_scores`` [n_rows] where it is among the session's best."""
    calls = _beam_call(stream)
    if calls:
        status = calls.select_beams(logits, scores, cu_rows, cu_next, max_next, parents, tokens, next_scores, end_token, end_scores,
                                    workspace)
        if status is not None:
            return _check(status, "symph_beam_select")
    torch = _torch()
    i32, f32 = torch.int32, torch.float32
    if logits.dim() != 2 or logits.dtype not in (torch.bfloat16, f32):
        raise ValueError("logits must be a bfloat16 or float32 tensor [n_rows][vocab]")
    if not logits.is_cuda:
        raise ValueError("logits must be a device tensor")
    (rows, vocab), (row_stride, step) = logits.shape, logits.stride()
    if (vocab > 1 and step != 1) or (rows > 1 and row_stride < vocab):
        raise ValueError("logits must be dense along the vocabulary, rows apart")
    _on_this_device(stream, logits=logits, scores=scores, cu_rows=cu_rows, cu_next=cu_next, parents=parents, tokens=tokens,
                    next_scores=next_scores, end_scores=end_scores, workspace=workspace)
    n, total = cu_rows.shape[0] - 1, parents.shape[0]
    wp, ws_bytes = _scratch(workspace)
    _check(load_library().symph_beam_select(
        logits.data_ptr(), max(row_stride, vocab), SYMPH_BF16 if logits.dtype == torch.bfloat16 else SYMPH_FP32, rows, vocab,
        _vector(scores, "scores", f32, rows), _vector(cu_rows, "cu_rows", i32, 1), _vector(cu_next, "cu_next", i32, n + 1), n, total,
        int(max_next), int(end_token), _vector(parents, "parents", i32), _vector(tokens, "tokens", i32, total),
        _vector(next_scores, "next_scores", f32, total), _vector(end_scores, "end_scores", f32, rows, True), wp, ws_bytes,
        _stream_ptr(stream)), "symph_beam_select")


def _rows_table(t, name: str, rows: int, stride: Optional[int] = None):
    """(pointer, row stride) of a block table of at least ``rows`` rows."""
    if t is None:
        raise ValueError(f"{name} is required")
    tp, width = _table(t, name)
    if t.shape[0] < rows or (stride is not None and width != stride):
        raise ValueError(f"{name} must be [{rows}][{'max_blocks' if stride is None else stride}], not {list(t.shape)}")
    return tp, width


def kv_fork(parents, lens, block_table, refs, free_blocks, block_size: int, table_out, lens_out, refs_after, copy_src, copy_dst,
            copy_tokens, held_blocks=None, held_out=None, free_begin=None, blocks_taken=None, stream=None) -> None:
    """Rows that continue rows ``parents`` of ``block_table``: full blocks shared, the last one kept by a row's first child and
    replaced by a block of ``free_blocks`` for the others (``copy_*``: what kv_copy_blocks has to copy); ``refs_after`` <- how many
    rows hold each block.  A parent outside the table makes an empty row.  Behind a kv_free that dropped rows: its ``lens_after`` and
    ``held_after``, or those rows give their blocks up again."""
    calls = _beam_call(stream)
    if calls:
        status = calls.fork_rows(parents, lens, block_table, refs, free_blocks, block_size, table_out, lens_out, refs_after, copy_src,
                                 copy_dst, copy_tokens, held_blocks, held_out, free_begin, blocks_taken)
        if status is not None:
            return _check(status, "symph_kv_fork")
    _on_this_device(stream, parents=parents, lens=lens, block_table=block_table, refs=refs, free_blocks=free_blocks, table_out=table_out,
                    lens_out=lens_out, refs_after=refs_after, copy_src=copy_src, copy_dst=copy_dst, copy_tokens=copy_tokens,
                    held_blocks=held_blocks, held_out=held_out, free_begin=free_begin, blocks_taken=blocks_taken)
    i32 = _torch().int32
    out, n, n_blocks = parents.shape[0], lens.shape[0], refs.shape[0]
    tp, stride = _rows_table(block_table, "block_table", n)
    op, _ = _rows_table(table_out, "table_out", out, stride)
    _check(load_library().symph_kv_fork(
        _vector(parents, "parents", i32), out, _vector(lens, "lens", i32), _vector(held_blocks, "held_blocks", i32, n, True), n, tp,
        stride, int(block_size), n_blocks, _vector(refs, "refs", i32), _vector(free_blocks, "free_blocks", i32),
        free_blocks.shape[0], _vector(free_begin, "free_begin", i32, 1, True), op, _vector(lens_out, "lens_out", i32, out),
        _vector(held_out, "held_out", i32, out, True), _vector(refs_after, "refs_after", i32, n_blocks),
        _vector(copy_src, "copy_src", i32, out), _vector(copy_dst, "copy_dst", i32, out),
        _vector(copy_tokens, "copy_tokens", i32, out), _vector(blocks_taken, "blocks_taken", i32, 1, True), _stream_ptr(stream)),
        "symph_kv_fork")


def kv_copy_blocks(cache: KVCache, src_blocks, dst_blocks, tokens=None, stream=None) -> None:
    """The first ``tokens[i]`` slots (None: all) of block ``src_blocks[i]`` of every layer into block ``dst_blocks[i]``, for every i
    where both are blocks of the cache."""
    calls = type(cache) is KVCache and _beam_call(stream)
    if calls:
        status = calls.copy_blocks(cache.k_pool, cache.v_pool, src_blocks, dst_blocks, tokens)
        if status is not None:
            return _check(status, "symph_kv_copy_blocks")
    _on_this_device(stream, k_pool=cache.k_pool, v_pool=cache.v_pool, src_blocks=src_blocks, dst_blocks=dst_blocks, tokens=tokens)
    if not (cache.k_pool.is_cuda and cache.v_pool.is_cuda):
        raise ValueError("the pools must be device tensors")
    st = cache.struct()
    i32, n = _torch().int32, src_blocks.shape[0]
    _check(load_library().symph_kv_copy_blocks(
        C.byref(st), _vector(src_blocks, "src_blocks", i32), _vector(dst_blocks, "dst_blocks", i32, n),
        _vector(tokens, "tokens", i32, n, True), n, _stream_ptr(stream)), "symph_kv_copy_blocks")


def kv_free_workspace_bytes(n_blocks: int) -> int:
    n = load_library().symph_kv_free_workspace_bytes(int(n_blocks))
    if n < 0:
        raise SymphError(-1, "symph_kv_free_workspace_bytes")
    return int(n)


def kv_free(drop, lens, block_table, refs, block_size: int, refs_after, free_blocks, n_free, held_blocks=None, lens_after=None,
            held_after=None, workspace=None, taken_blocks=None, taken_begin=None, taken_end=None, stream=None) -> None:
    """``refs_after`` <- ``refs`` without what rows with ``drop[r] != 0`` hold; ``free_blocks`` <- the blocks that nobody holds then,
    ascending, -1 behind them; ``n_free`` <- how many.  ``taken_blocks``: the list that build_tables has taken entries
    ``taken_begin`` .. ``taken_end`` - 1 of since ``refs`` was made, which then count as held by a row.  ``drop``, ``lens`` and
    ``block_table`` may be None: the list alone."""
    calls = _beam_call(stream)
    if calls:
        status = calls.free_rows(drop, lens, block_table, refs, block_size, refs_after, free_blocks, n_free, held_blocks, lens_after,
                                 held_after, workspace, taken_blocks, taken_begin, taken_end)
        if status is not None:
            return _check(status, "symph_kv_free")
    _on_this_device(stream, drop=drop, lens=lens, block_table=block_table, refs=refs, refs_after=refs_after, free_blocks=free_blocks,
                    n_free=n_free, held_blocks=held_blocks, lens_after=lens_after, held_after=held_after, workspace=workspace,
                    taken_blocks=taken_blocks, taken_begin=taken_begin, taken_end=taken_end)
    i32 = _torch().int32
    n, n_blocks = 0 if drop is None else drop.shape[0], refs.shape[0]
    tp, stride = _rows_table(block_table, "block_table", n) if n else (None, 0)
    wp, ws_bytes = _scratch(workspace)
    _check(load_library().symph_kv_free(
        _vector(drop, "drop", i32, n, n == 0), _vector(lens, "lens", i32, n, n == 0),
        _vector(held_blocks, "held_blocks", i32, n, True), n, tp, stride, int(block_size), n_blocks, _vector(refs, "refs", i32),
        _vector(refs_after, "refs_after", i32, n_blocks), _vector(free_blocks, "free_blocks", i32, n_blocks),
        _vector(n_free, "n_free", i32, 1), _vector(lens_after, "lens_after", i32, n, True),
        _vector(held_after, "held_after", i32, n, True), _vector(taken_blocks, "taken_blocks", i32, None, True),
        0 if taken_blocks is None else taken_blocks.shape[0], _vector(taken_begin, "taken_begin", i32, 1, True),
        _vector(taken_end, "taken_end", i32, 1, taken_blocks is None), wp, ws_bytes, _stream_ptr(stream)), "symph_kv_free")


def kv_compact_workspace_bytes(n_blocks: int) -> int:
    n = load_library().symph_kv_compact_workspace_bytes(int(n_blocks))
    if n < 0:
        raise SymphError(-1, "symph_kv_compact_workspace_bytes")
    return int(n)


def kv_compact(refs, n_keep: int, lens, block_table, block_size: int, table_out, refs_after, block_map, copy_src, copy_dst, counts,
               held_blocks=None, workspace=None, stream=None) -> None:
    """The moves after which the blocks from ``n_keep`` on are free (negative: all blocks in use move to the front), as lists for
    kv_copy_blocks, and the table (``table_out`` may be ``block_table``), counts and ``block_map`` after them.  ``counts`` <- blocks
    in use, moves, blocks that stay behind."""
    calls = _beam_call(stream)
    if calls:
        status = calls.compact_pool(refs, n_keep, lens, block_table, block_size, table_out, refs_after, block_map, copy_src, copy_dst,
                                    counts, held_blocks, workspace)
        if status is not None:
            return _check(status, "symph_kv_compact")
    _on_this_device(stream, refs=refs, lens=lens, block_table=block_table, table_out=table_out, refs_after=refs_after, block_map=block_map,
                    copy_src=copy_src, copy_dst=copy_dst, counts=counts, held_blocks=held_blocks, workspace=workspace)
    i32 = _torch().int32
    n, n_blocks, n_pairs = lens.shape[0], refs.shape[0], copy_src.shape[0]
    tp, stride = _rows_table(block_table, "block_table", n)
    op, _ = _rows_table(table_out, "table_out", n, stride)
    wp, ws_bytes = _scratch(workspace)
    _check(load_library().symph_kv_compact(
        _vector(refs, "refs", i32), n_blocks, int(n_keep), _vector(lens, "lens", i32),
        _vector(held_blocks, "held_blocks", i32, n, True), n, tp, stride, int(block_size), op,
        _vector(refs_after, "refs_after", i32, n_blocks), _vector(block_map, "block_map", i32, n_blocks),
        _vector(copy_src, "copy_src", i32), _vector(copy_dst, "copy_dst", i32, n_pairs), n_pairs, _vector(counts, "counts", i32, 3),
        wp, ws_bytes, _stream_ptr(stream)), "symph_kv_compact")


def debug_attn_flags(workspace, stream=None) -> int:
    """Flags of the device-side scheduler of the last attention call on ``workspace`` (synchronises the stream)."""
    flags = C.c_int32(0)
    _check(load_library().symph_debug_attn_flags(_dev(workspace, "workspace", allow_none=True), _stream_ptr(stream),
                                                 C.byref(flags)), "symph_debug_attn_flags")
    return flags.value


def stage_to_host(h_pinned, d_buf, nbytes: int, producer_stream, side_stream, event) -> None:
    _check(load_library().symph_stage_to_host(_ptr(h_pinned), _ptr(d_buf), int(nbytes), _stream_ptr(producer_stream),
                                              _stream_ptr(side_stream), _event_ptr(event)), "symph_stage_to_host")


def stage_to_device(d_buf, h_pinned, nbytes: int, consumer_stream, side_stream, event) -> None:
    _check(load_library().symph_stage_to_device(_ptr(d_buf), _ptr(h_pinned), int(nbytes),
                                                _stream_ptr(consumer_stream), _stream_ptr(side_stream),
                                                _event_ptr(event)), "symph_stage_to_device")


def stage_layer_to_host(h_pinned, d_buf, cache: KVCache, layer: int, h_prefix_lens, h_buf_token_offsets,
                        producer_stream, side_stream, event) -> None:
    """``h_prefix_lens`` (int32) and ``h_buf_token_offsets`` (int64) are HOST tensors (CPU, contiguous)."""
    st = cache.struct()
    _check(load_library().symph_stage_layer_to_host(
        _ptr(h_pinned), _ptr(d_buf), C.byref(st), int(layer), _ptr(h_prefix_lens), _ptr(h_buf_token_offsets),
        h_prefix_lens.shape[0], _stream_ptr(producer_stream), _stream_ptr(side_stream), _event_ptr(event)),
        "symph_stage_layer_to_host")


def stage_layer_to_device(d_buf, h_pinned, cache: KVCache, layer: int, h_prefix_lens, h_buf_token_offsets,
                          consumer_stream, side_stream, event) -> None:
    st = cache.struct()
    _check(load_library().symph_stage_layer_to_device(
        _ptr(d_buf), _ptr(h_pinned), C.byref(st), int(layer), _ptr(h_prefix_lens), _ptr(h_buf_token_offsets),
        h_prefix_lens.shape[0], _stream_ptr(consumer_stream), _stream_ptr(side_stream), _event_ptr(event)),
        "symph_stage_layer_to_device")


def mfma_reference(iters: int, sink, stream=None) -> int:
    """Launch the MFMA-only reference kernel; returns the floating-point operations of the launch."""
    flops = C.c_int64(0)
    _check(load_library().symph_mfma_reference(int(iters), C.byref(flops), _ptr(sink), _stream_ptr(stream)),
           "symph_mfma_reference")
    return int(flops.value)


def device_copy(dst, src, nbytes: int, stream=None) -> None:
    _check(load_library().symph_device_copy(_ptr(dst), _ptr(src), int(nbytes), _stream_ptr(stream)),
           "symph_device_copy")


class KvPool:
    """The pool object of ``include/symph_pool.h`` (host code): which layers of which announced sessions hold slots lent
    by the framework.  Every method is one C call plus marshalling; failures raise SymphError and change nothing."""

    EVICTED, LOAD = 0, 1

    def __init__(self, n_layers: int, n_slots: int, block_size: int):
        self._lib = load_library()
        self._h = C.c_void_p()
        self.n_layers, self.n_slots, self.block_size = n_layers, n_slots, block_size
        st = self._lib.symph_pool_create(n_layers, n_slots, block_size, C.byref(self._h))
        if st != 0:
            raise SymphError(st, "symph_pool_create")

    @property
    def handle(self):
        """The symph_pool* as a ctypes void pointer, for callers that drive the C entry points with arrays of their own
        (``PoolChange`` is the change record)."""
        return self._h

    def close(self):
        if self._h:
            self._lib.symph_pool_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, where: str) -> int:
        if st < 0:
            raise SymphError(st, where)
        return st

    def advise(self, session: int, n_tokens: int) -> None:
        self._check(self._lib.symph_pool_advise(self._h, session, n_tokens), "symph_pool_advise")

    def drop(self, session: int) -> None:
        self._check(self._lib.symph_pool_drop(self._h, session), "symph_pool_drop")

    def resident_layers(self, session: int) -> int:
        return self._check(self._lib.symph_pool_resident_layers(self._h, session), "symph_pool_resident_layers")

    def counts(self) -> tuple[int, int, int]:
        f, l, w = C.c_int32(), C.c_int32(), C.c_int32()
        self._check(self._lib.symph_pool_counts(self._h, C.byref(f), C.byref(l), C.byref(w)), "symph_pool_counts")
        return f.value, l.value, w.value

    def unit_slots(self, session: int) -> int:
        """Slots one layer of the session takes."""
        return self._check(self._lib.symph_pool_unit_slots(self._h, session), "symph_pool_unit_slots")

    def table(self, session: int, layer: int) -> list[int]:
        cap = self.unit_slots(session)
        buf = (C.c_int32 * max(cap, 1))()
        n = self._check(self._lib.symph_pool_table(self._h, session, layer, buf, cap), "symph_pool_table")
        return list(buf[:n])

    def claim(self, session: int) -> list[list[int]]:
        """Tables of the resident layers, which now belong to the framework."""
        b = self.unit_slots(session)
        cap = b * self.resident_layers(session)
        buf = (C.c_int32 * max(cap, 1))()
        r = C.c_int32()
        self._check(self._lib.symph_pool_claim(self._h, session, buf, cap, C.byref(r)), "symph_pool_claim")
        return [list(buf[i * b:(i + 1) * b]) for i in range(r.value)]

    def framework_take(self, n: int) -> list[int]:
        buf = (C.c_int32 * max(n, 1))()
        self._check(self._lib.symph_pool_framework_take(self._h, n, buf), "symph_pool_framework_take")
        return list(buf[:n])

    def framework_give(self, slots) -> None:
        n = len(slots)
        buf = (C.c_int32 * max(n, 1))(*slots)
        self._check(self._lib.symph_pool_framework_give(self._h, n, buf), "symph_pool_framework_give")

    def settle(self) -> list[tuple[int, int, int, list[int]]]:
        """[(kind, session, layer, slots)] — evictions first (slots empty), then loads, the most important first."""
        nc, ns = C.c_int32(), C.c_int32()
        st = self._lib.symph_pool_settle(self._h, None, 0, None, 0, C.byref(nc), C.byref(ns))
        if st == 0:
            return []
        if st != -4:
            raise SymphError(st, "symph_pool_settle")
        changes = (_PoolChange * max(nc.value, 1))()
        slots = (C.c_int32 * max(ns.value, 1))()
        self._check(self._lib.symph_pool_settle(self._h, changes, nc.value, slots, ns.value, C.byref(nc), C.byref(ns)),
                    "symph_pool_settle")
        out = []
        for c in changes[:nc.value]:
            own = list(slots[c.slot_begin:c.slot_begin + c.n_slots]) if c.kind == self.LOAD else []
            out.append((c.kind, c.session, c.layer, own))
        return out
