"""Thin Python binding of the C-ABI in include/hisparse.h (argument marshalling only).

Every step of the path runs in the CUDA library `_hisparse.so`; this module passes pointers of
torch tensors and stream handles to it.  There is no fallback: if the library is missing, import
of the binding fails loudly.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np

from . import build as _build

OK, EINVAL, ENOTPINNED, ENOMEM, ECUDA, ESTATE, ETOOBIG = 0, -1, -2, -3, -4, -5, -6
NOALLOC_MAX_REQUESTS, NOALLOC_MAX_SELECTIONS = 1024, 65536
FLAG_SKIP_IO, FLAG_DEBUG_VALIDATE, FLAG_INLINE_WRITE_THROUGH, FLAG_PHASE_TIMERS, FLAG_NO_PDL = 1, 2, 4, 8, 16
FLAG_EAGER_ORDER, FLAG_WIDE_BLOCKS, FLAG_NARROW_BLOCKS = 32, 64, 128
STATUS_OUT_OF_RANGE, STATUS_DUPLICATE, STATUS_CAPACITY, STATUS_INCONSISTENT, STATUS_TIMEOUT = 1, 2, 4, 8, 16
MAX_CACHE_SLOTS, MAX_TOP_K = 16384, 4096
POLICY_LRU, POLICY_FIFO, POLICY_RANDOM = 0, 1, 2
MAX_RECORD_DIMS, MAX_HEADS = 4096, 1024
BF16, FP16, FP32 = 0, 1, 2

EXPORTS = [
    "hisparse_create", "hisparse_destroy", "hisparse_append", "hisparse_resolve", "hisparse_prefetch", "hisparse_prefetch_hint",
    "hisparse_join", "hisparse_layer_pool", "hisparse_gather", "hisparse_gather_check", "hisparse_status",
    "hisparse_clear_status", "hisparse_dump_state", "hisparse_order_lag", "hisparse_load_state", "hisparse_load_appends", "hisparse_dump_plan", "hisparse_device_bytes",
    "hisparse_launch_geometry", "hisparse_phase_times", "hisparse_layer_times", "hisparse_selftest_wait_timeout", "hisparse_host_alloc", "hisparse_host_free", "hisparse_host_link_probe",
    "hisparse_scatter_read_probe", "hisparse_resolve_noalloc", "hisparse_strerror", "hisparse_last_cuda_error",
    "hisparse_attention_workspace_bytes", "hisparse_sparse_attention",
    "hisparse_record_bytes", "hisparse_write_records", "hisparse_read_records",
    "hisparse_record_attention_workspace_bytes", "hisparse_record_attention", "hisparse_status_word",
]


class HiSparseError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        msg = lib().hisparse_strerror(code).decode()
        if code == ECUDA:
            msg += " (cudaError %d)" % lib().hisparse_last_cuda_error()
        super().__init__("%s: %s" % (what, msg))


class Config(ctypes.Structure):
    _fields_ = [
        ("num_requests", ctypes.c_int32), ("num_layers", ctypes.c_int32), ("layers_per_group", ctypes.c_int32),
        ("cache_slots", ctypes.c_int32), ("top_k", ctypes.c_int32), ("entry_bytes", ctypes.c_int64),
        ("capacity", ctypes.c_void_p), ("init_len", ctypes.c_void_p), ("host_history", ctypes.c_void_p),
        ("device", ctypes.c_int32), ("flags", ctypes.c_uint32), ("ctas_per_request", ctypes.c_int32),
        ("policy", ctypes.c_int32), ("policy_seed", ctypes.c_uint64),
    ]


class ExternalState(ctypes.Structure):
    """hisparse_external_state_t: caller-owned state of one layer's caches (see hisparse_resolve_noalloc)."""
    _fields_ = [
        ("num_requests", ctypes.c_int32), ("cache_slots", ctypes.c_int32), ("top_k", ctypes.c_int32),
        ("entry_bytes", ctypes.c_int64), ("device", ctypes.c_int32), ("pool_dev", ctypes.c_void_p),
        ("slot_pos_dev", ctypes.c_void_p), ("last_use_dev", ctypes.c_void_p), ("lru_order_dev", ctypes.c_void_p),
        ("pos2slot_dev", ctypes.c_void_p), ("capacity_dev", ctypes.c_void_p), ("init_len_dev", ctypes.c_void_p),
        ("p2s_offset_dev", ctypes.c_void_p), ("host_layer_dev", ctypes.c_void_p), ("resolves_dev", ctypes.c_void_p),
        ("num_appends_dev", ctypes.c_void_p),
    ]


class _RecordFormat(ctypes.Structure):
    """hisparse_record_format_t"""
    _fields_ = [("dims", ctypes.c_int32), ("quant_dims", ctypes.c_int32)]


class _RecordAttention(ctypes.Structure):
    """hisparse_record_attention_t"""
    _fields_ = [
        ("device", ctypes.c_int32), ("format", _RecordFormat), ("records_dev", ctypes.c_void_p), ("num_records", ctypes.c_int64),
        ("table_dev", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("table_width", ctypes.c_int32),
        ("page_size", ctypes.c_int32), ("num_requests", ctypes.c_int32), ("num_heads", ctypes.c_int32),
        ("value_dims", ctypes.c_int32), ("q_dev", ctypes.c_void_p), ("q_token_stride", ctypes.c_int64),
        ("q_head_stride", ctypes.c_int64), ("total_q", ctypes.c_int64), ("q_start_dev", ctypes.c_void_p),
        ("max_q_len", ctypes.c_int32), ("kv_len_dev", ctypes.c_void_p), ("max_kv_len", ctypes.c_int32),
        ("causal", ctypes.c_int32), ("scale", ctypes.c_float), ("out_dev", ctypes.c_void_p), ("lse_dev", ctypes.c_void_p),
        ("status_dev", ctypes.c_void_p),
    ]


_lib = None


def lib() -> ctypes.CDLL:
    """The CUDA library; raises if it has not been built (see build.build_cuda / __graft_entry__.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.SO):
            raise RuntimeError("CUDA library %s is missing: run `python -m paper_2608_07009_b200.build` "
                               "(there is no CPU fallback)" % _build.SO)
        L = ctypes.CDLL(_build.SO)
        vp, i32, i64, u32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint32, ctypes.c_size_t
        P = ctypes.POINTER
        sig = {
            "hisparse_create": ([P(Config), P(vp)], i32),
            "hisparse_destroy": ([vp], i32),
            "hisparse_append": ([vp, vp, vp], i32),
            "hisparse_resolve": ([vp, i32, vp, vp, vp, vp, vp], i32),
            "hisparse_prefetch": ([vp, i32, vp], i32),
            "hisparse_prefetch_hint": ([vp, i32, vp, vp, vp], i32),
            "hisparse_join": ([vp, vp], i32),
            "hisparse_layer_pool": ([vp, i32], vp),
            "hisparse_gather": ([vp, i32, vp, vp, vp], i32),
            "hisparse_gather_check": ([vp, i32, vp, vp, vp, vp], i32),
            "hisparse_status": ([vp, P(u32)], i32),
            "hisparse_status_word": ([vp], vp),
            "hisparse_clear_status": ([vp], i32),
            "hisparse_dump_state": ([vp, i32, i32, vp, vp, vp, vp, P(i64), P(i64), P(u32)], i32),
            "hisparse_load_state": ([vp, i32, i32, vp, vp, u32], i32),
            "hisparse_order_lag": ([vp, i32, i32, P(u32)], i32),
            "hisparse_load_appends": ([vp, ctypes.c_int32], i32),
            "hisparse_dump_plan": ([vp, i32, i32, vp, vp, P(ctypes.c_int32)], i32),
            "hisparse_device_bytes": ([P(Config), P(sz), P(sz)], i32),
            "hisparse_launch_geometry": ([vp, P(ctypes.c_int32), P(ctypes.c_int32), P(ctypes.c_int32)], i32),
            "hisparse_phase_times": ([vp, vp], i32),
            "hisparse_layer_times": ([vp, vp], i32),
            "hisparse_selftest_wait_timeout": ([vp, ctypes.c_uint64, P(ctypes.c_uint64)], i32),
            "hisparse_host_alloc": ([sz, P(vp)], i32),
            "hisparse_host_free": ([vp], i32),
            "hisparse_host_link_probe": ([i32, sz, i32, P(ctypes.c_double)], i32),
            "hisparse_scatter_read_probe": ([i32, vp, sz, i64, ctypes.c_int32, ctypes.c_int32, i32, P(ctypes.c_double)], i32),
            "hisparse_resolve_noalloc": ([P(ExternalState), vp, vp, vp, vp, vp, vp], i32),
            "hisparse_attention_workspace_bytes": ([vp, i32, i32, P(sz)], i32),
            "hisparse_sparse_attention": ([vp, i32, vp, i32, i32, vp, ctypes.c_float, vp, vp, vp, sz, vp], i32),
            "hisparse_record_bytes": ([P(_RecordFormat), P(i64)], i32),
            "hisparse_write_records": ([P(_RecordFormat), i32, vp, i32, i64, i64, vp, vp, i64, vp, vp], i32),
            "hisparse_read_records": ([P(_RecordFormat), i32, vp, i64, vp, i64, vp, vp, vp], i32),
            "hisparse_record_attention_workspace_bytes": ([P(_RecordAttention), P(sz)], i32),
            "hisparse_record_attention": ([P(_RecordAttention), vp, sz, vp], i32),
            "hisparse_strerror": ([i32], ctypes.c_char_p),
            "hisparse_last_cuda_error": ([], i32),
        }
        for name, (args, res) in sig.items():
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, res
        _lib = L
    return _lib


def _check(code: int, what: str) -> None:
    if code != OK:
        raise HiSparseError(code, what)


def _stream_ptr(stream) -> int:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _dev_ptr(t, dtype_name: str, numel: Optional[int] = None) -> int:
    import torch
    want = getattr(torch, dtype_name)
    if not (t.is_cuda and t.dtype == want and t.is_contiguous()):
        raise ValueError("expected a contiguous CUDA %s tensor" % dtype_name)
    if numel is not None and t.numel() != numel:
        raise ValueError("expected %d elements, got %d" % (numel, t.numel()))
    return t.data_ptr()


class HostHistory:
    """Pinned, device-mapped host memory for one request's KV history, laid out [L][capacity][E]."""

    def __init__(self, num_layers: int, capacity: int, entry_bytes: int):
        self.shape = (num_layers, capacity, entry_bytes)
        self.nbytes = num_layers * capacity * entry_bytes
        p = ctypes.c_void_p()
        _check(lib().hisparse_host_alloc(self.nbytes, ctypes.byref(p)), "hisparse_host_alloc")
        self.ptr = p.value

    def numpy(self) -> np.ndarray:
        buf = (ctypes.c_uint8 * self.nbytes).from_address(self.ptr)
        return np.frombuffer(buf, dtype=np.uint8).reshape(self.shape)

    def free(self) -> None:
        if self.ptr:
            _check(lib().hisparse_host_free(self.ptr), "hisparse_host_free")
            self.ptr = None


def device_bytes(num_requests, num_layers, layers_per_group, cache_slots, top_k, entry_bytes, capacity):
    cap = np.asarray(capacity, dtype=np.int64)
    il = np.zeros_like(cap)
    cfg = Config(num_requests, num_layers, layers_per_group, cache_slots, top_k, entry_bytes,
                 cap.ctypes.data, il.ctypes.data, None, 0, 0, 0, 0, 0)
    kv, meta = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().hisparse_device_bytes(ctypes.byref(cfg), ctypes.byref(kv), ctypes.byref(meta)), "hisparse_device_bytes")
    return kv.value, meta.value


def host_link_probe(device: int = 0, nbytes: int = 1 << 30, reps: int = 10) -> float:
    """Best-of-reps bulk pinned H2D memcpy bandwidth in GB/s (the host-link peak)."""
    out = ctypes.c_double()
    _check(lib().hisparse_host_link_probe(device, nbytes, reps, ctypes.byref(out)), "hisparse_host_link_probe")
    return out.value


def scatter_read_probe(host_ptr: int, host_bytes: int, entry_bytes: int, num_records: int, num_ctas: int,
                       reps: int = 5, device: int = 0) -> float:
    out = ctypes.c_double()
    _check(lib().hisparse_scatter_read_probe(device, host_ptr, host_bytes, entry_bytes, num_records, num_ctas, reps,
                                             ctypes.byref(out)), "hisparse_scatter_read_probe")
    return out.value


def resolve_noalloc(state: ExternalState, sel, slot_table, hits, misses, status=None, stream=None) -> None:
    """Resolve on caller-owned state without any device allocation (hisparse_resolve_noalloc).

    For callers that may not call cudaMalloc (all of HBM handed to their own allocator, or a stream capture in
    progress): every tensor is the caller's; the kernel's scratch is a fixed array inside the library.  Calls
    on one device share that array, so do not let two of them overlap on the GPU.
    """
    n, k = state.num_requests, state.top_k
    _check(lib().hisparse_resolve_noalloc(ctypes.byref(state), _dev_ptr(sel, "int32", n * k),
                                          _dev_ptr(slot_table, "int32", n * k), _dev_ptr(hits, "int32", n),
                                          _dev_ptr(misses, "int32", n),
                                          status.data_ptr() if status is not None else None, _stream_ptr(stream)),
           "hisparse_resolve_noalloc")


# ---- records of numbers: quantised format, attention over a pool that the caller owns ----
#
# These calls take a few microseconds on the device, so the checks in front of them are kept to plain attribute reads.

def _int32(*numbers) -> None:
    """Refuses what an int32 field would cut off."""
    for n in numbers:
        if not -(1 << 31) <= n < 1 << 31:
            raise HiSparseError(EINVAL, "%d does not fit 32 bits" % n)


class RecordFormat:
    """Layout of a record of `dims` numbers: the first `quant_dims` (a multiple of 128) as e4m3 codes with a power-of-two
    scale per 128, the others bf16; quant_dims = 0 is the plain bf16 record.  `entry_bytes` is its size, and what a
    HiSparse handle for such records is created with."""

    __slots__ = ("dims", "quant_dims", "entry_bytes", "_c")
    _made: dict = {}

    def __new__(cls, dims: int, quant_dims: int = 0):
        f = cls._made.get((dims, quant_dims))
        if f is None:
            _int32(dims, quant_dims)
            f = object.__new__(cls)
            f.dims, f.quant_dims, f._c = dims, quant_dims, _RecordFormat(dims, quant_dims)
            n = ctypes.c_int64()
            _check(lib().hisparse_record_bytes(f._c, n), "hisparse_record_bytes")
            f.entry_bytes = n.value
            cls._made[(dims, quant_dims)] = f
        return f

    def __repr__(self) -> str:
        return "RecordFormat(dims=%d, quant_dims=%d)" % (self.dims, self.quant_dims)


_types: tuple = ()


def _torch_types():
    """(uint8, int32, int64, bfloat16, float32, {source type: its number})"""
    global _types
    if not _types:
        import torch
        _types = (torch.uint8, torch.int32, torch.int64, torch.bfloat16, torch.float32,
                  {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32})
    return _types


def _on_device(t, dtype, device: int, what: str) -> int:
    """Checks a contiguous CUDA tensor of this type and device and returns its address."""
    if not (t.dtype is dtype and t.is_cuda and t.get_device() == device and t.is_contiguous()):
        raise ValueError("%s: expected a contiguous %s tensor on cuda:%d" % (what, dtype, device))
    return t.data_ptr()


def _records_of(fmt: RecordFormat, records):
    """(address, records, device) of a pool."""
    if not (records.dtype is _torch_types()[0] and records.is_cuda and records.dim() == 2 and records.shape[1] == fmt.entry_bytes
            and records.is_contiguous()):
        raise ValueError("records: expected a contiguous CUDA uint8 tensor [records][%d]" % fmt.entry_bytes)
    return records.data_ptr(), records.shape[0], records.get_device()


def _status_of(status, device: int):
    """Address of a status word: None, an address (a handle's word) or one int32 on the device."""
    if status is None or isinstance(status, int):
        return status
    import torch
    if status.dtype not in (torch.int32, torch.uint32) or status.numel() != 1 or not status.is_cuda or status.get_device() != device:
        raise ValueError("status: expected one int32 on cuda:%d" % device)
    return status.data_ptr()


class _Launch:
    """The stream of one call: `stream`, or the current stream of the tensors' device.  Tensors made for the call inside
    `with` come from that stream's pool, so that memory freed on another stream is not written while that one still reads
    it, and scratch that the call drops is not handed out before its kernels are done."""

    __slots__ = ("ptr", "_ctx")

    def __init__(self, stream, device: int):
        import torch
        if stream is None:
            self.ptr, self._ctx = torch._C._cuda_getCurrentRawStream(device), None
            return
        s = stream
        if isinstance(stream, int):
            # (0 and 1 are the legacy default stream; torch takes a number of 0 for none and makes a stream of its own)
            s = torch.cuda.default_stream(device) if stream in (0, 1) else torch.cuda.ExternalStream(stream, device=device)
        if s.device.index != device:
            raise ValueError("stream: expected a stream of cuda:%d" % device)
        self.ptr, self._ctx = s.cuda_stream, torch.cuda.stream(s)

    def __enter__(self):
        if self._ctx is not None:
            self._ctx.__enter__()
        return self

    def __exit__(self, *exc):
        if self._ctx is not None:
            self._ctx.__exit__(*exc)


def write_records(fmt: RecordFormat, values, records, slots=None, status=None, stream=None):
    """Writes `values` [T][dims] (bf16, fp16 or fp32; rows may be strided) as records: row i becomes records[slots[i]]
    (int64; negative = skipped; without slots records[i]).  Slots that are not negative must differ.  Returns `records`."""
    _, _, int64, _, _, sources = _torch_types()
    ptr, count, device = _records_of(fmt, records)
    kind = sources.get(values.dtype)
    if kind is None or values.dim() != 2 or values.shape[1] != fmt.dims or not values.is_cuda or values.get_device() != device:
        raise ValueError("values: expected a bf16, fp16 or fp32 tensor [T][%d] on cuda:%d" % (fmt.dims, device))
    T = values.shape[0]
    if T == 0:
        return records
    if values.stride(1) != 1:
        raise ValueError("values: the numbers of a row have to be neighbours")
    slot_ptr = None
    if slots is not None:
        slot_ptr = _on_device(slots, int64, device, "slots")
        if slots.numel() != T:
            raise ValueError("slots: expected %d entries, got %d" % (T, slots.numel()))
    elif T > count:
        raise ValueError("%d rows for %d records" % (T, count))
    rc = lib().hisparse_write_records(fmt._c, device, values.data_ptr(), kind, values.stride(0) if T > 1 else fmt.dims, T, slot_ptr,
                                      ptr, count, _status_of(status, device), _Launch(stream, device).ptr)
    if rc:
        raise HiSparseError(rc, "hisparse_write_records")
    return records


def _read(fmt, ptr, count, device, table, out, status, stream):
    _, int32, _, bf16, _, _ = _torch_types()
    table_ptr = _on_device(table, int32, device, "table")
    with _Launch(stream, device) as on:
        if out is None:
            out = table.new_empty((*table.shape, fmt.dims), dtype=bf16)
        elif out.numel() != table.numel() * fmt.dims:
            raise ValueError("out: expected %d numbers, got %d" % (table.numel() * fmt.dims, out.numel()))
        rc = lib().hisparse_read_records(fmt._c, device, ptr, count, table_ptr, table.numel(), _on_device(out, bf16, device, "out"),
                                         _status_of(status, device), on.ptr)
    if rc:
        raise HiSparseError(rc, "hisparse_read_records")
    return out


def read_records(fmt: RecordFormat, records, table, out=None, status=None, stream=None):
    """bf16 [*table.shape][dims]: the numbers of records[table[...]] (int32 entries; a negative one gives zeros)."""
    ptr, count, device = _records_of(fmt, records)
    return _read(fmt, ptr, count, device, table, out, status, stream)


def _attend(fmt, ptr, count, device, table, q, value_dims, scale, page_size, q_start, kv_len, max_q_len, max_kv_len, causal,
            out, lse, workspace, status, stream):
    uint8, int32, _, bf16, f32, _ = _torch_types()
    if not (table.dtype is int32 and table.is_cuda and table.dim() == 2 and table.get_device() == device
            and (table.stride(1) == 1 or table.shape[1] <= 1)):
        raise ValueError("table: expected an int32 tensor [requests][entries] on cuda:%d" % device)
    if not (q.dtype is bf16 and q.is_cuda and q.dim() == 3 and q.get_device() == device and q.shape[2] == fmt.dims and q.stride(2) == 1):
        raise ValueError("q: expected a bfloat16 tensor [tokens][heads][%d] on cuda:%d" % (fmt.dims, device))
    _int32(value_dims, page_size, max_q_len, max_kv_len)
    N, width = table.shape
    T, H, _ = q.shape
    q_token, q_head, _ = q.stride()
    start_ptr = kv_ptr = None
    if q_start is not None:
        start_ptr = _on_device(q_start, int32, device, "q_start")
        if q_start.numel() != N + 1:
            raise ValueError("q_start: expected %d entries, got %d" % (N + 1, q_start.numel()))
    if kv_len is not None:
        kv_ptr = _on_device(kv_len, int32, device, "kv_len")
        if kv_len.numel() != N:
            raise ValueError("kv_len: expected %d entries, got %d" % (N, kv_len.numel()))
    if N == 0 and (T == 0 or q_start is not None):   # no request, no row to write
        out = q.new_empty((T, H, value_dims)) if out is None else out
        return out, q.new_empty((T, H), dtype=f32) if lse is None else lse
    # (an axis of one has any stride)
    p = _RecordAttention(device, fmt._c, ptr, count, table.data_ptr(), table.stride(0) if N > 1 else width, width, page_size, N, H,
                         value_dims, q.data_ptr(), q_token if T > 1 else 0, q_head if H > 1 else 0, T, start_ptr, max_q_len, kv_ptr, max_kv_len, causal, scale,
                         None, None, _status_of(status, device))
    need = ctypes.c_size_t()
    rc = lib().hisparse_record_attention_workspace_bytes(p, need)
    if rc:
        raise HiSparseError(rc, "hisparse_record_attention")
    with _Launch(stream, device) as on:
        if out is None:
            out = q.new_empty((T, H, value_dims))
        elif out.shape != (T, H, value_dims):
            raise ValueError("out: expected [%d][%d][%d]" % (T, H, value_dims))
        if lse is None:
            lse = q.new_empty((T, H), dtype=f32)
        elif lse.shape != (T, H):
            raise ValueError("lse: expected [%d][%d]" % (T, H))
        p.out_dev = _on_device(out, bf16, device, "out")
        p.lse_dev = _on_device(lse, f32, device, "lse")
        room = space = None
        if workspace is not None:
            if not (workspace.is_cuda and workspace.get_device() == device and workspace.is_contiguous()):
                raise ValueError("workspace: expected a contiguous tensor on cuda:%d" % device)
            space, room = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        elif need.value:
            workspace = q.new_empty(need.value, dtype=uint8)
            space, room = workspace.data_ptr(), need.value
        rc = lib().hisparse_record_attention(p, space, room or 0, on.ptr)
    if rc:
        raise HiSparseError(rc, "hisparse_record_attention")
    return out, lse


def record_attention(fmt: RecordFormat, records, table, q, value_dims: int, scale: float, out=None, lse=None, workspace=None,
                     status=None, stream=None):
    """Attention of one new token a request over the records of a slot table, int32 [N][k] as resolve emits it (negative =
    padding), in a pool uint8 [records][entry_bytes] that the caller owns.  q bf16 [N][H][dims]; returns (out bf16
    [N][H][value_dims], lse float32 [N][H]).  Two calls that may overlap must not share a workspace."""
    ptr, count, device = _records_of(fmt, records)
    return _attend(fmt, ptr, count, device, table, q, value_dims, scale, 1, None, None, 1, 0, 0, out, lse, workspace, status, stream)


def chunk_attention(fmt: RecordFormat, records, page_table, kv_len, q, q_start, value_dims: int, scale: float, *, page_size: int,
                    max_q_len: int, max_kv_len: int = 0, causal: bool = True, out=None, lse=None, workspace=None, status=None,
                    stream=None):
    """Attention of chunks of new tokens over a paged cache: request n's tokens are rows q_start[n] .. q_start[n + 1] - 1
    (int32 [N + 1]) of q, bf16 [tokens][H][dims], and the last ones of its kv_len[n] keys (int32 [N]), which are records
    page_table[n][j // page_size] * page_size + j % page_size (int32 [N][pages], negative = absent) of `records`.  With
    `causal`, token t of m sees the keys up to kv_len[n] - m + t, its own.  max_q_len and max_kv_len
    (0: the table's width) bound chunks and contexts.  A batch of no requests writes nothing; a table without entries is
    refused.  Returns (out bf16 [tokens][H][value_dims], lse float32 [tokens][H]);
    rows that belong to no request are left as they were."""
    ptr, count, device = _records_of(fmt, records)
    return _attend(fmt, ptr, count, device, page_table, q, value_dims, scale, page_size, q_start, kv_len, max_q_len, max_kv_len,
                   int(causal), out, lse, workspace, status, stream)


class HiSparse:
    """One handle = the caches and metadata of N requests on one GPU (see include/hisparse.h)."""

    def __init__(self, num_requests: int, num_layers: int, layers_per_group: int, cache_slots: int, top_k: int,
                 entry_bytes: int, capacity: Sequence[int], init_len: Sequence[int], host_history: Sequence,
                 device: int = 0, flags: int = 0, ctas_per_request: int = 0, policy: int = 0, policy_seed: int = 0):
        self.N, self.L, self.lpg, self.B, self.k, self.E = (num_requests, num_layers, layers_per_group, cache_slots,
                                                            top_k, entry_bytes)
        self.device = device
        self.capacity = np.ascontiguousarray(capacity, dtype=np.int64)
        self.init_len = np.ascontiguousarray(init_len, dtype=np.int64)
        if len(self.capacity) != num_requests or len(self.init_len) != num_requests or len(host_history) != num_requests:
            raise ValueError("capacity, init_len and host_history need one entry per request")
        self._hist = list(host_history)          # keep the pinned buffers alive
        ptrs = (ctypes.c_void_p * num_requests)(*[h.ptr if isinstance(h, HostHistory) else int(h) for h in host_history])
        cfg = Config(num_requests, num_layers, layers_per_group, cache_slots, top_k, entry_bytes,
                     self.capacity.ctypes.data, self.init_len.ctypes.data, ctypes.addressof(ptrs), device, flags,
                     ctas_per_request, policy, policy_seed)
        h = ctypes.c_void_p()
        _check(lib().hisparse_create(ctypes.byref(cfg), ctypes.byref(h)), "hisparse_create")
        self._h = h

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().hisparse_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- the path ----
    def append(self, new_kv, stream=None) -> None:
        _check(lib().hisparse_append(self._h, _dev_ptr(new_kv, "uint8", self.N * self.L * self.E), _stream_ptr(stream)),
               "hisparse_append")

    def resolve(self, layer: int, sel, slot_table=None, hits=None, misses=None, stream=None):
        import torch
        dev = "cuda:%d" % self.device
        if slot_table is None:
            slot_table = torch.empty((self.N, self.k), dtype=torch.int32, device=dev)
        if hits is None:
            hits = torch.empty(self.N, dtype=torch.int32, device=dev)
        if misses is None:
            misses = torch.empty(self.N, dtype=torch.int32, device=dev)
        sel_ptr = _dev_ptr(sel, "int32", self.N * self.k) if sel is not None else None
        _check(lib().hisparse_resolve(self._h, layer, sel_ptr, _dev_ptr(slot_table, "int32", self.N * self.k),
                                      _dev_ptr(hits, "int32", self.N), _dev_ptr(misses, "int32", self.N),
                                      _stream_ptr(stream)), "hisparse_resolve")
        return slot_table, hits, misses

    def prefetch(self, layer: int, side_stream) -> None:
        _check(lib().hisparse_prefetch(self._h, layer, _stream_ptr(side_stream)), "hisparse_prefetch")

    def prefetch_hint(self, layer: int, hint_sel, side_stream, stream=None) -> None:
        _check(lib().hisparse_prefetch_hint(self._h, layer, _dev_ptr(hint_sel, "int32", self.N * self.k),
                                            _stream_ptr(stream), _stream_ptr(side_stream)), "hisparse_prefetch_hint")

    def join(self, stream=None) -> None:
        _check(lib().hisparse_join(self._h, _stream_ptr(stream)), "hisparse_join")

    # ---- the sparse-attention consumer ----
    def attention_workspace_bytes(self, num_heads: int, value_dims: int) -> int:
        n = ctypes.c_size_t()
        _check(lib().hisparse_attention_workspace_bytes(self._h, num_heads, value_dims, ctypes.byref(n)),
               "hisparse_attention_workspace_bytes")
        return n.value

    def sparse_attention(self, layer: int, q, slot_table, value_dims: int, scale: float, out=None, lse=None,
                         workspace=None, stream=None):
        """q: bf16 CUDA tensor [N][H][E/2]; returns (out float32 [N][H][value_dims], lse float32 [N][H])."""
        import torch
        dev = "cuda:%d" % self.device
        H = q.shape[1]
        if not (q.is_cuda and q.dtype == torch.bfloat16 and q.is_contiguous() and q.shape == (self.N, H, self.E // 2)):
            raise ValueError("expected a contiguous CUDA bfloat16 tensor [N][H][E/2]")
        if out is None:
            out = torch.empty((self.N, H, value_dims), dtype=torch.float32, device=dev)
        if lse is None:
            lse = torch.empty((self.N, H), dtype=torch.float32, device=dev)
        need = self.attention_workspace_bytes(H, value_dims)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        _check(lib().hisparse_sparse_attention(self._h, layer, q.data_ptr(), H, value_dims,
                                               _dev_ptr(slot_table, "int32", self.N * self.k), scale,
                                               _dev_ptr(out, "float32", self.N * H * value_dims),
                                               _dev_ptr(lse, "float32", self.N * H), workspace.data_ptr(),
                                               workspace.numel() * workspace.element_size(), _stream_ptr(stream)),
               "hisparse_sparse_attention")
        return out, lse

    # ---- records of numbers (RecordFormat with this handle's entry_bytes) ----
    def _pool_of(self, layer: int, fmt: "RecordFormat"):
        """(address, records, device, address of the handle's status word)"""
        if fmt.entry_bytes != self.E:
            raise ValueError("%r has %d bytes, the handle's records %d" % (fmt, fmt.entry_bytes, self.E))
        return self.layer_pool(layer), self.N * (self.B + 1), self.device, lib().hisparse_status_word(self._h)

    def append_values(self, fmt: "RecordFormat", values, stream=None) -> None:
        """append of bf16, fp16 or fp32 numbers [N][L][dims], written as records of `fmt`."""
        import torch
        if fmt.entry_bytes != self.E:
            raise ValueError("%r has %d bytes, the handle's records %d" % (fmt, fmt.entry_bytes, self.E))
        if tuple(values.shape) != (self.N, self.L, fmt.dims):
            raise ValueError("values: expected [%d][%d][%d]" % (self.N, self.L, fmt.dims))
        with _Launch(stream, self.device) as on:
            records = torch.empty((self.N * self.L, self.E), dtype=torch.uint8, device="cuda:%d" % self.device)
            write_records(fmt, values.reshape(self.N * self.L, fmt.dims), records, stream=on.ptr)
            self.append(records, stream=on.ptr)

    def gather_values(self, layer: int, fmt: "RecordFormat", slot_table, out=None, stream=None):
        """bf16 [N][k][dims]: the numbers of the records that a slot table addresses (gather, expanded).  A slot beyond the
        cache gives zeros and STATUS_OUT_OF_RANGE in status()."""
        ptr, count, device, word = self._pool_of(layer, fmt)
        with _Launch(stream, device) as on:
            self.join(on.ptr)
            return _read(fmt, ptr, count, device, slot_table, out, word, stream)

    def record_attention(self, layer: int, fmt: "RecordFormat", q, slot_table, value_dims: int, scale: float, out=None, lse=None,
                         workspace=None, stream=None):
        """record_attention over this layer's cache: any number of heads, either record format, bf16 out; errors of the kernels
        appear in status()."""
        ptr, count, device, word = self._pool_of(layer, fmt)
        if tuple(slot_table.shape) != (self.N, self.k):
            raise ValueError("slot_table: expected [%d][%d]" % (self.N, self.k))
        with _Launch(stream, device) as on:
            self.join(on.ptr)                # a prefetch replay or a write-through may still be filling this layer's cache
            return _attend(fmt, ptr, count, device, slot_table, q, value_dims, scale, 1, None, None, 1, 0, 0, out, lse, workspace,
                           word, stream)

    # ---- consumer stand-ins ----
    def layer_pool(self, layer: int) -> int:
        p = lib().hisparse_layer_pool(self._h, layer)
        if not p:
            raise ValueError("bad layer")
        return p

    def gather(self, layer: int, slot_table, out=None, stream=None):
        import torch
        if out is None:
            out = torch.empty((self.N, self.k, self.E), dtype=torch.uint8, device="cuda:%d" % self.device)
        _check(lib().hisparse_gather(self._h, layer, _dev_ptr(slot_table, "int32", self.N * self.k),
                                     _dev_ptr(out, "uint8", self.N * self.k * self.E), _stream_ptr(stream)),
               "hisparse_gather")
        return out

    def gather_check(self, layer: int, sel, slot_table, mismatches, stream=None) -> None:
        _check(lib().hisparse_gather_check(self._h, layer, _dev_ptr(sel, "int32", self.N * self.k),
                                           _dev_ptr(slot_table, "int32", self.N * self.k),
                                           _dev_ptr(mismatches, "int32", 1), _stream_ptr(stream)),
               "hisparse_gather_check")

    # ---- inspection (synchronising) ----
    def status(self) -> int:
        bits = ctypes.c_uint32()
        _check(lib().hisparse_status(self._h, ctypes.byref(bits)), "hisparse_status")
        return bits.value

    def clear_status(self) -> None:
        _check(lib().hisparse_clear_status(self._h), "hisparse_clear_status")

    def dump_state(self, req: int, layer: int, with_pos2slot: bool = True) -> dict:
        B = self.B
        slot_pos = np.empty(B, dtype=np.int32)
        last_use = np.empty(B, dtype=np.uint32)
        order = np.empty(B, dtype=np.int32)
        p2s = np.empty(int(self.capacity[req]), dtype=np.int32) if with_pos2slot else None
        ln, newest, t = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_uint32()
        _check(lib().hisparse_dump_state(self._h, req, layer, slot_pos.ctypes.data, last_use.ctypes.data,
                                         order.ctypes.data, p2s.ctypes.data if with_pos2slot else None,
                                         ctypes.byref(ln), ctypes.byref(newest), ctypes.byref(t)),
               "hisparse_dump_state")
        return dict(slot_pos=slot_pos, last_use=last_use, lru_order=order, pos2slot=p2s, len=ln.value,
                    newest=newest.value, resolves=t.value)

    def load_appends(self, appends: int) -> None:
        _check(lib().hisparse_load_appends(self._h, appends), "hisparse_load_appends")

    def load_state(self, req: int, layer: int, slot_pos: np.ndarray, last_use: np.ndarray, resolves: int) -> None:
        sp = np.ascontiguousarray(slot_pos, dtype=np.int32)
        lu = np.ascontiguousarray(last_use, dtype=np.uint32)
        assert sp.size == self.B and lu.size == self.B
        _check(lib().hisparse_load_state(self._h, req, layer, sp.ctypes.data, lu.ctypes.data, resolves),
               "hisparse_load_state")

    def order_lag(self, req: int, layer: int) -> int:
        """Resolves of (req, layer's group) the recency list has not absorbed yet (0 = dump_state's lru_order is the
        slots sorted by (last_use, slot))."""
        lag = ctypes.c_uint32()
        _check(lib().hisparse_order_lag(self._h, req, layer, ctypes.byref(lag)), "hisparse_order_lag")
        return int(lag.value)

    def dump_plan(self, req: int, layer: int):
        pos = np.empty(self.k, dtype=np.int32)
        slot = np.empty(self.k, dtype=np.int32)
        n = ctypes.c_int32()
        _check(lib().hisparse_dump_plan(self._h, req, layer, pos.ctypes.data, slot.ctypes.data, ctypes.byref(n)),
               "hisparse_dump_plan")
        return pos[: n.value].copy(), slot[: n.value].copy()

    def phase_times(self) -> np.ndarray:
        """uint64 [N][16] stamps of the last anchor resolve (needs FLAG_PHASE_TIMERS): 8 in ns, 8 in SM cycles."""
        out = np.zeros((self.N, 16), dtype=np.uint64)
        _check(lib().hisparse_phase_times(self._h, out.ctypes.data), "hisparse_phase_times")
        return out

    def layer_times(self) -> np.ndarray:
        """uint64 [L][2]: start and end (ns) of each layer's last resolve kernel since the previous call (needs
        FLAG_PHASE_TIMERS); a layer without one reads (2**64 - 1, 0).  Synchronises and clears the stamps."""
        out = np.zeros((2, self.L), dtype=np.uint64)
        _check(lib().hisparse_layer_times(self._h, out.ctypes.data), "hisparse_layer_times")
        return np.ascontiguousarray(out.T)

    def selftest_wait_timeout(self, limit_ns: int) -> int:
        """Runs the library's bounded wait on a barrier that never completes; returns the nanoseconds waited."""
        out = ctypes.c_uint64()
        _check(lib().hisparse_selftest_wait_timeout(self._h, limit_ns, ctypes.byref(out)), "hisparse_selftest_wait_timeout")
        return out.value

    def launch_geometry(self):
        s, t, m = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
        _check(lib().hisparse_launch_geometry(self._h, ctypes.byref(s), ctypes.byref(t), ctypes.byref(m)),
               "hisparse_launch_geometry")
        return dict(ctas_per_request=s.value, threads=t.value, smem_bytes=m.value)
