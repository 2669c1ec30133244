"""Python binding of libfq (fused outlier-aware W4A16 decode matmul, MI355X, and
the operators around it in a decoder layer: paged KV cache, attention, norms).

Argument marshalling only: every step of the computation runs in the HIP
kernels of libfq.so, behind the C ABI declared in include/fq.h.  PyTorch
provides device memory and streams.  Function names follow the C names.

There is no CPU fallback: if libfq.so has not been built, every call raises.
"""

from __future__ import annotations

import contextlib
import ctypes as C
import os
import threading
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfq.so")

FQ_OK = 0
_FQ_ERR_WORKSPACE = 8
_FQ_ERR_HIP = 9
STATUS_NAMES = {0: "FQ_OK", 1: "FQ_ERR_NULL", 2: "FQ_ERR_SHAPE", 3: "FQ_ERR_RANGE",
                4: "FQ_ERR_DUPLICATE", 5: "FQ_ERR_ZERO_VALUE", 6: "FQ_ERR_FORMAT",
                7: "FQ_ERR_UNSUPPORTED", 8: "FQ_ERR_WORKSPACE", 9: "FQ_ERR_HIP",
                10: "FQ_ERR_ALIGN", 11: "FQ_ERR_SCRATCH_LIMIT"}
# static device scratch of fq_w4a16_outlier_matmul_noalloc (FQ_NOALLOC_SCRATCH_BYTES)
NOALLOC_SCRATCH_BYTES = 256 * 1024 + (8 << 20)
FQ_GROUP_BY_COLUMN = 0
FQ_GROUP_BY_BUCKET = 1
FQ_REORDER_COLUMNS = 1
FQ_REORDER_ELEMENTS = 2
FQ_Y_BF16 = 0
FQ_Y_F32 = 1
FQ_SPARSE_AUTO = 0
FQ_SPARSE_GATHER = 1
FQ_SPARSE_MFMA = 2
_SPARSE_MODES = {"auto": FQ_SPARSE_AUTO, "gather": FQ_SPARSE_GATHER, "mfma": FQ_SPARSE_MFMA}
FQ_SCHED_STREAM_K = 4
FQ_FOUR_WAVES = 8
FQ_STRIP_32 = 16
FQ_STRIP_64 = 32
FQ_SPARSE_WAVES = 64
FQ_DENSE_VALU = 128
FQ_KV_BF16 = 0
FQ_KV_INT8 = 1
FQ_KV_INT4 = 2
_KV_KINDS = {"bf16": FQ_KV_BF16, "int8": FQ_KV_INT8, "int4": FQ_KV_INT4}
FQ_ATTN_ROWS = 0
FQ_ATTN_TILES = 1
_ATTN_KERNELS = {FQ_ATTN_ROWS: "rows", FQ_ATTN_TILES: "tiles"}


class FqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        self.name = STATUS_NAMES.get(status, f"status {status}")
        super().__init__(f"{where}: {self.name}")


class fq_tilecoo_params(C.Structure):
    _fields_ = [("k_tile", C.c_int32), ("n_tile", C.c_int32), ("buckets_per_tile", C.c_int32),
                ("group_mode", C.c_int32), ("reorder", C.c_int32),
                ("elems_per_bank", C.c_int32), ("n_bank_groups", C.c_int32)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


class fq_tilecoo_sizes(C.Structure):
    _fields_ = [("n_tiles", C.c_int64), ("n_buckets", C.c_int64), ("n_groups", C.c_int64),
                ("nnz", C.c_int64), ("n_pad", C.c_int64), ("bytes", C.c_int64),
                ("max_tile_groups", C.c_int64)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


class fq_tilecoo_dev(C.Structure):
    _fields_ = [("tile_indptr", C.c_void_p), ("bucket_info", C.c_void_p),
                ("packed", C.c_void_p), ("params", fq_tilecoo_params),
                ("n_groups", C.c_int64), ("max_tile_groups", C.c_int64)]


class fq_problem(C.Structure):
    _fields_ = [("M", C.c_int32), ("K", C.c_int32), ("N", C.c_int32),
                ("group_size", C.c_int32), ("y_dtype", C.c_int32), ("split_k", C.c_int32),
                ("flags", C.c_int32)]


class fq_kv_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_meta", C.c_void_p),
                ("v_meta", C.c_void_p), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("token_stride", C.c_int64), ("meta_page_stride", C.c_int64),
                ("meta_head_stride", C.c_int64), ("n_pages", C.c_int64),
                ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("kind", C.c_int32)]


class fq_attention(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_heads", C.c_int32), ("max_q", C.c_int32),
                ("max_kv", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32),
                ("total_q", C.c_int64), ("q_token_stride", C.c_int64),
                ("q_head_stride", C.c_int64), ("o_token_stride", C.c_int64),
                ("o_head_stride", C.c_int64), ("table_stride", C.c_int64),
                ("table_cols", C.c_int32), ("scale", C.c_float)]


class fq_norm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("x_dtype", C.c_int32),
                ("residual_dtype", C.c_int32), ("eps", C.c_float), ("residual_scale", C.c_float),
                ("x_stride", C.c_int64), ("residual_stride", C.c_int64),
                ("gate_stride", C.c_int64), ("residual_out_stride", C.c_int64),
                ("h_stride", C.c_int64)]


_lib = None
_lock = threading.Lock()

_P = C.c_void_p
_SIGS = {
    "fq_default_tilecoo_params": ([], fq_tilecoo_params),
    "fq_pack_tile_coo": ([C.c_int32, C.c_int32, C.c_int64, _P, _P, _P,
                          C.POINTER(fq_tilecoo_params), C.POINTER(fq_tilecoo_sizes), _P, _P, _P],
                         C.c_int),
    "fq_unpack_tile_coo": ([C.c_int32, C.c_int32, C.POINTER(fq_tilecoo_params), C.c_int64,
                            _P, _P, _P, C.POINTER(C.c_int64), _P, _P, _P], C.c_int),
    "fq_validate_tile_coo": ([C.c_int32, C.c_int32, C.POINTER(fq_tilecoo_params), C.c_int64,
                              _P, _P, _P], C.c_int),
    "fq_workspace_bytes": ([C.POINTER(fq_problem), C.POINTER(C.c_size_t)], C.c_int),
    "fq_workspace_bytes_unfused": ([C.POINTER(fq_problem), C.POINTER(C.c_size_t)], C.c_int),
    "fq_w4a16_outlier_matmul": ([C.POINTER(fq_problem), _P, _P, _P, _P,
                                 C.POINTER(fq_tilecoo_dev), _P, _P, C.c_size_t, _P], C.c_int),
    "fq_w4a16_outlier_matmul_unfused": ([C.POINTER(fq_problem), _P, _P, _P, _P,
                                         C.POINTER(fq_tilecoo_dev), _P, _P, C.c_size_t, _P],
                                        C.c_int),
    "fq_w4a16_outlier_matmul_noalloc": ([C.POINTER(fq_problem), _P, _P, _P, _P,
                                         C.POINTER(fq_tilecoo_dev), _P, _P], C.c_int),
    "fq_w4a16_matmul": ([C.POINTER(fq_problem), _P, _P, _P, _P, _P, _P, C.c_size_t, _P],
                        C.c_int),
    "fq_debug_decode_tile_coo": ([C.POINTER(fq_tilecoo_dev), C.c_int32, C.c_int32, _P, _P, _P,
                                  _P], C.c_int),
    "fq_status_string": ([C.c_int], C.c_char_p),
    "fq_launch_kernel": ([C.POINTER(fq_problem), C.POINTER(fq_tilecoo_dev), C.c_size_t,
                          C.POINTER(C.c_int32)], C.c_int),
    "fq_launch_config": ([C.POINTER(fq_problem), C.c_int32, C.c_int32, C.POINTER(C.c_int32)],
                         C.c_int),
    "fq_quantize_outlier_aware": ([C.c_int32, C.c_int32, _P, C.c_int32, C.c_double,
                                   C.POINTER(C.c_int64), _P, _P, _P, _P, _P, _P], C.c_int),
    "fq_fill_padding_slots": ([C.c_int32, C.c_int32, _P, C.c_int32,
                               C.POINTER(fq_tilecoo_params), C.c_int64, _P, _P, _P, _P, _P,
                               C.POINTER(C.c_int64)], C.c_int),
    "fq_kv_cache_write": ([C.POINTER(fq_kv_cache), _P, _P, C.c_int64, C.c_int64, C.c_int64,
                           C.c_int64, _P, C.c_int64, _P], C.c_int),
    "fq_kv_cache_read": ([C.POINTER(fq_kv_cache), _P, C.c_int64, _P, _P, C.c_int32, _P], C.c_int),
    "fq_paged_attention_workspace_bytes": ([C.POINTER(fq_attention), C.POINTER(fq_kv_cache),
                                            C.POINTER(C.c_size_t)], C.c_int),
    "fq_paged_attention_launch": ([C.POINTER(fq_attention), C.POINTER(fq_kv_cache),
                                   C.POINTER(C.c_int32)], C.c_int),
    "fq_paged_attention": ([C.POINTER(fq_attention), _P, C.POINTER(fq_kv_cache), _P, _P, _P, _P,
                            _P, _P, C.c_size_t, _P], C.c_int),
    "fq_gated_residual_norm": ([C.POINTER(fq_norm), _P, _P, _P, _P, _P, _P, _P, _P], C.c_int),
}
EXPORTS = tuple(_SIGS)


def load() -> C.CDLL:
    """Load libfq.so (built in-tree by build.py); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise ImportError(f"libfq.so is not built ({LIB_PATH}); run "
                                  "paper_2608_15531_amd.build.build() first")
            lib = C.CDLL(LIB_PATH)
            for name, (args, res) in _SIGS.items():
                fn = getattr(lib, name)
                fn.argtypes = args
                fn.restype = res
            _lib = lib
    return _lib


STAMPS_LIB_PATH = os.path.join(os.path.dirname(LIB_PATH), "libfq_stamps.so")


def use_instrumented_build() -> C.CDLL:
    """Switch this process to libfq_stamps.so, the build of the same sources
    in which every wave of a matmul launch records timestamps
    (include/fq_debug.h), for measurement only.  Call it before anything else
    uses the library; raises if that build is missing."""
    global _lib
    with _lock:
        if not os.path.exists(STAMPS_LIB_PATH):
            raise ImportError(f"libfq_stamps.so is not built ({STAMPS_LIB_PATH})")
        lib = C.CDLL(STAMPS_LIB_PATH)
        for name, (args, res) in _SIGS.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = res
        lib.fq_debug_wave_stamps.argtypes = [C.c_void_p, C.c_int64]
        lib.fq_debug_wave_stamps.restype = C.c_int
        _lib = lib
    return _lib


def fq_debug_wave_stamps(n_waves: int) -> np.ndarray:
    """The per-wave timestamps of the last matmul launch (instrumented build
    only): uint64 [n_waves][4] = start, first tile's data, end of the tile
    loop, exit, in ticks of the 100 MHz s_memrealtime counter."""
    lib = load()
    if not hasattr(lib, "fq_debug_wave_stamps") or lib.fq_debug_wave_stamps.argtypes is None:
        raise RuntimeError("fq_debug_wave_stamps: call use_instrumented_build() first")
    out = np.zeros((n_waves, 4), np.uint64)
    if lib.fq_debug_wave_stamps(out.ctypes.data, n_waves) != 0:
        raise RuntimeError("fq_debug_wave_stamps failed")
    return out


def _check(status: int, where: str) -> None:
    if status != FQ_OK:
        raise FqError(status, where)


def _ptr(a: np.ndarray) -> int | None:
    return a.ctypes.data if a.size else None


def _params(p) -> fq_tilecoo_params:
    if p is None:
        return load().fq_default_tilecoo_params()
    if isinstance(p, fq_tilecoo_params):
        return p
    d = load().fq_default_tilecoo_params().as_dict()
    d.update(p if isinstance(p, dict) else vars(p))
    return fq_tilecoo_params(**{k: int(d[k]) for k, _ in fq_tilecoo_params._fields_})


def fq_default_tilecoo_params() -> fq_tilecoo_params:
    return load().fq_default_tilecoo_params()


def fq_status_string(status: int) -> str:
    return load().fq_status_string(status).decode()


# ------------------------------------------------------------------ host --

@dataclass
class TileCOOHost:
    params: fq_tilecoo_params
    sizes: fq_tilecoo_sizes
    tile_indptr: np.ndarray   # uint32
    bucket_info: np.ndarray   # uint16
    packed: np.ndarray        # uint32


def fq_pack_tile_coo(K: int, N: int, k, n, v, params=None) -> TileCOOHost:
    """Encode COO outliers (k, n int32; v bf16 bits uint16) into Tile-COO."""
    lib = load()
    k = np.ascontiguousarray(k, dtype=np.int32)
    n = np.ascontiguousarray(n, dtype=np.int32)
    v = np.ascontiguousarray(v, dtype=np.uint16)
    if not (k.shape == n.shape == v.shape):
        raise ValueError("k, n, v must have the same length")
    p = _params(params)
    sizes = fq_tilecoo_sizes()
    _check(lib.fq_pack_tile_coo(K, N, k.size, _ptr(k), _ptr(n), _ptr(v), C.byref(p),
                                C.byref(sizes), None, None, None), "fq_pack_tile_coo")
    tile_indptr = np.empty(sizes.n_tiles + 1, dtype=np.uint32)
    bucket_info = np.empty(2 * sizes.n_buckets, dtype=np.uint16)
    packed = np.empty(max(4 * sizes.n_groups, 4), dtype=np.uint32)
    _check(lib.fq_pack_tile_coo(K, N, k.size, _ptr(k), _ptr(n), _ptr(v), C.byref(p),
                                C.byref(sizes), tile_indptr.ctypes.data,
                                bucket_info.ctypes.data, packed.ctypes.data), "fq_pack_tile_coo")
    return TileCOOHost(p, sizes, tile_indptr, bucket_info, packed[:4 * sizes.n_groups])


def fq_validate_tile_coo(K: int, N: int, params, tile_indptr, bucket_info, packed) -> None:
    lib = load()
    p = _params(params)
    ti = np.ascontiguousarray(tile_indptr, dtype=np.uint32)
    bi = np.ascontiguousarray(bucket_info, dtype=np.uint16)
    pk = np.ascontiguousarray(packed, dtype=np.uint32)
    _check(lib.fq_validate_tile_coo(K, N, C.byref(p), pk.size // 4, _ptr(ti), _ptr(bi),
                                    _ptr(pk)), "fq_validate_tile_coo")


def fq_unpack_tile_coo(K: int, N: int, params, tile_indptr, bucket_info, packed):
    """Decode Tile-COO on the host; returns (k, n, v) sorted by (k, n)."""
    lib = load()
    p = _params(params)
    ti = np.ascontiguousarray(tile_indptr, dtype=np.uint32)
    bi = np.ascontiguousarray(bucket_info, dtype=np.uint16)
    pk = np.ascontiguousarray(packed, dtype=np.uint32)
    nnz = C.c_int64(0)
    _check(lib.fq_unpack_tile_coo(K, N, C.byref(p), pk.size // 4, _ptr(ti), _ptr(bi), _ptr(pk),
                                  C.byref(nnz), None, None, None), "fq_unpack_tile_coo")
    k = np.empty(max(nnz.value, 1), np.int32)
    n = np.empty(max(nnz.value, 1), np.int32)
    v = np.empty(max(nnz.value, 1), np.uint16)
    _check(lib.fq_unpack_tile_coo(K, N, C.byref(p), pk.size // 4, _ptr(ti), _ptr(bi), _ptr(pk),
                                  C.byref(nnz), k.ctypes.data, n.ctypes.data, v.ctypes.data),
           "fq_unpack_tile_coo")
    return k[:nnz.value], n[:nnz.value], v[:nnz.value]


@dataclass
class QuantizedWeight:
    K: int
    N: int
    group: int
    Wq: np.ndarray       # uint32 [K/8][N]
    scales: np.ndarray   # uint16 [K/G][N] fp16 bits
    zeros: np.ndarray    # uint32 [K/G][N/8]
    k: np.ndarray        # int32 [nnz] outlier rows
    n: np.ndarray        # int32 [nnz] outlier columns
    v: np.ndarray        # uint16 [nnz] bf16 bits


def fq_quantize_outlier_aware(W, outlier_frac: float, group: int = 128) -> QuantizedWeight:
    """Split fp32 W [K][N] into INT4 W_Q (per-group affine) and bf16 outliers."""
    lib = load()
    W = np.ascontiguousarray(W, dtype=np.float32)
    K, N = W.shape
    nnz = C.c_int64(0)
    _check(lib.fq_quantize_outlier_aware(K, N, W.ctypes.data, group, float(outlier_frac),
                                         C.byref(nnz), None, None, None, None, None, None),
           "fq_quantize_outlier_aware")
    Wq = np.empty((K // 8, N), np.uint32)
    scales = np.empty((K // group, N), np.uint16)
    zeros = np.empty((K // group, N // 8), np.uint32)
    m = max(nnz.value, 1)
    k, n, v = np.empty(m, np.int32), np.empty(m, np.int32), np.empty(m, np.uint16)
    _check(lib.fq_quantize_outlier_aware(K, N, W.ctypes.data, group, float(outlier_frac),
                                         C.byref(nnz), Wq.ctypes.data, scales.ctypes.data,
                                         zeros.ctypes.data, k.ctypes.data, n.ctypes.data,
                                         v.ctypes.data), "fq_quantize_outlier_aware")
    c = nnz.value
    return QuantizedWeight(K, N, group, Wq, scales, zeros, k[:c], n[:c], v[:c])


def fq_fill_padding_slots(W, qw: QuantizedWeight, host: TileCOOHost) -> int:
    """Store original weights in the padding slots of `host` (in place) and set
    the matching codes of qw.Wq to their zero-points; returns the slots filled."""
    lib = load()
    W = np.ascontiguousarray(W, dtype=np.float32)
    K, N = W.shape
    filled = C.c_int64(0)
    pk = host.packed if host.packed.size else np.zeros(4, np.uint32)
    _check(lib.fq_fill_padding_slots(K, N, W.ctypes.data, qw.group, C.byref(host.params),
                                     int(host.sizes.n_groups), host.tile_indptr.ctypes.data,
                                     host.bucket_info.ctypes.data, pk.ctypes.data,
                                     qw.Wq.ctypes.data, qw.zeros.ctypes.data, C.byref(filled)),
           "fq_fill_padding_slots")
    return int(filled.value)


# ---------------------------------------------------------------- device --

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


class TileCOODevice:
    """Tile-COO arrays resident in device memory (torch tensors)."""

    def __init__(self, host: TileCOOHost, device="cuda"):
        torch = _torch()
        self.params = host.params
        self.sizes = host.sizes
        self.tile_indptr = torch.from_numpy(host.tile_indptr.view(np.int32).copy()).to(device)
        self.bucket_info = torch.from_numpy(host.bucket_info.view(np.int16).copy()).to(device)
        pk = host.packed if host.packed.size else np.zeros(4, np.uint32)
        self.packed = torch.from_numpy(pk.view(np.int32).copy()).to(device)
        self.n_groups = int(host.sizes.n_groups)
        self.max_tile_groups = int(host.sizes.max_tile_groups)

    def struct(self) -> fq_tilecoo_dev:
        return fq_tilecoo_dev(self.tile_indptr.data_ptr(), self.bucket_info.data_ptr(),
                              self.packed.data_ptr(), self.params, self.n_groups,
                              self.max_tile_groups)

    @property
    def nbytes(self) -> int:
        return int(self.sizes.bytes)


_workspaces: dict = {}
_captured: dict = {}       # of graphs: (capture, workspace) by stream, the last capture only
_COUNTER_BYTES = 256 * 1024   # of a workspace, which have to be zero before its first use


def _stream_handle(stream, device) -> int:
    torch = _torch()
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return int(stream.cuda_stream)


_raw_stream = None


def _current_device() -> int:
    return _torch()._C._cuda_getDevice()   # as torch.cuda.current_device, once a tensor is there


def _elsewhere(index: int) -> bool:
    """Whether device `index` is not the current one.  Its default stream has the handle of
    every device's, and the library would launch on the current device's."""
    return _current_device() != index


def _stream_of(stream, index: int) -> int:
    """_stream_handle by device index, without making a torch Stream object of the current
    stream (1.5 us a call) where torch offers its handle."""
    global _raw_stream
    if stream is not None:
        if stream.device_index != index:
            raise ValueError(f"the stream is on device {stream.device_index}, the tensors on {index}")
        return int(stream.cuda_stream)
    if _raw_stream is None:
        torch = _torch()
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda i: int(torch.cuda.current_stream(i).cuda_stream))
    return _raw_stream(index)


def _capture_of(stream, stream_handle: int):
    """Number of the graph capture that the stream is part of, or None."""
    if stream is None and not _torch().cuda.is_current_stream_capturing():
        return None
    if not stream_handle:
        return None   # the default stream cannot be captured
    status, number = C.c_int(0), C.c_ulonglong(0)
    if load().hipStreamGetCaptureInfo(C.c_void_p(stream_handle), C.byref(status), C.byref(number)):
        raise FqError(_FQ_ERR_HIP, "hipStreamGetCaptureInfo")
    return number.value if status.value else None


def _kept(key, capture):
    """The workspace kept for (device index, stream), in a capture that of the capture."""
    if capture is None:
        return _workspaces.get(key)
    number, buf = _captured.get(key, (None, None))
    return buf if number == capture else None


def workspace(nbytes: int, device, stream_handle: int, capture=None):
    """Zero-filled workspace kept per (device, stream); the kernels leave it zeroed.
    Call it with the kernel's stream current (see _on_stream): the allocation
    and its zero fill are then ordered before the kernel on that stream.

    capture: number of the graph capture that the call is recorded in (_capture_of).  The
    workspace then comes from the graph's memory, no eager call and no other graph uses it,
    and its counters' zero fill is recorded with it, so each replay starts with it: a kept
    one may be gone when the graph is replayed, or never have been cleared."""
    torch = _torch()
    key = (torch.device(device).index, stream_handle)
    buf = _kept(key, capture)
    if buf is None or buf.numel() < nbytes:
        if capture is None:
            buf = torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=device)
            _workspaces[key] = buf
        else:
            buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
            buf[:_COUNTER_BYTES].zero_()
            _captured[key] = (capture, buf)
    return buf


_NO_STREAM = contextlib.nullcontext()
_STRIP_ROWS = 16   # up to so many rows, one kernel and one workspace size per problem


def _on_stream(stream):
    """Makes `stream` current while Y and the workspace are allocated, so the
    caching allocator ties them to the stream the kernel runs on and the
    workspace's zero fill precedes the kernel there."""
    if stream is None:
        return _NO_STREAM
    return _torch().cuda.stream(stream)


def _launch(call, sizer, pr, ws, device, stream, where):
    """call(workspace tensor, stream handle) -> status.  Without a workspace from
    the caller the one kept for the stream is tried first; the library checks its
    size against the launch before it enqueues anything, and only when that check
    fails (or none is kept yet) is the size asked for and a larger one made.  With
    more than 16 rows the size is always asked for: there a smaller workspace may
    pass the check and get the strip kernel in the row-block kernel's place, so the
    kernel would depend on the calls before.  Calls recorded in a graph share one of the
    graph's own (workspace)."""
    sh = _stream_handle(stream, device)
    if ws is None:
        capture = _capture_of(stream, sh)
        ws = _kept((device.index, sh), capture) if pr.M <= _STRIP_ROWS else None
        if ws is not None:
            status = call(ws, sh)
            if status != _FQ_ERR_WORKSPACE:
                _check(status, where)
                return
        need = C.c_size_t(0)
        _check(sizer(C.byref(pr), C.byref(need)), sizer.__name__)
        with _on_stream(stream):
            ws = workspace(need.value, device, sh, capture)
    _check(call(ws, sh), where)


def _problem(M, K, N, y_dtype, split_k, group=128, sparse="auto", flags=0) -> fq_problem:
    return fq_problem(M, K, N, group, y_dtype, split_k, _SPARSE_MODES[sparse] | flags)


def _check_tensor(t, dtype, shape, name):
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)}, got "
                         f"{t.dtype} {tuple(t.shape)}")


def _matmul_args(X, Wq, scales, zeros, Y, y_dtype, group):
    torch = _torch()
    M, K = X.shape
    N = Wq.shape[1]
    _check_tensor(X, torch.bfloat16, (M, K), "X")
    _check_tensor(Wq, torch.int32, (K // 8, N), "Wq")
    _check_tensor(scales, torch.float16, (K // group, N), "scales")
    _check_tensor(zeros, torch.int32, (K // group, N // 8), "zeros")
    ydt = FQ_Y_F32 if y_dtype in ("f32", "fp32", torch.float32) else FQ_Y_BF16
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float32 if ydt == FQ_Y_F32 else torch.bfloat16,
                        device=X.device)
    else:
        _check_tensor(Y, torch.float32 if ydt == FQ_Y_F32 else torch.bfloat16, (M, N), "Y")
    return M, K, N, ydt, Y


def fq_w4a16_outlier_matmul(X, Wq, scales, zeros, tc: TileCOODevice, Y=None, y_dtype="bf16",
                            split_k: int = 0, stream=None, ws=None, group: int = 128,
                            sparse: str = "auto", flags: int = 0):
    """Fused Y = X dequant(W_Q) + X W_O on the GPU; returns Y.  flags: any of
    FQ_SCHED_STREAM_K, FQ_FOUR_WAVES."""
    lib = load()
    with _on_stream(stream):
        M, K, N, ydt, Y = _matmul_args(X, Wq, scales, zeros, Y, y_dtype, group)
    pr = _problem(M, K, N, ydt, split_k, group, sparse, flags)
    tcs = tc.struct()
    _launch(lambda w, sh: lib.fq_w4a16_outlier_matmul(
                C.byref(pr), X.data_ptr(), Wq.data_ptr(), scales.data_ptr(), zeros.data_ptr(),
                C.byref(tcs), Y.data_ptr(), w.data_ptr(), w.numel(), sh),
            lib.fq_workspace_bytes, pr, ws, X.device, stream, "fq_w4a16_outlier_matmul")
    return Y


def fq_w4a16_outlier_matmul_noalloc(X, Wq, scales, zeros, tc: TileCOODevice, Y,
                                    y_dtype="bf16", split_k: int = 0, stream=None,
                                    group: int = 128, sparse: str = "auto", flags: int = 0):
    """Fused Y = X dequant(W_Q) + X W_O without a workspace: the library's
    static device scratch serves as one.  Y is the caller's output tensor
    (nothing is allocated here either); returns Y."""
    lib = load()
    if Y is None:
        raise ValueError("fq_w4a16_outlier_matmul_noalloc: pass the output tensor Y")
    M, K, N, ydt, Y = _matmul_args(X, Wq, scales, zeros, Y, y_dtype, group)
    pr = _problem(M, K, N, ydt, split_k, group, sparse, flags)
    tcs = tc.struct()
    _check(lib.fq_w4a16_outlier_matmul_noalloc(C.byref(pr), X.data_ptr(), Wq.data_ptr(),
                                               scales.data_ptr(), zeros.data_ptr(),
                                               C.byref(tcs), Y.data_ptr(),
                                               _stream_handle(stream, X.device)),
           "fq_w4a16_outlier_matmul_noalloc")
    return Y


def fq_w4a16_outlier_matmul_unfused(X, Wq, scales, zeros, tc: TileCOODevice, Y=None,
                                    y_dtype="bf16", split_k: int = 0, stream=None, ws=None,
                                    group: int = 128, sparse: str = "auto", flags: int = 0):
    """Two-kernel baseline (dense W4A16 then Tile-COO SpMM); returns Y."""
    lib = load()
    with _on_stream(stream):
        M, K, N, ydt, Y = _matmul_args(X, Wq, scales, zeros, Y, y_dtype, group)
    pr = _problem(M, K, N, ydt, split_k, group, sparse, flags)
    tcs = tc.struct()
    _launch(lambda w, sh: lib.fq_w4a16_outlier_matmul_unfused(
                C.byref(pr), X.data_ptr(), Wq.data_ptr(), scales.data_ptr(), zeros.data_ptr(),
                C.byref(tcs), Y.data_ptr(), w.data_ptr(), w.numel(), sh),
            lib.fq_workspace_bytes_unfused, pr, ws, X.device, stream,
            "fq_w4a16_outlier_matmul_unfused")
    return Y


def fq_w4a16_matmul(X, Wq, scales, zeros, Y=None, y_dtype="bf16", split_k: int = 0,
                    stream=None, ws=None, group: int = 128, flags: int = 0):
    """Dense-only Y = X dequant(W_Q) (outliers ignored); returns Y."""
    lib = load()
    with _on_stream(stream):
        M, K, N, ydt, Y = _matmul_args(X, Wq, scales, zeros, Y, y_dtype, group)
    pr = _problem(M, K, N, ydt, split_k, group, flags=flags)
    _launch(lambda w, sh: lib.fq_w4a16_matmul(
                C.byref(pr), X.data_ptr(), Wq.data_ptr(), scales.data_ptr(), zeros.data_ptr(),
                Y.data_ptr(), w.data_ptr(), w.numel(), sh),
            lib.fq_workspace_bytes, pr, ws, X.device, stream, "fq_w4a16_matmul")
    return Y


def fq_debug_decode_tile_coo(tc: TileCOODevice, K: int, N: int, stream=None):
    """Device decode of every group; returns (k, n, v) torch tensors of 4*n_groups."""
    torch = _torch()
    lib = load()
    dev = tc.packed.device
    G = tc.n_groups
    with _on_stream(stream):
        k = torch.empty(max(4 * G, 1), dtype=torch.int32, device=dev)
        n = torch.empty(max(4 * G, 1), dtype=torch.int32, device=dev)
        v = torch.empty(max(4 * G, 1), dtype=torch.int16, device=dev)
    tcs = tc.struct()
    _check(lib.fq_debug_decode_tile_coo(C.byref(tcs), K, N, k.data_ptr(), n.data_ptr(),
                                        v.data_ptr(), _stream_handle(stream, dev)),
           "fq_debug_decode_tile_coo")
    return k[:4 * G], n[:4 * G], v[:4 * G]


def fq_launch_kernel(M: int, K: int, N: int, tc=None, split_k: int = 0, sparse: str = "auto",
                     flags: int = 0, workspace_bytes: int | None = None) -> dict:
    """The kernel and grid of a matmul call (nothing is launched).  tc: a TileCOOHost
    or TileCOODevice, or None for the dense-only entry point.  workspace_bytes: the
    workspace's size (default: any size that is needed)."""
    lib = load()
    pr = _problem(M, K, N, FQ_Y_BF16, split_k, 128, sparse, flags)
    dev = None
    if tc is not None:
        dev = C.byref(fq_tilecoo_dev(None, None, None, tc.params, tc.sizes.n_groups,
                                     tc.sizes.max_tile_groups))
    if workspace_bytes is None:
        workspace_bytes = C.c_size_t(-1).value
    out = (C.c_int32 * 10)()
    _check(lib.fq_launch_kernel(C.byref(pr), dev, workspace_bytes, out), "fq_launch_kernel")
    return {"kernel": "rows" if out[0] else "strip", "block_cols": out[1], "block_rows": out[2],
            "row_blocks": out[3], "split_k": out[4], "workgroups": out[5], "waves": out[6],
            "group_loads": out[7], "lds_bytes": out[8], "partial_kib": out[9]}


def fq_launch_config(M: int, K: int, N: int, split_k: int = 0, sparse: str = "auto",
                     flags: int = 0, buckets_per_tile: int | None = None,
                     group_mode: int | None = None) -> dict:
    """The strip kernel's launch (nothing is launched; fq_launch_kernel says when it runs) for a
    Tile-COO packed with the given bucket count and grouping (default: the
    library's default packing)."""
    lib = load()
    if buckets_per_tile is None or group_mode is None:
        d = lib.fq_default_tilecoo_params()
        buckets_per_tile = d.buckets_per_tile if buckets_per_tile is None else buckets_per_tile
        group_mode = d.group_mode if group_mode is None else group_mode
    pr = _problem(M, K, N, FQ_Y_BF16, split_k, 128, sparse, flags)
    cfg = (C.c_int32 * 10)()
    _check(lib.fq_launch_config(C.byref(pr), buckets_per_tile, group_mode, cfg),
           "fq_launch_config")
    return {"strip_cols": cfg[0], "split_k": cfg[1], "dense_waves": cfg[2],
            "outlier_waves": cfg[3], "mapping": "gather" if cfg[4] == FQ_SPARSE_GATHER else "mfma",
            "workgroups": cfg[5], "stream_k": bool(cfg[6]), "lds_bytes": cfg[7],
            "x_staged": bool(cfg[8]), "x_stage_loads": cfg[8], "bulk_scales": bool(cfg[9])}


def fq_workspace_bytes(M: int, K: int, N: int, y_dtype=FQ_Y_BF16, split_k: int = 0,
                       group: int = 128, flags: int = 0) -> int:
    lib = load()
    pr = _problem(M, K, N, y_dtype, split_k, group, flags=flags)
    need = C.c_size_t(0)
    _check(lib.fq_workspace_bytes(C.byref(pr), C.byref(need)), "fq_workspace_bytes")
    return need.value


def fq_workspace_bytes_unfused(M: int, K: int, N: int, y_dtype=FQ_Y_BF16, split_k: int = 0,
                               group: int = 128, flags: int = 0) -> int:
    lib = load()
    pr = _problem(M, K, N, y_dtype, split_k, group, flags=flags)
    need = C.c_size_t(0)
    _check(lib.fq_workspace_bytes_unfused(C.byref(pr), C.byref(need)),
           "fq_workspace_bytes_unfused")
    return need.value


# ------------------------------------------- the rest of a decoder layer --

def _check_rows(t, dtype, shape, name, index=None):
    """The strides of a CUDA tensor whose last dimension is contiguous; the others may have
    any.  index: the device that it has to be on."""
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} "
                         f"{tuple(t.shape)}")
    if index is not None and t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on device {index}")
    st = t.stride()
    if st[-1] != 1 and shape[-1] != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return st


def _rows(t, dtype, shape, name, index):
    """_check_rows, quick where all is well."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == index:
            st = t.stride()
            if st[-1] == 1:
                return st
    except AttributeError:
        pass   # no tensor
    return _check_rows(t, dtype, shape, name, index)


def _check_slots(slots, index):
    if not isinstance(slots, _torch().Tensor) or slots.dim() != 1:
        raise ValueError("slots: expected int64 [n_tokens]")
    n = slots.shape[0]
    _rows(slots, _torch().int64, (n,), "slots", index)
    return n


def _check_workspace(ws, index):
    """A workspace of the caller; returns its bytes."""
    if not isinstance(ws, _torch().Tensor) or ws.get_device() != index or not ws.is_contiguous():
        raise ValueError(f"ws: expected a contiguous tensor on device {index}")
    return ws.numel() * ws.element_size()


def _any_stride(t):
    """Strides with 0 for dimensions of one, of which torch keeps any number."""
    return tuple(0 if n == 1 else s for n, s in zip(t.shape, t.stride()))


class KVCache:
    """A paged KV cache over device tensors (fq.h, fq_kv_cache).

    k, v: [n_pages][n_kv_heads][page_size][row], bf16 with kind "bf16" (row =
    head_dim), uint8 with "int8" (row = head_dim) and "int4" (row = head_dim / 2);
    k_meta, v_meta: bf16 [n_pages][n_kv_heads][page_size][2], scale and zero-point.
    The tensors may be views with other strides (k and v with the same ones), such as
    pools ordered [n_pages][page_size][n_kv_heads][row] seen through transpose(1, 2)."""

    def __init__(self, k, v, k_meta=None, v_meta=None, kind: str = "bf16"):
        torch = _torch()
        if kind not in _KV_KINDS:
            raise ValueError(f"kind: one of {sorted(_KV_KINDS)}, got {kind!r}")
        dtype = torch.bfloat16 if kind == "bf16" else torch.uint8
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("k: expected [n_pages][n_kv_heads][page_size][row]")
        _check_rows(k, dtype, k.shape, "k")
        _check_rows(v, dtype, k.shape, "v")
        st = _any_stride(k)
        if _any_stride(v) != st:
            raise ValueError("k and v must have the same strides")
        P, H, T, row = k.shape
        size = k.element_size()
        mst = (0, 0, 1)
        if kind == "bf16":
            if k_meta is not None or v_meta is not None:
                raise ValueError("a bf16 cache has no k_meta and v_meta")
        else:
            if k_meta is None or v_meta is None:
                raise ValueError(f"a cache of kind {kind} needs k_meta and v_meta")
            _check_rows(k_meta, torch.bfloat16, (P, H, T, 2), "k_meta")
            _check_rows(v_meta, torch.bfloat16, (P, H, T, 2), "v_meta")
            m = _any_stride(k_meta)
            if _any_stride(v_meta) != m:
                raise ValueError("k_meta and v_meta must have the same strides")
            if (T > 1 and m[2] != 2) or m[0] % 2 or m[1] % 2:
                raise ValueError("k_meta, v_meta: the tokens of a page must be contiguous")
            mst = (m[0] // 2, m[1] // 2, 1)
        for t, name in ((v, "v"), (k_meta, "k_meta"), (v_meta, "v_meta")):
            if t is not None and t.device != k.device:
                raise ValueError(f"{name} is on {t.device}, k on {k.device}")
        self.k, self.v, self.k_meta, self.v_meta, self.kind = k, v, k_meta, v_meta, kind
        self.device = k.device
        self._index = k.get_device()
        self.n_pages, self.n_kv_heads, self.page_size = P, H, T
        self.head_dim = 2 * row if kind == "int4" else row
        self._struct = fq_kv_cache(
            k.data_ptr(), v.data_ptr(), None if k_meta is None else k_meta.data_ptr(),
            None if v_meta is None else v_meta.data_ptr(), st[0] * size, st[1] * size,
            st[2] * size, mst[0], mst[1], P, T, H, self.head_dim, _KV_KINDS[kind])
        self._ref = C.byref(self._struct)

    @classmethod
    def empty(cls, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int,
              kind: str = "bf16", device="cuda") -> "KVCache":
        """A cache whose pages hold nothing yet."""
        torch = _torch()
        if kind not in _KV_KINDS:
            raise ValueError(f"kind: one of {sorted(_KV_KINDS)}, got {kind!r}")
        row = head_dim // 2 if kind == "int4" else head_dim
        dtype = torch.bfloat16 if kind == "bf16" else torch.uint8
        k, v = (torch.empty((n_pages, n_kv_heads, page_size, row), dtype=dtype, device=device)
                for _ in range(2))
        if kind == "bf16":
            return cls(k, v, kind=kind)
        km, vm = (torch.empty((n_pages, n_kv_heads, page_size, 2), dtype=torch.bfloat16,
                              device=device) for _ in range(2))
        return cls(k, v, km, vm, kind=kind)

    def struct(self) -> fq_kv_cache:
        return self._struct

    @property
    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size()
                   for t in (self.k, self.v, self.k_meta, self.v_meta) if t is not None)


class PagedBatch:
    """The sequences of one step: cu_q int32 [n_seqs + 1] (first new token of each),
    kv_lens int32 [n_seqs] (tokens in the cache, the new ones included), block_table
    int32 [n_seqs][pages], and upper bounds max_q and max_kv of the new tokens and of
    kv_lens.  Made once for all layers of a step; the tensors' contents may change
    between calls, and between replays of a graph, within the bounds."""

    def __init__(self, cu_q, kv_lens, block_table, max_q: int, max_kv: int):
        torch = _torch()
        if not isinstance(kv_lens, torch.Tensor) or kv_lens.dim() != 1:
            raise ValueError("kv_lens: expected [n_seqs]")
        n = kv_lens.shape[0]
        _check_tensor(kv_lens, torch.int32, (n,), "kv_lens")
        _check_tensor(cu_q, torch.int32, (n + 1,), "cu_q")
        if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
            raise ValueError("block_table: expected [n_seqs][pages]")
        _check_rows(block_table, torch.int32, (n, block_table.shape[1]), "block_table")
        st = _any_stride(block_table)
        for t, name in ((kv_lens, "kv_lens"), (block_table, "block_table")):
            if t.device != cu_q.device:
                raise ValueError(f"{name} is on {t.device}, cu_q on {cu_q.device}")
        self.cu_q, self.kv_lens, self.block_table = cu_q, kv_lens, block_table
        self.n_seqs, self.max_q, self.max_kv = n, int(max_q), int(max_kv)
        self.table_stride = st[0]
        self.device = cu_q.device
        self._index = cu_q.get_device()
        self._table_cols = block_table.shape[1]
        self._pointers = (cu_q.data_ptr(), kv_lens.data_ptr(), block_table.data_ptr())


def fq_kv_cache_write(cache: KVCache, k, v, slots, stream=None) -> None:
    """Store the rows k, v (bf16 [n_tokens][n_kv_heads][head_dim], any token and head
    stride) at `slots` (int64 [n_tokens]: page * page_size + place; a token whose slot is
    out of range, such as -1, is not stored), quantised as the cache's kind asks."""
    lib = load()
    index, bf16 = cache._index, _torch().bfloat16
    if _elsewhere(index):
        with _torch().cuda.device(index):
            return fq_kv_cache_write(cache, k, v, slots, stream)
    n = _check_slots(slots, index)
    shape = (n, cache.n_kv_heads, cache.head_dim)
    ks = _rows(k, bf16, shape, "k", index)
    vs = _rows(v, bf16, shape, "v", index)
    status = lib.fq_kv_cache_write(cache._ref, k.data_ptr(), v.data_ptr(), ks[0], ks[1], vs[0],
                                   vs[1], slots.data_ptr(), n, _stream_of(stream, index))
    if status:
        raise FqError(status, "fq_kv_cache_write")


def fq_kv_cache_read(cache: KVCache, slots, k=None, v=None, dtype="bf16", stream=None):
    """The rows at `slots` (int64 [n_tokens]; out of range: zeros) as the values they
    stand for; returns K, V of [n_tokens][n_kv_heads][head_dim], bf16 or fp32 ("f32")."""
    torch = _torch()
    lib = load()
    index = cache._index
    f32 = dtype in ("f32", "fp32", torch.float32)
    if not f32 and dtype not in ("bf16", "bfloat16", torch.bfloat16):
        raise ValueError(f"dtype: bf16 or f32, got {dtype!r}")
    if _elsewhere(index):
        with torch.cuda.device(index):
            return fq_kv_cache_read(cache, slots, k, v, dtype, stream)
    n = _check_slots(slots, index)
    shape = (n, cache.n_kv_heads, cache.head_dim)
    dt = torch.float32 if f32 else torch.bfloat16
    for t, name in ((k, "k"), (v, "v")):
        if t is not None:
            _check_tensor(t, dt, shape, name)
            _rows(t, dt, shape, name, index)
    if k is None or v is None:
        with _on_stream(stream):
            k = torch.empty(shape, dtype=dt, device=cache.device) if k is None else k
            v = torch.empty_like(k) if v is None else v
    status = lib.fq_kv_cache_read(cache._ref, slots.data_ptr(), n, k.data_ptr(), v.data_ptr(),
                                  FQ_Y_F32 if f32 else FQ_Y_BF16, _stream_of(stream, index))
    if status:
        raise FqError(status, "fq_kv_cache_read")
    return k, v


def _attention(n_heads, q_strides, o_strides, total_q, cache, batch, scale, window, sinks):
    # ctypes would cut wider numbers to 32 bits
    numbers = (batch.max_q, batch.max_kv, window, sinks)
    if max(numbers) > 0x7FFFFFFF or min(numbers) < -0x80000000:
        raise ValueError("max_q, max_kv, window and sinks: below 2^31, and not negative")
    return fq_attention(batch.n_seqs, n_heads, batch.max_q, batch.max_kv, window, sinks, total_q,
                        q_strides[0], q_strides[1], o_strides[0], o_strides[1],
                        batch.table_stride, batch._table_cols,
                        cache.head_dim ** -0.5 if scale is None else scale)


def fq_paged_attention(q, cache: KVCache, batch: PagedBatch, scale: float | None = None,
                       window: int = 0, sinks: int = 0, out=None, return_lse: bool = False,
                       stream=None, ws=None):
    """Attention of the new tokens q (bf16 [total_q][n_heads][head_dim], any token and
    head stride) over the cache, which holds their K and V already.  scale: default
    1 / sqrt(head_dim).  window W > 0: a token sees the last W keys up to its own and the
    first `sinks` keys.  Returns out (bf16, like q), and with return_lse also the ln of
    the softmax sums, fp32 [total_q][n_heads].  A token that sees no key gets zeros and
    -infinity; rows of q that belong to no sequence are left as they are in `out`
    (unspecified in a new one).

    ws: a zero-filled workspace of fq_paged_attention_workspace_bytes or more on the cache's
    device, for calls that do not overlap in time.  Without one the workspace kept for the stream is used, which
    grows to the largest call's (277 MB of partial sums at most) and is not given back; a
    call recorded in a graph uses one in the graph's memory."""
    torch = _torch()
    lib = load()
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q: expected [total_q][n_heads][head_dim]")
    index, bf16 = cache._index, torch.bfloat16
    if _elsewhere(index):
        with torch.cuda.device(index):
            return fq_paged_attention(q, cache, batch, scale, window, sinks, out, return_lse, stream, ws)
    total, heads, _ = q.shape
    shape = (total, heads, cache.head_dim)
    qs = _rows(q, bf16, shape, "q", index)
    if batch._index != index:
        raise ValueError(f"the batch is on {batch.device}, the cache on {cache.device}")
    lse = None
    if out is not None:
        os_ = _rows(out, bf16, shape, "out", index)
    if out is None or return_lse:
        with _on_stream(stream):
            if out is None:
                out = torch.empty_like(q, memory_format=torch.contiguous_format)
                os_ = out.stride()
            if return_lse:
                lse = torch.empty((total, heads), dtype=torch.float32, device=cache.device)
    ref = C.byref(_attention(heads, qs, os_, total, cache, batch, scale, window, sinks))
    cu, lens, table = batch._pointers
    sh = _stream_of(stream, index)
    pq, po = q.data_ptr(), out.data_ptr()
    pl = None if lse is None else lse.data_ptr()
    capture = _capture_of(stream, sh) if ws is None else None
    w = _kept((index, sh), capture) if ws is None else ws
    size = 0 if w is None else w.numel() if ws is None else _check_workspace(ws, index)
    status = lib.fq_paged_attention(ref, pq, cache._ref, cu, lens, table, po, pl,
                                    None if w is None else w.data_ptr(), size, sh)
    if status == _FQ_ERR_WORKSPACE and ws is None:
        # checked before anything is enqueued: none is kept yet, or too small a one
        need = C.c_size_t(0)
        _check(lib.fq_paged_attention_workspace_bytes(ref, cache._ref, C.byref(need)),
               "fq_paged_attention_workspace_bytes")
        with _on_stream(stream):
            w = workspace(need.value, cache.device, sh, capture)
        status = lib.fq_paged_attention(ref, pq, cache._ref, cu, lens, table, po, pl,
                                        w.data_ptr(), w.numel(), sh)
    if status:
        raise FqError(status, "fq_paged_attention")
    return (out, lse) if return_lse else out


def fq_paged_attention_workspace_bytes(n_heads: int, total_q: int, cache: KVCache,
                                       batch: PagedBatch, window: int = 0, sinks: int = 0) -> int:
    a = _attention(n_heads, (0, 0), (0, 0), total_q, cache, batch, None, window, sinks)
    need = C.c_size_t(0)
    _check(load().fq_paged_attention_workspace_bytes(C.byref(a), cache._ref, C.byref(need)),
           "fq_paged_attention_workspace_bytes")
    return need.value


def fq_paged_attention_launch(n_heads: int, total_q: int, cache: KVCache, batch: PagedBatch,
                              window: int = 0, sinks: int = 0) -> dict:
    """The kernel and grid of a call (nothing is launched)."""
    a = _attention(n_heads, (0, 0), (0, 0), total_q, cache, batch, None, window, sinks)
    out = (C.c_int32 * 8)()
    _check(load().fq_paged_attention_launch(C.byref(a), cache._ref, out),
           "fq_paged_attention_launch")
    return {"kernel": _ATTN_KERNELS[out[0]], "rows": out[1], "row_blocks": out[2],
            "split": out[3], "split_keys": out[4], "workgroups": out[5], "lds_bytes": out[6],
            "partial_kib": out[7]}


def _dtype_code(dtype, name):
    torch = _torch()
    if dtype == torch.bfloat16:
        return FQ_Y_BF16
    if dtype == torch.float32:
        return FQ_Y_F32
    raise ValueError(f"{name}: expected bfloat16 or float32, got {dtype}")


def fq_gated_residual_norm(x, residual=None, pre_weight=None, post_weight=None, gate=None,
                           residual_scale: float = 1.0, eps: float = 1e-5, residual_out=None,
                           h=None, stream=None):
    """u = RMSNorm(x) post_weight (x itself without post_weight), r = residual_scale
    residual + gate u, h = RMSNorm(r) pre_weight, each rounded once; returns (r, h).

    x [rows][cols] bf16 or fp32; residual the same shape, bf16 or fp32 (None: r = gate u,
    of x's type); gate bf16 [cols] or [rows][cols] (None: 1); weights bf16 [cols].
    Without pre_weight only r is computed and h is None.  residual_out may be residual.
    Rows may have any stride; columns are contiguous."""
    torch = _torch()
    lib = load()
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x: expected [rows][cols]")
    if not x.is_cuda:   # below, the others are only compared with its device
        raise TypeError("x must be a CUDA (HIP) tensor")
    index, bf16, shape, xt = x.get_device(), torch.bfloat16, x.shape, x.dtype
    if _elsewhere(index):
        with torch.cuda.device(index):
            return fq_gated_residual_norm(x, residual, pre_weight, post_weight, gate, residual_scale, eps,
                                          residual_out, h, stream)
    M, H = shape
    xs = _rows(x, xt, shape, "x", index)
    rt, rs, gs, pr, pg = xt, 0, 0, None, None
    if residual is not None:
        rt = residual.dtype
        rs = _rows(residual, rt, shape, "residual", index)[0]
        pr = residual.data_ptr()
    if gate is not None:
        if gate.dim() == 1:
            _rows(gate, bf16, (H,), "gate", index)
        else:
            gs = _rows(gate, bf16, shape, "gate", index)[0]
        pg = gate.data_ptr()
    if post_weight is not None:
        _rows(post_weight, bf16, (H,), "post_weight", index)
    if pre_weight is not None:
        _rows(pre_weight, bf16, (H,), "pre_weight", index)
    elif h is not None:
        raise ValueError("h needs pre_weight")
    ros = hs = H
    if residual_out is not None:
        ros = _rows(residual_out, rt, shape, "residual_out", index)[0]
    if h is not None:
        hs = _rows(h, bf16, shape, "h", index)[0]
    if residual_out is None or (h is None and pre_weight is not None):
        with _on_stream(stream):
            like = torch.contiguous_format
            if residual_out is None:
                residual_out = torch.empty_like(x if residual is None else residual,
                                                memory_format=like)
            if h is None and pre_weight is not None:
                h = torch.empty_like(x, memory_format=like) if xt is bf16 else \
                    torch.empty(shape, dtype=bf16, device=x.device)
    n = fq_norm(M, H, _dtype_code(xt, "x"), _dtype_code(rt, "residual"), eps, residual_scale, xs[0],
                rs, gs, ros, hs)
    status = lib.fq_gated_residual_norm(
        C.byref(n), x.data_ptr(), pr, None if post_weight is None else post_weight.data_ptr(), pg,
        None if pre_weight is None else pre_weight.data_ptr(), residual_out.data_ptr(),
        None if h is None else h.data_ptr(), _stream_of(stream, index))
    if status:
        raise FqError(status, "fq_gated_residual_norm")
    return residual_out, h


# ---------------------------------------------------- numpy -> device --

def to_device(problem, device="cuda"):
    """Upload a synth.Problem's dense arrays as torch tensors in the library layout."""
    torch = _torch()
    X = torch.from_numpy(problem.X.view(np.int16).copy()).view(torch.bfloat16).to(device)
    Wq = torch.from_numpy(problem.Wq.view(np.int32).copy()).to(device)
    scales = torch.from_numpy(problem.scales.view(np.int16).copy()).view(torch.float16).to(device)
    zeros = torch.from_numpy(problem.zeros.view(np.int32).copy()).to(device)
    return X, Wq, scales, zeros
