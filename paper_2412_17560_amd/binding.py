"""ctypes marshalling for libgqsa.so -- same names as the C ABI, no arithmetic here."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

from . import build as _build

_LIB = None


class GqsaError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {gqsa_status_string(status)} (status {status})")
        self.status = status


class _Info(C.Structure):
    _fields_ = [("N", C.c_int64), ("K", C.c_int64), ("G", C.c_int32), ("bits", C.c_int32),
                ("nnz_groups", C.c_int64), ("values_bytes", C.c_int64), ("n_blocks", C.c_int64),
                ("n_workgroups", C.c_int32), ("waves_per_workgroup", C.c_int32),
                ("needs_fixup", C.c_int32), ("span_tiles", C.c_int32), ("n_empty_rows", C.c_int64),
                ("device_bytes", C.c_int64), ("algorithmic_bytes", C.c_int64),
                ("on_device", C.c_int32), ("panel_integer_zeros", C.c_int32), ("panel_bytes", C.c_int64),
                ("tile_blocks", C.c_int32), ("tile_lanes", C.c_int32), ("span_per_worker", C.c_int32),
                ("reserved0", C.c_int32)]


class _CacheInfo(C.Structure):
    _fields_ = [("n_pages", C.c_int64), ("page_tokens", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("token_bytes", C.c_int32), ("device_bytes", C.c_int64), ("workspace_bytes", C.c_int64)]


def library_path() -> str:
    return _build.LIB


def _lib():
    global _LIB
    if _LIB is not None:
        return _LIB
    # PyTorch ships its own HIP runtime (same SONAME as the system one).  Streams and device
    # pointers handed to libgqsa come from PyTorch, so both must live in ONE runtime: import
    # torch first, and the loader resolves libgqsa's libamdhip64 to the copy already mapped.
    # (A host-only build named by GQSA_LIBRARY has no HIP runtime to share.)
    if not _build.HOST_ONLY:
        import torch  # noqa: F401
    path = _build.LIB
    if not os.path.exists(path):
        _build.build()           # nothing built yet: build once, in-tree
    if not os.path.exists(path):
        raise ImportError(f"libgqsa.so is missing at {path}; run `python -m paper_2412_17560_amd.build`")
    lib = C.CDLL(path)
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int
    lib.gqsa_pack.restype = C.c_int
    lib.gqsa_pack.argtypes = [vp, i64, i64, i32, i32, C.c_double, C.POINTER(vp)]
    lib.gqsa_pack_rows.restype = C.c_int
    lib.gqsa_pack_rows.argtypes = [vp, i64, i64, i32, i32, vp, C.POINTER(vp)]
    lib.gqsa_pack_hessian.restype = C.c_int
    lib.gqsa_pack_hessian.argtypes = [vp, i64, i64, i32, i32, C.c_double, vp, C.POINTER(vp)]
    lib.gqsa_pack_device.restype = C.c_int
    lib.gqsa_pack_device.argtypes = [vp, i64, i64, i32, i32, C.c_double, vp, vp, vp, C.POINTER(vp)]
    lib.gqsa_save.restype = C.c_int
    lib.gqsa_save.argtypes = [vp, C.c_char_p]
    lib.gqsa_load.restype = C.c_int
    lib.gqsa_load.argtypes = [C.c_char_p, C.POINTER(vp)]
    lib.gqsa_import.restype = C.c_int
    lib.gqsa_import.argtypes = [vp, vp, vp, vp, vp, i64, i64, i32, i32, C.POINTER(vp)]
    lib.gqsa_set_partition.restype = C.c_int
    lib.gqsa_set_partition.argtypes = [vp, i32, i32]
    lib.gqsa_build_panels.restype = C.c_int
    lib.gqsa_build_panels.argtypes = [vp]
    lib.gqsa_export_panel_blob.restype = C.c_int
    lib.gqsa_export_panel_blob.argtypes = [vp, vp, C.c_size_t]
    lib.gqsa_set_partition_aligned.restype = C.c_int
    lib.gqsa_set_partition_aligned.argtypes = [vp, i32, i32, i32]
    lib.gqsa_upload.restype = C.c_int
    lib.gqsa_upload.argtypes = [vp]
    lib.gqsa_gemv.restype = C.c_int
    lib.gqsa_gemv.argtypes = [vp, vp, vp, i32, vp]
    lib.gqsa_gemv_static.restype = C.c_int
    lib.gqsa_gemv_static.argtypes = [vp, vp, vp, i32, vp]
    lib.gqsa_default_partition.restype = C.c_int
    lib.gqsa_default_partition.argtypes = [vp, i64, i64, i32, i32, C.POINTER(C.c_int32 * 6)]
    lib.gqsa_set_partition_rows.restype = C.c_int
    lib.gqsa_set_partition_rows.argtypes = [vp, i32, i32, i32, i32, i32]
    lib.gqsa_gemv_panels.restype = C.c_int
    lib.gqsa_gemv_panels.argtypes = [vp, vp, vp, i32, vp]
    lib.gqsa_gemv_multi.restype = C.c_int
    lib.gqsa_gemv_multi.argtypes = [C.POINTER(vp), i32, vp, C.POINTER(vp), i32, vp]
    lib.gqsa_info.restype = C.c_int
    lib.gqsa_info.argtypes = [vp, C.POINTER(_Info)]
    lib.gqsa_export.restype = C.c_int
    lib.gqsa_export.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.gqsa_export_device_blob.restype = C.c_int
    lib.gqsa_export_device_blob.argtypes = [vp, vp, C.c_size_t]
    lib.gqsa_free.restype = None
    lib.gqsa_free.argtypes = [vp]
    lib.gqsa_status_string.restype = C.c_char_p
    lib.gqsa_status_string.argtypes = [C.c_int]
    lib.gqsa_dense_f16_gemv.restype = C.c_int
    lib.gqsa_dense_f16_gemv.argtypes = [vp, vp, vp, i64, i64, i32, vp]
    lib.gqsa_stream_read.restype = C.c_int
    lib.gqsa_stream_read.argtypes = [vp, C.c_size_t, vp, vp]
    lib.gqsa_copy.restype = C.c_int
    lib.gqsa_copy.argtypes = [vp, vp, C.c_size_t, vp]
    lib.gqsa_launch_floor.restype = C.c_int
    lib.gqsa_launch_floor.argtypes = [i32, i32, vp, vp]
    heads = [vp, i64, i64]                               # an array [rows, heads, head_dim]: pointer, distances
    sequences = [vp, i32, vp, vp, i32]                   # pages, max_pages, lengths, row_starts, n_seqs
    lib.gqsa_qk_norm_rotate.restype = C.c_int
    lib.gqsa_qk_norm_rotate.argtypes = [*heads, i32, *heads, i32, i64, i32, vp, vp, C.c_float, vp, i64, i32, i32, vp, *heads, *heads, vp]
    lib.gqsa_cache_create.restype = C.c_int
    lib.gqsa_cache_create.argtypes = [i64, i32, i32, i32, C.POINTER(vp)]
    lib.gqsa_cache_info.restype = C.c_int
    lib.gqsa_cache_info.argtypes = [vp, C.POINTER(_CacheInfo)]
    lib.gqsa_cache_free.restype = None
    lib.gqsa_cache_free.argtypes = [vp]
    for name in ("gqsa_cache_append", "gqsa_cache_read"):
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = [vp, *heads, *heads, i64, *sequences, vp]
    lib.gqsa_cache_attend.restype = C.c_int
    lib.gqsa_cache_attend.argtypes = [vp, *heads, i32, i64, *sequences, C.c_float, *heads, vp]
    lib.gqsa_prompt_attend.restype = C.c_int
    lib.gqsa_prompt_attend.argtypes = [*heads, i32, i64, *heads, *heads, i32, i64, i32, vp, vp, i32, C.c_float, *heads, vp]
    lib.gqsa_cache_append_rotated.restype = C.c_int
    lib.gqsa_cache_append_rotated.argtypes = [vp, *heads, i32, *heads, *heads, i64, vp, vp, C.c_float, vp, i64, i32, i32, vp, *heads, *heads, *sequences, vp]
    lib.gqsa_cache_attend_tree.restype = C.c_int
    lib.gqsa_cache_attend_tree.argtypes = [vp, *heads, i32, i64, *sequences, vp, i32, C.c_float, *heads, vp]
    lib.gqsa_cache_keep.restype = C.c_int
    lib.gqsa_cache_keep.argtypes = [vp, i64, *sequences, vp, vp, vp]
    lib.gqsa_verify_create.restype = C.c_int
    lib.gqsa_verify_create.argtypes = [i32, i32, C.POINTER(vp)]
    lib.gqsa_verify_free.restype = None
    lib.gqsa_verify_free.argtypes = [vp]
    lib.gqsa_verify.restype = C.c_int
    lib.gqsa_verify.argtypes = [vp, vp, i64, vp, i64, i32, i64, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
    lib.gqsa_stream_read_workgroups.restype = C.c_int
    lib.gqsa_stream_read_workgroups.argtypes = []
    _LIB = lib
    return lib


def gqsa_status_string(status: int) -> str:
    return _lib().gqsa_status_string(int(status)).decode()


def _check(status: int, what: str):
    if status != 0:
        raise GqsaError(status, what)


class GqsaHandle:
    """Owns one gqsa_handle_t; freed on gqsa_free() or garbage collection."""

    def __init__(self, ptr: int):
        self.ptr = C.c_void_p(ptr)
        self.shape = None        # (N, K), which a handle keeps for life: asked for by the first call that needs it

    def __del__(self):
        try:
            gqsa_free(self)
        except Exception:
            pass


def _np_ptr(a):
    return None if a is None else C.c_void_p(a.ctypes.data)


def gqsa_pack(W: np.ndarray, G: int = 16, bits: int = 4, sparsity: float = 0.5) -> GqsaHandle:
    W = np.ascontiguousarray(W, dtype=np.float32)
    if W.ndim != 2:
        raise ValueError("W must be [N, K]")
    out = C.c_void_p()
    _check(_lib().gqsa_pack(_np_ptr(W), W.shape[0], W.shape[1], G, bits, float(sparsity),
                            C.byref(out)), "gqsa_pack")
    return GqsaHandle(out.value)


def gqsa_pack_hessian(W: np.ndarray, hinv_diag: np.ndarray, G: int = 16, bits: int = 4,
                      sparsity: float = 0.5) -> GqsaHandle:
    W = np.ascontiguousarray(W, dtype=np.float32)
    d = np.ascontiguousarray(hinv_diag, dtype=np.float32)
    if W.ndim != 2 or d.shape != (W.shape[1],):
        raise ValueError("W must be [N, K] and hinv_diag [K]")
    out = C.c_void_p()
    _check(_lib().gqsa_pack_hessian(_np_ptr(W), W.shape[0], W.shape[1], G, bits, float(sparsity),
                                    _np_ptr(d), C.byref(out)), "gqsa_pack_hessian")
    return GqsaHandle(out.value)


def gqsa_pack_device(W, G: int = 16, bits: int = 4, sparsity: float = 0.5, keep_per_row=None, hinv_diag=None,
                     stream=None) -> GqsaHandle:
    """gqsa_pack / gqsa_pack_rows / gqsa_pack_hessian on the GPU: W a float32 device tensor [N, K],
    hinv_diag a float32 device tensor [K] or None, keep_per_row a host int32 array [N] or None."""
    if W.dim() != 2:
        raise ValueError("W must be [N, K]")
    keep = None
    if keep_per_row is not None:
        keep = np.ascontiguousarray(keep_per_row, dtype=np.int32)
        if keep.shape != (W.shape[0],):
            raise ValueError("keep_per_row must be [N]")
    if hinv_diag is not None and tuple(hinv_diag.shape) != (W.shape[1],):
        raise ValueError("hinv_diag must be [K]")
    out = C.c_void_p()
    _check(_lib().gqsa_pack_device(_dev_ptr(W, "torch.float32", "W"), W.shape[0], W.shape[1], G, bits, float(sparsity),
                                   _np_ptr(keep) if keep is not None else None,
                                   _dev_ptr(hinv_diag, "torch.float32", "hinv_diag") if hinv_diag is not None else None,
                                   _stream_ptr(stream), C.byref(out)), "gqsa_pack_device")
    return GqsaHandle(out.value)


def gqsa_save(h: GqsaHandle, path: str) -> None:
    _check(_lib().gqsa_save(h.ptr, os.fsencode(path)), "gqsa_save")


def gqsa_load(path: str) -> GqsaHandle:
    out = C.c_void_p()
    _check(_lib().gqsa_load(os.fsencode(path), C.byref(out)), "gqsa_load")
    return GqsaHandle(out.value)


def gqsa_pack_rows(W: np.ndarray, keep_per_row: np.ndarray, G: int = 16, bits: int = 4) -> GqsaHandle:
    W = np.ascontiguousarray(W, dtype=np.float32)
    keep = np.ascontiguousarray(keep_per_row, dtype=np.int32)
    if W.ndim != 2 or keep.shape != (W.shape[0],):
        raise ValueError("W must be [N, K] and keep_per_row [N]")
    out = C.c_void_p()
    _check(_lib().gqsa_pack_rows(_np_ptr(W), W.shape[0], W.shape[1], G, bits, _np_ptr(keep),
                                 C.byref(out)), "gqsa_pack_rows")
    return GqsaHandle(out.value)


def gqsa_import(rowIndex, groups, values, scales_f16, zeros_f16, N: int, K: int, G: int = 16,
                bits: int = 4) -> GqsaHandle:
    ri = np.ascontiguousarray(rowIndex, dtype=np.int32)
    gr = np.ascontiguousarray(groups, dtype=np.int32)
    va = np.ascontiguousarray(values, dtype=np.uint8)
    sc = np.ascontiguousarray(scales_f16, dtype=np.uint16)
    ze = np.ascontiguousarray(zeros_f16, dtype=np.uint16)
    if ri.shape != (N + 1,):
        raise ValueError("rowIndex must have N+1 entries")
    nnz = int(ri[-1])
    if gr.size != nnz or sc.size != nnz or ze.size != nnz or va.size != nnz * G * bits // 8:
        raise ValueError("array sizes do not match rowIndex[N]")
    out = C.c_void_p()
    _check(_lib().gqsa_import(_np_ptr(ri), _np_ptr(gr), _np_ptr(va), _np_ptr(sc), _np_ptr(ze),
                              N, K, G, bits, C.byref(out)), "gqsa_import")
    return GqsaHandle(out.value)


def gqsa_set_partition(h: GqsaHandle, n_workgroups: int, waves_per_workgroup: int = 16) -> None:
    _check(_lib().gqsa_set_partition(h.ptr, int(n_workgroups), int(waves_per_workgroup)),
           "gqsa_set_partition")


def gqsa_set_partition_aligned(h: GqsaHandle, span_tiles: int, n_workgroups: int = 0,
                               waves_per_workgroup: int = 4) -> None:
    _check(_lib().gqsa_set_partition_aligned(h.ptr, int(span_tiles), int(n_workgroups), int(waves_per_workgroup)),
           "gqsa_set_partition_aligned")


def gqsa_set_partition_rows(h: GqsaHandle, tile_blocks: int, tile_lanes: int = 64, tiles_per_worker: int = 1,
                            n_workgroups: int = 0, waves_per_workgroup: int = 4) -> None:
    _check(_lib().gqsa_set_partition_rows(h.ptr, int(tile_blocks), int(tile_lanes), int(tiles_per_worker),
                                          int(n_workgroups), int(waves_per_workgroup)), "gqsa_set_partition_rows")


def gqsa_build_panels(h: GqsaHandle) -> None:
    _check(_lib().gqsa_build_panels(h.ptr), "gqsa_build_panels")


def gqsa_export_panel_blob(h: GqsaHandle) -> bytes:
    n = gqsa_info(h)["panel_bytes"]
    buf = np.zeros(max(n, 1), dtype=np.uint8)
    _check(_lib().gqsa_export_panel_blob(h.ptr, _np_ptr(buf), n), "gqsa_export_panel_blob")
    return buf[:n].tobytes()


def gqsa_upload(h: GqsaHandle) -> None:
    _check(_lib().gqsa_upload(h.ptr), "gqsa_upload")


def gqsa_info(h: GqsaHandle) -> dict:
    info = _Info()
    _check(_lib().gqsa_info(h.ptr, C.byref(info)), "gqsa_info")
    return {name: getattr(info, name) for name, _ in _Info._fields_ if not name.startswith("reserved")}


def gqsa_export(h: GqsaHandle) -> dict:
    info = gqsa_info(h)
    nnz = info["nnz_groups"]
    ri = np.empty(info["N"] + 1, dtype=np.int32)        # (written in full by the call)
    gr = np.empty(nnz, dtype=np.int32)
    va = np.empty(info["values_bytes"], dtype=np.uint8)
    sc = np.empty(nnz, dtype=np.uint16)
    ze = np.empty(nnz, dtype=np.uint16)
    _check(_lib().gqsa_export(h.ptr, _np_ptr(ri), _np_ptr(gr) if nnz else None,
                              _np_ptr(va) if nnz else None, _np_ptr(sc) if nnz else None,
                              _np_ptr(ze) if nnz else None), "gqsa_export")
    return {"rowIndex": ri, "groups": gr, "values": va, "scales": sc, "zeros": ze}


def gqsa_export_device_blob(h: GqsaHandle) -> bytes:
    n = gqsa_info(h)["device_bytes"]
    buf = np.zeros(n, dtype=np.uint8)
    _check(_lib().gqsa_export_device_blob(h.ptr, _np_ptr(buf), n), "gqsa_export_device_blob")
    return buf.tobytes()


def gqsa_free(h: GqsaHandle) -> None:
    if h.ptr is not None and h.ptr.value:
        _lib().gqsa_free(h.ptr)
        h.ptr = C.c_void_p()
        h.shape = None


# What a call of the GEMV passes through -- eagerly issued it is bound by this host work, not by its kernel
# (1024x4096 at one row: the kernel takes 2.6 us).  With the handle's whole record fetched and turned into
# a dict, a Stream object made and dtypes compared by name on every call, a call took 10.2 us; now 5.4 us.

def _shape(h: GqsaHandle):
    """(N, K) of a handle."""
    if h.shape is None:
        info = gqsa_info(h)
        h.shape = (info["N"], info["K"])
    return h.shape


_TORCH = None


def _torch():
    global _TORCH
    import torch
    _TORCH = torch
    return torch


def _stream_ptr(stream, device=None):
    """(device: the current one's number, where the caller has it)"""
    if stream is None:
        torch = _TORCH or _torch()
        try:                 # (not public names, but torch.cuda.current_stream() makes an object a call)
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice() if device is None else device)
        except AttributeError:
            return torch.cuda.current_stream().cuda_stream
    return C.c_void_p(getattr(stream, "cuda_stream", stream))      # (an integer; as an argument itself ctypes would take a text too)


_DTYPES = {}      # name -> torch.dtype


def _dev_ptr(t, dtype_name: str, what: str) -> int:
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous device tensor")
    dtype = _DTYPES.get(dtype_name) or _DTYPES.setdefault(dtype_name, getattr(torch, dtype_name.removeprefix("torch.")))
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype_name}")
    return t.data_ptr()


def gqsa_default_partition(rowIndex, K: int, G: int = 16, bits: int = 4):
    """(n_workgroups, waves_per_workgroup, span_tiles, tile_blocks, tile_lanes, span_per_worker) the library would
    choose for these row pointers."""
    ri = np.ascontiguousarray(rowIndex, dtype=np.int32)
    out = (C.c_int32 * 6)()
    _check(_lib().gqsa_default_partition(C.c_void_p(ri.ctypes.data), ri.size - 1, K, G, bits, C.byref(out)),
           "gqsa_default_partition")
    return tuple(int(v) for v in out)


def gqsa_partition(h: GqsaHandle):
    """The handle's partition, in the order of gqsa_default_partition."""
    info = gqsa_info(h)
    return tuple(info[k] for k in ("n_workgroups", "waves_per_workgroup", "span_tiles", "tile_blocks", "tile_lanes",
                                   "span_per_worker"))


def gqsa_gemv_static(h: GqsaHandle, x, y, stream=None):
    """gqsa_gemv without any allocation: y must be given, the handle must be on the device."""
    N, K = _shape(h)
    if x.dim() != 2 or x.shape[1] != K or tuple(y.shape) != (x.shape[0], N):
        raise ValueError("x must be [batch, K] and y [batch, N]")
    _check(_lib().gqsa_gemv_static(h.ptr, _dev_ptr(x, "torch.float16", "x"), _dev_ptr(y, "torch.float16", "y"),
                                   x.shape[0], _stream_ptr(stream)), "gqsa_gemv_static")
    return y


def gqsa_gemv(h: GqsaHandle, x, y=None, stream=None, panels: bool = False):
    """y[batch,N] (fp16, device) = W^ x[batch,K]; enqueues on `stream` (default: torch's current).
    panels=True: gqsa_gemv_panels (the second image, whatever the batch)."""
    N, K = _shape(h)
    if x.dim() == 1:
        x = x.unsqueeze(0)
    shape = x.shape
    batch = shape[0]
    if shape[1] != K:
        raise ValueError("x must be [batch, K]")
    if y is None:
        import torch
        y = torch.empty((batch, N), dtype=torch.float16, device=x.device)
    if y.shape != (batch, N):
        raise ValueError("y must be [batch, N]")
    fn = _lib().gqsa_gemv_panels if panels else _lib().gqsa_gemv
    _check(fn(h.ptr, _dev_ptr(x, "torch.float16", "x"), _dev_ptr(y, "torch.float16", "y"), batch,
              _stream_ptr(stream)), "gqsa_gemv_panels" if panels else "gqsa_gemv")
    return y


def gqsa_gemv_multi(hs, x, ys=None, stream=None):
    """ys[i][batch,N_i] = W^_i x for several matrices sharing x, in one launch."""
    shapes = [_shape(h) for h in hs]
    if x.dim() == 1:
        x = x.unsqueeze(0)
    batch, columns = x.shape[0], x.shape[1]
    for _, K in shapes:
        if columns != K:
            raise ValueError("x must be [batch, K] for every matrix")
    if ys is None:
        import torch
        ys = [torch.empty((batch, N), dtype=torch.float16, device=x.device) for N, _ in shapes]
    if len(ys) != len(hs):
        raise ValueError("ys[i] must be [batch, N_i]")
    for y, (N, _) in zip(ys, shapes):
        if y.shape != (batch, N):
            raise ValueError("ys[i] must be [batch, N_i]")
    n = len(hs)
    harr = (C.c_void_p * n)(*[h.ptr.value for h in hs])
    yarr = (C.c_void_p * n)(*[_dev_ptr(y, "torch.float16", "y") for y in ys])
    _check(_lib().gqsa_gemv_multi(harr, n, _dev_ptr(x, "torch.float16", "x"), yarr, batch,
                                  _stream_ptr(stream)), "gqsa_gemv_multi")
    return ys


def gqsa_dense_f16_gemv(W, x, y=None, stream=None):
    import torch
    if x.dim() == 1:
        x = x.unsqueeze(0)
    N, K = W.shape
    batch = x.shape[0]
    if y is None:
        y = torch.empty((batch, N), dtype=torch.float16, device=x.device)
    _check(_lib().gqsa_dense_f16_gemv(_dev_ptr(W, "torch.float16", "W"),
                                      _dev_ptr(x, "torch.float16", "x"),
                                      _dev_ptr(y, "torch.float16", "y"), N, K, batch,
                                      _stream_ptr(stream)), "gqsa_dense_f16_gemv")
    return y


def gqsa_stream_read_workgroups() -> int:
    return int(_lib().gqsa_stream_read_workgroups())


def gqsa_copy(dst, src, stream=None) -> None:
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("dst and src must have the same size")
    _check(_lib().gqsa_copy(C.c_void_p(dst.data_ptr()), C.c_void_p(src.data_ptr()), nbytes,
                            _stream_ptr(stream)), "gqsa_copy")


def gqsa_launch_floor(n_workgroups: int, lds_bytes: int, sink, stream=None) -> None:
    _check(_lib().gqsa_launch_floor(int(n_workgroups), int(lds_bytes), C.c_void_p(sink.data_ptr()),
                                    _stream_ptr(stream)), "gqsa_launch_floor")


def gqsa_stream_read(buf, sink, stream=None) -> None:
    nbytes = buf.numel() * buf.element_size()
    _check(_lib().gqsa_stream_read(C.c_void_p(buf.data_ptr()), nbytes, C.c_void_p(sink.data_ptr()),
                                   _stream_ptr(stream)), "gqsa_stream_read")


# ----------------------------------------------------------------------------- between the q/k/v and the o product

# These calls, too, are bound by their host work where the kernels take a few microseconds: an attribute of a tensor costs 0.05 to 0.08 us, so each
# is asked for once (norm and rotation of one row: 11.1 us a call with the helpers above, 8.5 with these; 4 of them are the C call).

_HALF = _INT = _FLOAT = None      # torch's dtypes, looked up by the first call


def _names():
    global _HALF, _INT, _FLOAT
    import torch
    _HALF, _INT, _FLOAT = torch.float16, torch.int32, torch.float32


def _device_of(t) -> int:
    """Number of the device of a call's first tensor, where the others have to lie too, and which has to be the current one: the launch goes there, and nothing else would
    notice.  -2 for what is on no device, or no tensor: nothing lies there."""
    try:
        device = t.get_device()
    except AttributeError:
        return -2
    if device < 0:
        return -2
    torch = _TORCH or _torch()
    try:                 # (as in _stream_ptr)
        current = torch._C._cuda_getDevice()
    except AttributeError:
        current = torch.cuda.current_device()
    if device != current:
        raise ValueError(f"tensors on device {device}, but the current device is {current}")
    return device


def _heads(t, what: str, device: int):
    """(pointer, distance between rows, distance between heads, rows, heads, head_dim) of a float16 tensor [rows, heads, head_dim] on that device
    whose heads are contiguous; the other two dimensions may be strided."""
    if _HALF is None:
        _names()
    try:
        rows, heads, dim = t.shape
        row, head, one = t.stride()
        if (one == 1 or rows == 0) and t.dtype is _HALF and t.get_device() == device:
            # (torch lets the distance of a dimension of size 1 be anything, and all of them without rows)
            return t.data_ptr(), row if rows > 1 else 0, head if heads > 1 else 0, rows, heads, dim
    except (AttributeError, TypeError, ValueError):
        pass
    raise ValueError(f"{what} must be a float16 device tensor [rows, heads, head_dim] with contiguous heads, on the device of the others")


def _heads_like(t, what: str, rows: int, heads: int, dim: int, device: int):
    """The first three of _heads, of an array of that shape."""
    at, row, head, t_rows, t_heads, t_dim = _heads(t, what, device)
    if t_rows != rows or t_heads != heads or t_dim != dim:
        raise ValueError(f"{what} must be [{rows}, {heads}, {dim}]")
    return at, row, head


def _flat(t, dtype, what: str, device: int):
    """(pointer, shape) of a contiguous tensor of that dtype on that device."""
    if t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} device tensor, on the device of the others")
    return t.data_ptr(), t.shape


def _like(x, stream):
    """A new array of x's shape, for work on `stream` (memory is handed out, and taken back, in the order of a stream's work)."""
    import torch
    if stream is None:
        return torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream))
    with torch.cuda.stream(stream):
        return torch.empty(x.shape, dtype=x.dtype, device=x.device)


def _rotation(table, positions, rows: int, device: int, needs_positions: bool):
    """(table's pointer, its positions, rotary_dim, pointer of positions) of a rotation, or of none."""
    if table is None:
        return None, 0, 0, None
    at, shape = _flat(table, _FLOAT, "table", device)
    n_positions, half, two = shape if len(shape) == 3 else (0, 0, 0)
    if two != 2 or (positions is None and needs_positions):
        raise ValueError("table must be [n_positions, rotary_dim / 2, 2] and positions [rows]")
    positions_at = None
    if positions is not None:
        positions_at, shape = _flat(positions, _INT, "positions", device)
        if len(shape) != 1 or shape[0] != rows:
            raise ValueError("positions must be [rows]")
    return at, n_positions, 2 * half, positions_at


def _norm_weight(w, dim: int, device: int):
    at, shape = _flat(w, _HALF, "norm weights", device)
    if len(shape) != 1 or shape[0] != dim:
        raise ValueError("norm weights must be [head_dim]")
    return at


def gqsa_qk_norm_rotate(q, k, positions, table, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                        q_out=None, k_out=None, stream=None):
    """Norms of queries [rows, q_heads, head_dim] and keys [rows, k_heads, head_dim] per head (weights float16 [head_dim] or None: no norm)
    and their rotation: positions int32 [rows], table float32 [n_positions, rotary_dim / 2, 2] (cosine, sine), or both None: no
    rotation.  k None: queries only.  q_out = q, k_out = k: in place.  Returns (q_out, k_out)."""
    device = _device_of(q)
    q_at, q_row, q_head, rows, q_heads, dim = _heads(q, "q", device)
    if q_out is None:
        q_out = _like(q, stream)
    qo_at, qo_row, qo_head = _heads_like(q_out, "q_out", rows, q_heads, dim, device)
    k_at, k_row, k_head, k_heads, ko_at, ko_row, ko_head = None, 0, 0, 0, None, 0, 0
    if k is not None:
        k_at, k_row, k_head, k_rows, k_heads, k_dim = _heads(k, "k", device)
        if k_out is None:
            k_out = _like(k, stream)
        if k_rows != rows or k_dim != dim:
            raise ValueError("k must be [rows, k_heads, head_dim]")
        ko_at, ko_row, ko_head = _heads_like(k_out, "k_out", rows, k_heads, dim, device)
    table_at, n_positions, rotary, positions_at = _rotation(table, positions, rows, device, True)
    q_weight_at = None if q_weight is None else _norm_weight(q_weight, dim, device)
    k_weight_at = None if k_weight is None else _norm_weight(k_weight, dim, device)
    _check(_lib().gqsa_qk_norm_rotate(
        q_at, q_row, q_head, q_heads, k_at, k_row, k_head, k_heads, rows, dim, q_weight_at, k_weight_at, eps, table_at,
        n_positions, rotary, interleaved, positions_at, qo_at, qo_row, qo_head, ko_at, ko_row, ko_head, _stream_ptr(stream, device)), "gqsa_qk_norm_rotate")
    return q_out, k_out


class GqsaCache:
    """Owns one gqsa_cache_t; freed on gqsa_cache_free() or garbage collection."""

    def __init__(self, ptr: int, kv_heads: int, head_dim: int):
        self.ptr = C.c_void_p(ptr)
        self.kv_heads, self.head_dim = kv_heads, head_dim

    def __del__(self):
        try:
            gqsa_cache_free(self)
        except Exception:
            pass


def gqsa_cache_create(n_pages: int, page_tokens: int, kv_heads: int, head_dim: int) -> GqsaCache:
    out = C.c_void_p()
    _check(_lib().gqsa_cache_create(n_pages, page_tokens, kv_heads, head_dim, C.byref(out)), "gqsa_cache_create")
    return GqsaCache(out.value, kv_heads, head_dim)


def gqsa_cache_info(c: GqsaCache) -> dict:
    info = _CacheInfo()
    _check(_lib().gqsa_cache_info(c.ptr, C.byref(info)), "gqsa_cache_info")
    return {name: getattr(info, name) for name, _ in _CacheInfo._fields_}


def gqsa_cache_free(c: GqsaCache) -> None:
    """The pages must not be in use any more (as with gqsa_free, work that reads them has to be over)."""
    if c.ptr is not None and c.ptr.value:
        _lib().gqsa_cache_free(c.ptr)
        c.ptr = C.c_void_p()


def _sequences(pages, lengths, row_starts, device: int):
    """pages int32 [n_seqs, max_pages], lengths int32 [n_seqs], row_starts int32 [n_seqs + 1] or None (a row per sequence)."""
    pages_at, shape = _flat(pages, _INT, "pages", device)
    lengths_at, n_lengths = _flat(lengths, _INT, "lengths", device)
    if len(shape) != 2 or len(n_lengths) != 1 or n_lengths[0] != shape[0]:
        raise ValueError("pages must be [n_seqs, max_pages] and lengths [n_seqs]")
    n, max_pages = shape
    starts_at = None
    if row_starts is not None:
        starts_at, shape = _flat(row_starts, _INT, "row_starts", device)
        if len(shape) != 1 or shape[0] != n + 1:
            raise ValueError("row_starts must be [n_seqs + 1]")
    return pages_at, max_pages, lengths_at, starts_at, n


def _cache_rows(c: GqsaCache, k, v, k_what: str, v_what: str, device: int):
    """Pointers and distances of keys and values of the cache's heads, and their rows."""
    k_at, k_row, k_head, rows, heads, dim = _heads(k, k_what, device)
    if heads != c.kv_heads or dim != c.head_dim:
        raise ValueError("keys and values must be [rows, kv_heads, head_dim] of the cache")
    v_at, v_row, v_head = _heads_like(v, v_what, rows, heads, dim, device)
    return k_at, k_row, k_head, v_at, v_row, v_head, rows


def gqsa_cache_append(c: GqsaCache, k, v, pages, lengths, row_starts=None, stream=None) -> None:
    """New keys and values [rows, kv_heads, head_dim] become the last tokens of their sequences; lengths counts them in."""
    device = _device_of(k)
    _check(_lib().gqsa_cache_append(c.ptr, *_cache_rows(c, k, v, "k", "v", device), *_sequences(pages, lengths, row_starts, device),
                                    _stream_ptr(stream, device)), "gqsa_cache_append")


def gqsa_cache_append_rotated(c: GqsaCache, q, k, v, positions, table, pages, lengths, row_starts=None, q_weight=None, k_weight=None, eps: float = 1e-6,
                              interleaved: bool = False, q_out=None, k_out=None, stream=None):
    """gqsa_qk_norm_rotate of queries [rows, q_heads, head_dim] (or None) and keys and gqsa_cache_append of keys and values in one launch.  positions None: a
    token's place in its sequence; table None: no rotation; k_out None: the rotated keys go to the cache only.  Returns (q_out, k_out)."""
    device = _device_of(k)
    k_at, k_row, k_head, v_at, v_row, v_head, rows = _cache_rows(c, k, v, "k", "v", device)
    dim = c.head_dim
    q_at, q_row, q_head, q_heads, qo_at, qo_row, qo_head = None, 0, 0, 0, None, 0, 0
    if q is not None:
        q_at, q_row, q_head, q_rows, q_heads, q_dim = _heads(q, "q", device)
        if q_rows != rows or q_dim != dim:
            raise ValueError("q must be [rows, q_heads, head_dim] of the cache")
        if q_out is None:
            q_out = _like(q, stream)
        qo_at, qo_row, qo_head = _heads_like(q_out, "q_out", rows, q_heads, dim, device)
    ko_at, ko_row, ko_head = (None, 0, 0) if k_out is None else _heads_like(k_out, "k_out", rows, c.kv_heads, dim, device)
    table_at, n_positions, rotary, positions_at = _rotation(table, positions, rows, device, False)
    q_weight_at = None if q_weight is None else _norm_weight(q_weight, dim, device)
    k_weight_at = None if k_weight is None else _norm_weight(k_weight, dim, device)
    _check(_lib().gqsa_cache_append_rotated(
        c.ptr, q_at, q_row, q_head, q_heads, k_at, k_row, k_head, v_at, v_row, v_head, rows, q_weight_at, k_weight_at, eps, table_at, n_positions, rotary,
        interleaved, positions_at, qo_at, qo_row, qo_head, ko_at, ko_row, ko_head, *_sequences(pages, lengths, row_starts, device),
        _stream_ptr(stream, device)), "gqsa_cache_append_rotated")
    return q_out, k_out


def gqsa_cache_keep(c: GqsaCache, pages, lengths, row_starts, path, accepted, stream=None) -> None:
    """Of the newest rows of each sequence, those of path (int32 [rows], as gqsa_verify gives it) become the first accepted + 1 (accepted int32 [n_seqs])."""
    device = _device_of(path)
    if _INT is None:
        _names()
    path_at, path_shape = _flat(path, _INT, "path", device)
    where = _sequences(pages, lengths, row_starts, device)
    accepted_at, accepted_shape = _flat(accepted, _INT, "accepted", device)
    if len(path_shape) != 1 or len(accepted_shape) != 1 or accepted_shape[0] != where[4]:
        raise ValueError("path must be [rows] and accepted [n_seqs]")
    _check(_lib().gqsa_cache_keep(c.ptr, path_shape[0], *where, path_at, accepted_at, _stream_ptr(stream, device)), "gqsa_cache_keep")


def gqsa_cache_read(c: GqsaCache, pages, lengths, row_starts, k_out, v_out, stream=None):
    """The values of the last tokens of each sequence, as many as it has rows in k_out and v_out [rows, kv_heads, head_dim]."""
    device = _device_of(k_out)
    _check(_lib().gqsa_cache_read(c.ptr, *_cache_rows(c, k_out, v_out, "k_out", "v_out", device), *_sequences(pages, lengths, row_starts, device),
                                  _stream_ptr(stream, device)), "gqsa_cache_read")
    return k_out, v_out


def gqsa_cache_attend(c: GqsaCache, q, pages, lengths, row_starts=None, scale: float = None, out=None, stream=None):
    """Attention of the newest rows q [rows, q_heads, head_dim] of each sequence over its cache; scale None: head_dim ** -0.5."""
    device = _device_of(q)
    q_at, q_row, q_head, rows, heads, dim = _heads(q, "q", device)
    if dim != c.head_dim:
        raise ValueError("q must be [rows, q_heads, head_dim] of the cache")
    if out is None:
        out = _like(q, stream)
    out_at, out_row, out_head = _heads_like(out, "out", rows, heads, dim, device)
    _check(_lib().gqsa_cache_attend(c.ptr, q_at, q_row, q_head, heads, rows, *_sequences(pages, lengths, row_starts, device),
                                    dim ** -0.5 if scale is None else scale, out_at, out_row, out_head, _stream_ptr(stream, device)),
           "gqsa_cache_attend")
    return out


def gqsa_cache_attend_tree(c: GqsaCache, q, pages, lengths, row_starts, masks, scale: float = None, out=None, stream=None):
    """gqsa_cache_attend where a row sees the tokens before all rows of its sequence, and of these rows those that its mask names: masks int32
    [rows, mask_words], bit j % 32 of word j / 32 for row j of the sequence."""
    device = _device_of(q)
    q_at, q_row, q_head, rows, heads, dim = _heads(q, "q", device)
    if dim != c.head_dim:
        raise ValueError("q must be [rows, q_heads, head_dim] of the cache")
    masks_at, shape = _flat(masks, _INT, "masks", device)
    if len(shape) != 2 or shape[0] != rows:
        raise ValueError("masks must be [rows, mask_words]")
    if out is None:
        out = _like(q, stream)
    out_at, out_row, out_head = _heads_like(out, "out", rows, heads, dim, device)
    _check(_lib().gqsa_cache_attend_tree(c.ptr, q_at, q_row, q_head, heads, rows, *_sequences(pages, lengths, row_starts, device), masks_at, shape[1],
                                         dim ** -0.5 if scale is None else scale, out_at, out_row, out_head, _stream_ptr(stream, device)),
           "gqsa_cache_attend_tree")
    return out


class GqsaVerifier:
    """Owns one gqsa_verifier_t; freed on gqsa_verify_free() or garbage collection."""

    def __init__(self, ptr: int):
        self.ptr = C.c_void_p(ptr)

    def __del__(self):
        try:
            gqsa_verify_free(self)
        except Exception:
            pass


def gqsa_verify_create(max_seqs: int, max_vocab: int) -> GqsaVerifier:
    out = C.c_void_p()
    _check(_lib().gqsa_verify_create(max_seqs, max_vocab, C.byref(out)), "gqsa_verify_create")
    return GqsaVerifier(out.value)


def gqsa_verify_free(v: GqsaVerifier) -> None:
    """The workspace must not be in use any more (as with gqsa_free, calls that use it have to be over)."""
    if v.ptr is not None and v.ptr.value:
        _lib().gqsa_verify_free(v.ptr)
        v.ptr = C.c_void_p()


def _probabilities(t, what: str, device: int):
    """(pointer, distance between rows, rows, vocabulary) of a float32 tensor [rows, vocabulary] on that device with contiguous rows."""
    try:
        rows, vocab = t.shape
        row, one = t.stride()
        if (one == 1 or vocab == 1 or rows == 0) and t.dtype is _FLOAT and t.get_device() == device:
            return t.data_ptr(), row if rows > 1 else vocab, rows, vocab
    except (AttributeError, TypeError, ValueError):
        pass
    raise ValueError(f"{what} must be a float32 device tensor [rows, vocabulary] with contiguous rows, on the device of the others")


def _numbers(t, dtype, what: str, n: int, device: int):
    at, shape = _flat(t, dtype, what, device)
    if len(shape) != 1 or shape[0] != n:
        raise ValueError(f"{what} must be [{n}]")
    return at


def gqsa_verify(v: GqsaVerifier, target, tokens, uniforms, finals, row_starts=None, parents=None, draft=None, path=None, out=None, accepted=None, stream=None):
    """Which drafted tokens (int32 [rows], row 0 of a sequence the last certain one) the target's probabilities (float32 [rows, vocabulary]) let stand, and
    one more token behind them.  parents int32 [rows] (None: chains), draft float32 [rows, vocabulary] what chains were drawn from (or None), uniforms
    float32 [rows] and finals float32 [n_seqs] from [0, 1).  Returns (path, out, accepted), int32 [rows], [rows], [n_seqs]."""
    device = _device_of(target)
    if _INT is None:
        _names()
    target_at, target_row, rows, vocab = _probabilities(target, "target", device)
    draft_at, draft_row = None, 0
    if draft is not None:
        draft_at, draft_row, d_rows, d_vocab = _probabilities(draft, "draft", device)
        if d_rows != rows or d_vocab != vocab:
            raise ValueError("draft must be like target")
    tokens_at = _numbers(tokens, _INT, "tokens", rows, device)
    uniforms_at = _numbers(uniforms, _FLOAT, "uniforms", rows, device)
    finals_at, shape = _flat(finals, _FLOAT, "finals", device)
    n_seqs = shape[0] if len(shape) == 1 else -1
    parents_at = None if parents is None else _numbers(parents, _INT, "parents", rows, device)
    starts_at = None if row_starts is None else _numbers(row_starts, _INT, "row_starts", n_seqs + 1, device)
    path = _like(tokens, stream) if path is None else path
    out = _like(tokens, stream) if out is None else out
    accepted = _like(finals, stream).view(_INT) if accepted is None else accepted
    _check(_lib().gqsa_verify(v.ptr, target_at, target_row, draft_at, draft_row, vocab, rows, tokens_at, parents_at, uniforms_at, finals_at, starts_at, n_seqs,
                              _numbers(path, _INT, "path", rows, device), _numbers(out, _INT, "out", rows, device),
                              _numbers(accepted, _INT, "accepted", n_seqs, device), _stream_ptr(stream, device)), "gqsa_verify")
    return path, out, accepted


def gqsa_prompt_attend(q, k, v, q_starts, k_starts, scale: float = None, out=None, stream=None):
    """Causal attention over packed prompts: q [q_rows, q_heads, head_dim], k and v [k_rows, kv_heads, head_dim], starts int32
    [n_seqs + 1] of each sequence's rows; scale None: head_dim ** -0.5."""
    device = _device_of(q)
    q_at, q_row, q_head, rows, heads, dim = _heads(q, "q", device)
    k_at, k_row, k_head, k_rows, kv_heads, k_dim = _heads(k, "k", device)
    if k_dim != dim:
        raise ValueError("k and v must be [k_rows, kv_heads, head_dim]")
    v_at, v_row, v_head = _heads_like(v, "v", k_rows, kv_heads, dim, device)
    q_starts_at, n_starts = _flat(q_starts, _INT, "q_starts", device)
    k_starts_at, shape = _flat(k_starts, _INT, "k_starts", device)
    if len(n_starts) != 1 or shape != n_starts:
        raise ValueError("q_starts and k_starts must be [n_seqs + 1]")
    if out is None:
        out = _like(q, stream)
    out_at, out_row, out_head = _heads_like(out, "out", rows, heads, dim, device)
    _check(_lib().gqsa_prompt_attend(q_at, q_row, q_head, heads, rows, k_at, k_row, k_head, v_at, v_row, v_head, kv_heads, k_rows, dim,
                                     q_starts_at, k_starts_at, n_starts[0] - 1, dim ** -0.5 if scale is None else scale,
                                     out_at, out_row, out_head, _stream_ptr(stream, device)), "gqsa_prompt_attend")
    return out
