"""ctypes binding of libmmvseg.so: argument marshalling only.

Every function here has the name of the C entry point it calls
(include/mmvseg.h) and takes torch tensors that live on the GPU; torch only
provides the device memory and the HIP stream.  No step of the computation
runs in Python or in torch, and there is no fallback: if the library has not
been built, loading raises.
"""
from __future__ import annotations

import ctypes
import importlib
import math
import os
from typing import NamedTuple

import torch  # imported before the library so that both share one HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmmvseg.so")
MARSHAL_PATH = os.path.join(_HERE, "_marshal.so")

MMV_OK = 0
MMV_F32_F32, MMV_F16_F32, MMV_BF16_F32, MMV_I8_I32, MMV_U8_XOR = 0, 1, 2, 3, 4
MMV_FLAGS_U8, MMV_FLAGS_PACKED32 = 0, 1
MMV_VARIANT_MFMA, MMV_VARIANT_SHUFFLE = 0, 1
MMV_OP_SEGSCAN, MMV_OP_SEGSUM, MMV_OP_SPMV_COO = 0, 1, 2
MMV_OP_SCAN, MMV_OP_COMPRESS, MMV_OP_SEGSUM_SCD, MMV_OP_SEGSCAN_SSCR, MMV_OP_SPMV_CSR = 3, 4, 5, 6, 7
MMV_ELEM_I32, MMV_ELEM_F32 = 0, 1
MMV_TYPE_F16, MMV_TYPE_BF16, MMV_TYPE_E4M3, MMV_TYPE_I8 = 1, 2, 5, 6

EXPORTS = [
    "mmv_workspace_bytes", "mmv_segscan", "mmv_segsum", "mmv_spmv_coo", "mmv_workspace_status",
    "mmv_stream_copy", "mmv_gather_reference", "mmv_status_string", "mmv_tile_elems", "mmv_set_kernel_events",
    "mmv_spmv_csr_workspace_bytes", "mmv_spmv_csr", "mmv_scan", "mmv_compress", "mmv_diff", "mmv_revert",
    "mmv_segsum_scd", "mmv_segscan_sscr", "mmv_segscan_static",
    "mmv_spmv_coo_prepare", "mmv_spmv_coo_run", "mmv_spmv_csr_prepare", "mmv_spmv_csr_run",
    "mmv_page_tables_workspace_bytes", "mmv_page_tables", "mmv_cache_append", "mmv_paged_attention_workspace_bytes", "mmv_paged_attention",
    "mmv_decay_attention_workspace_bytes", "mmv_decay_attention", "mmv_decay_step",
    "mmv_block_append", "mmv_block_read", "mmv_block_attention", "mmv_delta_attention_workspace_bytes", "mmv_delta_attention", "mmv_delta_step",
]
STATIC_SCRATCH_BYTES = 1 << 20   # MMV_STATIC_SCRATCH_BYTES

_DTYPES = {torch.float32: MMV_F32_F32, torch.float16: MMV_F16_F32, torch.bfloat16: MMV_BF16_F32,
           torch.int8: MMV_I8_I32, torch.uint8: MMV_U8_XOR}   # uint8 values: bytes under bit-wise exclusive or
_OUT_DTYPE = {MMV_F32_F32: torch.float32, MMV_F16_F32: torch.float32, MMV_BF16_F32: torch.float32,
              MMV_I8_I32: torch.int32, MMV_U8_XOR: torch.int32}
_VARIANTS = {"mfma": MMV_VARIANT_MFMA, "shuffle": MMV_VARIANT_SHUFFLE}

_lib = None
# The calls that programs make over and over go through csrc/marshal.cpp where all their arguments are given: it does what the
# lines below each of them do, and answers None where they have to (arguments left out, errors).  Where it is not built, or for another
# torch, they do it all.  Host time of a call on 3000 values, us:
# segmented scan 4.7 -> 3.3, segmented sum 5.1 -> 3.5, scan 4.3 -> 3.5, COMPRESS 5.1 -> 3.6 (the launch itself takes 2.9).
_marshal = None


class MmvError(RuntimeError):
    pass


def load() -> ctypes.CDLL:
    """Loads libmmvseg.so; raises if it has not been built (there is no fallback path)."""
    global _lib, _marshal
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise MmvError("libmmvseg.so is not built: run `python -m paper_2506_23906_amd.build` "
                       "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(LIB_PATH)
    vp, u64, sz, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int
    lib.mmv_workspace_bytes.argtypes = [i32, i32, i32, u64]
    lib.mmv_workspace_bytes.restype = sz
    lib.mmv_segscan.argtypes = [vp, vp, u64, vp, i32, i32, i32, vp, sz, vp]
    lib.mmv_segscan.restype = i32
    lib.mmv_segscan_static.argtypes = [vp, vp, u64, vp, i32, i32, i32, vp]
    lib.mmv_segscan_static.restype = i32
    lib.mmv_segsum.argtypes = [vp, vp, u64, vp, u64, vp, i32, i32, i32, vp, sz, vp]
    lib.mmv_segsum.restype = i32
    lib.mmv_spmv_coo.argtypes = [u64, u64, u64, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    lib.mmv_spmv_coo.restype = i32
    lib.mmv_workspace_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.mmv_workspace_status.restype = i32
    lib.mmv_stream_copy.argtypes = [vp, sz, vp, sz, vp]
    lib.mmv_stream_copy.restype = i32
    lib.mmv_gather_reference.argtypes = [u64, vp, vp, u64, vp, vp, vp]
    lib.mmv_gather_reference.restype = i32
    lib.mmv_status_string.argtypes = [i32]
    lib.mmv_status_string.restype = ctypes.c_char_p
    lib.mmv_set_kernel_events.argtypes = [vp, vp]
    lib.mmv_set_kernel_events.restype = i32
    lib.mmv_tile_elems.argtypes = [i32, i32, u64]
    lib.mmv_tile_elems.restype = ctypes.c_uint32
    lib.mmv_spmv_csr_workspace_bytes.argtypes = [u64, u64]
    lib.mmv_spmv_csr_workspace_bytes.restype = sz
    lib.mmv_spmv_csr.argtypes = [u64, u64, u64, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    lib.mmv_spmv_csr.restype = i32
    for name in ("mmv_spmv_coo_prepare", "mmv_spmv_csr_prepare"):
        getattr(lib, name).argtypes = [u64, u64, u64, vp, vp, vp, sz, vp]
        getattr(lib, name).restype = i32
    for name in ("mmv_spmv_coo_run", "mmv_spmv_csr_run"):
        getattr(lib, name).argtypes = [u64, u64, u64, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        getattr(lib, name).restype = i32
    lib.mmv_scan.argtypes = [vp, u64, vp, i32, i32, vp, sz, vp]
    lib.mmv_scan.restype = i32
    lib.mmv_compress.argtypes = [vp, vp, u64, vp, u64, vp, i32, vp, sz, vp]
    lib.mmv_compress.restype = i32
    lib.mmv_diff.argtypes = [vp, u64, vp, i32, vp]
    lib.mmv_diff.restype = i32
    lib.mmv_revert.argtypes = [vp, vp, vp, u64, u64, vp, i32, vp]
    lib.mmv_revert.restype = i32
    lib.mmv_segsum_scd.argtypes = [vp, vp, u64, vp, u64, vp, i32, i32, i32, vp, sz, vp]
    lib.mmv_segsum_scd.restype = i32
    lib.mmv_segscan_sscr.argtypes = [vp, vp, u64, vp, i32, i32, i32, vp, sz, vp]
    lib.mmv_segscan_sscr.restype = i32
    u32, f32 = ctypes.c_uint32, ctypes.c_float
    lib.mmv_page_tables_workspace_bytes.argtypes = [u64]
    lib.mmv_page_tables_workspace_bytes.restype = sz
    lib.mmv_page_tables.argtypes = [u64, vp, vp, vp, u64, vp, u64, u64, u32, u64, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.mmv_page_tables.restype = i32
    lib.mmv_cache_append.argtypes = [u64, vp, u64, vp, u64, i32, vp, vp, vp]
    lib.mmv_cache_append.restype = i32
    lib.mmv_paged_attention_workspace_bytes.argtypes = [u64, u32, u32, u32, u64]
    lib.mmv_paged_attention_workspace_bytes.restype = sz
    lib.mmv_paged_attention.argtypes = [u64, u32, vp, u64, i32, vp, vp, u64, u64, vp, f32, u32, vp, vp, vp, sz, vp]
    lib.mmv_paged_attention.restype = i32
    lib.mmv_decay_attention_workspace_bytes.argtypes = [u64, u64, u32, u32, u32]
    lib.mmv_decay_attention_workspace_bytes.restype = sz
    lib.mmv_decay_attention.argtypes = [u64, u64, u32, u32, u32, u32, vp, u64, vp, u64, vp, u64, i32, vp, vp, f32, vp, vp, u64, vp, vp, vp, sz, vp]
    lib.mmv_decay_attention.restype = i32
    lib.mmv_decay_step.argtypes = [u64, u32, u32, u32, u32, vp, u64, vp, u64, vp, u64, i32, vp, f32, vp, vp, u64, vp, vp, vp]
    lib.mmv_decay_step.restype = i32
    lib.mmv_block_append.argtypes = [u64, vp, u64, vp, u64, i32, vp, vp, vp]
    lib.mmv_block_append.restype = i32
    lib.mmv_block_read.argtypes = [u64, u64, vp, vp, vp, u64, u64, vp, i32, vp, u64, vp, u64, vp]
    lib.mmv_block_read.restype = i32
    lib.mmv_block_attention.argtypes = lib.mmv_paged_attention.argtypes
    lib.mmv_block_attention.restype = i32
    lib.mmv_delta_attention_workspace_bytes.argtypes = [u64, u64, u32, u32, u32]
    lib.mmv_delta_attention_workspace_bytes.restype = sz
    lib.mmv_delta_attention.argtypes = [u64, u64, u32, u32, u32, u32, vp, u64, vp, u64, vp, u64, i32, vp, vp, vp, f32, vp, vp, u64, vp, vp, vp, sz, vp]
    lib.mmv_delta_attention.restype = i32
    lib.mmv_delta_step.argtypes = [u64, u32, u32, u32, u32, vp, u64, vp, u64, vp, u64, i32, vp, vp, f32, vp, vp, u64, vp, vp, vp]
    lib.mmv_delta_step.restype = i32
    try:
        marshal = importlib.import_module(__package__ + "._marshal")
    except ImportError:
        marshal = None
    if getattr(marshal, "torch_version", None) != torch.__version__:
        marshal = None
    if marshal is not None:
        marshal.bind(*(ctypes.cast(getattr(lib, name), vp).value for name in
                       ("mmv_segscan", "mmv_segsum", "mmv_scan", "mmv_compress", "mmv_spmv_coo", "mmv_spmv_csr", "mmv_spmv_coo_run", "mmv_spmv_csr_run")))
        marshal.bind_serving(*(ctypes.cast(getattr(lib, name), vp).value for name in
                               ("mmv_page_tables", "mmv_cache_append", "mmv_paged_attention", "mmv_decay_attention", "mmv_decay_step",
                                "mmv_block_append", "mmv_block_read", "mmv_block_attention", "mmv_delta_attention", "mmv_delta_step")))
    _lib, _marshal = lib, marshal
    return lib


def _check(status: int, what: str) -> None:
    if status != MMV_OK:
        raise MmvError("%s failed: %s (status %d)" % (what, load().mmv_status_string(status).decode(), status))


# The handle of torch.cuda.current_stream() without the Stream object around it: that takes 2.7 us to make, a quarter of a
# small call (the two queries 0.2 us).  None where this torch does not have them.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device_index = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _device_index is not None:
            return _raw_stream(_device_index())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _dev(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda or not t.is_contiguous():
        raise MmvError("%s must be a contiguous tensor in GPU memory" % name)
    return t.data_ptr()


def _flag_fmt(flags: torch.Tensor) -> int:
    if flags.dtype == torch.uint8:
        return MMV_FLAGS_U8
    if flags.dtype == torch.int32:
        return MMV_FLAGS_PACKED32
    raise MmvError("flags must be uint8 (one byte per element) or int32 (bit-packed words)")


def mmv_tile_elems(op: int = MMV_OP_SEGSCAN, dt: int = MMV_I8_I32, n: int = 1 << 40) -> int:
    """Elements per workgroup tile; the default arguments give the largest tile there is."""
    return int(load().mmv_tile_elems(op, dt, n))


def mmv_workspace_bytes(op: int, dt: int, ff: int, n: int) -> int:
    return int(load().mmv_workspace_bytes(op, dt, ff, n))


def workspace(nbytes: int, device=None) -> torch.Tensor:
    """Scratch of at least `nbytes` bytes (torch allocations are 256-byte aligned)."""
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device=device or "cuda")


def new_workspace(op: int, dt: int, ff: int, n: int, device=None) -> torch.Tensor:
    return workspace(mmv_workspace_bytes(op, dt, ff, n), device)


def mmv_segscan(x: torch.Tensor, flags: torch.Tensor, n: int | None = None, z: torch.Tensor | None = None,
                variant: str = "mfma", ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Segmented inclusive scan of x under segment-start flags; returns z (fp32 or int32)."""
    if _marshal is not None:
        st = _marshal.segscan(x, flags, n, z, variant, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_segscan")
            return z
    lib = load()
    n = x.numel() if n is None else n
    dt, ff = _DTYPES[x.dtype], _flag_fmt(flags)
    if z is None:
        z = torch.empty(n, dtype=_OUT_DTYPE[dt], device=x.device)
    if ws is None:
        ws = new_workspace(MMV_OP_SEGSCAN, dt, ff, n, x.device)
    st = lib.mmv_segscan(_dev(x, "x"), _dev(flags, "flags"), n, _dev(z, "z"), dt, ff, _VARIANTS[variant],
                         _dev(ws, "ws"), ws.numel(), _stream_ptr(stream))
    _check(st, "mmv_segscan")
    return z


def mmv_segscan_static(x: torch.Tensor, flags: torch.Tensor, z: torch.Tensor, n: int | None = None,
                       variant: str = "mfma", stream=None) -> torch.Tensor:
    """mmv_segscan on the library's built-in scratch array: the caller passes inputs and the output, nothing
    is allocated (neither here nor in the library)."""
    n = x.numel() if n is None else n
    st = load().mmv_segscan_static(_dev(x, "x"), _dev(flags, "flags"), n, _dev(z, "z"), _DTYPES[x.dtype],
                                   _flag_fmt(flags), _VARIANTS[variant], _stream_ptr(stream))
    _check(st, "mmv_segscan_static")
    return z


def mmv_segsum(x: torch.Tensor, flags: torch.Tensor, n: int | None = None, out: torch.Tensor | None = None,
               nseg: torch.Tensor | None = None, variant: str = "mfma", ws: torch.Tensor | None = None,
               stream=None):
    """Segmented sum; returns (out, nseg) where nseg is a one-element int64 device tensor."""
    if _marshal is not None:
        st = _marshal.segsum(x, flags, n, out, nseg, variant, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_segsum")
            return out, nseg
    lib = load()
    n = x.numel() if n is None else n
    dt, ff = _DTYPES[x.dtype], _flag_fmt(flags)
    if out is None:
        out = torch.empty(max(n, 1), dtype=_OUT_DTYPE[dt], device=x.device)
    if nseg is None:
        nseg = torch.empty(1, dtype=torch.int64, device=x.device)
    if ws is None:
        ws = new_workspace(MMV_OP_SEGSUM, dt, ff, n, x.device)
    st = lib.mmv_segsum(_dev(x, "x"), _dev(flags, "flags"), n, _dev(out, "out"), out.numel(), _dev(nseg, "nseg"),
                        dt, ff, _VARIANTS[variant], _dev(ws, "ws"), ws.numel(), _stream_ptr(stream))
    _check(st, "mmv_segsum")
    return out, nseg


def mmv_spmv_coo(n_rows: int, n_cols: int, row: torch.Tensor, col: torch.Tensor, val: torch.Tensor,
                 x: torch.Tensor, y: torch.Tensor | None = None, variant: str = "mfma",
                 ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y = A x for a row-sorted COO matrix (int32 indices, fp32 values)."""
    if _marshal is not None:
        st = _marshal.spmv_coo(n_rows, n_cols, None, row, col, val, x, y, variant, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_spmv_coo")
            return y
    lib = load()
    nnz = val.numel()
    if y is None:
        y = torch.empty(n_rows, dtype=torch.float32, device=val.device)
    if ws is None:
        ws = new_workspace(MMV_OP_SPMV_COO, MMV_F32_F32, MMV_FLAGS_PACKED32, nnz, val.device)
    st = lib.mmv_spmv_coo(n_rows, n_cols, nnz, _dev(row, "row"), _dev(col, "col"), _dev(val, "val"), _dev(x, "x"),
                          _dev(y, "y"), _VARIANTS[variant], _dev(ws, "ws"), ws.numel(), _stream_ptr(stream))
    _check(st, "mmv_spmv_coo")
    return y


def mmv_spmv_coo_prepare(n_rows: int, n_cols: int, row: torch.Tensor, col: torch.Tensor,
                         ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """First step of the two-step COO SpMV: returns the workspace that holds the plan for this matrix."""
    nnz = row.numel()
    if ws is None:
        ws = new_workspace(MMV_OP_SPMV_COO, MMV_F32_F32, MMV_FLAGS_PACKED32, nnz, row.device)
    st = load().mmv_spmv_coo_prepare(n_rows, n_cols, nnz, _dev(row, "row"), _dev(col, "col"), _dev(ws, "ws"), ws.numel(),
                                     _stream_ptr(stream))
    _check(st, "mmv_spmv_coo_prepare")
    return ws


def mmv_spmv_coo_run(n_rows: int, n_cols: int, row: torch.Tensor, col: torch.Tensor, val: torch.Tensor,
                     x: torch.Tensor, ws: torch.Tensor, y: torch.Tensor | None = None, variant: str = "mfma",
                     stream=None) -> torch.Tensor:
    """Second step: y = A x with the plan that mmv_spmv_coo_prepare left in ws."""
    if _marshal is not None:
        st = _marshal.spmv_coo_run(n_rows, n_cols, None, row, col, val, x, y, variant, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_spmv_coo_run")
            return y
    if y is None:
        y = torch.empty(n_rows, dtype=torch.float32, device=val.device)
    st = load().mmv_spmv_coo_run(n_rows, n_cols, val.numel(), _dev(row, "row"), _dev(col, "col"), _dev(val, "val"),
                                 _dev(x, "x"), _dev(y, "y"), _VARIANTS[variant], _dev(ws, "ws"), ws.numel(),
                                 _stream_ptr(stream))
    _check(st, "mmv_spmv_coo_run")
    return y


def mmv_spmv_csr_prepare(n_rows: int, n_cols: int, rowptr: torch.Tensor, col: torch.Tensor,
                         ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """First step of the two-step CSR SpMV: returns the workspace that holds the plan for this matrix."""
    nnz = col.numel()
    if ws is None:
        ws = workspace(mmv_spmv_csr_workspace_bytes(n_rows, nnz), col.device)
    st = load().mmv_spmv_csr_prepare(n_rows, n_cols, nnz, _dev(rowptr, "rowptr"), _dev(col, "col"), _dev(ws, "ws"),
                                     ws.numel(), _stream_ptr(stream))
    _check(st, "mmv_spmv_csr_prepare")
    return ws


def mmv_spmv_csr_run(n_rows: int, n_cols: int, rowptr: torch.Tensor, col: torch.Tensor, val: torch.Tensor,
                     x: torch.Tensor, ws: torch.Tensor, y: torch.Tensor | None = None, variant: str = "mfma",
                     stream=None) -> torch.Tensor:
    """Second step: y = A x with the plan that mmv_spmv_csr_prepare left in ws."""
    if _marshal is not None:
        st = _marshal.spmv_csr_run(n_rows, n_cols, None, rowptr, col, val, x, y, variant, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_spmv_csr_run")
            return y
    if y is None:
        y = torch.empty(n_rows, dtype=torch.float32, device=val.device)
    st = load().mmv_spmv_csr_run(n_rows, n_cols, val.numel(), _dev(rowptr, "rowptr"), _dev(col, "col"), _dev(val, "val"),
                                 _dev(x, "x"), _dev(y, "y"), _VARIANTS[variant], _dev(ws, "ws"), ws.numel(),
                                 _stream_ptr(stream))
    _check(st, "mmv_spmv_csr_run")
    return y


def mmv_workspace_status(ws: torch.Tensor, stream=None) -> int:
    h = ctypes.c_uint32(0)
    _check(load().mmv_workspace_status(_dev(ws, "ws"), _stream_ptr(stream), ctypes.byref(h)), "mmv_workspace_status")
    return int(h.value)


def mmv_stream_copy(src: torch.Tensor, dst: torch.Tensor, in_bytes: int | None = None,
                    out_bytes: int | None = None, stream=None) -> None:
    ib = src.numel() * src.element_size() if in_bytes is None else in_bytes
    ob = dst.numel() * dst.element_size() if out_bytes is None else out_bytes
    _check(load().mmv_stream_copy(_dev(src, "src"), ib, _dev(dst, "dst"), ob, _stream_ptr(stream)),
           "mmv_stream_copy")


GATHER_REFERENCE_PARTIALS = 8192 * 256


def mmv_gather_reference(val: torch.Tensor, col: torch.Tensor, x: torch.Tensor, partial: torch.Tensor,
                         nnz: int | None = None, stream=None) -> None:
    if partial.numel() < GATHER_REFERENCE_PARTIALS:
        raise MmvError("mmv_gather_reference: partial needs %d floats" % GATHER_REFERENCE_PARTIALS)
    _check(load().mmv_gather_reference(val.numel() if nnz is None else nnz, _dev(val, "val"), _dev(col, "col"),
                                       x.numel(), _dev(x, "x"), _dev(partial, "partial"), _stream_ptr(stream)),
           "mmv_gather_reference")


def mmv_set_kernel_events(ev_start: int | None, ev_stop: int | None) -> None:
    """ev_start / ev_stop are hipEvent_t handles as integers (or None to switch off)."""
    _check(load().mmv_set_kernel_events(ev_start, ev_stop), "mmv_set_kernel_events")


# ---- CSR SpMV, the stand-alone primitives of Sec. 4.1 and the un-fused compositions ------------------------

_ELEMS = {torch.int32: MMV_ELEM_I32, torch.float32: MMV_ELEM_F32}


def mmv_spmv_csr_workspace_bytes(n_rows: int, nnz: int) -> int:
    return int(load().mmv_spmv_csr_workspace_bytes(n_rows, nnz))


def mmv_spmv_csr(n_rows: int, n_cols: int, rowptr: torch.Tensor, col: torch.Tensor, val: torch.Tensor,
                 x: torch.Tensor, y: torch.Tensor | None = None, variant: str = "mfma",
                 ws: torch.Tensor | None = None, stream=None, nnz: int | None = None) -> torch.Tensor:
    """y = A x for a CSR matrix (int32 row pointers and column indices, fp32 values)."""
    if _marshal is not None:
        st = _marshal.spmv_csr(n_rows, n_cols, nnz, rowptr, col, val, x, y, variant, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_spmv_csr")
            return y
    lib = load()
    nnz = val.numel() if nnz is None else nnz
    if y is None:
        y = torch.empty(n_rows, dtype=torch.float32, device=val.device)
    if ws is None:
        ws = workspace(mmv_spmv_csr_workspace_bytes(n_rows, nnz), val.device)
    st = lib.mmv_spmv_csr(n_rows, n_cols, nnz, _dev(rowptr, "rowptr"), _dev(col, "col"), _dev(val, "val"),
                          _dev(x, "x"), _dev(y, "y"), _VARIANTS[variant], _dev(ws, "ws"), ws.numel(),
                          _stream_ptr(stream))
    _check(st, "mmv_spmv_csr")
    return y


def mmv_scan(x: torch.Tensor, n: int | None = None, z: torch.Tensor | None = None, variant: str = "mfma",
             ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Unsegmented inclusive scan; returns z (fp32 or int32)."""
    if _marshal is not None:
        st = _marshal.scan(x, n, z, variant, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_scan")
            return z
    lib = load()
    n = x.numel() if n is None else n
    dt = _DTYPES[x.dtype]
    if z is None:
        z = torch.empty(n, dtype=_OUT_DTYPE[dt], device=x.device)
    if ws is None:
        ws = new_workspace(MMV_OP_SCAN, dt, MMV_FLAGS_PACKED32, n, x.device)
    st = lib.mmv_scan(_dev(x, "x"), n, _dev(z, "z"), dt, _VARIANTS[variant], _dev(ws, "ws"), ws.numel(),
                      _stream_ptr(stream))
    _check(st, "mmv_scan")
    return z


def mmv_compress(x: torch.Tensor | None, mask: torch.Tensor, n: int, out: torch.Tensor | None = None,
                 count: torch.Tensor | None = None, ws: torch.Tensor | None = None, stream=None):
    """COMPRESS of a 32-bit vector (or of the positions, x=None); returns (out, count)."""
    if _marshal is not None:
        st = _marshal.compress(x, mask, n, out, count, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_compress")
            return out, count
    lib = load()
    ff = _flag_fmt(mask)
    if x is not None and x.element_size() != 4:
        raise MmvError("mmv_compress works on 32-bit elements")
    if out is None:
        out = torch.empty(max(n, 1), dtype=torch.int32 if x is None else x.dtype, device=mask.device)
    if count is None:
        count = torch.empty(1, dtype=torch.int64, device=mask.device)
    if ws is None:
        ws = new_workspace(MMV_OP_COMPRESS, MMV_I8_I32, ff, n, mask.device)
    st = lib.mmv_compress(None if x is None else _dev(x, "x"), _dev(mask, "mask"), n, _dev(out, "out"), out.numel(),
                          _dev(count, "count"), ff, _dev(ws, "ws"), ws.numel(), _stream_ptr(stream))
    _check(st, "mmv_compress")
    return out, count


def mmv_diff(x: torch.Tensor, n: int | None = None, z: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """DIFF of an int32 or fp32 vector."""
    n = x.numel() if n is None else n
    if z is None:
        z = torch.empty(max(n, 1), dtype=x.dtype, device=x.device)
    _check(load().mmv_diff(_dev(x, "x"), n, _dev(z, "z"), _ELEMS[x.dtype], _stream_ptr(stream)), "mmv_diff")
    return z


def mmv_revert(xhat: torch.Tensor, fhat: torch.Tensor, w: torch.Tensor, n: int | None = None,
               nw: int | None = None, z: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """REVERT: xhat(i) - w(fhat(i) - 2) where fhat(i) >= 2; int32 or fp32, fhat int32."""
    n = xhat.numel() if n is None else n
    nw = w.numel() if nw is None else nw
    if fhat.dtype != torch.int32 or w.dtype != xhat.dtype:
        raise MmvError("fhat must be int32 and w must have the type of xhat")
    if z is None:
        z = torch.empty(max(n, 1), dtype=xhat.dtype, device=xhat.device)
    _check(load().mmv_revert(_dev(xhat, "xhat"), _dev(fhat, "fhat"), _dev(w, "w"), n, nw, _dev(z, "z"),
                             _ELEMS[xhat.dtype], _stream_ptr(stream)), "mmv_revert")
    return z


def mmv_segsum_scd(x: torch.Tensor, flags: torch.Tensor, n: int | None = None, out: torch.Tensor | None = None,
                   nseg: torch.Tensor | None = None, variant: str = "mfma", ws: torch.Tensor | None = None,
                   stream=None):
    """Segmented sum through the un-fused Algorithm SCD; returns (out, nseg) like mmv_segsum."""
    lib = load()
    n = x.numel() if n is None else n
    dt, ff = _DTYPES[x.dtype], _flag_fmt(flags)
    if out is None:
        out = torch.empty(max(n, 1), dtype=_OUT_DTYPE[dt], device=x.device)
    if nseg is None:
        nseg = torch.empty(1, dtype=torch.int64, device=x.device)
    if ws is None:
        ws = new_workspace(MMV_OP_SEGSUM_SCD, dt, ff, n, x.device)
    st = lib.mmv_segsum_scd(_dev(x, "x"), _dev(flags, "flags"), n, _dev(out, "out"), out.numel(), _dev(nseg, "nseg"),
                            dt, ff, _VARIANTS[variant], _dev(ws, "ws"), ws.numel(), _stream_ptr(stream))
    _check(st, "mmv_segsum_scd")
    return out, nseg


def mmv_segscan_sscr(x: torch.Tensor, flags: torch.Tensor, n: int | None = None, z: torch.Tensor | None = None,
                     variant: str = "mfma", ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Segmented scan through the un-fused Algorithm SSCR; returns z like mmv_segscan."""
    lib = load()
    n = x.numel() if n is None else n
    dt, ff = _DTYPES[x.dtype], _flag_fmt(flags)
    if z is None:
        z = torch.empty(n, dtype=_OUT_DTYPE[dt], device=x.device)
    if ws is None:
        ws = new_workspace(MMV_OP_SEGSCAN_SSCR, dt, ff, n, x.device)
    st = lib.mmv_segscan_sscr(_dev(x, "x"), _dev(flags, "flags"), n, _dev(z, "z"), dt, ff, _VARIANTS[variant],
                              _dev(ws, "ws"), ws.numel(), _stream_ptr(stream))
    _check(st, "mmv_segscan_sscr")
    return z


# ---- a serving step over a ragged batch ---------------------------------------------------------------------------

_VALUE_TYPES = {torch.float16: MMV_TYPE_F16, torch.bfloat16: MMV_TYPE_BF16}
_CACHE_TYPES = {**_VALUE_TYPES, torch.float8_e4m3fn: MMV_TYPE_E4M3}


class PageTables(NamedTuple):
    """What mmv_page_tables leaves for the other calls of a step (beside the table itself)."""
    offsets: torch.Tensor    # int32 [n + 1]: first token of every request, and their number
    context: torch.Tensor    # int32 [n]: positions of every request, the new ones among them
    slots: torch.Tensor      # int64 [max_tokens]: every token's slot in the cache, -1: none
    positions: torch.Tensor  # int32 [max_tokens]: every token's position in its request, -1 behind the last one
    used: torch.Tensor       # int64 [2]: free pages that the batch needs, tokens that it has


class _CacheStruct(ctypes.Structure):   # mmv_paged_cache
    _fields_ = [("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p), ("type", ctypes.c_int), ("page", ctypes.c_uint32), ("heads", ctypes.c_uint32),
                ("dim", ctypes.c_uint32), ("pages", ctypes.c_uint64), ("page_stride", ctypes.c_uint64), ("head_stride", ctypes.c_uint64),
                ("slot_stride", ctypes.c_uint64), ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)]


class PagedCache:
    """The keys and values of a layer in pages: two tensors [pages, heads, slots of a page, dim] of fp16, bf16 or e4m3 (any order of the first
    three dimensions in memory: both tensors with the same strides).  An e4m3 cache holds key / k_scale and value / v_scale.  mmv_paged_attention takes
    pages of a multiple of 8 slots."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: float = 1.0, v_scale: float = 1.0):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device or k.stride() != v.stride():
            raise MmvError("a cache is two tensors [pages, heads, slots, dim] of the same shape, type and strides")
        if k.dtype not in _CACHE_TYPES:
            raise MmvError("a cache holds float16, bfloat16 or float8_e4m3fn")
        if not k.is_cuda or k.stride(3) != 1 or min(k.stride()) < 0:
            raise MmvError("a cache lies in GPU memory, the values of a slot one after the other")
        self.k, self.v, self.k_scale, self.v_scale = k, v, float(k_scale), float(v_scale)
        self._struct = _CacheStruct(k.data_ptr(), v.data_ptr(), _CACHE_TYPES[k.dtype], k.shape[2], k.shape[1], k.shape[3], k.shape[0],
                                    k.stride(0), k.stride(1), k.stride(2), self.k_scale, self.v_scale)
        self._ref = ctypes.addressof(self._struct)


def _ints(t: torch.Tensor, name: str, dtype: torch.dtype, numel: int) -> int:
    if t.dtype != dtype or t.numel() < numel:
        raise MmvError("%s must hold %d values of %s" % (name, numel, dtype))
    return _dev(t, name)


def _tokens(t: torch.Tensor, name: str, shape: tuple, dtype: torch.dtype) -> tuple:
    """(address, elements from token to token) of [tokens, heads, dim], the heads of a token one after the other."""
    if not t.is_cuda or t.dtype != dtype or tuple(t.shape) != shape:
        raise MmvError("%s must be %s of %s in GPU memory" % (name, list(shape), dtype))
    if t.numel() and ((t.shape[2] > 1 and t.stride(2) != 1) or (t.shape[1] > 1 and t.stride(1) != t.shape[2])):
        raise MmvError("%s: the heads of a token must lie one after the other" % name)
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else shape[1] * shape[2]


def _u32(v: int, name: str) -> int:   # (ctypes would cut it off)
    if v != int(v) or not 0 <= v < 1 << 32:
        raise MmvError("%s must be a whole number below 2^32, not negative" % name)
    return int(v)


def _table(t: torch.Tensor, n: int) -> tuple:
    if not t.is_cuda or t.dtype != torch.int32 or t.dim() != 2 or t.shape[0] < n or (t.shape[1] > 1 and t.stride(1) != 1):
        raise MmvError("table must be int32 [%d, pages] in GPU memory, the entries of a row one after the other" % n)
    return t.data_ptr(), t.shape[1], t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _out(out, name: str, shape: tuple, dtype: torch.dtype, device) -> torch.Tensor:
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if tuple(out.shape) != shape or out.dtype != dtype:
        raise MmvError("%s must be %s of %s" % (name, list(shape), dtype))
    return out


def _made_current(stream):
    """For a call on another stream than the current one: what it allocates (results, scratch) then belongs to that stream, so that no work on
    the current one has it before or gets it while the call's kernels run."""
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream.cuda_stream)))


def _ws(ws, nbytes: int, device) -> tuple:
    if ws is None and nbytes:
        ws = workspace(nbytes, device)
    return (None, 0, None) if ws is None else (_dev(ws, "ws"), ws.numel() * ws.element_size(), ws)


def mmv_page_tables_workspace_bytes(n: int) -> int:
    return int(load().mmv_page_tables_workspace_bytes(n))


def mmv_page_tables(cached: torch.Tensor, new: torch.Tensor, free: torch.Tensor, table: torch.Tensor, page: int, max_tokens: int,
                    out: PageTables | None = None, ws: torch.Tensor | None = None, stream=None) -> PageTables:
    """Pages for the new tokens of every request (written into `table`) and the slot of every one; returns PageTables."""
    if stream is not None:
        with _made_current(stream):
            return mmv_page_tables(cached, new, free, table, page, max_tokens, out, ws)
    if _marshal is not None:
        st = _marshal.page_tables(cached, new, free, table, page, max_tokens, out, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_page_tables")
            return out
    page = _u32(page, "page")
    lib, n, device = load(), new.numel(), new.device
    if out is None:
        out = PageTables(*(torch.empty(k, dtype=d, device=device) for k, d in
                           ((n + 1, torch.int32), (n, torch.int32), (max_tokens, torch.int64), (max_tokens, torch.int32), (2, torch.int64))))
    row, width, stride = _table(table, n)
    w, w_bytes, ws = _ws(ws, mmv_page_tables_workspace_bytes(n), device)
    st = lib.mmv_page_tables(n, _ints(cached, "cached", torch.int32, n), _ints(new, "new", torch.int32, n), _ints(free, "free", torch.int32, 0), free.numel(),
                             row, width, stride, page, max_tokens, _ints(out.offsets, "offsets", torch.int32, n + 1),
                             _ints(out.context, "context", torch.int32, n), _ints(out.slots, "slots", torch.int64, max_tokens),
                             _ints(out.positions, "positions", torch.int32, max_tokens), _ints(out.used, "used", torch.int64, 2), w, w_bytes, _stream_ptr(stream))
    _check(st, "mmv_page_tables")
    return out


def mmv_cache_append(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache: PagedCache, stream=None) -> None:
    """The keys and values [tokens, heads, dim] of new tokens into their slots."""
    if _marshal is not None:
        st = _marshal.cache_append(k, v, slots, cache._ref, stream)
        if st is not None:
            if st:
                _check(st, "mmv_cache_append")
            return
    if k.dtype not in _VALUE_TYPES or k.dim() != 3:
        raise MmvError("k and v must be [tokens, heads, dim] of float16 or bfloat16")
    shape = (k.shape[0], cache.k.shape[1], cache.k.shape[3])
    (pk, sk), (pv, sv) = _tokens(k, "k", shape, k.dtype), _tokens(v, "v", shape, k.dtype)
    st = load().mmv_cache_append(shape[0], pk, sk, pv, sv, _VALUE_TYPES[k.dtype], _ints(slots, "slots", torch.int64, shape[0]), cache._ref, _stream_ptr(stream))
    _check(st, "mmv_cache_append")


def mmv_paged_attention_workspace_bytes(n: int, q_heads: int, heads: int, dim: int, max_context: int) -> int:
    """max_context: entries of a row of the table times the slots of a page."""
    return int(load().mmv_paged_attention_workspace_bytes(n, q_heads, heads, dim, max_context))


def _attention(name, ref, q, cache, table, context, scale, window, out, lse, ws, stream):
    window = _u32(window, "window")
    if q.dtype not in _VALUE_TYPES or q.dim() != 3:
        raise MmvError("q must be [rows, heads, dim] of float16 or bfloat16")
    lib, (n, heads, dim), own = load(), q.shape, cache.k.shape
    pq, sq = _tokens(q, "q", (n, heads, own[3]), q.dtype)
    out = _out(out, "out", (n, heads, dim), q.dtype, q.device)
    row, width, stride = _table(table, n)
    if lse is not None:
        lse = _out(lse, "lse", (n, heads), torch.float32, q.device)
    w, w_bytes, ws = _ws(ws, mmv_paged_attention_workspace_bytes(n, heads, own[1], dim, width * own[2]), q.device)
    st = getattr(lib, name)(n, heads, pq, sq, _VALUE_TYPES[q.dtype], ref, row, width, stride, _ints(context, "context", torch.int32, n),
                            1.0 / math.sqrt(dim) if scale is None else scale, window, _dev(out, "out"), None if lse is None else _dev(lse, "lse"),
                            w, w_bytes, _stream_ptr(stream))
    _check(st, name)
    return out


def mmv_paged_attention(q: torch.Tensor, cache: PagedCache, table: torch.Tensor, context: torch.Tensor, scale: float | None = None, window: int = 0,
                        out: torch.Tensor | None = None, lse: torch.Tensor | None = None, ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Attention of one token q[r] ([rows, query heads, dim]) over the first context[r] positions of every row of the table, or the last
    `window` of them; returns out like q.  scale: dim ** -0.5 if left out; lse: fp32 [rows, query heads], filled if given."""
    if stream is not None:
        with _made_current(stream):
            return mmv_paged_attention(q, cache, table, context, scale, window, out, lse, ws)
    if _marshal is not None:
        st = _marshal.paged_attention(q, cache._ref, table, context, scale, window, out, lse, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_paged_attention")
            return out
    return _attention("mmv_paged_attention", cache._ref, q, cache, table, context, scale, window, out, lse, ws, stream)


def _states(heads, dk, dv, state_in, state_out, state_index, n):
    states = None
    for name, s in (("state_in", state_in), ("state_out", state_out)):
        if s is not None:
            if s.dtype != torch.float32 or s.dim() != 4 or tuple(s.shape[1:]) != (heads, dk, dv) or s.shape[0] != (states or s.shape)[0]:
                raise MmvError("%s must be [states, %d, %d, %d] of float32" % (name, heads, dk, dv))
            states = s.shape
    return (None if state_in is None else _dev(state_in, "state_in"), None if state_out is None else _dev(state_out, "state_out"), states[0] if states else 0,
            None if state_index is None else _ints(state_index, "state_index", torch.int32, n))


def _decay_arguments(q, k, v, log_decay, state_in, state_out, state_index, n, out):
    if q.dtype not in _VALUE_TYPES or q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise MmvError("q, k and v must be [tokens, heads, dim] of float16 or bfloat16")
    (t, heads, dk), (kv, dv) = q.shape, v.shape[1:]
    (pq, sq), (pk, sk), (pv, sv) = _tokens(q, "q", (t, heads, dk), q.dtype), _tokens(k, "k", (t, kv, dk), q.dtype), _tokens(v, "v", (t, kv, dv), q.dtype)
    state = _states(heads, dk, dv, state_in, state_out, state_index, n)
    out = _out(out, "out", (t, heads, dv), q.dtype, q.device)
    head = (heads, kv, dk, dv, pq, sq, pk, sk, pv, sv, _VALUE_TYPES[q.dtype])
    tail = (_ints(log_decay, "log_decay", torch.float32, heads),)
    return t, head, tail, state + (_dev(out, "out"),), out


def mmv_decay_attention_workspace_bytes(n: int, tokens: int, heads: int, dk: int, dv: int) -> int:
    return int(load().mmv_decay_attention_workspace_bytes(n, tokens, heads, dk, dv))


def mmv_decay_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, log_decay: torch.Tensor, scale: float | None = None,
                        state_in: torch.Tensor | None = None, state_out: torch.Tensor | None = None, state_index: torch.Tensor | None = None,
                        out: torch.Tensor | None = None, ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Linear attention with a decay for each head over packed requests; q [tokens, heads, dk], k [tokens, kv heads, dk], v [tokens, kv heads,
    dv], states [states, heads, dk, dv] of fp32; returns out [tokens, heads, dv].  scale: dk ** -0.5 if left out."""
    if stream is not None:
        with _made_current(stream):
            return mmv_decay_attention(q, k, v, offsets, log_decay, scale, state_in, state_out, state_index, out, ws)
    if _marshal is not None:
        st = _marshal.decay_attention(q, k, v, offsets, log_decay, scale, state_in, state_out, state_index, out, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_decay_attention")
            return out
    n = offsets.numel() - 1
    if n < 0:
        raise MmvError("offsets must hold the first token of every request, and their number")
    t, head, decay, state, out = _decay_arguments(q, k, v, log_decay, state_in, state_out, state_index, n, out)
    w, w_bytes, ws = _ws(ws, mmv_decay_attention_workspace_bytes(n, t, head[0], head[2], head[3]), q.device)
    st = load().mmv_decay_attention(n, t, *head, _ints(offsets, "offsets", torch.int32, n + 1), *decay, head[2] ** -0.5 if scale is None else scale, *state,
                                    w, w_bytes, _stream_ptr(stream))
    _check(st, "mmv_decay_attention")
    return out


def mmv_decay_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, state_in: torch.Tensor | None = None,
                   state_out: torch.Tensor | None = None, scale: float | None = None, state_index: torch.Tensor | None = None,
                   out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_decay_attention for one token of every request."""
    if stream is not None:
        with _made_current(stream):
            return mmv_decay_step(q, k, v, log_decay, state_in, state_out, scale, state_index, out)
    if _marshal is not None:
        st = _marshal.decay_step(q, k, v, log_decay, state_in, state_out, scale, state_index, out, stream)
        if st is not None:
            if st:
                _check(st, "mmv_decay_step")
            return out
    t, head, decay, state, out = _decay_arguments(q, k, v, log_decay, state_in, state_out, state_index, q.shape[0], out)
    st = load().mmv_decay_step(t, *head, *decay, head[2] ** -0.5 if scale is None else scale, *state, _stream_ptr(stream))
    _check(st, "mmv_decay_step")
    return out


# ---- a cache of 8-bit values with a scale for each block of slots and head ------------------------------------------

_BLOCK_TYPES = {torch.int8: MMV_TYPE_I8, torch.float8_e4m3fn: MMV_TYPE_E4M3}


class _BlockCacheStruct(ctypes.Structure):   # mmv_block_cache
    _fields_ = [("d_k", ctypes.c_void_p), ("d_v", ctypes.c_void_p), ("d_k_scales", ctypes.c_void_p), ("d_v_scales", ctypes.c_void_p), ("type", ctypes.c_int),
                ("page", ctypes.c_uint32), ("heads", ctypes.c_uint32), ("dim", ctypes.c_uint32), ("block", ctypes.c_uint32), ("pages", ctypes.c_uint64),
                ("page_stride", ctypes.c_uint64), ("head_stride", ctypes.c_uint64), ("slot_stride", ctypes.c_uint64)]


class BlockCache:
    """The keys and values of a layer in pages of 8-bit codes: two tensors [pages, heads, slots of a page, dim] of int8 or e4m3 (any order of the first three
    dimensions in memory: both with the same strides), and their scales, two fp32 tensors [pages, heads, blocks of a page] (zeros to begin with): a block is a
    multiple of 8 neighbouring slots, and its values are code * scale."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device or k.stride() != v.stride():
            raise MmvError("a cache is two tensors [pages, heads, slots, dim] of the same shape, type and strides")
        if k.dtype not in _BLOCK_TYPES:
            raise MmvError("a cache in blocks holds int8 or float8_e4m3fn")
        if not k.is_cuda or k.stride(3) != 1 or min(k.stride()) < 0:
            raise MmvError("a cache lies in GPU memory, the values of a slot one after the other")
        for name, s in (("k_scales", k_scales), ("v_scales", v_scales)):
            if s.dim() != 3 or s.dtype != torch.float32 or s.shape[:2] != k.shape[:2] or s.shape != k_scales.shape or s.device != k.device or not s.is_contiguous():
                raise MmvError("%s must be [%d, %d, blocks of a page] of float32 beside the cache, contiguous" % (name, k.shape[0], k.shape[1]))
        blocks = k_scales.shape[2]
        if blocks < 1 or k.shape[2] % blocks or k.shape[2] // blocks % 8:
            raise MmvError("a page has whole blocks of a multiple of 8 slots")
        self.k, self.v, self.k_scales, self.v_scales, self.block = k, v, k_scales, v_scales, k.shape[2] // blocks
        self._struct = _BlockCacheStruct(k.data_ptr(), v.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), _BLOCK_TYPES[k.dtype], k.shape[2], k.shape[1], k.shape[3],
                                         self.block, k.shape[0], k.stride(0), k.stride(1), k.stride(2))
        self._blocks_ref = ctypes.addressof(self._struct)   # (not PagedCache's name: neither is taken for the other)


def _blocks(cache) -> int:
    if type(cache) is not BlockCache:
        raise MmvError("cache must be a BlockCache")
    return cache._blocks_ref


def mmv_block_append(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache: BlockCache, stream=None) -> None:
    """The keys and values [tokens, heads, dim] of new tokens into their slots, quantised; tokens of one block are neighbours."""
    ref = _blocks(cache)
    if _marshal is not None:
        st = _marshal.block_append(k, v, slots, ref, stream)
        if st is not None:
            if st:
                _check(st, "mmv_block_append")
            return
    if k.dtype not in _VALUE_TYPES or k.dim() != 3:
        raise MmvError("k and v must be [tokens, heads, dim] of float16 or bfloat16")
    shape = (k.shape[0], cache.k.shape[1], cache.k.shape[3])
    (pk, sk), (pv, sv) = _tokens(k, "k", shape, k.dtype), _tokens(v, "v", shape, k.dtype)
    st = load().mmv_block_append(shape[0], pk, sk, pv, sv, _VALUE_TYPES[k.dtype], _ints(slots, "slots", torch.int64, shape[0]), ref, _stream_ptr(stream))
    _check(st, "mmv_block_append")


def mmv_block_read(cache: BlockCache, table: torch.Tensor, offsets: torch.Tensor, tokens: int | None = None, dtype: torch.dtype = torch.bfloat16,
                   first: torch.Tensor | None = None, out: tuple | None = None, stream=None) -> tuple:
    """Keys and values of every request's positions first[r] (0 if left out) to first[r] + offsets[r + 1] - offsets[r] - 1, packed; returns (k, v), two
    [tokens, heads, dim] of dtype, or `out` filled in: two such tensors, views of others too."""
    if stream is not None:
        with _made_current(stream):
            return mmv_block_read(cache, table, offsets, tokens, dtype, first, out)
    ref = _blocks(cache)
    if _marshal is not None:
        st = _marshal.block_read(ref, table, offsets, first, out, stream)
        if st is not None:
            if st:
                _check(st, "mmv_block_read")
            return out
    n = offsets.numel() - 1
    if n < 0:
        raise MmvError("offsets must hold the first token of every request, and their number")
    if out is None:
        if tokens is None or dtype not in _VALUE_TYPES:
            raise MmvError("without out, tokens must be their number and dtype float16 or bfloat16")
        out = tuple(torch.empty(tokens, cache.k.shape[1], cache.k.shape[3], dtype=dtype, device=cache.k.device) for _ in "kv")
    k, v = out
    if k.dtype not in _VALUE_TYPES or k.dim() != 3:
        raise MmvError("out must be two [tokens, heads, dim] of float16 or bfloat16")
    shape = (k.shape[0], cache.k.shape[1], cache.k.shape[3])
    (pk, sk), (pv, sv) = _tokens(k, "k", shape, k.dtype), _tokens(v, "v", shape, k.dtype)
    row, width, stride = _table(table, n)
    st = load().mmv_block_read(n, shape[0], _ints(offsets, "offsets", torch.int32, n + 1), None if first is None else _ints(first, "first", torch.int32, n),
                               row, width, stride, ref, _VALUE_TYPES[k.dtype], pk, sk, pv, sv, _stream_ptr(stream))
    _check(st, "mmv_block_read")
    return out


def mmv_block_attention(q: torch.Tensor, cache: BlockCache, table: torch.Tensor, context: torch.Tensor, scale: float | None = None, window: int = 0,
                        out: torch.Tensor | None = None, lse: torch.Tensor | None = None, ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_paged_attention over a cache in blocks (and the same workspace)."""
    if stream is not None:
        with _made_current(stream):
            return mmv_block_attention(q, cache, table, context, scale, window, out, lse, ws)
    ref = _blocks(cache)
    if _marshal is not None:
        st = _marshal.block_attention(q, ref, table, context, scale, window, out, lse, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_block_attention")
            return out
    return _attention("mmv_block_attention", ref, q, cache, table, context, scale, window, out, lse, ws, stream)


# ---- the gated delta rule -------------------------------------------------------------------------------------------


def _delta_arguments(q, k, v, log_decay, beta, state_in, state_out, state_index, n, out):
    if q.dtype not in _VALUE_TYPES or q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise MmvError("q, k and v must be [tokens, heads, dim] of float16 or bfloat16")
    (t, shared, dk), (heads, dv) = q.shape, v.shape[1:]
    (pq, sq), (pk, sk), (pv, sv) = _tokens(q, "q", (t, shared, dk), q.dtype), _tokens(k, "k", (t, shared, dk), q.dtype), _tokens(v, "v", (t, heads, dv), q.dtype)
    for name, x in (("log_decay", log_decay), ("beta", beta)):
        if tuple(x.shape) != (t, heads):
            raise MmvError("%s must be [%d, %d] of float32" % (name, t, heads))
    state = _states(heads, dk, dv, state_in, state_out, state_index, n)
    out = _out(out, "out", (t, heads, dv), q.dtype, q.device)
    head = (heads, shared, dk, dv, pq, sq, pk, sk, pv, sv, _VALUE_TYPES[q.dtype])
    gates = (_ints(log_decay, "log_decay", torch.float32, t * heads), _ints(beta, "beta", torch.float32, t * heads))
    return t, head, gates, state + (_dev(out, "out"),), out


def mmv_delta_attention_workspace_bytes(n: int, tokens: int, heads: int, dk: int, dv: int) -> int:
    return int(load().mmv_delta_attention_workspace_bytes(n, tokens, heads, dk, dv))


def mmv_delta_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets: torch.Tensor, log_decay: torch.Tensor, beta: torch.Tensor,
                        scale: float | None = None, state_in: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
                        state_index: torch.Tensor | None = None, out: torch.Tensor | None = None, ws: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The gated delta rule over packed requests; q and k [tokens, key heads, dk], v [tokens, heads, dv], log_decay and beta [tokens, heads] of fp32, states
    [states, heads, dk, dv] of fp32; returns out [tokens, heads, dv].  scale: dk ** -0.5 if left out."""
    if stream is not None:
        with _made_current(stream):
            return mmv_delta_attention(q, k, v, offsets, log_decay, beta, scale, state_in, state_out, state_index, out, ws)
    if _marshal is not None:
        st = _marshal.delta_attention(q, k, v, offsets, log_decay, beta, scale, state_in, state_out, state_index, out, ws, stream)
        if st is not None:
            if st:
                _check(st, "mmv_delta_attention")
            return out
    n = offsets.numel() - 1
    if n < 0:
        raise MmvError("offsets must hold the first token of every request, and their number")
    t, head, gates, state, out = _delta_arguments(q, k, v, log_decay, beta, state_in, state_out, state_index, n, out)
    w, w_bytes, ws = _ws(ws, mmv_delta_attention_workspace_bytes(n, t, head[0], head[2], head[3]), q.device)
    st = load().mmv_delta_attention(n, t, *head, _ints(offsets, "offsets", torch.int32, n + 1), *gates, head[2] ** -0.5 if scale is None else scale, *state,
                                    w, w_bytes, _stream_ptr(stream))
    _check(st, "mmv_delta_attention")
    return out


def mmv_delta_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, beta: torch.Tensor, state_in: torch.Tensor | None = None,
                   state_out: torch.Tensor | None = None, scale: float | None = None, state_index: torch.Tensor | None = None,
                   out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """mmv_delta_attention for one token of every request."""
    if stream is not None:
        with _made_current(stream):
            return mmv_delta_step(q, k, v, log_decay, beta, state_in, state_out, scale, state_index, out)
    if _marshal is not None:
        st = _marshal.delta_step(q, k, v, log_decay, beta, state_in, state_out, scale, state_index, out, stream)
        if st is not None:
            if st:
                _check(st, "mmv_delta_step")
            return out
    t, head, gates, state, out = _delta_arguments(q, k, v, log_decay, beta, state_in, state_out, state_index, q.shape[0], out)
    st = load().mmv_delta_step(t, *head, *gates, head[2] ** -0.5 if scale is None else scale, *state, _stream_ptr(stream))
    _check(st, "mmv_delta_step")
    return out
