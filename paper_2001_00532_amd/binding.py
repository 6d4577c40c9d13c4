"""Thin ctypes binding of libpsk.so: argument marshalling only.

Function names match include/psk.h.  Tensors are torch CUDA tensors (device memory and streams are
PyTorch's only role); every computation happens inside the library's kernels.  There is no CPU
fallback: a missing library raises at import of this module's first use.
"""
from __future__ import annotations

import ctypes
import os
import warnings

import torch

from .build import built_for

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpsk.so")
TRACE_LIB_PATH = os.path.join(_HERE, "libpsk_trace.so")

PSK_OK = 0
PSK_OP_SPMV_CSR, PSK_OP_SPMM_CSR, PSK_OP_SPMV_BCSR, PSK_OP_SPMM_BCSR, PSK_OP_MTTKRP_CSF3 = 0, 1, 2, 3, 4
PSK_OP_SPMV_CSR_F64 = 5
PSK_CUT_POSITIONS, PSK_CUT_ROWS = 0, 1
PSK_SCHEDULE_POSITIONS, PSK_SCHEDULE_ROWS = 0, 1
PSK_PHASE_PARTITION, PSK_PHASE_MAIN, PSK_PHASE_FIXUP, PSK_PHASE_ALL = 1, 2, 4, 7
PSK_ROWSPLIT_THREAD_PER_ROW, PSK_ROWSPLIT_WAVE_PER_ROW = 0, 1

EXPORTS = [
    "psk_status_string", "psk_version", "psk_default_tile", "psk_num_tiles", "psk_workspace_bytes",
    "psk_partition_csr", "psk_analyze_csr", "psk_spmv_csr", "psk_spmm_csr", "psk_spmv_bcsr", "psk_spmm_bcsr",
    "psk_spmv_csr_rowsplit", "psk_spmm_csr_rowsplit", "psk_spmv_csr_atomics", "psk_mttkrp_csf3",
    "psk_partition_csf3", "psk_spmv_csr_notemp", "psk_spmv_csr_f64", "psk_spmv_dcsr", "psk_spmv_csr_divide", "psk_suggest_schedule_csr", "psk_default_tile_bcsr", "psk_validate_csr",
    "psk_spmv_csr_static", "psk_static_scratch_bytes", "psk_spmv_dcsr_workspace_bytes",
    "psk_slab_mem_bytes", "psk_slab_build_workspace_bytes", "psk_slab_spmv_workspace_bytes", "psk_slab_build_csr",
    "psk_spmv_slab", "psk_slab_mem_bytes_f64", "psk_slab_build_workspace_bytes_f64", "psk_slab_build_csr_f64",
    "psk_spmv_slab_f64", "psk_cu_trace_set", "psk_calibrate_stream_read", "psk_calibrate_gather", "psk_calibrate_gather_lds",
    "psk_gemm_q4_workspace_bytes", "psk_gemm_q4", "psk_moe_route_workspace_bytes", "psk_moe_route", "psk_moe_workspace_bytes",
    "psk_moe_experts", "psk_moe_experts_q4",
    "psk_quant_i8", "psk_gemm_i8_workspace_bytes", "psk_gemm_i8", "psk_linear_i8_workspace_bytes", "psk_linear_i8",
    "psk_embed", "psk_embed_i8", "psk_embed_grad_workspace_bytes", "psk_embed_grad",
]


PSK_SLAB_COLS, PSK_SLAB_CHUNK = 32736, 512


class psk_slab(ctypes.Structure):
    """Mirror of the C struct psk_slab (host memory; the pointers are device addresses)."""
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "cols", "nnz", "nslabs", "nslots", "nchunks", "npairs", "nq")] + \
               [(n, ctypes.c_int32) for n in ("slab_cols", "chunk", "tile", "value_bytes")] + \
               [(n, ctypes.c_void_p) for n in ("svals", "scol", "chunk_pair", "slab_chunk", "qpos", "qidx", "qtile_row")]


PSK_F32, PSK_F16, PSK_BF16 = 0, 1, 2
PSK_SCORE_SOFTMAX, PSK_SCORE_SIGMOID = 0, 1
PSK_ACT_SILU, PSK_ACT_GELU = 0, 1
PSK_MAX_VECTORS, PSK_MOE_MAX_EXPERTS, PSK_MOE_MAX_TOP_K = 1 << 19, 1024, 64


class psk_q4(ctypes.Structure):
    """Mirror of the C struct psk_q4 (host memory; the pointers are device addresses)."""
    _fields_ = [(n, ctypes.c_int64) for n in ("count", "rows", "cols")] + [(n, ctypes.c_int32) for n in ("group", "scale_type")] + \
               [(n, ctypes.c_void_p) for n in ("codes", "scales", "zeros")] + \
               [(n, ctypes.c_int64) for n in ("ld_codes", "ld_scales", "stride_codes", "stride_scales")]


PSK_I8_MAX_COLS, PSK_I8_MAX_LD, PSK_MAX_TOKENS = 131071, 1 << 23, 1 << 24


class psk_i8(ctypes.Structure):
    """Mirror of the C struct psk_i8 (host memory; the pointers are device addresses)."""
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "cols", "ld")] + [(n, ctypes.c_void_p) for n in ("codes", "scales")]


class PskError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__("%s failed: status %d (%s)" % (what, status, status_string(status)))
        self.status = status


_lib = None
_lib_path = LIB_PATH
_marshal = None                                  # the native side of a call (csrc/marshal.cpp), None: the Python functions do its work
_spmv_address = {}


def _spmv(*args):                                # lib() puts the native one here; None: not done
    return None


def _native_side():
    """_marshal.so if it is there and was built for this torch and Python (it reads tensors through their C++ objects).  Without
    it everything works as with it, a small CSR product takes 6.4 us in place of 3.9."""
    try:
        from . import _marshal as native
        if native.built_for == built_for():
            return native
        why = "it was built for %s, this is %s" % (native.built_for, built_for())
    except (ImportError, AttributeError) as e:
        why = str(e)
    warnings.warn("the native side of a call is not used (%s); `python -m paper_2001_00532_amd.build` builds it" % why)
    return None


def use_instrumented_library() -> None:
    """Selects libpsk_trace.so (the build with per-workgroup records, see psk_cu_trace_set) instead of libpsk.so.
    Must be called before the first operation of the process."""
    global _lib_path
    if _lib is not None:
        raise RuntimeError("the library is already loaded")
    _lib_path = TRACE_LIB_PATH


def lib() -> ctypes.CDLL:
    """The loaded library.  Raises if it has not been built (python -m paper_2001_00532_amd.build)."""
    global _lib, _marshal, _ptr, _spmv
    if _lib is None:
        if not os.path.exists(_lib_path):
            raise RuntimeError("%s is not built; run `python -m paper_2001_00532_amd.build`" % os.path.basename(_lib_path))
        L = ctypes.CDLL(_lib_path)
        i64, i32, p, ci, sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.psk_status_string.argtypes, L.psk_status_string.restype = [ci], ctypes.c_char_p
        L.psk_version.argtypes, L.psk_version.restype = [], ci
        L.psk_default_tile.argtypes, L.psk_default_tile.restype = [ci], i32
        L.psk_num_tiles.argtypes, L.psk_num_tiles.restype = [i64, i32], i64
        L.psk_workspace_bytes.argtypes, L.psk_workspace_bytes.restype = [ci, i64, i64, i32, i32, i32], sz
        L.psk_partition_csr.argtypes, L.psk_partition_csr.restype = [i64, i64, p, i32, ci, p, p], ci
        L.psk_analyze_csr.argtypes = [i64, i64, i64, p, p, p, sz, ctypes.POINTER(i32), p]
        L.psk_analyze_csr.restype = ci
        L.psk_spmv_csr.argtypes = [i64, i64, i64, p, p, p, p, p, i32, i32, ci, p, sz, p]
        L.psk_spmv_csr.restype = ci
        L.psk_spmv_csr_static.argtypes = [i64, i64, i64, p, p, p, p, p, i32, i32, p]
        L.psk_spmv_csr_static.restype = ci
        L.psk_static_scratch_bytes.argtypes, L.psk_static_scratch_bytes.restype = [], sz
        L.psk_slab_mem_bytes.argtypes, L.psk_slab_mem_bytes.restype = [i64, i64, i64], sz
        L.psk_slab_build_workspace_bytes.argtypes, L.psk_slab_build_workspace_bytes.restype = [i64, i64, i64], sz
        L.psk_slab_spmv_workspace_bytes.argtypes = [ctypes.POINTER(psk_slab)]
        L.psk_slab_spmv_workspace_bytes.restype = sz
        L.psk_slab_build_csr.argtypes = [i64, i64, i64, p, p, p, p, sz, p, sz, ctypes.POINTER(psk_slab), p]
        L.psk_slab_build_csr.restype = ci
        L.psk_spmv_slab.argtypes = [ctypes.POINTER(psk_slab), p, p, ci, p, sz, p]
        L.psk_spmv_slab.restype = ci
        L.psk_slab_mem_bytes_f64.argtypes, L.psk_slab_mem_bytes_f64.restype = [i64, i64, i64], sz
        L.psk_slab_build_workspace_bytes_f64.argtypes, L.psk_slab_build_workspace_bytes_f64.restype = [i64, i64, i64], sz
        L.psk_slab_build_csr_f64.argtypes = [i64, i64, i64, p, p, p, p, sz, p, sz, ctypes.POINTER(psk_slab), p]
        L.psk_slab_build_csr_f64.restype = ci
        L.psk_spmv_slab_f64.argtypes = [ctypes.POINTER(psk_slab), p, p, ci, p, sz, p]
        L.psk_spmv_slab_f64.restype = ci
        L.psk_cu_trace_set.argtypes, L.psk_cu_trace_set.restype = [p, sz], ci
        L.psk_calibrate_stream_read.argtypes, L.psk_calibrate_stream_read.restype = [p, sz, p, p], ci
        L.psk_calibrate_gather.argtypes, L.psk_calibrate_gather.restype = [p, i64, p, i64, p, p], ci
        L.psk_calibrate_gather_lds.argtypes, L.psk_calibrate_gather_lds.restype = [p, i32, p, i64, p, p], ci
        L.psk_spmm_csr.argtypes = [i64, i64, i64, p, p, p, p, i32, i64, p, i64, i32, ci, p, sz, p]
        L.psk_spmm_csr.restype = ci
        L.psk_spmv_bcsr.argtypes = [i64, i64, i64, i32, p, p, p, p, p, i32, ci, p, sz, p]
        L.psk_spmv_bcsr.restype = ci
        L.psk_spmm_bcsr.argtypes = [i64, i64, i64, i32, p, p, p, p, i32, i64, p, i64, i32, ci, p, sz, p]
        L.psk_spmm_bcsr.restype = ci
        L.psk_partition_csf3.argtypes = [i64, i64, i64, p, p, i32, p, p, p]
        L.psk_partition_csf3.restype = ci
        L.psk_mttkrp_csf3.argtypes = [i64, i64, i64, i64, i64, i64, p, p, p, p, p, p, p, i64, p, i64, i32, p, i64, i32,
                                      ci, p, sz, p]
        L.psk_mttkrp_csf3.restype = ci
        L.psk_spmv_csr_atomics.argtypes = [i64, i64, i64, p, p, p, p, p, i32, ci, p, sz, p]
        L.psk_spmv_csr_atomics.restype = ci
        L.psk_spmv_csr_notemp.argtypes = [i64, i64, i64, p, p, p, p, p, i32, ci, p, sz, p]
        L.psk_spmv_csr_notemp.restype = ci
        L.psk_spmv_csr_f64.argtypes = [i64, i64, i64, p, p, p, p, p, i32, i32, ci, p, sz, p]
        L.psk_spmv_csr_f64.restype = ci
        L.psk_spmv_dcsr.argtypes = [i64, i64, i64, i64, p, p, p, p, p, p, ci, i32, i32, ci, p, sz, p]
        L.psk_spmv_dcsr.restype = ci
        L.psk_spmv_dcsr_workspace_bytes.argtypes, L.psk_spmv_dcsr_workspace_bytes.restype = [i64, i64, i32], sz
        L.psk_default_tile_bcsr.argtypes = [ci, i32]
        L.psk_default_tile_bcsr.restype = i32
        L.psk_suggest_schedule_csr.argtypes = [i64, i64, p, p, sz, p, p]
        L.psk_suggest_schedule_csr.restype = ci
        L.psk_validate_csr.argtypes = [i64, i64, i64, p, p, p, sz, p, p]
        L.psk_validate_csr.restype = ci
        L.psk_spmv_csr_divide.argtypes = [i64, i64, i64, p, p, p, p, p, i32, ci, p, sz, p]
        L.psk_spmv_csr_divide.restype = ci
        L.psk_spmv_csr_rowsplit.argtypes = [i64, i64, i64, p, p, p, p, p, ci, p]
        L.psk_spmv_csr_rowsplit.restype = ci
        L.psk_spmm_csr_rowsplit.argtypes = [i64, i64, i64, p, p, p, p, i32, i64, p, i64, p]
        L.psk_spmm_csr_rowsplit.restype = ci
        q4, f32 = ctypes.POINTER(psk_q4), ctypes.c_float
        L.psk_gemm_q4_workspace_bytes.argtypes, L.psk_gemm_q4_workspace_bytes.restype = [i64, i64, i64, ci], sz
        L.psk_gemm_q4.argtypes, L.psk_gemm_q4.restype = [q4, i64, ci, p, i64, p, i64, p, sz, p], ci
        L.psk_moe_route_workspace_bytes.argtypes, L.psk_moe_route_workspace_bytes.restype = [i64, i64], sz
        L.psk_moe_route.argtypes = [i64, i64, i64, i32, ci, ci, f32, ci, p, i64, ci, p, i64, p, p, p, p, sz, p]
        L.psk_moe_route.restype = ci
        L.psk_moe_workspace_bytes.argtypes, L.psk_moe_workspace_bytes.restype = [i64, i64, i64, i64, i32], sz
        L.psk_moe_experts.argtypes = [i64, i64, i64, i64, i32, ci, ci, p, i64, p, p, p, p, i64, i64, p, i64, i64, p, i64, p, sz, p]
        L.psk_moe_experts.restype = ci
        L.psk_moe_experts_q4.argtypes = [i64, i32, ci, ci, p, i64, p, p, q4, q4, q4, p, i64, p, sz, p]
        L.psk_moe_experts_q4.restype = ci
        i8 = ctypes.POINTER(psk_i8)
        L.psk_quant_i8.argtypes, L.psk_quant_i8.restype = [i64, i64, ci, p, i64, p, i64, p, p], ci
        L.psk_gemm_i8_workspace_bytes.argtypes, L.psk_gemm_i8_workspace_bytes.restype = [i64, i64, i64], sz
        L.psk_gemm_i8.argtypes, L.psk_gemm_i8.restype = [i8, i64, p, i64, p, p, ci, p, i64, p, sz, p], ci
        L.psk_linear_i8_workspace_bytes.argtypes, L.psk_linear_i8_workspace_bytes.restype = [i64, i64, i64, ci], sz
        L.psk_linear_i8.argtypes, L.psk_linear_i8.restype = [i8, i64, ci, p, i64, p, p, i64, p, sz, p], ci
        L.psk_embed.argtypes, L.psk_embed.restype = [i64, i64, i64, p, f32, ci, p, i64, ci, p, i64, p], ci
        L.psk_embed_i8.argtypes, L.psk_embed_i8.restype = [i8, i64, p, f32, ci, p, i64, p], ci
        L.psk_embed_grad_workspace_bytes.argtypes, L.psk_embed_grad_workspace_bytes.restype = [i64, i64, i64], sz
        L.psk_embed_grad.argtypes = [i64, i64, i64, p, i32, f32, ci, p, i64, ci, p, i64, ci, p, sz, p]
        L.psk_embed_grad.restype = ci
        if _marshal is None:
            native = _native_side()
            if native is not None:
                native.use(_ptr_checked, _stream)
                _marshal, _ptr, _spmv = native, native.ptr, native.spmv
        for f64, f in ((0, L.psk_spmv_csr), (1, L.psk_spmv_csr_f64)):
            _spmv_address[f64] = ctypes.cast(f, ctypes.c_void_p).value
        _lib = L
    return _lib


def _ptr_checked(t, dtype=None):
    """Device address of a tensor (None -> NULL).  Checks device, dtype and contiguity of the last dim.  (An int: ctypes
    converts it by the declared argument types; making a c_void_p of it first costs as much as the checks.)"""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError("expected dtype %s, got %s" % (dtype, t.dtype))
    if t.stride(-1) != 1 and t.numel():
        raise ValueError("innermost dimension must be contiguous")
    return t.data_ptr()


_ptr = _ptr_checked                              # lib() puts the native one here


def _stream(stream=None):
    """Address of the stream's hipStream_t.  The current one is asked for without building a Stream object."""
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _temporary_ws_ok(phases: int, what: str):
    """A workspace made for one call holds no table: the main and fix-up steps on their own would read garbage
    row numbers (and run out of bounds), so a partial product must bring the workspace the table was built in."""
    if int(phases) & PSK_PHASE_PARTITION == 0:
        raise ValueError("%s: phases without PSK_PHASE_PARTITION need the workspace (ws=...) that holds the table" % what)


def _check(status: int, what: str):
    if status != PSK_OK:
        raise PskError(status, what)


def status_string(status: int) -> str:
    return lib().psk_status_string(int(status)).decode()


def psk_version() -> int:
    return int(lib().psk_version())


def psk_default_tile(op: int) -> int:
    return int(lib().psk_default_tile(int(op)))


def psk_default_tile_bcsr(op: int, bs: int) -> int:
    return int(lib().psk_default_tile_bcsr(int(op), int(bs)))


def psk_num_tiles(nnz: int, tile: int) -> int:
    return int(lib().psk_num_tiles(int(nnz), int(tile)))


def psk_workspace_bytes(op: int, rows: int, nnz: int, k: int = 1, bs: int = 1, tile: int = 0) -> int:
    return int(lib().psk_workspace_bytes(int(op), int(rows), int(nnz), int(k), int(bs), int(tile)))


def psk_spmv_dcsr_workspace_bytes(nstored: int, nnz: int, tile: int = 0) -> int:
    return int(lib().psk_spmv_dcsr_workspace_bytes(int(nstored), int(nnz), int(tile)))


DCSR_ROOM_ROWS = 1 << 22


def workspace(op: int, rows: int, nnz: int, k: int = 1, bs: int = 1, tile: int = 0, device="cuda", stream=None):
    """A byte tensor that suits the operation (torch allocations are 256-byte aligned).

    One made for PSK_OP_SPMV_CSR is also what psk_spmv_dcsr takes, so up to DCSR_ROOM_ROWS rows it has the room for row
    sums that the faster route of that product wants (at most 16 MiB; with more stored rows ask
    psk_spmv_dcsr_workspace_bytes).

    `stream`: the stream the kernels that use it will run on.  The block is allocated under that stream, so
    torch's caching allocator hands it out again only to work that is ordered after those kernels; a
    temporary workspace dropped right after an asynchronous call stays valid until the call has run."""
    n = psk_workspace_bytes(op, rows, nnz, k, bs, tile)
    if n == 0:
        raise ValueError("invalid arguments for psk_workspace_bytes")
    if op == PSK_OP_SPMV_CSR and 0 <= rows <= DCSR_ROOM_ROWS:
        n = max(n, psk_spmv_dcsr_workspace_bytes(rows, nnz, tile))
    return _alloc_bytes(n, device, stream)


def _csr_ws(rows, nnz, tile, device, stream):
    """What one CSR product needs, no more (for workspaces that live for one call)."""
    n = psk_workspace_bytes(PSK_OP_SPMV_CSR, rows, nnz, tile=tile)
    if n == 0:
        raise ValueError("invalid arguments for psk_workspace_bytes")
    return _alloc_bytes(n, device, stream)


def _alloc_bytes(n: int, device, stream=None):
    if stream is None:
        return torch.empty(n, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(n, dtype=torch.uint8, device=device)


PSK_PARTITION_AUTO, PSK_PARTITION_SEARCH, PSK_PARTITION_SCAN = 0, 1, 2


def psk_partition_csr(pos, nnz: int, tile: int, method: int = 0, tile_row=None, stream=None):
    """tile_row (int32, num_tiles+1) for the position cut of `pos` (int32 device tensor, rows+1)."""
    rows = pos.numel() - 1
    nt = max(psk_num_tiles(nnz, tile), 0)
    if tile_row is None:
        tile_row = torch.empty(nt + 1, dtype=torch.int32, device=pos.device)
    st = lib().psk_partition_csr(rows, int(nnz), _ptr(pos, torch.int32), int(tile), int(method),
                                 _ptr(tile_row, torch.int32), _stream(stream))
    _check(st, "psk_partition_csr")
    return tile_row


def psk_analyze_csr(rows, cols, nnz, pos, crd, ws=None, stream=None) -> int:
    """Suggested col_passes for psk_spmv_csr (synchronises the stream)."""
    if ws is None:
        ws = _alloc_bytes(256, pos.device, stream)
    out = ctypes.c_int32(0)
    st = lib().psk_analyze_csr(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                               _ptr(ws), ws.numel(), ctypes.byref(out), _stream(stream))
    _check(st, "psk_analyze_csr")
    return int(out.value)


def psk_validate_csr(rows, cols, nnz, pos, crd, ws=None, stream=None) -> int:
    """0 if the index structure is well formed, else the number (1..4) of the first failing condition
    (synchronises the stream)."""
    if ws is None:
        ws = _alloc_bytes(256, pos.device, stream)
    out = ctypes.c_int32(-1)
    st = lib().psk_validate_csr(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                _ptr(ws), ws.numel(), ctypes.byref(out), _stream(stream))
    _check(st, "psk_validate_csr")
    return int(out.value)


def psk_suggest_schedule_csr(rows, nnz, pos, ws=None, stream=None) -> int:
    """PSK_SCHEDULE_POSITIONS or PSK_SCHEDULE_ROWS for y = A x on this matrix (may synchronise the stream)."""
    if ws is None:
        ws = _alloc_bytes(256, pos.device, stream)
    out = ctypes.c_int32(-1)
    st = lib().psk_suggest_schedule_csr(int(rows), int(nnz), _ptr(pos, torch.int32), _ptr(ws), ws.numel(),
                                        ctypes.byref(out), _stream(stream))
    _check(st, "psk_suggest_schedule_csr")
    return int(out.value)


def psk_spmv_csr(rows, cols, nnz, pos, crd, vals, x, y, tile=0, col_passes=1, phases=PSK_PHASE_ALL, ws=None,
                 stream=None):
    if ws is None:
        _temporary_ws_ok(phases, "psk_spmv_csr")
        ws = _csr_ws(rows, nnz, tile, pos.device, stream)
    L = _lib or lib()
    st = _spmv(0, _spmv_address[0], rows, cols, nnz, pos, crd, vals, x, y, tile, col_passes, phases, ws,
               None if stream is None else stream.cuda_stream)
    if st is None:                               # something that is not a plain tensor, or no native side
        st = L.psk_spmv_csr(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                _ptr(vals, torch.float32), _ptr(x, torch.float32), _ptr(y, torch.float32), int(tile),
                                int(col_passes), int(phases), _ptr(ws), ws.numel(), _stream(stream))
    if st:
        _check(st, "psk_spmv_csr")
    return y


def psk_static_scratch_bytes() -> int:
    return int(lib().psk_static_scratch_bytes())


def psk_spmv_csr_static(rows, cols, nnz, pos, crd, vals, x, y, tile=0, col_passes=1, stream=None):
    """psk_spmv_csr without a workspace: the library's built-in scratch array is used; nothing is allocated."""
    st = lib().psk_spmv_csr_static(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                   _ptr(vals, torch.float32), _ptr(x, torch.float32), _ptr(y, torch.float32),
                                   int(tile), int(col_passes), _stream(stream))
    _check(st, "psk_spmv_csr_static")
    return y


class PreparedCall:
    """A call whose arguments are already marshalled: calling it only crosses into the library.  For loops that
    repeat one product on the same buffers and are bound by the host side of the call (small matrices)."""

    def __init__(self, fn, what, cargs, keep):
        self._fn, self._what, self._cargs, self._keep = fn, what, cargs, keep      # `keep` holds the tensors alive

    def __call__(self):
        st = self._fn(*self._cargs)
        if st != PSK_OK:
            raise PskError(st, self._what)


def psk_spmv_csr_prepared(rows, cols, nnz, pos, crd, vals, x, y, tile=0, col_passes=1, phases=PSK_PHASE_ALL, ws=None,
                          stream=None) -> PreparedCall:
    """psk_spmv_csr with the marshalling done once; the returned object repeats the call."""
    if ws is None:
        ws = _csr_ws(rows, nnz, tile, pos.device, stream)
    cargs = (int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32), _ptr(vals, torch.float32),
             _ptr(x, torch.float32), _ptr(y, torch.float32), int(tile), int(col_passes), int(phases), _ptr(ws), ws.numel(),
             _stream(stream))
    return PreparedCall(lib().psk_spmv_csr, "psk_spmv_csr", cargs, (pos, crd, vals, x, y, ws, stream))


def psk_spmm_csr(rows, cols, nnz, pos, crd, vals, B, C, tile=0, phases=PSK_PHASE_ALL, ws=None, stream=None):
    k = B.shape[1]
    if ws is None:
        _temporary_ws_ok(phases, "psk_spmm_csr")
        ws = workspace(PSK_OP_SPMM_CSR, rows, nnz, k=k, tile=tile, device=pos.device, stream=stream)
    st = lib().psk_spmm_csr(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                            _ptr(vals, torch.float32), _ptr(B, torch.float32), int(k), int(B.stride(0)),
                            _ptr(C, torch.float32), int(C.stride(0)), int(tile), int(phases), _ptr(ws),
                            ws.numel(), _stream(stream))
    _check(st, "psk_spmm_csr")
    return C


def psk_spmv_bcsr(brows, bcols, nblocks, bs, pos, crd, vals, x, y, tile=0, phases=PSK_PHASE_ALL, ws=None,
                  stream=None):
    if ws is None:
        _temporary_ws_ok(phases, "psk_spmv_bcsr")
        ws = workspace(PSK_OP_SPMV_BCSR, brows, nblocks, bs=bs, tile=tile, device=pos.device, stream=stream)
    st = lib().psk_spmv_bcsr(int(brows), int(bcols), int(nblocks), int(bs), _ptr(pos, torch.int32),
                             _ptr(crd, torch.int32), _ptr(vals, torch.float32), _ptr(x, torch.float32),
                             _ptr(y, torch.float32), int(tile), int(phases), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "psk_spmv_bcsr")
    return y


def psk_spmm_bcsr(brows, bcols, nblocks, bs, pos, crd, vals, B, C, tile=0, phases=PSK_PHASE_ALL, ws=None,
                  stream=None):
    k = B.shape[1]
    if ws is None:
        _temporary_ws_ok(phases, "psk_spmm_bcsr")
        ws = workspace(PSK_OP_SPMM_BCSR, brows, nblocks, k=k, bs=bs, tile=tile, device=pos.device, stream=stream)
    st = lib().psk_spmm_bcsr(int(brows), int(bcols), int(nblocks), int(bs), _ptr(pos, torch.int32),
                             _ptr(crd, torch.int32), _ptr(vals, torch.float32), _ptr(B, torch.float32), int(k),
                             int(B.stride(0)), _ptr(C, torch.float32), int(C.stride(0)), int(tile), int(phases),
                             _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "psk_spmm_bcsr")
    return C


def psk_partition_csf3(pos_k, pos_l, nnz: int, tile: int, stream=None):
    """(tile_slice, tile_fiber), each int32 with num_tiles+1 entries."""
    nslices, nfibers = pos_k.numel() - 1, pos_l.numel() - 1
    nt = max(psk_num_tiles(nnz, tile), 0)
    ts = torch.empty(nt + 1, dtype=torch.int32, device=pos_k.device)
    tf = torch.empty(nt + 1, dtype=torch.int32, device=pos_k.device)
    st = lib().psk_partition_csf3(nslices, nfibers, int(nnz), _ptr(pos_k, torch.int32), _ptr(pos_l, torch.int32),
                                  int(tile), _ptr(ts, torch.int32), _ptr(tf, torch.int32), _stream(stream))
    _check(st, "psk_partition_csf3")
    return ts, tf


def psk_mttkrp_csf3(dims, crd_i, pos_k, crd_k, pos_l, crd_l, vals, C, D, A, tile=0, phases=PSK_PHASE_ALL, ws=None,
                    stream=None):
    """A (dims[0] x j) = MTTKRP of the three-level tensor with C (dims[1] x j) and D (dims[2] x j)."""
    nslices, nfibers, nnz, j = pos_k.numel() - 1, pos_l.numel() - 1, crd_l.numel(), C.shape[1]
    if ws is None:
        _temporary_ws_ok(phases, "psk_mttkrp_csf3")
        ws = workspace(PSK_OP_MTTKRP_CSF3, nslices, nnz, k=j, tile=tile, device=pos_k.device, stream=stream)
    st = lib().psk_mttkrp_csf3(int(dims[0]), int(dims[1]), int(dims[2]), nslices, nfibers, nnz,
                               _ptr(crd_i, torch.int32), _ptr(pos_k, torch.int32), _ptr(crd_k, torch.int32),
                               _ptr(pos_l, torch.int32), _ptr(crd_l, torch.int32), _ptr(vals, torch.float32),
                               _ptr(C, torch.float32), int(C.stride(0)), _ptr(D, torch.float32), int(D.stride(0)),
                               int(j), _ptr(A, torch.float32), int(A.stride(0)), int(tile), int(phases), _ptr(ws),
                               ws.numel(), _stream(stream))
    _check(st, "psk_mttkrp_csf3")
    return A


def psk_spmv_csr_atomics(rows, cols, nnz, pos, crd, vals, x, y, tile=0, phases=PSK_PHASE_ALL, ws=None, stream=None):
    if ws is None:
        _temporary_ws_ok(phases, "psk_spmv_csr_atomics")
        ws = _csr_ws(rows, nnz, tile, pos.device, stream)
    st = lib().psk_spmv_csr_atomics(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                    _ptr(vals, torch.float32), _ptr(x, torch.float32), _ptr(y, torch.float32),
                                    int(tile), int(phases), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "psk_spmv_csr_atomics")
    return y


def psk_spmv_csr_f64(rows, cols, nnz, pos, crd, vals, x, y, tile=0, col_passes=1, phases=PSK_PHASE_ALL, ws=None,
                     stream=None):
    if ws is None:
        _temporary_ws_ok(phases, "psk_spmv_csr_f64")
        ws = workspace(PSK_OP_SPMV_CSR_F64, rows, nnz, tile=tile, device=pos.device, stream=stream)
    L = _lib or lib()
    st = _spmv(1, _spmv_address[1], rows, cols, nnz, pos, crd, vals, x, y, tile, col_passes, phases, ws,
               None if stream is None else stream.cuda_stream)
    if st is None:                               # something that is not a plain tensor, or no native side
        st = L.psk_spmv_csr_f64(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                    _ptr(vals, torch.float64), _ptr(x, torch.float64), _ptr(y, torch.float64),
                                    int(tile), int(col_passes), int(phases), _ptr(ws), ws.numel(), _stream(stream))
    if st:
        _check(st, "psk_spmv_csr_f64")
    return y


def psk_spmv_dcsr(rows, cols, nnz, crd_i, pos, crd, vals, x, y, cut=PSK_CUT_POSITIONS, tile=0, col_passes=1,
                  phases=PSK_PHASE_ALL, ws=None, stream=None):
    nstored = int(crd_i.numel())
    if ws is None and cut == PSK_CUT_POSITIONS:
        _temporary_ws_ok(phases, "psk_spmv_dcsr")
    if ws is None:
        n = psk_spmv_dcsr_workspace_bytes(nstored, nnz, tile)
        if n == 0:
            raise ValueError("invalid arguments for psk_spmv_dcsr_workspace_bytes")
        ws = _alloc_bytes(n, pos.device, stream)
    st = lib().psk_spmv_dcsr(int(rows), int(cols), nstored, int(nnz), _ptr(crd_i, torch.int32), _ptr(pos, torch.int32),
                             _ptr(crd, torch.int32), _ptr(vals, torch.float32), _ptr(x, torch.float32),
                             _ptr(y, torch.float32), int(cut), int(tile), int(col_passes), int(phases), _ptr(ws),
                             ws.numel(), _stream(stream))
    _check(st, "psk_spmv_dcsr")
    return y


def psk_spmv_csr_divide(rows, cols, nnz, pos, crd, vals, x, y, parts=0, phases=PSK_PHASE_ALL, ws=None, stream=None):
    if ws is None:
        if int(phases) & 6 != 6:      # no table here, but main and fix-up share the carry records
            raise ValueError("psk_spmv_csr_divide: main and fix-up on their own need a workspace that outlives the call")
        ws = _csr_ws(rows, nnz, 2048, pos.device, stream)
    st = lib().psk_spmv_csr_divide(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                   _ptr(vals, torch.float32), _ptr(x, torch.float32), _ptr(y, torch.float32),
                                   int(parts), int(phases), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "psk_spmv_csr_divide")
    return y


def psk_spmv_csr_notemp(rows, cols, nnz, pos, crd, vals, x, y, tile=0, phases=PSK_PHASE_ALL, ws=None, stream=None):
    if ws is None:
        _temporary_ws_ok(phases, "psk_spmv_csr_notemp")
        ws = _csr_ws(rows, nnz, tile, pos.device, stream)
    st = lib().psk_spmv_csr_notemp(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                   _ptr(vals, torch.float32), _ptr(x, torch.float32), _ptr(y, torch.float32),
                                   int(tile), int(phases), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "psk_spmv_csr_notemp")
    return y


def psk_spmv_csr_rowsplit(rows, cols, nnz, pos, crd, vals, x, y, variant=PSK_ROWSPLIT_WAVE_PER_ROW, stream=None):
    st = lib().psk_spmv_csr_rowsplit(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                     _ptr(vals, torch.float32), _ptr(x, torch.float32), _ptr(y, torch.float32),
                                     int(variant), _stream(stream))
    _check(st, "psk_spmv_csr_rowsplit")
    return y


def psk_spmm_csr_rowsplit(rows, cols, nnz, pos, crd, vals, B, C, stream=None):
    st = lib().psk_spmm_csr_rowsplit(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                     _ptr(vals, torch.float32), _ptr(B, torch.float32), int(B.shape[1]),
                                     int(B.stride(0)), _ptr(C, torch.float32), int(C.stride(0)), _stream(stream))
    _check(st, "psk_spmm_csr_rowsplit")
    return C


class Slab:
    """A built column-slab structure: the C struct (`desc`) plus the device memory that holds its arrays."""

    def __init__(self, desc, mem):
        self.desc, self.mem = desc, mem

    def array(self, name):
        """Device view of one array of the structure (for inspection and tests)."""
        d = self.desc
        dtype, n = {"svals": (torch.float64 if d.value_bytes == 8 else torch.float32, d.nslots), "scol": (torch.int16, d.nslots),
                    "chunk_pair": (torch.int32, d.nchunks + 1), "slab_chunk": (torch.int32, d.nslabs + 1),
                    "qpos": (torch.int32, d.rows + 1), "qidx": (torch.int32, d.nq),
                    "qtile_row": (torch.int32, psk_num_tiles(d.nq, d.tile) + 1)}[name]
        off = int(getattr(d, name)) - self.mem.data_ptr()
        size = n * torch.empty((), dtype=dtype).element_size()
        return self.mem[off:off + size].view(dtype)


def psk_slab_mem_bytes(rows, cols, nnz) -> int:
    return int(lib().psk_slab_mem_bytes(int(rows), int(cols), int(nnz)))


def psk_slab_build_workspace_bytes(rows, cols, nnz) -> int:
    return int(lib().psk_slab_build_workspace_bytes(int(rows), int(cols), int(nnz)))


def psk_slab_build_csr(rows, cols, nnz, pos, crd, vals, mem=None, ws=None, stream=None) -> Slab:
    """Builds the column-slab structure of a CSR matrix on the device (synchronises the stream)."""
    nm, nw = psk_slab_mem_bytes(rows, cols, nnz), psk_slab_build_workspace_bytes(rows, cols, nnz)
    if nm == 0 or nw == 0:
        raise PskError(5, "psk_slab_build_csr (sizes outside the limits of the slab structure)")
    if mem is None:
        mem = _alloc_bytes(nm, pos.device, stream)
    if ws is None:
        ws = _alloc_bytes(nw, pos.device, stream)
    desc = psk_slab()
    st = lib().psk_slab_build_csr(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                  _ptr(vals, torch.float32), _ptr(mem), mem.numel(), _ptr(ws), ws.numel(),
                                  ctypes.byref(desc), _stream(stream))
    _check(st, "psk_slab_build_csr")
    return Slab(desc, mem)


def psk_slab_mem_bytes_f64(rows, cols, nnz) -> int:
    return int(lib().psk_slab_mem_bytes_f64(int(rows), int(cols), int(nnz)))


def psk_slab_build_workspace_bytes_f64(rows, cols, nnz) -> int:
    return int(lib().psk_slab_build_workspace_bytes_f64(int(rows), int(cols), int(nnz)))


def psk_slab_build_csr_f64(rows, cols, nnz, pos, crd, vals, mem=None, ws=None, stream=None) -> Slab:
    """The structure with fp64 values (synchronises the stream)."""
    nm, nw = psk_slab_mem_bytes_f64(rows, cols, nnz), psk_slab_build_workspace_bytes_f64(rows, cols, nnz)
    if nm == 0 or nw == 0:
        raise PskError(5, "psk_slab_build_csr_f64 (sizes outside the limits of the slab structure)")
    if mem is None:
        mem = _alloc_bytes(nm, pos.device, stream)
    if ws is None:
        ws = _alloc_bytes(nw, pos.device, stream)
    desc = psk_slab()
    st = lib().psk_slab_build_csr_f64(int(rows), int(cols), int(nnz), _ptr(pos, torch.int32), _ptr(crd, torch.int32),
                                      _ptr(vals, torch.float64), _ptr(mem), mem.numel(), _ptr(ws), ws.numel(),
                                      ctypes.byref(desc), _stream(stream))
    _check(st, "psk_slab_build_csr_f64")
    return Slab(desc, mem)


def psk_spmv_slab_f64(S: Slab, x, y, phases=PSK_PHASE_ALL, ws=None, stream=None):
    if ws is None:
        if int(phases) != PSK_PHASE_ALL:
            raise ValueError("psk_spmv_slab_f64: a partial product needs the workspace (ws=...) of the earlier steps")
        ws = psk_slab_spmv_workspace(S, x.device if x is not None else y.device, stream)
    st = lib().psk_spmv_slab_f64(ctypes.byref(S.desc), _ptr(x, torch.float64), _ptr(y, torch.float64), int(phases), _ptr(ws),
                                 ws.numel(), _stream(stream))
    _check(st, "psk_spmv_slab_f64")
    return y


def psk_slab_spmv_workspace(S: Slab, device="cuda", stream=None):
    n = int(lib().psk_slab_spmv_workspace_bytes(ctypes.byref(S.desc)))
    return _alloc_bytes(max(n, 256), device, stream)


def psk_spmv_slab(S: Slab, x, y, phases=PSK_PHASE_ALL, ws=None, stream=None):
    if ws is None:
        if int(phases) != PSK_PHASE_ALL:
            raise ValueError("psk_spmv_slab: a partial product needs the workspace (ws=...) of the earlier steps")
        ws = psk_slab_spmv_workspace(S, x.device if x is not None else y.device, stream)
    st = lib().psk_spmv_slab(ctypes.byref(S.desc), _ptr(x, torch.float32), _ptr(y, torch.float32), int(phases), _ptr(ws), ws.numel(),
                             _stream(stream))
    _check(st, "psk_spmv_slab")
    return y


def psk_calibrate_stream_read(src, sink, stream=None):
    st = lib().psk_calibrate_stream_read(_ptr(src), src.numel() * src.element_size(), _ptr(sink, torch.float32), _stream(stream))
    _check(st, "psk_calibrate_stream_read")


def psk_calibrate_gather(table, idx, out, stream=None):
    st = lib().psk_calibrate_gather(_ptr(table, torch.float32), table.numel(), _ptr(idx, torch.int32), idx.numel(),
                                    _ptr(out, torch.float32), _stream(stream))
    _check(st, "psk_calibrate_gather")


def psk_calibrate_gather_lds(table, idx, out, stream=None):
    st = lib().psk_calibrate_gather_lds(_ptr(table, torch.float32), table.numel(), _ptr(idx, torch.int16), idx.numel(),
                                        _ptr(out, torch.float32), _stream(stream))
    _check(st, "psk_calibrate_gather_lds")


def psk_cu_trace_set(records) -> None:
    """records: int64 device tensor with 3 entries per workgroup, more than 1024 records (None switches tracing off).
    Instrumented build only."""
    n = 0 if records is None else records.numel() // 3
    st = lib().psk_cu_trace_set(_ptr(records, torch.int64) if records is not None else None, n)
    _check(st, "psk_cu_trace_set")


_TYPES = {torch.float32: PSK_F32, torch.float16: PSK_F16, torch.bfloat16: PSK_BF16}


def _type(t, what):
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise ValueError("%s: dtype %s is not one of float32, float16, bfloat16" % (what, t.dtype)) from None


def _rows(t, rows, cols, dtype, what):
    """(address, leading dimension) of a matrix of rows x cols."""
    if t.shape != (rows, cols):
        raise ValueError("%s: expected a tensor of %d x %d, got %s" % (what, rows, cols, tuple(t.shape)))
    return _ptr(t, dtype), (t.stride(0) if rows > 1 else max(t.stride(0), cols))


def _gating_ptrs(crd, vals, n, top_k, what):
    for t, dtype in ((crd, torch.int32), (vals, torch.float32)):
        if tuple(t.shape) != (n, top_k) or not t.is_contiguous():
            raise ValueError("%s: crd and vals must be contiguous tensors of %d x %d" % (what, n, top_k))
    return _ptr(crd, torch.int32), _ptr(vals, torch.float32)


def _one_device(what, *tensors):
    """A call runs on the current device: all of its tensors have to be there."""
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here and t.is_cuda:
            raise ValueError("%s: a tensor is on cuda:%d, the current device is cuda:%d" % (what, t.get_device(), here))


class Q4:
    """One or more matrices in 4 bits: the C struct (`desc`) and the tensors it points into.

    codes: uint8, rows x bytes or count x rows x bytes, two columns to a byte, the low half first; a row holds a multiple of 16
    bytes, ceil(cols / 32) * 16 at least.  scales: (count x) rows x ceil(cols / group).  zeros: uint8 laid out as the scales, or
    None for 8 everywhere."""

    def __init__(self, codes, scales, zeros=None, cols=None, group=128):
        if codes.dtype != torch.uint8 or (zeros is not None and zeros.dtype != torch.uint8):
            raise ValueError("codes and zeros must be uint8")
        if codes.dim() not in (2, 3) or scales.dim() != codes.dim():
            raise ValueError("codes and scales must both have two dimensions, or three for several matrices")
        if group < 32 or group & (group - 1):
            raise ValueError("group must be a power of two, 32 or more")
        cols = 2 * codes.shape[-1] if cols is None else int(cols)
        groups = (cols + group - 1) // group
        if cols < 0 or codes.shape[-1] < (cols + 31) // 32 * 16:
            raise ValueError("a row of codes must hold %d bytes for %d columns" % ((cols + 31) // 32 * 16, cols))
        if tuple(scales.shape) != tuple(codes.shape[:-1]) + (groups,):
            raise ValueError("scales must have the shape %s" % (tuple(codes.shape[:-1]) + (groups,),))
        if zeros is not None and (zeros.shape != scales.shape or zeros.stride() != scales.stride()):
            raise ValueError("zeros must be laid out as the scales")
        self.codes, self.scales, self.zeros = codes, scales, zeros
        d = self.desc = psk_q4()
        d.count, d.rows, d.cols, d.group, d.scale_type = codes.shape[0] if codes.dim() == 3 else 1, codes.shape[-2], cols, group, _type(scales, "scales")
        d.codes, d.scales, d.zeros = _ptr(codes, torch.uint8), _ptr(scales), _ptr(zeros)
        d.ld_codes = max(int(codes.stride(-2)), codes.shape[-1]) if codes.shape[-2] <= 1 else int(codes.stride(-2))
        d.ld_scales = max(int(scales.stride(-2)), groups) if codes.shape[-2] <= 1 else int(scales.stride(-2))
        if codes.dim() == 3 and codes.shape[0] > 1:
            d.stride_codes, d.stride_scales = int(codes.stride(0)), int(scales.stride(0))
        if any(t is not None and t.device != codes.device for t in (scales, zeros)):
            raise ValueError("codes, scales and zeros must be on one device")
        self.rows, self.cols, self._ref = d.rows, d.cols, ctypes.byref(d)      # (a field of the struct costs a call ten times as much)


def psk_gemm_q4_workspace_bytes(rows: int, cols: int, n: int, type: int) -> int:
    return int(lib().psk_gemm_q4_workspace_bytes(int(rows), int(cols), int(n), int(type)))


def psk_gemm_q4_workspace(A: Q4, X, stream=None):
    """A byte tensor that suits psk_gemm_q4 with vectors like X (n x cols)."""
    n = psk_gemm_q4_workspace_bytes(A.desc.rows, A.desc.cols, X.shape[0], _type(X, "X"))
    if n == 0:
        raise ValueError("invalid arguments for psk_gemm_q4_workspace_bytes")
    return _alloc_bytes(n, X.device, stream)


def psk_gemm_q4(A: Q4, X, Y, ws=None, stream=None):
    """Y (n x rows) = X (n x cols) A^T for one matrix in 4 bits."""
    n, dtype, type = X.shape[0], X.dtype, _type(X, "psk_gemm_q4")
    x, ldx = _rows(X, n, A.cols, dtype, "psk_gemm_q4: X")
    y, ldy = _rows(Y, n, A.rows, dtype, "psk_gemm_q4: Y")
    _one_device("psk_gemm_q4", X, Y, A.codes, ws)
    if ws is None:
        ws = psk_gemm_q4_workspace(A, X, stream)
    st = lib().psk_gemm_q4(A._ref, n, type, x, ldx, y, ldy, _ptr(ws), ws.numel(), _stream(stream))
    if st:
        _check(st, "psk_gemm_q4")
    return Y


def psk_moe_route_workspace_bytes(n: int, experts: int) -> int:
    return int(lib().psk_moe_route_workspace_bytes(int(n), int(experts)))


def psk_moe_route_workspace(n, experts, device="cuda", stream=None):
    b = psk_moe_route_workspace_bytes(n, experts)
    if b == 0:
        raise ValueError("invalid arguments for psk_moe_route_workspace_bytes")
    return _alloc_bytes(b, device, stream)


def psk_moe_route(X, W, crd, vals, score=PSK_SCORE_SOFTMAX, bias=None, normalise=True, factor=1.0, ws=None, stream=None):
    """(crd, vals): the gating matrix of the tokens X (n x dim) for the router weights W (experts x dim); top_k = crd.shape[1]."""
    n, dim, experts = X.shape[0], X.shape[1], W.shape[0]
    type, wtype, top_k = _type(X, "psk_moe_route"), _type(W, "psk_moe_route"), crd.shape[1]
    x, ldx = _rows(X, n, dim, X.dtype, "psk_moe_route: X")
    w, ldw = _rows(W, experts, dim, W.dtype, "psk_moe_route: W")
    c, v = _gating_ptrs(crd, vals, n, top_k, "psk_moe_route")
    if bias is not None and (tuple(bias.shape) != (experts,) or not bias.is_contiguous()):
        raise ValueError("psk_moe_route: bias must be a contiguous tensor of %d" % experts)
    _one_device("psk_moe_route", X, W, crd, vals, bias, ws)
    if ws is None:
        ws = psk_moe_route_workspace(n, experts, X.device, stream)
    st = lib().psk_moe_route(n, dim, experts, top_k, int(score), int(bool(normalise)), float(factor), type, x, ldx, wtype, w, ldw,
                             _ptr(bias, torch.float32), c, v, _ptr(ws), ws.numel(), _stream(stream))
    if st:
        _check(st, "psk_moe_route")
    return crd, vals


def psk_moe_workspace_bytes(n: int, dim: int, inter: int, experts: int, top_k: int) -> int:
    return int(lib().psk_moe_workspace_bytes(int(n), int(dim), int(inter), int(experts), int(top_k)))


def psk_moe_workspace(n, dim, inter, experts, top_k, device="cuda", stream=None):
    b = psk_moe_workspace_bytes(n, dim, inter, experts, top_k)
    if b == 0:
        raise ValueError("invalid arguments for psk_moe_workspace_bytes")
    return _alloc_bytes(b, device, stream)


def _experts_of(W, experts, rows, cols, dtype, what):
    """(address, leading dimension, stride between experts)."""
    if tuple(W.shape) != (experts, rows, cols):
        raise ValueError("%s: expected a tensor of %d x %d x %d, got %s" % (what, experts, rows, cols, tuple(W.shape)))
    return _ptr(W, dtype), (int(W.stride(1)) if rows > 1 else (cols + 7) // 8 * 8), (int(W.stride(0)) if experts > 1 else 0)


def psk_moe_experts(X, crd, vals, W1, W3, W2, Y, act=PSK_ACT_SILU, ws=None, stream=None):
    """Y (n x dim) = the layer for the tokens X with the gating matrix (crd, vals), weights of the type of X: W1, W3 experts x inter x dim
    (strided alike), W2 experts x dim x inter."""
    n, dim = X.shape
    experts, inter = W1.shape[0], W1.shape[1]
    type, top_k = _type(X, "psk_moe_experts"), crd.shape[1]
    x, ldx = _rows(X, n, dim, X.dtype, "psk_moe_experts: X")
    y, ldy = _rows(Y, n, dim, X.dtype, "psk_moe_experts: Y")
    c, v = _gating_ptrs(crd, vals, n, top_k, "psk_moe_experts")
    w1, ld1, stride1 = _experts_of(W1, experts, inter, dim, X.dtype, "psk_moe_experts: W1")
    w3, ld3, stride3 = _experts_of(W3, experts, inter, dim, X.dtype, "psk_moe_experts: W3")
    w2, ld2, stride2 = _experts_of(W2, experts, dim, inter, X.dtype, "psk_moe_experts: W2")
    if (ld1, stride1) != (ld3, stride3):
        raise ValueError("psk_moe_experts: W1 and W3 must have the same strides")
    _one_device("psk_moe_experts", X, crd, vals, W1, W3, W2, Y, ws)
    if ws is None:
        ws = psk_moe_workspace(n, dim, inter, experts, top_k, X.device, stream)
    st = lib().psk_moe_experts(n, dim, inter, experts, top_k, int(act), type, x, ldx, c, v, w1, w3, ld1, stride1, w2, ld2, stride2, y, ldy,
                               _ptr(ws), ws.numel(), _stream(stream))
    if st:
        _check(st, "psk_moe_experts")
    return Y


def psk_moe_experts_q4(X, crd, vals, W1: Q4, W3: Q4, W2: Q4, Y, act=PSK_ACT_SILU, ws=None, stream=None):
    """The layer with weights in 4 bits."""
    n, dim = X.shape
    type, top_k = _type(X, "psk_moe_experts_q4"), crd.shape[1]
    x, ldx = _rows(X, n, W1.cols, X.dtype, "psk_moe_experts_q4: X")
    y, ldy = _rows(Y, n, W2.rows, X.dtype, "psk_moe_experts_q4: Y")
    c, v = _gating_ptrs(crd, vals, n, top_k, "psk_moe_experts_q4")
    _one_device("psk_moe_experts_q4", X, crd, vals, Y, W1.codes, W3.codes, W2.codes, ws)
    if ws is None:
        ws = psk_moe_workspace(n, dim, W1.desc.rows, W1.desc.count, top_k, X.device, stream)
    st = lib().psk_moe_experts_q4(n, top_k, int(act), type, x, ldx, c, v, W1._ref, W3._ref, W2._ref, y,
                                  ldy, _ptr(ws), ws.numel(), _stream(stream))
    if st:
        _check(st, "psk_moe_experts_q4")
    return Y


class I8:
    """A matrix in 8 bits with a scale per row: the C struct (`desc`) and the tensors it points into.

    codes: int8, rows x bytes, a row begins at a multiple of 16 bytes and holds ceil(cols / 16) * 16 at least.  scales: float32, rows.
    psk_quant_i8 makes both from weights (row by row), or from tokens."""

    def __init__(self, codes, scales, cols=None):
        if codes.dtype != torch.int8 or scales.dtype != torch.float32:
            raise ValueError("codes must be int8 and scales float32")
        if codes.dim() != 2 or tuple(scales.shape) != (codes.shape[0],) or not scales.is_contiguous():
            raise ValueError("codes must have two dimensions, and scales must be a contiguous tensor of one per row")
        cols = codes.shape[1] if cols is None else int(cols)
        if cols < 0 or codes.shape[1] < (cols + 15) // 16 * 16:
            raise ValueError("a row of codes must hold %d bytes for %d columns" % ((cols + 15) // 16 * 16, cols))
        if scales.device != codes.device:
            raise ValueError("codes and scales must be on one device")
        self.codes, self.scales = codes, scales
        d = self.desc = psk_i8()
        d.rows, d.cols, d.ld = codes.shape[0], cols, _ld_codes(codes)
        d.codes, d.scales = _ptr(codes, torch.int8), _ptr(scales, torch.float32)
        self.rows, self.cols, self._ref = d.rows, d.cols, ctypes.byref(d)


def _ld_codes(codes):
    return int(codes.stride(0)) if codes.shape[0] > 1 else (max(int(codes.stride(0)), codes.shape[1]) + 15) // 16 * 16


def _vector(t, n, dtype, what):
    """Address of a contiguous vector of n."""
    if t is not None and (t.shape != (n,) or not t.is_contiguous()):
        raise ValueError("%s: expected a contiguous tensor of %d, got %s" % (what, n, tuple(t.shape)))
    return _ptr(t, dtype)


def psk_quant_i8(X, codes, scales, stream=None):
    """(codes, scales): the rows of X (n x cols) in 8 bits; codes int8 of n x bytes, whose rows hold ceil(cols / 16) * 16 bytes at least (I8)."""
    if X.dim() != 2 or codes.dim() != 2:
        raise ValueError("psk_quant_i8: X and codes must have two dimensions")
    n, cols = X.shape
    x, ldx = _rows(X, n, cols, X.dtype, "psk_quant_i8: X")
    if codes.shape[0] != n or codes.shape[1] < (cols + 15) // 16 * 16:
        raise ValueError("psk_quant_i8: codes must have %d rows of %d bytes at least" % (n, (cols + 15) // 16 * 16))
    s = _vector(scales, n, torch.float32, "psk_quant_i8: scales")
    _one_device("psk_quant_i8", X, codes, scales)
    st = lib().psk_quant_i8(n, cols, _type(X, "psk_quant_i8"), x, ldx, _ptr(codes, torch.int8), _ld_codes(codes), s, _stream(stream))
    if st:
        _check(st, "psk_quant_i8")
    return codes, scales


def psk_gemm_i8_workspace_bytes(rows: int, cols: int, n: int) -> int:
    return int(lib().psk_gemm_i8_workspace_bytes(int(rows), int(cols), int(n)))


def psk_gemm_i8_workspace(A: I8, n: int, stream=None):
    """A byte tensor that suits psk_gemm_i8 with n tokens."""
    b = psk_gemm_i8_workspace_bytes(A.rows, A.cols, n)
    if b == 0:
        raise ValueError("invalid arguments for psk_gemm_i8_workspace_bytes")
    return _alloc_bytes(b, A.codes.device, stream)


def psk_gemm_i8(A: I8, X, scales, Y, bias=None, ws=None, stream=None):
    """Y (n x rows) = X A^T for tokens in 8 bits: X int8 of n x bytes (as the codes of I8) and a scale per token."""
    n, type = Y.shape[0], _type(Y, "psk_gemm_i8")
    if X.dim() != 2 or X.shape[0] != n or X.shape[1] < (A.cols + 15) // 16 * 16:
        raise ValueError("psk_gemm_i8: X must have %d rows of %d bytes at least" % (n, (A.cols + 15) // 16 * 16))
    y, ldy = _rows(Y, n, A.rows, Y.dtype, "psk_gemm_i8: Y")
    s, b = _vector(scales, n, torch.float32, "psk_gemm_i8: scales"), _vector(bias, A.rows, torch.float32, "psk_gemm_i8: bias")
    _one_device("psk_gemm_i8", X, scales, Y, A.codes, bias, ws)
    if ws is None:
        ws = psk_gemm_i8_workspace(A, n, stream)
    st = lib().psk_gemm_i8(A._ref, n, _ptr(X, torch.int8), _ld_codes(X), s, b, type, y, ldy, _ptr(ws), ws.numel(), _stream(stream))
    if st:
        _check(st, "psk_gemm_i8")
    return Y


def psk_linear_i8_workspace_bytes(rows: int, cols: int, n: int, type: int) -> int:
    return int(lib().psk_linear_i8_workspace_bytes(int(rows), int(cols), int(n), int(type)))


def psk_linear_i8_workspace(A: I8, X, stream=None):
    """A byte tensor that suits psk_linear_i8 with tokens like X (n x cols)."""
    b = psk_linear_i8_workspace_bytes(A.rows, A.cols, X.shape[0], _type(X, "X"))
    if b == 0:
        raise ValueError("invalid arguments for psk_linear_i8_workspace_bytes")
    return _alloc_bytes(b, X.device, stream)


def psk_linear_i8(A: I8, X, Y, bias=None, ws=None, stream=None):
    """Y (n x rows) = X (n x cols) A^T, the tokens quantised in the call."""
    n, dtype = X.shape[0], X.dtype
    type = _type(X, "psk_linear_i8")
    x, ldx = _rows(X, n, A.cols, dtype, "psk_linear_i8: X")
    y, ldy = _rows(Y, n, A.rows, dtype, "psk_linear_i8: Y")
    b = None if bias is None else _vector(bias, A.rows, torch.float32, "psk_linear_i8: bias")
    _one_device("psk_linear_i8", X, Y, A.codes, bias, ws)
    if ws is None:
        ws = psk_linear_i8_workspace(A, X, stream)
    st = lib().psk_linear_i8(A._ref, n, type, x, ldx, b, y, ldy, _ptr(ws), ws.numel(), _stream(stream))
    if st:
        _check(st, "psk_linear_i8")
    return Y


def psk_embed(ids, E, Y, factor=1.0, stream=None):
    """Y (n x dim) = factor * the rows of E that the tokens `ids` (int32, n) name, zeros for a token outside the table.  E: rows x dim of
    any of the three types, or an I8."""
    n, ytype = Y.shape[0], _type(Y, "psk_embed")
    i = _vector(ids, n, torch.int32, "psk_embed: ids")
    if isinstance(E, I8):
        y, ldy = _rows(Y, n, E.cols, Y.dtype, "psk_embed: Y")
        _one_device("psk_embed", ids, E.codes, Y)
        st = lib().psk_embed_i8(E._ref, n, i, float(factor), ytype, y, ldy, _stream(stream))
    else:
        rows, dim = E.shape
        y, ldy = _rows(Y, n, dim, Y.dtype, "psk_embed: Y")
        e, lde = _rows(E, rows, dim, E.dtype, "psk_embed: E")
        _one_device("psk_embed", ids, E, Y)
        st = lib().psk_embed(n, rows, dim, i, float(factor), _type(E, "psk_embed"), e, lde, ytype, y, ldy, _stream(stream))
    if st:
        _check(st, "psk_embed")
    return Y


def psk_embed_grad_workspace_bytes(n: int, rows: int, dim: int) -> int:
    return int(lib().psk_embed_grad_workspace_bytes(int(n), int(rows), int(dim)))


def psk_embed_grad_workspace(dY, dE, stream=None):
    """A byte tensor that suits psk_embed_grad with gradients like dY (n x dim) and dE (rows x dim)."""
    b = psk_embed_grad_workspace_bytes(dY.shape[0], dE.shape[0], dE.shape[1])
    if b == 0:
        raise ValueError("invalid arguments for psk_embed_grad_workspace_bytes")
    return _alloc_bytes(b, dE.device, stream)


def psk_embed_grad(ids, dY, dE, factor=1.0, padding=-1, accumulate=False, ws=None, stream=None):
    """dE (rows x dim) = (dE if accumulate) + factor * the sums of the rows of dY (n x dim) whose tokens are the same, in an order that
    depends on the sizes, the type of dY and the tokens alone.  Tokens outside the table, and those equal to `padding`, add nothing."""
    (n, dim), rows = dY.shape, dE.shape[0]
    type, gtype = _type(dY, "psk_embed_grad"), _type(dE, "psk_embed_grad")
    i = _vector(ids, n, torch.int32, "psk_embed_grad: ids")
    y, ldy = _rows(dY, n, dim, dY.dtype, "psk_embed_grad: dY")
    e, lde = _rows(dE, rows, dim, dE.dtype, "psk_embed_grad: dE")
    _one_device("psk_embed_grad", ids, dY, dE, ws)
    if ws is None:
        ws = psk_embed_grad_workspace(dY, dE, stream)
    st = lib().psk_embed_grad(n, rows, dim, i, int(padding), float(factor), type, y, ldy, gtype, e, lde, int(bool(accumulate)), _ptr(ws), ws.numel(),
                              _stream(stream))
    if st:
        _check(st, "psk_embed_grad")
    return dE
