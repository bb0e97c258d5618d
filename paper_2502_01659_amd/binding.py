"""ctypes binding of libsga.so: argument marshalling only.

The `sga_*` functions mirror the C entry points one to one (raw addresses and
sizes in, status code out).  The un-prefixed helpers take torch tensors, check
shapes, allocate outputs and raise SgaError on a non-zero status.  There is no
CPU fallback: if the library is missing or cannot be built, loading raises.
"""
import ctypes
import os

from sga_inputs.masks import MaskSpec

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("SGA_LIB", os.path.join(_HERE, "libsga.so"))
_lib = None

PATH_AUTO, PATH_GATHER, PATH_TILE, PATH_TILE_SPLIT = 0, 1, 2, 3
_DTYPE_CODE = {"f32": 0, "f16": 1}


class SgaError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {sga_status_string(status)} (status {status})")


class _MaskDesc(ctypes.Structure):
    _fields_ = [
        ("struct_bytes", ctypes.c_uint32), ("kind", ctypes.c_int32),
        ("L", ctypes.c_int64), ("window", ctypes.c_int32), ("stride", ctypes.c_int32),
        ("n_global", ctypes.c_int32), ("block", ctypes.c_int32),
        ("window_blocks", ctypes.c_int32), ("n_global_blocks", ctypes.c_int32),
        ("n_random_blocks", ctypes.c_int32), ("seed", ctypes.c_uint64),
    ]


class GraphPlan(ctypes.Structure):
    """sga_graph_plan: host record of a prepared tile graph (see include/sga.h)."""
    _fields_ = [
        ("struct_bytes", ctypes.c_uint32), ("magic", ctypes.c_uint32),
        ("L", ctypes.c_int64), ("nnz", ctypes.c_int64),
        ("H", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("tiles_left", ctypes.c_uint32), ("multi_tiles", ctypes.c_uint32),
        ("tile_parts", ctypes.c_uint32), ("long_rows", ctypes.c_uint32),
        ("row_chunks", ctypes.c_uint32), ("flags", ctypes.c_uint32),
        ("row_ptr", ctypes.c_void_p), ("col_idx", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("head_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class _RotaryDesc(ctypes.Structure):
    _fields_ = [("struct_bytes", ctypes.c_uint32), ("layout", ctypes.c_int32), ("channels", ctypes.c_int32),
                ("magnitude", ctypes.c_float), ("frequencies", ctypes.c_void_p)]


class _PagedBatch(ctypes.Structure):
    _fields_ = [("struct_bytes", ctypes.c_uint32), ("n_seqs", ctypes.c_int32), ("n_tokens", ctypes.c_int64),
                ("n_pages", ctypes.c_int64), ("page_stride", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("pages_per_seq", ctypes.c_int32), ("page_table", ctypes.c_void_p), ("seq_ptr", ctypes.c_void_p),
                ("seq_len", ctypes.c_void_p)]


GRAPH_TILES_COVER_ALL, GRAPH_TILE_PARTS_FIT, GRAPH_ROW_CHUNKS_FIT, GRAPH_ROWS_SHARE_KEYS, GRAPH_ROWS_EVEN = 1, 2, 4, 8, 16


def lib_path():
    return _LIB_PATH


def load():
    """Load libsga.so (building it first only if no built library exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        from .build import build_lib
        build_lib()
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    P = ctypes.POINTER
    lib.sga_status_string.restype = ctypes.c_char_p
    lib.sga_status_string.argtypes = [ctypes.c_int]
    lib.sga_mask_nnz.restype = ctypes.c_int
    lib.sga_mask_nnz.argtypes = [P(_MaskDesc), P(ctypes.c_int64)]
    lib.sga_build_mask.restype = ctypes.c_int
    lib.sga_build_mask.argtypes = [P(_MaskDesc), vp, vp, i64, vp]
    lib.sga_validate_csr.restype = ctypes.c_int
    lib.sga_validate_csr.argtypes = [vp, vp, i64, i64, vp, P(ctypes.c_int64), vp]
    lib.sga_workspace_bytes.restype = ctypes.c_int
    lib.sga_workspace_bytes.argtypes = [i64, i32, i32, i32, i64, P(ctypes.c_size_t)]
    lib.sga_attention_forward.restype = ctypes.c_int
    lib.sga_attention_forward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, i32, f32, vp,
                                          i32, vp, vp, ctypes.c_size_t, i32]
    lib.sga_attention_forward_implicit.restype = ctypes.c_int
    lib.sga_attention_forward_implicit.argtypes = [vp, vp, vp, P(_MaskDesc), vp, i64, i32, i32,
                                                   f32, vp, i32, vp, vp, ctypes.c_size_t, i32]
    lib.sga_attention_accumulate.restype = ctypes.c_int
    lib.sga_attention_accumulate.argtypes = lib.sga_attention_forward.argtypes
    lib.sga_attention_accumulate_implicit.restype = ctypes.c_int
    lib.sga_attention_accumulate_implicit.argtypes = lib.sga_attention_forward_implicit.argtypes
    lib.sga_graph_prepare.restype = ctypes.c_int
    lib.sga_graph_prepare.argtypes = [vp, vp, i64, i32, i32, i32, vp, ctypes.c_size_t, vp, P(GraphPlan)]
    lib.sga_attention_forward_prepared.restype = ctypes.c_int
    lib.sga_attention_forward_prepared.argtypes = lib.sga_attention_forward.argtypes + [P(GraphPlan)]
    lib.sga_attention_accumulate_prepared.restype = ctypes.c_int
    lib.sga_attention_accumulate_prepared.argtypes = lib.sga_attention_forward.argtypes + [P(GraphPlan)]
    lib.sga_profile_enable.restype = ctypes.c_int
    lib.sga_profile_enable.argtypes = [i32]
    lib.sga_profile_collect.restype = ctypes.c_int
    lib.sga_profile_collect.argtypes = [P(ctypes.c_float), i32, P(ctypes.c_int32)]
    lib.sga_static_scratch_init.restype = ctypes.c_int
    lib.sga_static_scratch_init.argtypes = []
    lib.sga_static_scratch_bytes.restype = ctypes.c_size_t
    lib.sga_static_scratch_bytes.argtypes = []
    lib.sga_attention_forward_static.restype = ctypes.c_int
    lib.sga_attention_forward_static.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, i32, f32, vp,
                                                 i32, vp, i64, i32]
    rows, batch, rotary_desc = P(_Rows), P(_PagedBatch), P(_RotaryDesc)
    lib.sga_rotary.restype = ctypes.c_int
    lib.sga_rotary.argtypes = [rows, rows, vp, i64, i64, i32, i32, rotary_desc, i32, i32, vp]
    lib.sga_cache_append.restype = ctypes.c_int
    lib.sga_cache_append.argtypes = [rows, rows, vp, vp, batch, i32, i32, rotary_desc, rows, rows, i32, i32, vp]
    lib.sga_paged_workspace_bytes.restype = ctypes.c_int
    lib.sga_paged_workspace_bytes.argtypes = [batch, P(_MaskDesc), i32, i32, i32, i32, P(ctypes.c_size_t)]
    lib.sga_attention_paged.restype = ctypes.c_int
    lib.sga_attention_paged.argtypes = [rows, vp, vp, batch, P(_MaskDesc), i32, rows, i32, i32, i32, f32, i32, vp, vp,
                                        ctypes.c_size_t, vp]
    lib.sga_profile_last_kernel.restype = ctypes.c_char_p
    lib.sga_profile_last_kernel.argtypes = []
    _lib = lib
    return lib


def _desc(spec: MaskSpec) -> _MaskDesc:
    return _MaskDesc(ctypes.sizeof(_MaskDesc), spec.kind, spec.L, spec.window, spec.stride,
                     spec.n_global, spec.block, spec.window_blocks, spec.n_global_blocks,
                     spec.n_random_blocks, spec.seed & ((1 << 64) - 1))


# ---- raw entry points (same names and argument order as include/sga.h) ----------
def sga_status_string(status):
    return load().sga_status_string(int(status)).decode()


def sga_mask_nnz(spec: MaskSpec):
    """-> (status, nnz)"""
    d = _desc(spec)
    out = ctypes.c_int64(0)
    st = load().sga_mask_nnz(ctypes.byref(d), ctypes.byref(out))
    return st, out.value


def sga_build_mask(spec: MaskSpec, row_ptr_addr, col_idx_addr, col_capacity, stream):
    d = _desc(spec)
    return load().sga_build_mask(ctypes.byref(d), row_ptr_addr, col_idx_addr, col_capacity, stream)


def sga_validate_csr(row_ptr_addr, col_idx_addr, L, col_capacity, scratch_addr, stream):
    """-> (status, bad_row)"""
    bad = ctypes.c_int64(-2)
    st = load().sga_validate_csr(row_ptr_addr, col_idx_addr, L, col_capacity, scratch_addr, ctypes.byref(bad), stream)
    return st, bad.value


def sga_workspace_bytes(L, H, d, dtype_code, nnz):
    """-> (status, bytes)"""
    out = ctypes.c_size_t(0)
    st = load().sga_workspace_bytes(L, H, d, dtype_code, nnz, ctypes.byref(out))
    return st, out.value


def sga_attention_forward(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype_code,
                          lse, workspace, workspace_bytes_, path):
    return load().sga_attention_forward(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream,
                                        dtype_code, lse, workspace, workspace_bytes_, path)


def sga_attention_forward_implicit(Q, K, V, spec, O, L, H, d, scale, stream, dtype_code, lse,
                                   workspace, workspace_bytes_, path):
    dsc = _desc(spec)
    return load().sga_attention_forward_implicit(Q, K, V, ctypes.byref(dsc), O, L, H, d, scale,
                                                 stream, dtype_code, lse, workspace,
                                                 workspace_bytes_, path)


def sga_attention_accumulate(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype_code,
                             lse, workspace, workspace_bytes_, path):
    return load().sga_attention_accumulate(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream,
                                           dtype_code, lse, workspace, workspace_bytes_, path)


def sga_attention_accumulate_implicit(Q, K, V, spec, O, L, H, d, scale, stream, dtype_code, lse,
                                      workspace, workspace_bytes_, path):
    dsc = _desc(spec)
    return load().sga_attention_accumulate_implicit(Q, K, V, ctypes.byref(dsc), O, L, H, d, scale,
                                                    stream, dtype_code, lse, workspace,
                                                    workspace_bytes_, path)


def sga_graph_prepare(row_ptr, col_idx, L, H, d, dtype_code, workspace, workspace_bytes_, stream):
    """-> (status, GraphPlan)"""
    plan = GraphPlan()
    st = load().sga_graph_prepare(row_ptr, col_idx, L, H, d, dtype_code, workspace, workspace_bytes_,
                                  stream, ctypes.byref(plan))
    return st, plan


def sga_attention_forward_prepared(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype_code,
                                   lse, workspace, workspace_bytes_, path, plan):
    return load().sga_attention_forward_prepared(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream,
                                                 dtype_code, lse, workspace, workspace_bytes_, path,
                                                 ctypes.byref(plan))


def sga_attention_accumulate_prepared(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream,
                                      dtype_code, lse, workspace, workspace_bytes_, path, plan):
    return load().sga_attention_accumulate_prepared(Q, K, V, row_ptr, col_idx, O, L, H, d, scale,
                                                    stream, dtype_code, lse, workspace,
                                                    workspace_bytes_, path, ctypes.byref(plan))


def sga_static_scratch_init():
    return load().sga_static_scratch_init()


def sga_static_scratch_bytes():
    return int(load().sga_static_scratch_bytes())


def sga_attention_forward_static(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream, dtype_code,
                                 lse, nnz, path):
    return load().sga_attention_forward_static(Q, K, V, row_ptr, col_idx, O, L, H, d, scale, stream,
                                               dtype_code, lse, nnz, path)


def sga_profile_enable(on):
    return load().sga_profile_enable(int(on))


def sga_profile_collect(capacity=4096):
    """-> (status, [kernel durations in ms])"""
    buf = (ctypes.c_float * capacity)()
    n = ctypes.c_int32(0)
    st = load().sga_profile_collect(buf, capacity, ctypes.byref(n))
    return st, [buf[i] for i in range(min(n.value, capacity))]


def sga_profile_last_kernel():
    return load().sga_profile_last_kernel().decode()


def sga_rotary(X, Y, positions, first, L, H, d, rotary_desc, inverse, dtype_code, stream):
    """X, Y: _Rows or None; rotary_desc: _RotaryDesc or None"""
    return load().sga_rotary(X, Y, positions, first, L, H, d, rotary_desc, inverse, dtype_code, stream)


def sga_cache_append(K, V, cache_k, cache_v, batch, Hkv, d, rotary_desc, Q, Q_out, Hq, dtype_code, stream):
    return load().sga_cache_append(K, V, cache_k, cache_v, batch, Hkv, d, rotary_desc, Q, Q_out, Hq, dtype_code, stream)


def sga_paged_workspace_bytes(batch, spec: MaskSpec, Hq, Hkv, d, dtype_code):
    """-> (status, bytes)"""
    out = ctypes.c_size_t(0)
    st = load().sga_paged_workspace_bytes(batch, _desc(spec), Hq, Hkv, d, dtype_code, ctypes.byref(out))
    return st, out.value


def sga_attention_paged(Q, cache_k, cache_v, batch, spec, causal, O, Hq, Hkv, d, scale, dtype_code, lse, workspace,
                        workspace_bytes_, stream):
    return load().sga_attention_paged(Q, cache_k, cache_v, batch, _desc(spec), causal, O, Hq, Hkv, d, scale, dtype_code, lse,
                                      workspace, workspace_bytes_, stream)


# ---- tensor-level helpers ---------------------------------------------------------
def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return 0
    if t.dtype == torch.float16:
        return 1
    raise TypeError(f"unsupported storage dtype {t.dtype}")


def mask_nnz(spec: MaskSpec) -> int:
    st, n = sga_mask_nnz(spec)
    if st != 0:
        raise SgaError(st, "sga_mask_nnz")
    return n


def build_mask(spec: MaskSpec, device="cuda"):
    """Build the CSR of the mask on `device`.  Returns (row_ptr int64 [L+1], col_idx int32 [nnz])."""
    import torch
    nnz = mask_nnz(spec)
    row_ptr = torch.empty(spec.L + 1, dtype=torch.int64, device=device)
    col_idx = torch.empty(max(nnz, 1), dtype=torch.int32, device=device)
    with torch.cuda.device(row_ptr.device):
        st = sga_build_mask(spec, row_ptr.data_ptr(), col_idx.data_ptr(), col_idx.numel(), _stream())
    if st != 0:
        raise SgaError(st, "sga_build_mask")
    return row_ptr, col_idx[:nnz]


def validate_csr(row_ptr, col_idx) -> int:
    """-1 if (row_ptr, col_idx) is a valid mask for the forward calls, else the smallest row that
    breaks the contract (L if row_ptr[0] or row_ptr[L] does).  Waits for the current stream."""
    import torch
    if not (row_ptr.is_cuda and col_idx.is_cuda and row_ptr.device == col_idx.device):
        raise ValueError("row_ptr and col_idx must be tensors of one device")
    if row_ptr.dtype != torch.int64 or col_idx.dtype != torch.int32 or row_ptr.dim() != 1 or col_idx.dim() != 1:
        raise ValueError("row_ptr must be int64 [L+1], col_idx int32 [nnz]")
    if not (row_ptr.is_contiguous() and col_idx.is_contiguous()) or row_ptr.numel() < 2:
        raise ValueError("row_ptr and col_idx must be contiguous, L >= 1")
    scratch = torch.empty(2, dtype=torch.int64, device=row_ptr.device)
    with torch.cuda.device(row_ptr.device):
        st, bad = sga_validate_csr(row_ptr.data_ptr(), _col_ptr(row_ptr, col_idx), row_ptr.numel() - 1,
                                   col_idx.numel(), scratch.data_ptr(), _stream())
    if st != 0 and bad < 0:
        raise SgaError(st, "sga_validate_csr")
    return bad


def workspace_bytes(L, H, d, dtype, nnz=-1) -> int:
    st, n = sga_workspace_bytes(L, H, d, _DTYPE_CODE[dtype] if isinstance(dtype, str) else dtype, nnz)
    if st != 0:
        raise SgaError(st, "sga_workspace_bytes")
    return n


def alloc_workspace(L, H, d, dtype, nnz=-1, device="cuda"):
    import torch
    n = workspace_bytes(L, H, d, dtype, nnz)
    return torch.empty(n, dtype=torch.uint8, device=device)


def _check_qkv(Q, K, V):
    if not (Q.is_cuda and K.is_cuda and V.is_cuda):
        raise ValueError("Q, K, V must be device tensors")
    if Q.dim() != 3 or Q.shape != K.shape or Q.shape != V.shape:
        raise ValueError("Q, K, V must all be [H, L, d]")
    if not (Q.is_contiguous() and K.is_contiguous() and V.is_contiguous()):
        raise ValueError("Q, K, V must be contiguous")
    if not (Q.dtype == K.dtype == V.dtype):
        raise ValueError("Q, K, V must share a dtype")


def _col_ptr(row_ptr, col_idx):
    # a mask without edges has an empty col_idx, whose address is null; the entry points want a
    # device address even though they will not read through it
    return col_idx.data_ptr() if col_idx.numel() > 0 else row_ptr.data_ptr()


def _check_csr(Q, row_ptr, col_idx):
    import torch
    L = Q.shape[1]
    if row_ptr.dtype != torch.int64 or row_ptr.numel() != L + 1 or not row_ptr.is_contiguous():
        raise ValueError("row_ptr must be contiguous int64 [L+1]")
    if col_idx.dtype != torch.int32 or not col_idx.is_contiguous():
        raise ValueError("col_idx must be contiguous int32")
    if row_ptr.device != Q.device or (col_idx.numel() > 0 and col_idx.device != Q.device):
        raise ValueError("row_ptr and col_idx must be on Q's device")


def _check_outputs(Q, O, lse, workspace):
    """Caller-supplied output and scratch buffers: the kernels write H*L*d elements of O and H*L
    floats of lse without further checks, so a wrong shape here would be an out-of-bounds write."""
    import torch
    H, L, d = Q.shape
    if O is not None and (O.shape != Q.shape or O.dtype != Q.dtype or not O.is_contiguous()
                          or O.device != Q.device):
        raise ValueError("O must match Q in shape, dtype and device, and be contiguous")
    if lse is not None and (lse.shape != (H, L) or lse.dtype != torch.float32
                            or not lse.is_contiguous() or lse.device != Q.device):
        raise ValueError("lse must be contiguous float32 [H, L] on Q's device")
    if workspace is not None and (workspace.device != Q.device or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous tensor on Q's device")


def attention_forward(Q, K, V, row_ptr, col_idx, scale, O=None, lse=None, workspace=None,
                      path=PATH_AUTO, want_lse=False):
    """Masked attention over an explicit CSR mask.  Returns O (and lse if requested)."""
    import torch
    _check_qkv(Q, K, V)
    H, L, d = Q.shape
    _check_csr(Q, row_ptr, col_idx)
    _check_outputs(Q, O, lse, workspace)
    if O is None:
        O = torch.empty_like(Q)
    if want_lse and lse is None:
        lse = torch.empty((H, L), dtype=torch.float32, device=Q.device)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_n = workspace.numel() * workspace.element_size() if workspace is not None else 0
    with torch.cuda.device(Q.device):
        st = sga_attention_forward(Q.data_ptr(), K.data_ptr(), V.data_ptr(), row_ptr.data_ptr(),
                                   _col_ptr(row_ptr, col_idx), O.data_ptr(), L, H, d, float(scale),
                                   _stream(), _dtype_code(Q),
                                   lse.data_ptr() if lse is not None else None, ws_ptr, ws_n, path)
    if st != 0:
        raise SgaError(st, "sga_attention_forward")
    return (O, lse) if (want_lse or lse is not None) else O


def attention_forward_implicit(Q, K, V, spec: MaskSpec, scale, O=None, lse=None, workspace=None,
                               path=PATH_AUTO, want_lse=False):
    """Masked attention with neighbours generated in the kernel (sliding / dilated windows)."""
    import torch
    _check_qkv(Q, K, V)
    H, L, d = Q.shape
    _check_outputs(Q, O, lse, workspace)
    if O is None:
        O = torch.empty_like(Q)
    if want_lse and lse is None:
        lse = torch.empty((H, L), dtype=torch.float32, device=Q.device)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_n = workspace.numel() * workspace.element_size() if workspace is not None else 0
    with torch.cuda.device(Q.device):
        st = sga_attention_forward_implicit(Q.data_ptr(), K.data_ptr(), V.data_ptr(), spec,
                                            O.data_ptr(), L, H, d, float(scale), _stream(),
                                            _dtype_code(Q),
                                            lse.data_ptr() if lse is not None else None,
                                            ws_ptr, ws_n, path)
    if st != 0:
        raise SgaError(st, "sga_attention_forward_implicit")
    return (O, lse) if (want_lse or lse is not None) else O


def _check_state(Q, O, lse):
    import torch
    H, L, d = Q.shape
    if O.shape != Q.shape or O.dtype != Q.dtype or not O.is_contiguous() or O.device != Q.device:
        raise ValueError("O must match Q in shape, dtype and device")
    if (lse.shape != (H, L) or lse.dtype != torch.float32 or not lse.is_contiguous()
            or lse.device != Q.device):
        raise ValueError("lse must be contiguous float32 [H, L] on Q's device")


def attention_accumulate(Q, K, V, row_ptr, col_idx, scale, O, lse, workspace=None, path=PATH_AUTO):
    """Continue the (O, lse) state over the edges of an explicit CSR mask, in place."""
    import torch
    _check_qkv(Q, K, V)
    _check_state(Q, O, lse)
    H, L, d = Q.shape
    _check_csr(Q, row_ptr, col_idx)
    _check_outputs(Q, None, None, workspace)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_n = workspace.numel() * workspace.element_size() if workspace is not None else 0
    with torch.cuda.device(Q.device):
        st = sga_attention_accumulate(Q.data_ptr(), K.data_ptr(), V.data_ptr(), row_ptr.data_ptr(),
                                      _col_ptr(row_ptr, col_idx), O.data_ptr(), L, H, d, float(scale),
                                      _stream(), _dtype_code(Q), lse.data_ptr(), ws_ptr, ws_n, path)
    if st != 0:
        raise SgaError(st, "sga_attention_accumulate")
    return O, lse


def attention_accumulate_implicit(Q, K, V, spec: MaskSpec, scale, O, lse, workspace=None,
                                  path=PATH_AUTO):
    """Continue the (O, lse) state over the edges of an implicit mask, in place."""
    import torch
    _check_qkv(Q, K, V)
    _check_state(Q, O, lse)
    H, L, d = Q.shape
    _check_outputs(Q, None, None, workspace)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_n = workspace.numel() * workspace.element_size() if workspace is not None else 0
    with torch.cuda.device(Q.device):
        st = sga_attention_accumulate_implicit(Q.data_ptr(), K.data_ptr(), V.data_ptr(), spec,
                                               O.data_ptr(), L, H, d, float(scale), _stream(),
                                               _dtype_code(Q), lse.data_ptr(), ws_ptr, ws_n, path)
    if st != 0:
        raise SgaError(st, "sga_attention_accumulate_implicit")
    return O, lse


def graph_prepare(row_ptr, col_idx, H, d, dtype, workspace):
    """Prepare the tile graph of an explicit mask once (waits for the stream).  Returns the
    GraphPlan to pass to attention_forward_prepared / attention_accumulate_prepared together with
    the same row_ptr, col_idx and workspace."""
    import torch
    L = row_ptr.numel() - 1
    if row_ptr.dtype != torch.int64 or not row_ptr.is_contiguous() or not row_ptr.is_cuda:
        raise ValueError("row_ptr must be a contiguous int64 device tensor")
    if col_idx.dtype != torch.int32 or not col_idx.is_contiguous():
        raise ValueError("col_idx must be contiguous int32")
    if workspace is None or workspace.device != row_ptr.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on row_ptr's device")
    code = _DTYPE_CODE[dtype] if isinstance(dtype, str) else dtype
    with torch.cuda.device(row_ptr.device):
        st, plan = sga_graph_prepare(row_ptr.data_ptr(), _col_ptr(row_ptr, col_idx), L, H, d, code,
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                     _stream())
    if st != 0:
        raise SgaError(st, "sga_graph_prepare")
    return plan


def _prepared_call(fn, name, Q, K, V, row_ptr, col_idx, scale, plan, O, lse, workspace, path):
    import torch
    H, L, d = Q.shape
    with torch.cuda.device(Q.device):
        st = fn(Q.data_ptr(), K.data_ptr(), V.data_ptr(), row_ptr.data_ptr(), _col_ptr(row_ptr, col_idx),
                O.data_ptr(), L, H, d, float(scale), _stream(), _dtype_code(Q),
                lse.data_ptr() if lse is not None else None, workspace.data_ptr(),
                workspace.numel() * workspace.element_size(), path, plan)
    if st != 0:
        raise SgaError(st, name)


def attention_forward_prepared(Q, K, V, row_ptr, col_idx, scale, plan, workspace, O=None, lse=None,
                               path=PATH_AUTO, want_lse=False):
    """attention_forward on a graph prepared by graph_prepare (same row_ptr, col_idx, workspace)."""
    import torch
    _check_qkv(Q, K, V)
    H, L, d = Q.shape
    _check_csr(Q, row_ptr, col_idx)
    _check_outputs(Q, O, lse, workspace)
    if O is None:
        O = torch.empty_like(Q)
    if want_lse and lse is None:
        lse = torch.empty((H, L), dtype=torch.float32, device=Q.device)
    _prepared_call(sga_attention_forward_prepared, "sga_attention_forward_prepared", Q, K, V, row_ptr,
                   col_idx, scale, plan, O, lse, workspace, path)
    return (O, lse) if (want_lse or lse is not None) else O


def attention_accumulate_prepared(Q, K, V, row_ptr, col_idx, scale, plan, workspace, O, lse,
                                  path=PATH_AUTO):
    """attention_accumulate on a prepared graph, in place."""
    _check_qkv(Q, K, V)
    _check_state(Q, O, lse)
    _check_csr(Q, row_ptr, col_idx)
    _check_outputs(Q, None, None, workspace)
    _prepared_call(sga_attention_accumulate_prepared, "sga_attention_accumulate_prepared", Q, K, V,
                   row_ptr, col_idx, scale, plan, O, lse, workspace, path)
    return O, lse


# ---- serving: rotary positions, a paged cache, attention of new tokens over it --------------------
_SERVING_CODE = {"torch.float32": 0, "torch.float16": 1, "torch.bfloat16": 2, "f32": 0, "f16": 1, "bf16": 2}
_LAYOUT_CODE = {"half": 0, "interleaved": 1}


def _serving_code(dtype):
    code = _SERVING_CODE.get(str(dtype))
    if code is None:
        raise TypeError(f"unsupported storage dtype {dtype}")
    return code


def _enqueue(index, call, *args):
    """call(*args, stream) on the current stream of device `index`, made the current device meanwhile.  A step of generation is a
    few short calls, so what the host does for each counts: torch.cuda.current_stream() alone takes 2.7 us, the raw
    handle of the same stream 0.1."""
    import torch
    if torch._C._cuda_getDevice() == index:
        return call(*args, torch._C._cuda_getCurrentRawStream(index))
    with torch.cuda.device(index):
        return call(*args, torch._C._cuda_getCurrentRawStream(index))


def _strides(t, name, written=False):
    """_Rows of a [H, T, d] tensor whose channels lie side by side.  A written one has to hold each element once."""
    H, T, d = t.shape
    sh, st, sc = t.stride()
    if sc != 1 and d > 1:
        raise ValueError(f"the channels of {name} must be contiguous")
    if H == 1:
        sh = 0
    if T == 1:
        st = 0
    if written and not ((H == 1 or sh >= d) and (T == 1 or st >= d)
                        and (H == 1 or T == 1 or st >= sh * (H - 1) + d or sh >= st * (T - 1) + d)) and t.numel() > 0:
        raise ValueError(f"rows of {name} overlap")
    return _Rows(t.data_ptr(), sh, st)


def _check_tokens(t, name, T=None):
    if t.dim() != 3 or not t.is_cuda:
        raise ValueError(f"{name} must be a [H, T, d] device tensor")
    if T is not None and t.shape[1] != T:
        raise ValueError(f"{name} must have the batch's {T} tokens")


def rotary_frequencies(channels, base=10000.0, scaling=None, factor=1.0, original_length=0, slow_turns=1.0, fast_turns=32.0,
                       device="cuda"):
    """Frequencies base^(-2 i / channels), i < channels / 2, for Rotary, scaled for contexts `factor` times as long as the
    trained `original_length`.  Returns (float64 [channels / 2], magnitude).

    scaling  None        as they are
             "linear"    positions shrink: every frequency divided by factor
             "base"      the base grows by factor^(channels / (channels - 2)): the lowest frequency shrinks by
                         factor, the highest stays
             "parts"     by the turns that a pair makes over original_length: from fast_turns on its frequency
                         stays, up to slow_turns it is divided by factor, between them in proportion; the magnitude
                         is 1 + ln(factor) / 10

    The formulas are published: "linear" is the position interpolation of Chen et al. (2023, arXiv 2306.15595), "base" and "parts"
    with its magnitude are the scaled base and the interpolation by parts of Peng et al. (2023, arXiv 2309.00071).
    """
    import math
    import torch
    if channels < 2 or channels % 2 != 0 or not base > 0 or not factor >= 1:
        raise ValueError("channels must be even and positive, base positive, factor at least 1")
    magnitude = 1.0
    if scaling == "base":
        if channels == 2:
            raise ValueError("scaling of the base needs more than two channels")
        base = base * factor ** (channels / (channels - 2))
    f = base ** (-torch.arange(0, channels, 2, dtype=torch.float64) / channels)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if original_length < 1 or not 0 <= slow_turns < fast_turns:
            raise ValueError("scaling by parts needs the trained length and slow_turns < fast_turns")
        keep = ((original_length * f / (2 * math.pi) - slow_turns) / (fast_turns - slow_turns)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
        magnitude = 1.0 + 0.1 * math.log(factor)
    elif scaling not in (None, "base"):
        raise ValueError(f"unknown scaling {scaling!r}")
    return f.to(device), magnitude


class _Fixed:
    """Attributes are set once.  The records for the library, and what a captured graph has taken from them, hold addresses and
    sizes: they would not follow an attribute that is replaced (one that is given what it holds, as by `x.seq_len += 1`, is not)."""

    def __setattr__(self, name, value):
        if name in self.__dict__ and self.__dict__[name] is not value:
            raise AttributeError(f"{type(self).__name__}.{name} cannot be replaced: write into its tensor, or make a new {type(self).__name__}")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        raise AttributeError(f"{type(self).__name__}.{name} cannot be removed")


class Rotary(_Fixed):
    """Which channels turn, how fast, and in which layout (sga_rotary_desc).  frequencies: float64 [channels / 2] on the
    device, radians per position; layout "half" (channels i and i + channels / 2) or "interleaved" (2 i and 2 i + 1).
    New frequencies may be written into the tensor; the attributes cannot be replaced."""

    def __init__(self, frequencies, layout="half", magnitude=1.0):
        if str(frequencies.dtype) != "torch.float64" or frequencies.dim() != 1 or frequencies.numel() < 1 \
                or not frequencies.is_contiguous() or not frequencies.is_cuda:
            raise ValueError("frequencies must be a contiguous float64 device tensor [channels / 2]")
        if layout not in _LAYOUT_CODE:
            raise ValueError(f"unknown layout {layout!r}")
        self.frequencies = frequencies
        self.device_index = frequencies.get_device()
        self.channels = 2 * frequencies.numel()
        self._desc = _RotaryDesc(ctypes.sizeof(_RotaryDesc), _LAYOUT_CODE[layout], self.channels, float(magnitude),
                                 frequencies.data_ptr())

    def _check(self, t):
        if self.device_index != t.get_device():
            raise ValueError("the rotary frequencies are on another device")


def rotary(X, rotary, positions=None, first=0, inverse=False, out=None):
    """Rotate [H, L, d] by position: row t has positions[t] (int64 [L]), or first + t.  inverse=True turns back: of a
    gradient, that is the gradient of the input.  (Like the package's other calls it records no history: a backward pass calls it
    again with inverse=True.)  out may be X."""
    _check_tokens(X, "X")
    rotary._check(X)
    H, L, d = X.shape
    index = X.get_device()
    at = None
    if positions is not None:
        if str(positions.dtype) != "torch.int64" or positions.shape != (L,) or not positions.is_contiguous() \
                or positions.get_device() != index:
            raise ValueError("positions must be contiguous int64 [L] on X's device")
        at = positions.data_ptr()
    if out is None:
        import torch
        out = torch.empty_like(X)
    elif out.shape != X.shape or out.dtype != X.dtype or out.get_device() != index:
        raise ValueError("out must match X in shape, dtype and device")
    st = _enqueue(index, sga_rotary, _strides(X, "X"), _strides(out, "out", written=True), at, int(first), L, H, d, rotary._desc,
                  1 if inverse else 0, _serving_code(X.dtype))
    if st != 0:
        raise SgaError(st, "sga_rotary")
    return out


class PagedBatch(_Fixed):
    """New tokens of several sequences and the pages of their keys and values (sga_paged_batch).

    page_table  int32 [S, columns]: page of tokens c * page_size .. of a sequence, -1 where there is none
    seq_ptr     int64 [S + 1]: sequence s has rows seq_ptr[s] .. seq_ptr[s + 1] - 1 of the packed tensors
    seq_len     int32 [S]: tokens of the sequence, the new ones among them
    n_tokens    rows of the packed tensors (rows behind the last sequence are padding)
    page_size, n_pages   of the caches [n_pages, Hkv, page_size, d]
    The arrays are read when the calls run, so a program may write new lengths and pages into them (`batch.seq_len += 1`).
    The attributes themselves cannot be replaced: for other arrays or another number of tokens make a new batch.
    """

    def __init__(self, page_table, seq_ptr, seq_len, n_tokens, page_size, n_pages):
        if str(page_table.dtype) != "torch.int32" or page_table.dim() != 2 or not page_table.is_contiguous():
            raise ValueError("page_table must be contiguous int32 [S, columns]")
        S, columns = page_table.shape
        if str(seq_ptr.dtype) != "torch.int64" or seq_ptr.shape != (S + 1,) or not seq_ptr.is_contiguous():
            raise ValueError("seq_ptr must be contiguous int64 [S + 1]")
        if str(seq_len.dtype) != "torch.int32" or seq_len.shape != (S,) or not seq_len.is_contiguous():
            raise ValueError("seq_len must be contiguous int32 [S]")
        if not page_table.is_cuda or seq_ptr.device != page_table.device or seq_len.device != page_table.device:
            raise ValueError("page_table, seq_ptr and seq_len must be tensors of one device")
        # (one update: the check of __setattr__ for each would cost 2 us, and a program may make a batch per step)
        self.__dict__.update(page_table=page_table, seq_ptr=seq_ptr, seq_len=seq_len, n_tokens=int(n_tokens), page_size=int(page_size),
                             n_pages=int(n_pages), device=page_table.device, device_index=page_table.get_device(), _structs={})

    def _struct(self, page_stride):
        s = self._structs.get(page_stride)
        if s is None:
            S, columns = self.page_table.shape
            s = _PagedBatch(ctypes.sizeof(_PagedBatch), S, self.n_tokens, self.n_pages, page_stride, self.page_size, columns,
                            self.page_table.data_ptr(), self.seq_ptr.data_ptr(), self.seq_len.data_ptr())
            self._structs[page_stride] = s
        return s

    def _caches(self, like, cache_k, cache_v):
        """The batch's record for these caches, and their key heads."""
        if like.get_device() != self.device_index:
            raise ValueError("the batch is on another device")
        d, page, n_pages = like.shape[2], self.page_size, self.n_pages
        shape = cache_k.shape
        if len(shape) != 4 or cache_v.shape != shape or shape[0] != n_pages or shape[2] != page or shape[3] != d:
            raise ValueError("the caches must both be [n_pages, Hkv, page_size, d]")
        Hkv = shape[1]
        apart = 0
        for t in (cache_k, cache_v):
            if t.dtype != like.dtype or t.get_device() != self.device_index:
                raise ValueError("the caches must share dtype and device with the tokens")
            sp, sh, st, sc = t.stride()
            if sc != 1 or (st != d and page > 1) or (sh != page * d and Hkv > 1):
                raise ValueError("every page of a cache must be contiguous")
            if n_pages == 1:
                sp = Hkv * page * d
            if sp < Hkv * page * d or sp != (apart or sp):
                raise ValueError("the pages of a cache must not overlap, and both caches must have them at one distance")
            apart = sp
        return self._struct(apart), Hkv


def cache_append(K, V, cache_k, cache_v, batch, rotary=None, Q=None, Q_out=None):
    """Write the batch's new keys (rotated) and values, [Hkv, n_tokens, d], into their pages, and rotate the queries Q
    beside them.  Returns Q_out (which may be Q) if Q is given; one that is made here holds nothing in padding rows."""
    _check_tokens(K, "K", T=batch.n_tokens)
    struct, Hkv = batch._caches(K, cache_k, cache_v)
    index, shape, dtype = batch.device_index, K.shape, K.dtype
    if shape[0] != Hkv or V.shape != shape or V.dtype != dtype or V.get_device() != index:
        raise ValueError("K and V must be alike and have the caches' heads")
    q = q_out = None
    Hq = 0
    if rotary is not None:
        rotary._check(K)
    if Q is not None:
        if rotary is None:
            raise ValueError("queries are rotated: a call with Q needs rotary")
        if Q.dim() != 3 or Q.shape[1:] != shape[1:] or Q.dtype != dtype or Q.get_device() != index:
            raise ValueError("Q must be [Hq, n_tokens, d] and share dtype and device with K")
        if Q_out is None:
            import torch
            Q_out = torch.empty_like(Q)
        elif Q_out.shape != Q.shape or Q_out.dtype != dtype or Q_out.get_device() != index:
            raise ValueError("Q_out must match Q")
        q, q_out, Hq = _strides(Q, "Q"), _strides(Q_out, "Q_out", written=True), Q.shape[0]
    elif Q_out is not None:
        raise ValueError("Q_out without Q")
    st = _enqueue(index, sga_cache_append, _strides(K, "K"), _strides(V, "V"), cache_k.data_ptr(),
                  cache_v.data_ptr(), struct, Hkv, shape[2], rotary._desc if rotary is not None else None, q, q_out, Hq,
                  _serving_code(dtype))
    if st != 0:
        raise SgaError(st, "sga_cache_append")
    return Q_out


def paged_workspace_bytes(batch, spec: MaskSpec, Hq, Hkv, d, dtype) -> int:
    st, n = sga_paged_workspace_bytes(batch._struct(Hkv * batch.page_size * d), spec, Hq, Hkv, d, _serving_code(dtype))
    if st != 0:
        raise SgaError(st, "sga_paged_workspace_bytes")
    return n


def alloc_paged_workspace(batch, spec: MaskSpec, Hq, Hkv, d, dtype):
    """Workspace for attention_paged calls of this batch and mask (calls that overlap in time need one each).  A call under another
    mask may need more; with a smaller one than its own it runs without cutting long sequences, which is slower and as right."""
    import torch
    return torch.empty(paged_workspace_bytes(batch, spec, Hq, Hkv, d, dtype), dtype=torch.uint8, device=batch.device)


def attention_paged(Q, cache_k, cache_v, batch, spec: MaskSpec, scale, causal=True, O=None, lse=None, workspace=None,
                    want_lse=False):
    """Attention of the batch's new tokens, Q [Hq, n_tokens, d], over the paged cache under a sliding or global + local mask
    of spec.L tokens (window >= L: every token), of earlier tokens only if causal.  Consecutive Hq / Hkv query heads share
    a key head.  Returns O (and lse [Hq, n_tokens] if requested); a token that sees nothing has O = 0, lse = -inf; padding rows
    are left as they were, in tensors that are made here with whatever memory held."""
    _check_tokens(Q, "Q", T=batch.n_tokens)
    struct, Hkv = batch._caches(Q, cache_k, cache_v)
    Hq, T, d = Q.shape
    index = batch.device_index
    if O is None:
        import torch
        O = torch.empty_like(Q)
    elif O.shape != Q.shape or O.dtype != Q.dtype or O.get_device() != index:
        raise ValueError("O must match Q in shape, dtype and device")
    if want_lse and lse is None:
        import torch
        lse = torch.empty((Hq, T), dtype=torch.float32, device=Q.device)
    if lse is not None and (lse.shape != (Hq, T) or str(lse.dtype) != "torch.float32" or not lse.is_contiguous()
                            or lse.get_device() != index):
        raise ValueError("lse must be contiguous float32 [Hq, n_tokens] on Q's device")
    ws_ptr, ws_n = None, 0
    if workspace is not None and workspace.numel() > 0:
        if workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on Q's device")
        ws_ptr, ws_n = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    st = _enqueue(index, sga_attention_paged, _strides(Q, "Q"), cache_k.data_ptr(), cache_v.data_ptr(), struct, spec,
                  1 if causal else 0, _strides(O, "O", written=True), Hq, Hkv, d, float(scale), _serving_code(Q.dtype),
                  lse.data_ptr() if lse is not None else None, ws_ptr, ws_n)
    if st != 0:
        raise SgaError(st, "sga_attention_paged")
    return (O, lse) if lse is not None else O
