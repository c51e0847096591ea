"""Thin ctypes binding of libdgc (include/dgc.h): argument marshalling only.

Every step of the path runs inside the HIP library.  PyTorch supplies device memory and the
stream.  There is no CPU fallback: if the library has not been built, or no GPU is present,
the calls raise.
"""
from __future__ import annotations

import ctypes as ct
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdgc.so")

TIME_KIND = {"none": 0, "gru": 1, "lstm": 2, "self_attn": 3}
ACT = {"none": 0, "relu": 1}
LINEAR_ACT = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
LINEAR_EXACT = 16       # added to an activation in the backward calls
GATHER = {"in_place": 0, "staged": 1}
DENSE = {"auto": 0, "tile": 1, "wave": 2}
AGG = {"table": 0, "walk": 1}
STRUCT = {"gcn": 0, "evolve_gcn_o": 1, "gat": 2}
DTYPE = {"f32": 0, "bf16": 1}

STATUS = {0: "DGC_OK", 1: "DGC_ERR_INVALID_ARG", 2: "DGC_ERR_BAD_GRAPH", 3: "DGC_ERR_BAD_CHUNK",
          4: "DGC_ERR_UNSUPPORTED", 5: "DGC_ERR_OOM", 6: "DGC_ERR_DEVICE", 7: "DGC_ERR_STATE"}

EXPORTS = ["dgc_layer_create", "dgc_layer_destroy", "dgc_layer_set_param", "dgc_layer_get_param",
           "dgc_layer_forward", "dgc_layer_backward", "dgc_layer_aggregate", "dgc_layer_gather",
           "dgc_layer_packing", "dgc_layer_set_presence", "dgc_layer_set_labels", "dgc_layer_set_profiling", "dgc_layer_stage_times", "dgc_last_error",
           "dgc_version", "dgc_stale_theta_factor", "dgc_stale_workspace_bytes", "dgc_stale_filter",
           "dgc_stale_static_max_candidates", "dgc_stale_filter_static",
           "dgc_layer_shared_rows", "dgc_fusion_select", "dgc_chunk_assign", "dgc_chunk_generate",
           "dgc_norm_workspace_bytes", "dgc_norm_forward", "dgc_norm_backward",
           "dgc_linear_workspace_bytes", "dgc_linear_forward", "dgc_linear_backward",
           "dgc_decay_attn_workspace_bytes", "dgc_decay_attn_forward", "dgc_decay_attn_backward"]
THETA_VARIANT = {"printed": 0, "sigmoid": 1}
N_STAGES = 13


class DgcError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"{STATUS.get(code, code)}: {text}")
        self.code = code


class ChunkT(ct.Structure):
    _fields_ = [("v_lo", ct.c_int64), ("v_hi", ct.c_int64), ("t_lo", ct.c_int32), ("t_hi", ct.c_int32)]


class GraphT(ct.Structure):
    _fields_ = [("T", ct.c_int32), ("N", ct.c_int64),
                ("rowptr", ct.POINTER(ct.c_void_p)), ("colidx", ct.POINTER(ct.c_void_p))]


class DescT(ct.Structure):
    _fields_ = [(n, ct.c_int32) for n in
                ("struct_kind", "n_struct_layers", "time_kind", "dtype", "F", "S", "H", "act_hidden",
                 "act_out", "gather_mode", "validate_level", "rows_per_group", "long_nnz", "part_nnz",
                 "dense_kernel", "heads", "lstm_input_concat", "agg_kernel", "n_time_layers")]


_lib = None


def load() -> ct.CDLL:
    """Load libdgc.so (built in-tree by __graft_entry__.build()).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ct.CDLL(LIB_PATH)
    vp, i32, i64 = ct.c_void_p, ct.c_int32, ct.c_int64
    lib.dgc_layer_create.argtypes = [ct.POINTER(DescT), ct.POINTER(GraphT), ct.POINTER(ChunkT), i32, vp,
                                     ct.POINTER(vp)]
    lib.dgc_layer_destroy.argtypes = [vp]
    lib.dgc_layer_set_param.argtypes = [vp, ct.c_char_p, vp, i64]
    lib.dgc_layer_get_param.argtypes = [vp, ct.c_char_p, vp, i64]
    lib.dgc_layer_forward.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp]
    lib.dgc_layer_backward.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, vp, i64, vp]
    lib.dgc_layer_aggregate.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp]
    lib.dgc_layer_gather.argtypes = [vp, vp, i64, vp, i64, vp]
    lib.dgc_layer_packing.argtypes = [vp, ct.c_char_p, vp, i64, ct.POINTER(i64)]
    lib.dgc_layer_set_presence.argtypes = [vp, vp, vp]
    lib.dgc_layer_set_labels.argtypes = [vp, vp, vp]
    lib.dgc_layer_set_profiling.argtypes = [vp, i32]
    lib.dgc_layer_stage_times.argtypes = [vp, vp]
    lib.dgc_last_error.argtypes = [vp]
    lib.dgc_last_error.restype = ct.c_char_p
    lib.dgc_version.restype = ct.c_char_p
    lib.dgc_chunk_generate.argtypes = [ct.POINTER(GraphT), i32, i32, i64, i32, vp, ct.POINTER(i32), ct.POINTER(i32), vp]
    lib.dgc_layer_shared_rows.argtypes = [vp, vp, vp]
    lib.dgc_fusion_select.argtypes = [i32, vp, vp, i64, vp]
    lib.dgc_chunk_assign.argtypes = [i32, vp, vp, i32, vp]
    lib.dgc_stale_theta_factor.argtypes = [ct.c_double, ct.c_double, i32]
    lib.dgc_stale_theta_factor.restype = ct.c_double
    lib.dgc_stale_workspace_bytes.argtypes = [i64]
    lib.dgc_stale_workspace_bytes.restype = i64
    lib.dgc_stale_filter.argtypes = [vp, i64, vp, i64, i64, i32, i32, vp, i64, ct.c_double, ct.c_double, vp, vp, vp, i64,
                                     vp, vp, i64, vp]
    lib.dgc_stale_filter_static.argtypes = [vp, i64, vp, i64, i64, i32, i32, vp, i64, ct.c_double, ct.c_double, vp, vp, vp,
                                            i64, vp, vp]
    lib.dgc_stale_static_max_candidates.argtypes = []
    lib.dgc_stale_static_max_candidates.restype = i64
    f32 = ct.c_float
    lib.dgc_norm_forward.argtypes = [vp, i64, i64, i32, i32, vp, vp, f32, vp, i64, vp, vp, vp]
    lib.dgc_norm_backward.argtypes = [vp, i64, vp, i64, vp, vp, i64, i32, i32, vp, vp, i64, vp, i64, vp, vp, vp, i64, vp]
    lib.dgc_norm_workspace_bytes.argtypes = [i64, i32]
    lib.dgc_linear_forward.argtypes = [vp, i64, vp, i64, i64, i32, i32, i32, vp, i32, vp, i64, vp, i64, vp, i64, vp]
    lib.dgc_linear_backward.argtypes = [vp, i64, vp, i64, vp, i64, i64, i32, i32, i32, vp, i64, i32, vp, i64, vp, i64, vp, vp, i64, vp]
    lib.dgc_linear_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
    lib.dgc_decay_attn_workspace_bytes.argtypes = [i64, i64, i32, i32, i32, i32]
    seq = [vp, i64, i64]    # a tensor of rows (t, i): address, strides of t and i
    dims = [i64, i64, i32, i32, i32, i32]
    lib.dgc_decay_attn_forward.argtypes = seq * 3 + dims + [vp, f32, vp, vp, vp] + seq + [vp, vp, i64, vp]
    lib.dgc_decay_attn_backward.argtypes = seq * 4 + dims + [vp, f32, vp, vp, vp, vp] + seq * 3 + [vp, vp, i64, vp]
    sizes = ("dgc_norm_workspace_bytes", "dgc_linear_workspace_bytes", "dgc_decay_attn_workspace_bytes")
    for name in sizes:
        getattr(lib, name).restype = i64
    for name in EXPORTS:
        if name not in ("dgc_last_error", "dgc_version", "dgc_stale_theta_factor", "dgc_stale_workspace_bytes",
                        "dgc_stale_static_max_candidates") + sizes:
            getattr(lib, name).restype = ct.c_int
    _lib = lib
    return lib


def version() -> str:
    return load().dgc_version().decode()


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return ct.c_void_p(stream.cuda_stream)


def _dev(t, name: str):
    """Device pointer of a contiguous-in-the-last-dim CUDA tensor (or None)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    return ct.c_void_p(t.data_ptr())


def _ld(t, name: str) -> int:
    if t is None:
        return 0
    if t.dim() != 3 or t.stride(2) != 1 or t.stride(0) != t.shape[1] * t.stride(1):
        raise ValueError(f"{name} must be [T,N,ld] row-major (last dim contiguous, no gap between snapshots)")
    return int(t.stride(1))


_PACK_DTYPES = {"seg_row_off": np.int64, "seg_nnz_off": np.int64, "halo_ptr": np.int64,
                "halo_idx": np.int32, "col_local": np.int32, "work_short": np.int32,
                "work_long": np.int32, "deg_inv_sqrt": np.float32, "lane_ptr": np.int64, "slot_row": np.int64,
                "slot_reset": np.uint8}


class DgcLayer:
    """dgc_layer_create / forward / backward / destroy with torch tensors as arguments.

    rowptr, colidx: lists of T device tensors (int64 [N+1], int32 [nnz_t]).
    chunks: array-like [n,4] of (v_lo, v_hi, t_lo, t_hi).
    """

    def __init__(self, rowptr, colidx, N: int, chunks, *, F: int, S: int, H: int, time_kind: str = "gru",
                 n_struct_layers: int = 1, act_hidden: str = "relu", act_out: str = "none",
                 gather_mode: str = "in_place", validate_level: int = 0, rows_per_group: int = 0,
                 long_nnz: int = 0, part_nnz: int = 0, dense_kernel: str = "auto", struct_kind: str = "gcn",
                 dtype: str = "f32", heads: int = 0, lstm_input_concat: bool = False, agg_kernel: str = "table",
                 n_time_layers: int = 1, stream=None):
        import torch
        lib = load()
        self._lib = lib
        self._h = ct.c_void_p(None)
        T = len(rowptr)
        for r, c in zip(rowptr, colidx):
            if r.dtype != torch.int64 or c.dtype != torch.int32 or not r.is_cuda or not c.is_cuda:
                raise ValueError("rowptr must be int64 and colidx int32 device tensors")
            if not r.is_contiguous() or not c.is_contiguous():
                raise ValueError("CSR arrays must be contiguous")
        self._keep = (list(rowptr), list(colidx))  # the layer borrows the CSR arrays for its life
        rp = (ct.c_void_p * T)(*[r.data_ptr() for r in rowptr])
        cj = (ct.c_void_p * T)(*[c.data_ptr() for c in colidx])
        graph = GraphT(T, N, rp, cj)
        ch = np.asarray(chunks, np.int64).reshape(-1, 4)
        carr = (ChunkT * len(ch))(*[ChunkT(int(a), int(b), int(c), int(d)) for a, b, c, d in ch])
        desc = DescT(STRUCT[struct_kind], n_struct_layers, TIME_KIND[time_kind], DTYPE[dtype], F, S, H, ACT[act_hidden],
                     ACT[act_out],
                     GATHER[gather_mode], validate_level, rows_per_group, long_nnz, part_nnz, DENSE[dense_kernel],
                     heads, int(lstm_input_concat), AGG[agg_kernel], int(n_time_layers))
        rc = lib.dgc_layer_create(ct.byref(desc), ct.byref(graph), carr, len(ch), _stream_ptr(stream),
                                  ct.byref(self._h))
        if rc:
            raise DgcError(rc, lib.dgc_last_error(None).decode())
        self.T, self.N, self.F, self.S, self.H = T, N, F, S, H
        self.time_kind, self.n_struct_layers, self.n_time_layers = time_kind, n_struct_layers, n_time_layers
        self.chunks = ch
        self.out_dim = H if time_kind in ("gru", "lstm") else S

    # -- lifetime
    def destroy(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.dgc_layer_destroy(self._h)
            self._h = ct.c_void_p(None)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc:
            raise DgcError(rc, self._lib.dgc_last_error(self._h).decode())

    # -- parameters
    def set_param(self, name: str, value: np.ndarray):
        v = np.ascontiguousarray(value, np.float32)
        self._check(self._lib.dgc_layer_set_param(self._h, name.encode(), v.ctypes.data_as(ct.c_void_p), v.size))

    def set_params(self, params: dict):
        for k, v in params.items():
            self.set_param(k, v)

    def get_param(self, name: str, shape) -> np.ndarray:
        out = np.zeros(shape, np.float32)
        self._check(self._lib.dgc_layer_get_param(self._h, name.encode(), out.ctypes.data_as(ct.c_void_p), out.size))
        return out

    # -- the path
    def forward(self, X, C, Y, *, C1=None, H0=None, reset_mask=None, HN=None, stream=None):
        self._check(self._lib.dgc_layer_forward(
            self._h, _dev(X, "X"), _ld(X, "X"), _dev(C, "C"), _ld(C, "C"), _dev(C1, "C1"), _ld(C1, "C1"),
            _dev(H0, "H0"), _dev(reset_mask, "reset_mask"), _dev(Y, "Y"), _ld(Y, "Y"), _dev(HN, "HN"),
            _stream_ptr(stream)))
        return Y

    def backward(self, Y, *, dY=None, target=None, loss_out=None, dX=None, stream=None):
        self._check(self._lib.dgc_layer_backward(
            self._h, _dev(Y, "Y"), _ld(Y, "Y"), _dev(dY, "dY"), _ld(dY, "dY"), _dev(target, "target"),
            _ld(target, "target"), _dev(loss_out, "loss_out"), _dev(dX, "dX"), _ld(dX, "dX"), _stream_ptr(stream)))

    def set_presence(self, present, stream=None):
        """present: uint8 device tensor [T,N]; switches the layer to temporal fusion (on a layer that has
        labels: over the runs of present instances with one label; labels are set first)."""
        if not present.is_cuda or present.dtype.itemsize != 1 or not present.is_contiguous():
            raise ValueError("present must be a contiguous uint8 device tensor [T,N]")
        self._check(self._lib.dgc_layer_set_presence(self._h, _dev(present, "present"), _stream_ptr(stream)))

    def set_labels(self, labels, stream=None):
        """labels: int32 device tensor [T*N] (or [T,N]), e.g. chunk_generate's output; the layer then
        runs over the generated chunks."""
        import torch
        if not labels.is_cuda or labels.dtype != torch.int32 or not labels.is_contiguous() or labels.numel() != self.T * self.N:
            raise ValueError("labels must be a contiguous int32 device tensor with T*N entries")
        self._check(self._lib.dgc_layer_set_labels(self._h, _dev(labels, "labels"), _stream_ptr(stream)))

    def aggregate(self, X, C, M, stream=None):
        self._check(self._lib.dgc_layer_aggregate(self._h, _dev(X, "X"), _ld(X, "X"), _dev(C, "C"), _ld(C, "C"),
                                                  _dev(M, "M"), int(M.stride(0)), _stream_ptr(stream)))
        return M

    def gather(self, C, halo, stream=None):
        self._check(self._lib.dgc_layer_gather(self._h, _dev(C, "C"), _ld(C, "C"), _dev(halo, "halo"),
                                               int(halo.stride(0)), _stream_ptr(stream)))
        return halo

    def shared_rows(self, stream=None) -> np.ndarray:
        """int64 [n_chunks, n_chunks]: rows every pair of chunks would load twice."""
        n = len(self.chunks)
        out = np.zeros((n, n), np.int64)
        self._check(self._lib.dgc_layer_shared_rows(self._h, out.ctypes.data_as(ct.c_void_p), _stream_ptr(stream)))
        return out

    # -- measurement
    def set_profiling(self, enable: bool):
        self._check(self._lib.dgc_layer_set_profiling(self._h, int(bool(enable))))

    def stage_times(self) -> np.ndarray:
        """Milliseconds per stage of the last profiled forward (waits for it)."""
        out = np.zeros(N_STAGES, np.float32)
        self._check(self._lib.dgc_layer_stage_times(self._h, out.ctypes.data_as(ct.c_void_p)))
        return out

    # -- inspection
    def packing(self, what: str) -> np.ndarray:
        need = ct.c_int64(0)
        rc = self._lib.dgc_layer_packing(self._h, what.encode(), None, 0, ct.byref(need))
        if rc not in (0, 1):     # 1 = destination too small: the size query itself
            self._check(rc)
        dt = np.dtype(_PACK_DTYPES[what])
        out = np.zeros(need.value // dt.itemsize, dt)
        if out.size:
            self._check(self._lib.dgc_layer_packing(self._h, what.encode(), out.ctypes.data_as(ct.c_void_p),
                                                    out.nbytes, ct.byref(need)))
        if what == "work_short":
            out = out.reshape(-1, 3)
        if what == "work_long":
            out = out.reshape(-1, 4)
        return out


# --------------------------------------------------------------------------- stale filter

STALE_RESULT_DTYPE = np.dtype([("n_send", np.int64), ("D", np.float32), ("theta", np.float32),
                               ("n_invalid", np.int64)])


def stale_theta_factor(l1: float, l_prev: float, variant: str = "printed") -> float:
    f = load().dgc_stale_theta_factor(float(l1), float(l_prev), THETA_VARIANT[variant])
    if f < 0:
        raise ValueError("stale_theta_factor: l1 must be > 0 and l_prev finite")
    return f


def stale_workspace_bytes(n_candidates: int) -> int:
    return int(load().dgc_stale_workspace_bytes(int(n_candidates)))


def stale_static_max_candidates() -> int:
    return int(load().dgc_stale_static_max_candidates())


def stale_filter(E, L, *, F=None, rows=None, n_rows=None, factor=None, theta=None, dist, send_idx, send_buf=None, result,
                 workspace=None, stream=None):
    """dgc_stale_filter on device tensors: E, L [R, ld] fp32 or bfloat16; rows int64 or None (n_rows: how many of
    its entries count, default all; torch gives an empty tensor a NULL pointer, so an empty list is a
    non-empty tensor with n_rows = 0); dist fp32 and
    send_idx int64 with one entry per candidate; send_buf [n, ld] or None; result: 24-byte device
    tensor (view it with STALE_RESULT_DTYPE after a synchronisation); workspace: device bytes, or
    None for dgc_stale_filter_static (the library's own fixed scratch, nothing allocated).
    Exactly one of factor / theta.  Only enqueues."""
    if (factor is None) == (theta is None):
        raise ValueError("give exactly one of factor and theta")
    for name, t in (("E", E), ("L", L)):
        if t.dim() != 2 or t.stride(1) != 1:
            raise ValueError(f"{name} must be [R, ld] with a contiguous last dimension")
    if E.dtype != L.dtype or (send_buf is not None and send_buf.dtype != E.dtype):
        raise ValueError("E, L and send_buf must have the same element type")
    lib = load()
    head = (_dev(E, "E"), int(E.stride(0)), _dev(L, "L"), int(L.stride(0)), int(E.shape[0]),
            int(E.shape[1] if F is None else F), DTYPE["bf16" if E.element_size() == 2 else "f32"], _dev(rows, "rows"),
            0 if rows is None else int(rows.numel() if n_rows is None else n_rows),
            -1.0 if factor is None else float(factor), 0.0 if theta is None else float(theta), _dev(dist, "dist"),
            _dev(send_idx, "send_idx"), _dev(send_buf, "send_buf"), 0 if send_buf is None else int(send_buf.stride(0)),
            _dev(result, "result"))
    if workspace is None:
        rc = lib.dgc_stale_filter_static(*head, _stream_ptr(stream))
    else:
        rc = lib.dgc_stale_filter(*head, _dev(workspace, "workspace"),
                                  int(workspace.numel() * workspace.element_size()), _stream_ptr(stream))
    if rc != 0:
        raise DgcError(rc, lib.dgc_last_error(None).decode())


# --------------------------------------------------------------------------- fusion selection, assignment


def fusion_select(shared: np.ndarray, mem: np.ndarray, cap: int) -> np.ndarray:
    shared = np.ascontiguousarray(shared, np.int64)
    mem = np.ascontiguousarray(mem, np.int64)
    n = mem.size
    if shared.shape != (n, n):
        raise ValueError("shared must be [n, n]")
    out = np.zeros(n, np.int32)
    lib = load()
    rc = lib.dgc_fusion_select(n, shared.ctypes.data_as(ct.c_void_p), mem.ctypes.data_as(ct.c_void_p), int(cap),
                               out.ctypes.data_as(ct.c_void_p))
    if rc != 0:
        raise DgcError(rc, lib.dgc_last_error(None).decode())
    return out


def chunk_assign(g: np.ndarray, h: np.ndarray, n_gpus: int) -> np.ndarray:
    g = np.ascontiguousarray(g, np.float64)
    h = np.ascontiguousarray(h, np.float64)
    n = g.size
    if h.shape != (n, n):
        raise ValueError("h must be [n, n]")
    out = np.zeros(n, np.int32)
    lib = load()
    rc = lib.dgc_chunk_assign(n, g.ctypes.data_as(ct.c_void_p), h.ctypes.data_as(ct.c_void_p), int(n_gpus),
                              out.ctypes.data_as(ct.c_void_p))
    if rc != 0:
        raise DgcError(rc, lib.dgc_last_error(None).decode())
    return out


# --------------------------------------------------------------------------- chunk generation


def chunk_generate(rowptr, colidx, N: int, *, w_s: int, w_t: int, cap: int, max_iters: int, labels, stream=None):
    """dgc_chunk_generate: rowptr / colidx lists of T device tensors, labels int32 device tensor
    [T*N] (written).  Returns (iterations, converged)."""
    T = len(rowptr)
    rp = (ct.c_void_p * T)(*[r.data_ptr() for r in rowptr])
    cj = (ct.c_void_p * T)(*[c.data_ptr() for c in colidx])
    graph = GraphT(T, N, rp, cj)
    if labels.numel() != T * N or labels.element_size() != 4 or not labels.is_contiguous():
        raise ValueError("labels must be a contiguous int32 device tensor of T*N elements")
    it, conv = ct.c_int32(0), ct.c_int32(0)
    lib = load()
    rc = lib.dgc_chunk_generate(ct.byref(graph), int(w_s), int(w_t), int(cap), int(max_iters), _dev(labels, "labels"),
                                ct.byref(it), ct.byref(conv), _stream_ptr(stream))
    if rc != 0:
        raise DgcError(rc, lib.dgc_last_error(None).decode())
    return it.value, bool(conv.value)


# --------------------------------------------------------------------------- layer norm, products of rows, decaying attention
#
# Operators on plain device tensors: nothing is allocated, outputs and workspaces are the caller's, work is only
# enqueued on `stream` (default: the current stream of the tensors' device).


_torch = None
_raw_stream = None      # device index -> the current stream's handle
_device = None          # () -> the current device's index


def _op_init():
    global _torch, _raw_stream, _device
    import torch
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    _torch = torch
    return load()


def _op_first(t, name: str):
    """(library, element type, device index) of a call's first tensor."""
    lib = _lib if _torch is not None and _lib is not None else _op_init()
    dt = t.dtype
    if dt is _torch.bfloat16:
        code = 1
    elif dt is _torch.float32:
        code = 0
    else:
        raise ValueError(f"{name} must be float32 or bfloat16")
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a device tensor")
    return lib, code, dev


def _op_rows(t, name: str, dtype=None, dev=None, shape=None):
    """(address, pitch) of [..., F] rows at one pitch; dtype, dev: what the first tensor has; shape: (R, F)."""
    if t is None:
        return None, 0
    st, sh = t.stride(), t.shape
    n = len(sh)
    if n < 2 or (st[-1] != 1 and sh[-1] != 1):
        raise ValueError(f"{name} must be rows [..., F] with a contiguous last dimension")
    if dtype is not None and (t.dtype is not dtype or t.get_device() != dev):
        raise ValueError(f"{name} has another element type or device than the first tensor")
    F, rows, pitch = sh[-1], sh[-2], st[-2]
    if n > 2:
        step = pitch
        for d in range(n - 3, -1, -1):
            if sh[d] != 1:
                if rows == 1:
                    step = pitch = st[d]     # leading sizes of 1 leave their strides free
                elif st[d] != rows * step and rows and sh[d]:
                    raise ValueError(f"{name}: its rows must lie at one pitch")
                rows *= sh[d]
    if rows <= 1:
        pitch = -(-F // 8) * 8
    if shape is not None and (F != shape[1] or rows != shape[0]):
        raise ValueError(f"{name} must hold {shape[0]} rows of {shape[1]}, not {tuple(sh)}")
    return t.data_ptr(), pitch


def _op_count(t) -> int:
    """Rows of a [..., F] tensor."""
    n = 1
    for x in t.shape[:-1]:
        n *= x
    return n


def _op_flat(t, name: str, numel: int, dev: int, dtype=None):
    """Address of a contiguous device tensor of `numel` elements (fp32 unless `dtype` says otherwise), or None."""
    if t is None:
        return None
    if t.dtype is not (dtype or _torch.float32) or t.numel() != numel or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {str(dtype or _torch.float32)[6:]} tensor of {numel} elements on the first tensor's device")
    return t.data_ptr()


def _op_shape(t, name: str, shape, dev: int, dtype=None):
    """Address of a contiguous device tensor of just this shape (fp32 unless `dtype` says otherwise), or None."""
    if t is None:
        return None
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, not {list(t.shape)}")
    return _op_flat(t, name, t.numel(), dev, dtype)


def _op_workspace(t, dev: int):
    if t is None:
        return None, 0
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError("workspace must be contiguous and on the first tensor's device")
    return t.data_ptr(), t.numel() * t.element_size()


def _op_call(fn, dev: int, stream, *args):
    """Calls fn(*args, stream) with the tensors' device current."""
    if stream is None:
        handle = _raw_stream(dev)
    else:
        if stream.device.index != dev:
            raise ValueError("stream belongs to another device than the tensors")
        handle = stream.cuda_stream
    if _device() == dev:
        rc = fn(*args, handle)
    else:
        with _torch.cuda.device(dev):
            rc = fn(*args, handle)
    if rc:
        raise DgcError(rc, _lib.dgc_last_error(None).decode())


def norm_workspace_bytes(R: int, F: int) -> int:
    return int(load().dgc_norm_workspace_bytes(int(R), int(F)))


def norm_forward(x, y, *, gamma=None, beta=None, mean=None, rstd=None, eps: float = 1e-5, stream=None):
    """dgc_norm_forward: y = layer norm of the rows of x [..., F] (y may be x); gamma, beta fp32 [F] or None (1, 0);
    mean, rstd fp32, one entry a row, written if given."""
    lib, code, dev = _op_first(x, "x")
    dt = x.dtype
    px, ldx = _op_rows(x, "x")
    F, R = x.shape[-1], _op_count(x)
    py, ldy = _op_rows(y, "y", dt, dev, (R, F))
    _op_call(lib.dgc_norm_forward, dev, stream, px, ldx, R, F, code, _op_flat(gamma, "gamma", F, dev), _op_flat(beta, "beta", F, dev),
             float(eps), py, ldy, _op_flat(mean, "mean", R, dev), _op_flat(rstd, "rstd", R, dev))
    return y


def norm_backward(dy, x, mean, rstd, dx, *, gamma=None, add=None, dgamma=None, dbeta=None, workspace=None, stream=None):
    """dgc_norm_backward: dx = gradient of x, plus `add` if given (dx may be dy, x or add); dgamma, dbeta fp32 [F], written if
    given (they need `workspace`, norm_workspace_bytes(R, F) device bytes)."""
    lib, code, dev = _op_first(x, "x")
    dt = x.dtype
    px, ldx = _op_rows(x, "x")
    F, R = x.shape[-1], _op_count(x)
    pdy, lddy = _op_rows(dy, "dy", dt, dev, (R, F))
    padd, ldadd = _op_rows(add, "add", dt, dev, (R, F))
    pdx, lddx = _op_rows(dx, "dx", dt, dev, (R, F))
    ws, ws_bytes = _op_workspace(workspace, dev)
    _op_call(lib.dgc_norm_backward, dev, stream, pdy, lddy, px, ldx, _op_flat(mean, "mean", R, dev), _op_flat(rstd, "rstd", R, dev), R, F,
             code, _op_flat(gamma, "gamma", F, dev), padd, ldadd, pdx, lddx, _op_flat(dgamma, "dgamma", F, dev),
             _op_flat(dbeta, "dbeta", F, dev), ws, ws_bytes)
    return dx


def linear_workspace_bytes(R: int, K: int, M: int, *, dtype: str = "f32", act: str = "gelu", exact: bool = False) -> int:
    """Bytes that linear_backward needs; without an activation it needs less, with exact=True more."""
    return int(load().dgc_linear_workspace_bytes(int(R), int(K), int(M), DTYPE[dtype], LINEAR_ACT[act] + LINEAR_EXACT * bool(exact)))


def linear_forward(x, w, y, *, bias=None, act: str = "none", residual=None, pre=None, stream=None):
    """dgc_linear_forward: y = act(x w^T + bias) + residual for rows x [..., K], w [M, K] (out, in), y [..., M] of one element
    type; bias fp32 [M]; pre [..., M] receives the activation's argument; y may be residual itself."""
    lib, code, dev = _op_first(x, "x")
    dt = x.dtype
    px, ldx = _op_rows(x, "x")
    K, R, M = x.shape[-1], _op_count(x), w.shape[0]
    pw, ldw = _op_rows(w, "w", dt, dev, (M, K))
    py, ldy = _op_rows(y, "y", dt, dev, (R, M))
    pr, ldr = _op_rows(residual, "residual", dt, dev, (R, M))
    pp, ldp = _op_rows(pre, "pre", dt, dev, (R, M))
    _op_call(lib.dgc_linear_forward, dev, stream, px, ldx, pw, ldw, R, K, M, code, _op_flat(bias, "bias", M, dev), LINEAR_ACT[act], pr, ldr,
             py, ldy, pp, ldp)
    return y


def linear_backward(dy, x, w, *, pre=None, act: str = "none", dx=None, dw=None, dbias=None, workspace, exact: bool = False,
                    stream=None):
    """dgc_linear_backward: the wanted ones of dx [..., K], dw [M, K] and dbias fp32 [M] from dy [..., M]; `pre`: what
    linear_forward left, needed with an activation; workspace: linear_workspace_bytes device bytes.  exact=True: bfloat16's dy act'(pre)
    is not rounded to bfloat16 before it is multiplied."""
    lib, code, dev = _op_first(x, "x")
    dt = x.dtype
    px, ldx = _op_rows(x, "x")
    K, R, M = x.shape[-1], _op_count(x), w.shape[0]
    pw, ldw = _op_rows(w, "w", dt, dev, (M, K))
    pdy, lddy = _op_rows(dy, "dy", dt, dev, (R, M))
    pp, ldp = _op_rows(pre, "pre", dt, dev, (R, M))
    pdx, lddx = _op_rows(dx, "dx", dt, dev, (R, K))
    pdw, lddw = _op_rows(dw, "dw", dt, dev, (M, K))
    ws, ws_bytes = _op_workspace(workspace, dev)
    _op_call(lib.dgc_linear_backward, dev, stream, pdy, lddy, px, ldx, pw, ldw, R, K, M, code, pp, ldp, LINEAR_ACT[act] + (LINEAR_EXACT if exact else 0), pdx, lddx, pdw, lddw,
             _op_flat(dbias, "dbias", M, dev), ws, ws_bytes)


def decay_attn_workspace_bytes(T: int, N: int, heads: int, dk: int, dv: int, *, backward: bool = False) -> int:
    """Bytes that the calls need: none for short windows, segment states for few long sequences."""
    return int(load().dgc_decay_attn_workspace_bytes(int(T), int(N), int(heads), int(dk), int(dv), int(backward)))


def _op_seq(t, name: str, dtype, dev: int, T: int, N: int, F: int):
    """(address, stride of t, stride of i) of rows (t, i) in a [T, N, F] tensor or view."""
    if t is None:
        return None, 0, 0
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name} must be a device tensor of the first tensor's element type and device")
    st = t.stride()
    if tuple(t.shape) != (T, N, F) or st[2] != 1:
        raise ValueError(f"{name} must be [{T}, {N}, {F}] with a contiguous last dimension")
    return t.data_ptr(), (st[0] if T > 1 else 0), (st[1] if N > 1 else 0)


def _decay_sizes(q, v, heads: int):
    if q.dim() != 3 or v.dim() != 3 or heads < 1 or q.shape[2] % heads or v.shape[2] % heads:
        raise ValueError("q, k, v must be [T, N, heads * size of a head]")
    return q.shape[0], q.shape[1], q.shape[2] // heads, v.shape[2] // heads


def decay_attn_forward(q, k, v, decay, o, *, heads: int, scale: float = 1.0, s0=None, sn=None, lengths=None, reset=None,
                       workspace=None, stream=None):
    """dgc_decay_attn_forward: S_t = g S_{t-1} + k_t^T v_t, o_t = scale q_t S_t for every sequence i and head.  q, k [T, N,
    heads * dk], v, o [T, N, heads * dv], float32 or bfloat16, with any strides of t and i (a transposed [N, T, .] tensor is
    fine); decay fp32 [heads], each in [0, 1]; s0, sn fp32 [N, heads, dk, dv] or None (sn may be s0); lengths int32 [N]: tokens
    of each sequence, rows behind them are not written; reset uint8 [T, N]: a non-zero byte drops the state entering (t, i).
    workspace: decay_attn_workspace_bytes device bytes, None where that is 0.  T = 1 is the form for one new snapshot."""
    lib, code, dev = _op_first(q, "q")
    dt = q.dtype
    T, N, dk, dv = _decay_sizes(q, v, heads)
    state = (N, heads, dk, dv)
    ws, ws_bytes = _op_workspace(workspace, dev)
    _op_call(lib.dgc_decay_attn_forward, dev, stream, *_op_seq(q, "q", dt, dev, T, N, heads * dk), *_op_seq(k, "k", dt, dev, T, N, heads * dk),
             *_op_seq(v, "v", dt, dev, T, N, heads * dv), T, N, heads, dk, dv, code, _op_flat(decay, "decay", heads, dev), float(scale),
             _op_shape(s0, "s0", state, dev), _op_flat(lengths, "lengths", N, dev, _torch.int32), _op_shape(reset, "reset", (T, N), dev, _torch.uint8),
             *_op_seq(o, "o", dt, dev, T, N, heads * dv), _op_shape(sn, "sn", state, dev), ws, ws_bytes)
    return o


def decay_attn_backward(q, k, v, decay, do, dq, dk, dv, *, heads: int, scale: float = 1.0, s0=None, dsn=None, ds0=None, lengths=None,
                        reset=None, workspace=None, stream=None):
    """dgc_decay_attn_backward: the gradients of decay_attn_forward's q, k, v (each may be None: not wanted) and s0 (ds0) from
    do and the last state's gradient dsn (None: zero); ds0 may be dsn.  decay is a constant."""
    lib, code, dev = _op_first(q, "q")
    dt = q.dtype
    T, N, nk, nv = _decay_sizes(q, v, heads)
    state = (N, heads, nk, nv)
    ws, ws_bytes = _op_workspace(workspace, dev)
    _op_call(lib.dgc_decay_attn_backward, dev, stream, *_op_seq(q, "q", dt, dev, T, N, heads * nk), *_op_seq(k, "k", dt, dev, T, N, heads * nk),
             *_op_seq(v, "v", dt, dev, T, N, heads * nv), *_op_seq(do, "do", dt, dev, T, N, heads * nv), T, N, heads, nk, nv, code,
             _op_flat(decay, "decay", heads, dev), float(scale), _op_shape(s0, "s0", state, dev), _op_shape(dsn, "dsn", state, dev),
             _op_flat(lengths, "lengths", N, dev, _torch.int32), _op_shape(reset, "reset", (T, N), dev, _torch.uint8),
             *_op_seq(dq, "dq", dt, dev, T, N, heads * nk), *_op_seq(dk, "dk", dt, dev, T, N, heads * nk), *_op_seq(dv, "dv", dt, dev, T, N, heads * nv),
             _op_shape(ds0, "ds0", state, dev), ws, ws_bytes)
