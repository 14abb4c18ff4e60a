"""Thin Python binding of librairs.so: argument marshalling only.

Function names mirror include/rairs.h.  PyTorch supplies device memory and the stream; every
step of the search runs in the library's HIP kernels.  There is no CPU fallback: if the shared
library is missing, loading raises.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import NamedTuple, Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librairs.so")
_lib = None

STAGES = ("coarse", "lut", "scan", "refine", "scan_kernel")
MAX_REFINE_K = 1024
MAX_NPROBE = 4096

EXPORTS = ("rairs_index_upload", "rairs_search", "rairs_free", "rairs_workspace_bytes", "rairs_set_workspace",
           "rairs_search_noalloc", "rairs_graph_create", "rairs_graph_launch", "rairs_graph_free",
           "rairs_coarse", "rairs_lut",
           "rairs_scan", "rairs_refine", "rairs_set_scan_mode", "rairs_set_profiling", "rairs_get_stage_ms",
           "rairs_get_stage_ms_mean",
           "rairs_get_dco", "rairs_get_scan_stats", "rairs_scan_kernel_name", "rairs_index_bytes", "rairs_pq_encode", "rairs_assign",
           "rairs_project", "rairs_project_workspace_bytes", "rairs_project_backward", "rairs_project_backward_workspace_bytes",
           "rairs_search_projected", "rairs_index_table",
           "rairs_logprob", "rairs_logprob_workspace_bytes", "rairs_logprob_backward", "rairs_logprob_backward_workspace_bytes",
           "rairs_last_error")


PROFILE_STAGES, PROFILE_SCAN_KERNEL = 1, 2


class RairsError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"rairs error {code}: {msg}")
        self.code = code


class _HostIndex(C.Structure):
    _fields_ = [
        ("d", C.c_int32), ("M", C.c_int32), ("nbits", C.c_int32), ("nlist", C.c_int32),
        ("blk", C.c_int32), ("raw_is_u8", C.c_int32),
        ("ntotal", C.c_int64), ("nblocks", C.c_int64), ("nrefs", C.c_int64),
        ("centroids", C.c_void_p), ("codebook", C.c_void_p), ("codes", C.c_void_p),
        ("ids", C.c_void_p), ("other", C.c_void_p),
        ("list_shared_begin", C.c_void_p), ("list_shared_cnt", C.c_void_p),
        ("list_misc_begin", C.c_void_p), ("list_misc_cnt", C.c_void_p),
        ("list_ref_begin", C.c_void_p), ("list_ref_cnt", C.c_void_p),
        ("ref_owner", C.c_void_p), ("ref_block_begin", C.c_void_p), ("ref_nblocks", C.c_void_p),
        ("raw", C.c_void_p), ("metric", C.c_int32),
    ]


def load() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with "
                "`python -m paper_2601_07183_amd.build_ext` (there is no fallback path)")
        lib = C.CDLL(LIB_PATH)
        lib.rairs_last_error.restype = C.c_char_p
        lib.rairs_workspace_bytes.restype = C.c_size_t
        lib.rairs_scan_kernel_name.restype = C.c_char_p
        for name in ("rairs_project", "rairs_project_backward", "rairs_logprob", "rairs_logprob_backward"):
            getattr(lib, name + "_workspace_bytes").restype = C.c_size_t
        for name in EXPORTS:
            getattr(lib, name)
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != 0:
        raise RairsError(rc, load().rairs_last_error().decode())


def _stream_ptr(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _dev(t: torch.Tensor, dtype, name: str) -> C.c_void_p:
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise TypeError(f"{name}: expected a contiguous device tensor of {dtype}")
    return C.c_void_p(t.data_ptr())


_ARRAYS = [("centroids", np.float32), ("codebook", np.float32), ("codes", np.uint8),
           ("ids", np.int64), ("other", np.int32), ("list_shared_begin", np.int64),
           ("list_shared_cnt", np.int32), ("list_misc_begin", np.int64),
           ("list_misc_cnt", np.int32), ("list_ref_begin", np.int64), ("list_ref_cnt", np.int32),
           ("ref_owner", np.int32), ("ref_block_begin", np.int64), ("ref_nblocks", np.int32)]


def pq_encode(codebook: torch.Tensor, vectors: torch.Tensor, stream=None) -> torch.Tensor:
    """rairs_pq_encode: packed codes [n][M/2] of device vectors [n][d] for a device codebook [M][16][d/M]."""
    lib = load()
    M, ksub, dsub = codebook.shape
    if ksub != 16 or vectors.ndim != 2 or vectors.shape[1] != M * dsub:
        raise ValueError("codebook must be [M][16][d/M] and vectors [n][d]")
    n = vectors.shape[0]
    codes = torch.empty((n, M // 2), dtype=torch.uint8, device=vectors.device)
    _check(lib.rairs_pq_encode(_dev(codebook, torch.float32, "codebook"), C.c_int(M * dsub), C.c_int(M),
                               _dev(vectors, torch.float32, "vectors") if n else C.c_void_p(0),
                               C.c_int64(n), _dev(codes, torch.uint8, "codes") if n else C.c_void_p(0),
                               _stream_ptr(stream)))
    return codes


# --- the query side: projection with low-rank adapters, log probabilities -----------------------

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.uint8: 2}
MAX_TOP = 64


class _Projection(C.Structure):
    _fields_ = [("d_in", C.c_int32), ("d_out", C.c_int32), ("rank", C.c_int32), ("n_adapters", C.c_int32),
                ("dtype", C.c_int32), ("W", C.c_void_p), ("A", C.c_void_p), ("B", C.c_void_p), ("scale", C.c_void_p)]


class _Table(C.Structure):
    _fields_ = [("vectors", C.c_void_p), ("ld", C.c_int64), ("V", C.c_int64), ("d", C.c_int32), ("dtype", C.c_int32),
                ("scale", C.c_float), ("d_live", C.c_void_p), ("ld_live", C.c_int64)]


class _On:
    """The device of a call's tensors current, and `stream` the stream that its workspace and results are
    allocated for (None: the device's current one); its address.  (A small projection takes less time than
    switching to the device that is current already: that is left out.)"""
    __slots__ = ("device", "stream", "ctx")

    def __init__(self, device, stream):
        self.device, self.stream, self.ctx = device, stream, None

    def __enter__(self) -> C.c_void_p:
        if self.stream is not None and self.stream.device != self.device:
            raise ValueError(f"stream: expected one of {self.device}")
        if self.stream is not None or torch.cuda.current_device() != self.device.index:
            self.ctx = contextlib.ExitStack()
            self.ctx.enter_context(torch.cuda.device(self.device))
            if self.stream is not None:
                self.ctx.enter_context(torch.cuda.stream(self.stream))
                return C.c_void_p(self.stream.cuda_stream)
        return C.c_void_p(_raw_stream(self.device.index))

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.close()
        return False


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _rows(t: torch.Tensor, name: str, dtype, cols: int, device):
    """A device matrix whose rows are contiguous (any stride between them): pointer and row stride."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.device == device and t.ndim == 2 and t.dtype == dtype
            and t.shape[1] == cols and (cols == 1 or t.shape[0] == 0 or t.stride(1) == 1)):
        raise TypeError(f"{name}: expected a matrix of {dtype} with {cols} contiguous columns on {device}")
    ld = t.stride(0) if t.shape[0] > 1 else max(cols, t.stride(0))
    return C.c_void_p(t.data_ptr() if t.numel() else 0), C.c_int64(ld)


def _vec(t, name: str, dtype, n: int, device) -> C.c_void_p:
    if t is None:
        return C.c_void_p(0)
    if not (isinstance(t, torch.Tensor) and t.device == device and t.is_cuda and t.dtype == dtype and t.shape == (n,)
            and t.is_contiguous()):
        raise TypeError(f"{name}: expected {n} contiguous values of {dtype} on {device}")
    return C.c_void_p(t.data_ptr() if n else 0)


def _workspace(need: int, device):
    if need == 0:
        return None, C.c_void_p(0), C.c_size_t(0)
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    return ws, C.c_void_p(ws.data_ptr()), C.c_size_t(need)


class Projection:
    """A projection that all tenants share, W [d_out][d_in], and the low-rank adapters of each, A [n][rank][d_in],
    B [n][d_out][rank], scale [n] (None: 1): y = W x + scale[a] B[a] (A[a] x).  All of float32 or bfloat16,
    contiguous on one device; scale is float32.  Holds the tensors, copies nothing."""

    def __init__(self, W: torch.Tensor, A: Optional[torch.Tensor] = None, B: Optional[torch.Tensor] = None,
                 scale: Optional[torch.Tensor] = None):
        if W.ndim != 2 or W.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("W must be a matrix of float32 or bfloat16")
        if (A is None) != (B is None):
            raise ValueError("A and B: both or neither")
        self.W, self.A, self.B, self.scale = W, A, B, scale
        self.d_out, self.d_in = W.shape
        self.n_adapters, self.rank = (0, 0) if A is None else (A.shape[0], A.shape[1])
        s = self._s = _Projection()
        s.d_in, s.d_out, s.rank, s.n_adapters, s.dtype = self.d_in, self.d_out, self.rank, self.n_adapters, DTYPES[W.dtype]
        s.W = _dev(W, W.dtype, "W")
        if A is not None:
            if A.shape != (self.n_adapters, self.rank, self.d_in) or B.shape != (self.n_adapters, self.d_out, self.rank):
                raise ValueError("A must be [n][rank][d_in] and B [n][d_out][rank]")
            if A.device != W.device or B.device != W.device:
                raise TypeError("W, A and B must be on one device")
            s.A, s.B = _dev(A, W.dtype, "A"), _dev(B, W.dtype, "B")
            s.scale = _vec(scale, "scale", torch.float32, self.n_adapters, W.device)

    def project(self, x: torch.Tensor, adapter: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                out_dtype=None, stream=None) -> torch.Tensor:
        """rairs_project: rows [n][d_in] to [n][d_out], float32 (what a search takes) unless out or out_dtype
        says W's type; adapter [n] int32, a value outside [0, n_adapters) is none."""
        lib, dev, n = load(), self.W.device, x.shape[0]
        px, ldx = _rows(x, "x", self.W.dtype, self.d_in, dev)
        pa = _vec(adapter, "adapter", torch.int32, n, dev)
        with _On(dev, stream) as st:
            given = out is not None
            if not given:
                out = torch.empty((n, self.d_out), dtype=out_dtype or torch.float32, device=dev)
            elif out.shape[0] != n or (out_dtype is not None and out.dtype != out_dtype):
                raise ValueError("out does not fit")
            if out.dtype not in DTYPES:
                raise TypeError(f"out: unsupported type {out.dtype}")
            py, ldy = _rows(out, "out", out.dtype, self.d_out, dev) if given else (
                C.c_void_p(out.data_ptr() if n else 0), C.c_int64(self.d_out))
            need = lib.rairs_project_workspace_bytes(C.byref(self._s), C.c_int64(n))
            ws, pw, nw = _workspace(need, dev)
            _check(lib.rairs_project(C.byref(self._s), px, ldx, C.c_int64(n), pa, py, ldy, C.c_int(DTYPES[out.dtype]),
                                     pw, nw, st))
        return out

    def backward(self, x: torch.Tensor, adapter: Optional[torch.Tensor], dy: torch.Tensor, x_grad: bool = True,
                 adapter_grad: bool = True, stream=None):
        """rairs_project_backward: (dx, dA, dB) for dy [n][d_out] of W's type; None for what is not wanted."""
        lib, dev, n, t = load(), self.W.device, x.shape[0], self.W.dtype
        px, ldx = _rows(x, "x", t, self.d_in, dev)
        pg, ldg = _rows(dy, "dy", t, self.d_out, dev)
        if dy.shape[0] != n:
            raise ValueError("dy must have as many rows as x")
        pa = _vec(adapter, "adapter", torch.int32, n, dev)
        adapter_grad = adapter_grad and self.n_adapters > 0
        with _On(dev, stream) as st:
            dx = torch.empty((n, self.d_in), dtype=t, device=dev) if x_grad else None
            da = torch.empty_like(self.A) if adapter_grad else None
            db = torch.empty_like(self.B) if adapter_grad else None
            need = lib.rairs_project_backward_workspace_bytes(C.byref(self._s), C.c_int64(n))
            ws, pw, nw = _workspace(need, dev)
            _check(lib.rairs_project_backward(
                C.byref(self._s), px, ldx, C.c_int64(n), pa, pg, ldg,
                C.c_void_p(dx.data_ptr() if x_grad and n else 0), C.c_int64(self.d_in),
                C.c_void_p(da.data_ptr() if adapter_grad else 0), C.c_void_p(db.data_ptr() if adapter_grad else 0),
                pw, nw, st))
        return dx, da, db


class LogProb(NamedTuple):
    logp: torch.Tensor                       # [n] log p of each query's target
    lse: torch.Tensor                        # [n] log sum exp of its live rows
    entropy: Optional[torch.Tensor]          # [n]
    top_ids: Optional[torch.Tensor]          # [n][top] int64
    top_logp: Optional[torch.Tensor]         # [n][top]


def _table(table: torch.Tensor, scale: float, live, n: int):
    dev = table.device
    if table.dtype not in DTYPES:
        raise TypeError(f"table: unsupported type {table.dtype}")
    if table.ndim != 2:
        raise TypeError("table must be a matrix")
    t = _Table()
    t.vectors, ld = _rows(table, "table", table.dtype, table.shape[1], dev)
    t.ld, t.V, t.d, t.dtype, t.scale = ld.value, table.shape[0], table.shape[1], DTYPES[table.dtype], scale
    return _with_mask(t, live, n, dev)


def _with_mask(t, live, n: int, dev):
    if live is not None:
        words = (t.V + 31) // 32
        if live.ndim == 1:
            t.d_live, t.ld_live = _vec(live, "live", torch.int32, words, dev), 0
        else:
            if live.shape[0] != n:
                raise ValueError("live: one mask, or one per query")
            t.d_live, ld = _rows(live, "live", torch.int32, words, dev)
            t.ld_live = ld.value
    return t


def _logprob(t, q, targets, top, entropy, stream) -> LogProb:
    lib, dev, n = load(), q.device, q.shape[0]
    qt = _query_type(t)
    pq, ldq = _rows(q, "q", qt, t.d, dev)
    pt = _vec(targets, "targets", torch.int64, n, dev)
    with _On(dev, stream) as st:
        need = lib.rairs_logprob_workspace_bytes(C.byref(t), C.c_int64(n), C.c_int(DTYPES[qt]), C.c_int(top))
        ws, pw, nw = _workspace(need, dev)
        values = lambda *shape: torch.empty(shape, dtype=torch.float32, device=dev)     # (whatever torch's default type is)
        r = LogProb(values(n), values(n), values(n) if entropy else None,
                    torch.empty((n, top), dtype=torch.int64, device=dev) if top > 0 else None, values(n, top) if top > 0 else None)
        p = [C.c_void_p(x.data_ptr() if x is not None and n else 0) for x in r]
        _check(lib.rairs_logprob(C.byref(t), pq, ldq, C.c_int(DTYPES[qt]), C.c_int64(n), pt, p[0], p[1], p[2], C.c_int(top), p[3],
                                 p[4], pw, nw, st))
    return r


def logprob(q: torch.Tensor, table: torch.Tensor, targets: torch.Tensor, scale: float = 1.0, top: int = 0,
            live: Optional[torch.Tensor] = None, entropy: bool = True, stream=None) -> LogProb:
    """rairs_logprob: softmax over scale * <q, row> of the table's live rows.  q [n][d] and table [V][d] of
    float32 or bfloat16 (a uint8 table: float32 queries), rows may be strided; targets [n] int64 (outside
    [0, V): none); live: int32 words of 32 rows each, [words] for all queries or [n][words]."""
    return _logprob(_table(table, scale, live, q.shape[0]), q, targets, top, entropy, stream)


def _query_type(t):
    return torch.float32 if t.dtype == DTYPES[torch.uint8] else {v: k for k, v in DTYPES.items()}[t.dtype]


def _logprob_backward(t, q, targets, lse, dlogp, entropy, dentropy, q_grad, table_dtype, stream):
    """table_dtype: the type of the table's gradient, None: not wanted."""
    lib, dev, n, qt = load(), q.device, q.shape[0], _query_type(t)
    pq, ldq = _rows(q, "q", qt, t.d, dev)
    f = [_vec(x, name, torch.float32, n, dev) for x, name in
         ((lse, "lse"), (entropy, "entropy"), (dlogp, "dlogp"), (dentropy, "dentropy"))]
    pt = _vec(targets, "targets", torch.int64, n, dev)
    with _On(dev, stream) as st:
        need = lib.rairs_logprob_backward_workspace_bytes(C.byref(t), C.c_int64(n), C.c_int(DTYPES[qt]), C.c_int(int(table_dtype is not None)))
        ws, pw, nw = _workspace(need, dev)
        dq = torch.empty((n, t.d), dtype=qt, device=dev) if q_grad else None
        dt = torch.empty((t.V, t.d), dtype=table_dtype, device=dev) if table_dtype is not None else None
        _check(lib.rairs_logprob_backward(
            C.byref(t), pq, ldq, C.c_int(DTYPES[qt]), C.c_int64(n), pt, f[0], f[1], f[2], f[3],
            C.c_void_p(dq.data_ptr() if q_grad and n else 0), C.c_int64(t.d),
            C.c_void_p(dt.data_ptr() if dt is not None else 0), C.c_int64(t.d), pw, nw, st))
    return dq, dt


def logprob_backward(q: torch.Tensor, table: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, dlogp: torch.Tensor,
                     scale: float = 1.0, live: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                     dentropy: Optional[torch.Tensor] = None, q_grad: bool = True, table_grad: bool = False, stream=None):
    """rairs_logprob_backward: (dq, dtable) for the gradients dlogp, dentropy [n] of logprob's results; None for
    what is not wanted.  lse and entropy are logprob's."""
    return _logprob_backward(_table(table, scale, live, q.shape[0]), q, targets, lse, dlogp, entropy, dentropy, q_grad,
                             table.dtype if table_grad else None, stream)


def host_struct(hx):
    """ctypes view of a host index object (attributes named as in rairs_host_index_t)."""
    keep = []
    s = _HostIndex()
    s.d, s.M, s.nbits, s.nlist, s.blk = hx.d, hx.M, 4, hx.nlist, int(np.shape(hx.ids)[1])
    s.metric = {"l2": 0, "ip": 1}[getattr(hx, "metric", "l2")]
    s.ntotal, s.nblocks, s.nrefs = hx.ntotal, hx.ids.shape[0], hx.ref_owner.shape[0]
    for name, dt in _ARRAYS:
        a = np.ascontiguousarray(getattr(hx, name), dtype=dt)
        keep.append(a)
        setattr(s, name, a.ctypes.data)
    raw = np.ascontiguousarray(hx.raw)
    if raw.dtype not in (np.float32, np.uint8):
        raise TypeError("raw vectors must be float32 or uint8")
    s.raw_is_u8 = int(raw.dtype == np.uint8)
    s.raw = raw.ctypes.data
    keep.append(raw)
    return s, keep


class SearchGraph:
    """A captured search (rairs_graph_create ... rairs_graph_free); keeps its tensors alive."""

    def __init__(self, lib, g, tensors):
        self._lib, self._g, self._tensors = lib, g, tensors

    def launch(self, stream=None):
        _check(self._lib.rairs_graph_launch(self._g, _stream_ptr(stream)))

    def free(self):
        if self._g:
            _check(self._lib.rairs_graph_free(self._g))
            self._g = C.c_void_p()

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


class Index:
    """Device-resident RAIRS index (rairs_index_upload ... rairs_free)."""

    def __init__(self, hx, stream=None):
        self._h = C.c_void_p()
        self._lib = load()
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the search path has no CPU implementation")
        s, keep = host_struct(hx)
        _check(self._lib.rairs_index_upload(C.byref(s), _stream_ptr(stream), C.byref(self._h)))
        del keep
        self.d, self.M, self.nlist, self.ntotal = hx.d, hx.M, hx.nlist, hx.ntotal
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._ws = None                 # torch tensor that serves as the handle's workspace

    # --- workspace: device memory comes from PyTorch ------------------------------------------
    def workspace_bytes(self, nq: int, nprobe: int, refine_k: int) -> int:
        """rairs_workspace_bytes (0 for an empty batch; raises on arguments the search rejects)."""
        n = int(self._lib.rairs_workspace_bytes(self._h, C.c_int64(nq), C.c_int(nprobe), C.c_int(refine_k)))
        if n == 0 and nq > 0:
            raise RairsError(-1, self._lib.rairs_last_error().decode())
        return n

    def set_workspace(self, ws):
        """rairs_set_workspace: a uint8 device tensor (kept alive here), or None for the handle's own."""
        if ws is None:
            _check(self._lib.rairs_set_workspace(self._h, C.c_void_p(0), C.c_size_t(0)))
        else:
            _check(self._lib.rairs_set_workspace(self._h, _dev(ws, torch.uint8, "workspace"),
                                                 C.c_size_t(ws.numel())))
        self._ws = ws

    def _reserve(self, nq: int, nprobe: int, refine_k: int):
        """Give the handle a torch-allocated workspace large enough for this call (arguments that
        the library rejects are left to the call itself, which reports them)."""
        if nq <= 0 or self._ws is False:
            return
        need = int(self._lib.rairs_workspace_bytes(self._h, C.c_int64(nq), C.c_int(nprobe), C.c_int(refine_k)))
        if need and (self._ws is None or self._ws.numel() < need):
            torch.cuda.current_stream().synchronize()     # nothing of this handle is in flight
            self._ws = None
            self.set_workspace(torch.empty(need, dtype=torch.uint8, device="cuda"))

    def use_own_workspace(self):
        """Let the library allocate and grow its workspace itself (hipMalloc inside the handle)."""
        self.set_workspace(None)
        self._ws = False

    def free(self):
        if self._h:
            _check(self._lib.rairs_free(self._h))
            self._h = C.c_void_p()
            self._ws = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    # --- rairs_search ---------------------------------------------------------------------
    def search(self, queries: torch.Tensor, k: int, nprobe: int, refine_k: int, out_ids=None,
               out_dists=None, stream=None):
        nq = queries.shape[0]
        if out_ids is None:
            out_ids = torch.empty((nq, k), dtype=torch.int64, device=queries.device)
        if out_dists is None:
            out_dists = torch.empty((nq, k), dtype=torch.float32, device=queries.device)
        self._reserve(nq, nprobe, refine_k)
        _check(self._lib.rairs_search(
            self._h, _dev(queries, torch.float32, "queries"), C.c_int64(nq), C.c_int(k),
            C.c_int(nprobe), C.c_int(refine_k), _dev(out_ids, torch.int64, "out_ids"),
            _dev(out_dists, torch.float32, "out_dists"), _stream_ptr(stream)))
        return out_ids, out_dists

    def search_noalloc(self, queries: torch.Tensor, k: int, nprobe: int, refine_k: int, out_ids,
                       out_dists, stream=None):
        """rairs_search_noalloc: the caller supplies the outputs; scratch memory is the library's
        static device array."""
        _check(self._lib.rairs_search_noalloc(
            self._h, _dev(queries, torch.float32, "queries"), C.c_int64(queries.shape[0]), C.c_int(k),
            C.c_int(nprobe), C.c_int(refine_k), _dev(out_ids, torch.int64, "out_ids"),
            _dev(out_dists, torch.float32, "out_dists"), _stream_ptr(stream)))
        return out_ids, out_dists

    def graph(self, queries: torch.Tensor, k: int, nprobe: int, refine_k: int, out_ids, out_dists, stream):
        """rairs_graph_create: returns a SearchGraph that replays this search on the given tensors."""
        g = C.c_void_p()
        _check(self._lib.rairs_graph_create(
            self._h, _dev(queries, torch.float32, "queries"), C.c_int64(queries.shape[0]), C.c_int(k),
            C.c_int(nprobe), C.c_int(refine_k), _dev(out_ids, torch.int64, "out_ids"),
            _dev(out_dists, torch.float32, "out_dists"), _stream_ptr(stream), C.byref(g)))
        return SearchGraph(self._lib, g, (queries, out_ids, out_dists))

    # --- the query side -------------------------------------------------------------------
    def search_projected(self, projection: Projection, x: torch.Tensor, adapter, k: int, nprobe: int, refine_k: int,
                         stream=None):
        """rairs_search_projected: rows [n][d_in] through the projection and into the search; returns ids,
        distances and the queries that were searched with [n][d]."""
        n, dev = x.shape[0], self._on_device(projection.W, "the projection")
        px, ldx = _rows(x, "x", projection.W.dtype, projection.d_in, dev)
        pa = _vec(adapter, "adapter", torch.int32, n, dev)
        with _On(dev, stream) as st:
            self._reserve(n, nprobe, refine_k)
            ids = torch.empty((n, k), dtype=torch.int64, device=dev)
            dists = torch.empty((n, k), dtype=torch.float32, device=dev)
            q = torch.empty((n, self.d), dtype=torch.float32, device=dev)
            need = self._lib.rairs_project_workspace_bytes(C.byref(projection._s), C.c_int64(n))
            ws, pw, nw = _workspace(need, dev)
            _check(self._lib.rairs_search_projected(
                self._h, C.byref(projection._s), px, ldx, C.c_int64(n), pa, C.c_void_p(q.data_ptr() if n else 0), C.c_int(k),
                C.c_int(nprobe), C.c_int(refine_k), C.c_void_p(ids.data_ptr() if n else 0),
                C.c_void_p(dists.data_ptr() if n else 0), pw, nw, st))
        return ids, dists, q

    def logprob(self, q: torch.Tensor, targets: torch.Tensor, scale: float = 1.0, top: int = 0, live=None,
                entropy: bool = True, stream=None) -> LogProb:
        """logprob over the index's own vectors (rairs_index_table): float32 queries, targets are vector ids."""
        dev = self._on_device(q, "q")
        return _logprob(self._table(scale, live, q.shape[0], dev), q, targets, top, entropy, stream)

    def logprob_backward(self, q: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, dlogp: torch.Tensor, scale: float = 1.0,
                         live=None, entropy=None, dentropy=None, stream=None) -> torch.Tensor:
        """dq [n][d] float32 for the gradients dlogp, dentropy [n] of logprob's results (the index's vectors stay);
        lse and entropy are logprob's."""
        dev = self._on_device(q, "q")
        return _logprob_backward(self._table(scale, live, q.shape[0], dev), q, targets, lse, dlogp, entropy, dentropy, True, None, stream)[0]

    def _on_device(self, t: torch.Tensor, name: str):
        if t.device != self.device:
            raise TypeError(f"{name}: expected on the index's device {self.device}, got {t.device}")
        return self.device

    def _table(self, scale: float, live, n: int, dev):
        t = _Table()
        _check(self._lib.rairs_index_table(self._h, C.byref(t)))
        t.scale = scale
        return _with_mask(t, live, n, dev)

    # --- stages ---------------------------------------------------------------------------
    def coarse(self, queries: torch.Tensor, nprobe: int, stream=None):
        nq = queries.shape[0]
        self._reserve(nq, nprobe, 1)
        ids = torch.empty((nq, nprobe), dtype=torch.int32, device=queries.device)
        dists = torch.empty((nq, nprobe), dtype=torch.float32, device=queries.device)
        _check(self._lib.rairs_coarse(self._h, _dev(queries, torch.float32, "queries"),
                                      C.c_int64(nq), C.c_int(nprobe), _dev(ids, torch.int32, "ids"),
                                      _dev(dists, torch.float32, "dists"), _stream_ptr(stream)))
        return ids, dists

    def lut(self, queries: torch.Tensor, stream=None):
        nq = queries.shape[0]
        lut = torch.empty((nq, self.M, 16), dtype=torch.uint8, device=queries.device)
        bias = torch.empty((nq,), dtype=torch.float32, device=queries.device)
        scale = torch.empty((nq,), dtype=torch.float32, device=queries.device)
        _check(self._lib.rairs_lut(self._h, _dev(queries, torch.float32, "queries"), C.c_int64(nq),
                                   _dev(lut, torch.uint8, "lut"), _dev(bias, torch.float32, "bias"),
                                   _dev(scale, torch.float32, "scale"), _stream_ptr(stream)))
        return lut, bias, scale

    def scan(self, lut: torch.Tensor, probe_ids: torch.Tensor, refine_k: int, stream=None):
        nq, nprobe = probe_ids.shape
        self._reserve(nq, nprobe, refine_k)
        cand = torch.empty((nq, refine_k), dtype=torch.int64, device=lut.device)
        score = torch.empty((nq, refine_k), dtype=torch.int32, device=lut.device)
        dco = torch.empty((nq,), dtype=torch.int64, device=lut.device)
        _check(self._lib.rairs_scan(self._h, _dev(lut, torch.uint8, "lut"),
                                    _dev(probe_ids, torch.int32, "probe_ids"), C.c_int64(nq),
                                    C.c_int(nprobe), C.c_int(refine_k),
                                    _dev(cand, torch.int64, "cand"), _dev(score, torch.int32, "score"),
                                    _dev(dco, torch.int64, "dco"), _stream_ptr(stream)))
        return cand, score, dco

    def refine(self, queries: torch.Tensor, cand_ids: torch.Tensor, k: int, stream=None):
        nq, refine_k = cand_ids.shape
        ids = torch.empty((nq, k), dtype=torch.int64, device=queries.device)
        dists = torch.empty((nq, k), dtype=torch.float32, device=queries.device)
        _check(self._lib.rairs_refine(self._h, _dev(queries, torch.float32, "queries"),
                                      _dev(cand_ids, torch.int64, "cand_ids"), C.c_int64(nq),
                                      C.c_int(refine_k), C.c_int(k), _dev(ids, torch.int64, "ids"),
                                      _dev(dists, torch.float32, "dists"), _stream_ptr(stream)))
        return ids, dists

    def set_scan_mode(self, exact: bool, list_major: bool = False):
        """rairs_set_scan_mode: automatic, the exact kernel, or (list_major) the list-major search for small batches too."""
        _check(self._lib.rairs_set_scan_mode(self._h, C.c_int(1 if exact else 2 if list_major else 0)))

    # --- measurement ----------------------------------------------------------------------
    def set_profiling(self, level):
        """False / 0: off; True / PROFILE_STAGES: every stage; PROFILE_SCAN_KERNEL: the scan kernel only."""
        _check(self._lib.rairs_set_profiling(self._h, C.c_int(int(level))))

    def stage_ms(self) -> dict:
        ms = (C.c_float * len(STAGES))()
        _check(self._lib.rairs_get_stage_ms(self._h, ms))
        return dict(zip(STAGES, [float(x) for x in ms]))

    def stage_ms_mean(self, last_n: int) -> dict:
        ms = (C.c_float * len(STAGES))()
        _check(self._lib.rairs_get_stage_ms_mean(self._h, C.c_int(last_n), ms))
        return dict(zip(STAGES, [float(x) for x in ms]))

    def assign(self, vectors: torch.Tensor, n_cands: int = 10, lam: float = 0.5, strict: bool = True,
               stream=None) -> torch.Tensor:
        """rairs_assign: [n][2] list ids (smaller first) of device vectors [n][d]."""
        n = vectors.shape[0]
        self._reserve(n, max(1, min(n_cands, self.nlist)), 1)
        out = torch.empty((n, 2), dtype=torch.int32, device=vectors.device)
        _check(self._lib.rairs_assign(self._h, _dev(vectors, torch.float32, "vectors") if n else C.c_void_p(0),
                                      C.c_int64(n), C.c_int(n_cands), C.c_double(lam), C.c_int(int(strict)),
                                      _dev(out, torch.int32, "pairs") if n else C.c_void_p(0),
                                      _stream_ptr(stream)))
        return out

    def dco(self, nq: int) -> np.ndarray:
        out = np.empty(nq, dtype=np.int64)
        _check(self._lib.rairs_get_dco(self._h, C.c_void_p(out.ctypes.data), C.c_int64(nq)))
        return out

    def scan_stats(self) -> dict:
        st = (C.c_int64 * 5)()
        _check(self._lib.rairs_get_scan_stats(self._h, st))
        return dict(redone=int(st[0]), survivors=int(st[1]), max_survivors=int(st[2]),
                    queries=int(st[3]), logged=int(st[4]))

    def scan_kernel_name(self) -> str:
        return self._lib.rairs_scan_kernel_name(self._h).decode()

    def bytes(self):
        a, b = C.c_int64(), C.c_int64()
        _check(self._lib.rairs_index_bytes(self._h, C.byref(a), C.byref(b)))
        return a.value, b.value
