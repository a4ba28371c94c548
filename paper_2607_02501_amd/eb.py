"""Python binding of libeb (argument marshalling only).

Every computation runs in the HIP kernels of libeb.so; this module only
allocates outputs and workspaces with torch (the library allocates no device
memory), passes raw device pointers and the current HIP stream, and turns
status codes into exceptions.  It raises at import time if libeb.so has not
been built (there is no fallback path).

Names follow the C ABI in include/eb.h, include/eb_tuning.h, include/eb_multirate.h
and include/eb_attention.h.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libeb.so")

EB_OK = 0
EB_ERR_INVALID = -1
EB_ERR_ALIGN = -2
EB_ERR_UNSUPPORTED = -3
EB_ERR_HIP = -4

EB_Q8_0 = 1
EB_Q4_0 = 2
EB_Q6_S = 3
EB_F32 = 0
EB_F16 = 1
EB_BF16 = 2
EB_PATH_AUTO = 0
EB_PATH_GEMV = 1
EB_PATH_MFMA = 2
EB_PATH_MFMA_I8 = 3
EB_PRO_NONE = 0
EB_PRO_RMSNORM = 1
EB_EPI_NONE = 0
EB_EPI_ADD = 1
EB_EPI_GLU = 2

QTYPES = {"q8_0": EB_Q8_0, "q4_0": EB_Q4_0, "q6_s": EB_Q6_S}
# weights and canonical bytes per block of each format
BLOCK_ELEMS = {"q8_0": 32, "q4_0": 32, "q6_s": 256}
BLOCK_BYTES = {"q8_0": 34, "q4_0": 18, "q6_s": 210}
DTYPES = {torch.float32: EB_F32, torch.float16: EB_F16, torch.bfloat16: EB_BF16}
PATHS = {"auto": EB_PATH_AUTO, "gemv": EB_PATH_GEMV, "mfma": EB_PATH_MFMA, "mfma_i8": EB_PATH_MFMA_I8}
PROLOGUES = {None: EB_PRO_NONE, "none": EB_PRO_NONE, "rmsnorm": EB_PRO_RMSNORM}
EPILOGUES = {None: EB_EPI_NONE, "none": EB_EPI_NONE, "add": EB_EPI_ADD, "glu": EB_EPI_GLU}


class eb_qweights(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("reserved", ctypes.c_int32), ("n", ctypes.c_int64),
                ("k", ctypes.c_int64), ("data", ctypes.c_void_p)]


class eb_layout(ctypes.Structure):
    _fields_ = [("qs_offset", ctypes.c_int64), ("qs_row_bytes", ctypes.c_int64),
                ("d_offset", ctypes.c_int64), ("d_stride", ctypes.c_int64),
                ("total_bytes", ctypes.c_int64), ("canonical_bytes", ctypes.c_int64),
                ("sc_offset", ctypes.c_int64), ("sc_stride", ctypes.c_int64)]


class eb_qlinear_op(ctypes.Structure):
    _fields_ = [("w", eb_qweights), ("x", ctypes.c_void_p), ("y", ctypes.c_void_p),
                ("m", ctypes.c_int64), ("x_type", ctypes.c_int32), ("y_type", ctypes.c_int32),
                ("prologue", ctypes.c_int32), ("epilogue", ctypes.c_int32),
                ("norm_weight", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("norm_eps", ctypes.c_float), ("reserved", ctypes.c_int32)]


if not os.path.exists(LIB_PATH):
    raise ImportError(f"libeb.so not found at {LIB_PATH}: build it first "
                      "(python -m paper_2607_02501_amd.build); there is no fallback path")

lib = ctypes.CDLL(LIB_PATH)

_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
lib.eb_version.restype = ctypes.c_char_p
lib.eb_version.argtypes = []
lib.eb_status_str.restype = ctypes.c_char_p
lib.eb_status_str.argtypes = [_i32]
lib.eb_qweights_bytes.restype = ctypes.c_size_t
lib.eb_qweights_bytes.argtypes = [_i32, _i64, _i64]
lib.eb_qweights_layout.restype = _i32
lib.eb_qweights_layout.argtypes = [_i32, _i64, _i64, ctypes.POINTER(eb_layout)]
for _name in ("eb_quantize_q8_0", "eb_quantize_q4_0", "eb_quantize_q6_s"):
    getattr(lib, _name).restype = _i32
    getattr(lib, _name).argtypes = [_vp, _i64, _i64, _vp, _vp]
lib.eb_qweights_to_canonical.restype = _i32
lib.eb_qweights_to_canonical.argtypes = [ctypes.POINTER(eb_qweights), _vp, _vp]
lib.eb_qweights_from_canonical.restype = _i32
lib.eb_qweights_from_canonical.argtypes = [_i32, _vp, _i64, _i64, _vp, _vp]
lib.eb_qlinear.restype = _i32
lib.eb_qlinear.argtypes = [ctypes.POINTER(eb_qweights), _vp, _i32, _i64, _vp, _i32, _vp]
lib.eb_qlinear_ex.restype = _i32
lib.eb_qlinear_ex.argtypes = [ctypes.POINTER(eb_qweights), _vp, _i32, _i64, _vp, _i32, _i32, _vp]
lib.eb_qlinear_fused.restype = _i32
lib.eb_qlinear_fused.argtypes = [ctypes.POINTER(eb_qlinear_op), _i32, _vp]
lib.eb_qlinear_auto_path.restype = _i32
lib.eb_qlinear_auto_path.argtypes = [_i32, _i32, _i64, _i64, _i64]
lib.eb_qlinear_stack.restype = _i32
lib.eb_qlinear_stack.argtypes = [ctypes.POINTER(eb_qlinear_op), _i32, _vp, ctypes.c_size_t, _vp]
lib.eb_qlinear_stack_workspace_bytes.restype = ctypes.c_size_t
lib.eb_qlinear_stack_workspace_bytes.argtypes = [ctypes.POINTER(eb_qlinear_op), _i32]
lib.eb_qlinear_workspace_bytes.restype = ctypes.c_size_t
lib.eb_qlinear_workspace_bytes.argtypes = [ctypes.POINTER(eb_qlinear_op), _i32]
lib.eb_qlinear_fused_ws.restype = _i32
lib.eb_qlinear_fused_ws.argtypes = [ctypes.POINTER(eb_qlinear_op), _i32, _vp, ctypes.c_size_t, _vp]
lib.eb_qlinear_fused_static.restype = _i32
lib.eb_qlinear_fused_static.argtypes = [ctypes.POINTER(eb_qlinear_op), _i32, _vp]
lib.eb_qlinear_tuned.restype = _i32
lib.eb_qlinear_tuned.argtypes = [ctypes.POINTER(eb_qlinear_op), _i32, _i32, _vp, ctypes.c_size_t, _vp]
lib.eb_qlinear_stack_launches.restype = _i32
lib.eb_qlinear_stack_launches.argtypes = [ctypes.POINTER(eb_qlinear_op), _i32]


class eb_module(ctypes.Structure):
    _fields_ = [("ops", ctypes.POINTER(eb_qlinear_op)), ("n_ops", _i32), ("period", _i32),
                ("phase", _i32), ("repeats", _i32)]


lib.eb_multirate_workspace_bytes.restype = ctypes.c_size_t
lib.eb_multirate_workspace_bytes.argtypes = [ctypes.POINTER(eb_module), _i32]
lib.eb_multirate_tick.restype = _i32
lib.eb_multirate_tick.argtypes = [ctypes.POINTER(eb_module), _i32, _i64, _vp, ctypes.c_size_t, _vp]
lib.eb_multirate_launches.restype = _i32
lib.eb_multirate_launches.argtypes = [ctypes.POINTER(eb_module), _i32, _i64]
lib.eb_stack_cache_clear.restype = _i32
lib.eb_stack_cache_clear.argtypes = []
lib.eb_mfma_tile_count.restype = _i32
lib.eb_mfma_tile_count.argtypes = []


class EBError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {lib.eb_status_str(status).decode()}")
        self.status = status


def _check(status: int, what: str) -> None:
    if status != EB_OK:
        raise EBError(status, what)


def _stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def version() -> str:
    return lib.eb_version().decode()


def qweights_bytes(qtype: str, n: int, k: int) -> int:
    return int(lib.eb_qweights_bytes(QTYPES[qtype], n, k))


def layout(qtype: str, n: int, k: int) -> eb_layout:
    out = eb_layout()
    _check(lib.eb_qweights_layout(QTYPES[qtype], n, k, ctypes.byref(out)), "eb_qweights_layout")
    return out


class QWeights:
    """A quantized weight matrix W[n, k] held in a caller-owned device buffer."""

    def __init__(self, qtype: str, n: int, k: int, buf: torch.Tensor):
        assert buf.dtype == torch.uint8 and buf.is_cuda
        self.qtype, self.n, self.k, self.buf = qtype, n, k, buf

    @property
    def c(self) -> eb_qweights:
        return eb_qweights(QTYPES[self.qtype], 0, self.n, self.k, self.buf.data_ptr())

    @property
    def device(self):
        return self.buf.device

    def nbytes(self) -> int:
        return qweights_bytes(self.qtype, self.n, self.k)


def empty_qweights(qtype: str, n: int, k: int, device="cuda") -> QWeights:
    nbytes = qweights_bytes(qtype, n, k)
    if nbytes == 0:
        raise EBError(EB_ERR_INVALID, "eb_qweights_bytes")
    # torch's caching allocator returns 512-byte aligned blocks
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return QWeights(qtype, n, k, buf)


def quantize(w: torch.Tensor, qtype: str, out: QWeights | None = None) -> QWeights:
    """fp32 W[n, k] (device) -> QWeights in the planar layout."""
    assert w.dtype == torch.float32 and w.is_cuda and w.dim() == 2
    w = w.contiguous()
    n, k = w.shape
    out = out or empty_qweights(qtype, n, k, w.device)
    fn = {"q8_0": lib.eb_quantize_q8_0, "q4_0": lib.eb_quantize_q4_0,
          "q6_s": lib.eb_quantize_q6_s}[qtype]
    _check(fn(w.data_ptr(), n, k, out.buf.data_ptr(), _stream(w.device)), fn.__name__)
    return out


def to_canonical(qw: QWeights) -> torch.Tensor:
    """Canonical array-of-blocks bytes (device uint8 tensor [n, k/E, block_bytes],
    E = BLOCK_ELEMS[qtype])."""
    dst = torch.empty((qw.n, qw.k // BLOCK_ELEMS[qw.qtype], BLOCK_BYTES[qw.qtype]),
                      dtype=torch.uint8, device=qw.device)
    c = qw.c
    _check(lib.eb_qweights_to_canonical(ctypes.byref(c), dst.data_ptr(), _stream(qw.device)),
           "eb_qweights_to_canonical")
    return dst


def from_canonical(blocks: torch.Tensor, qtype: str, n: int, k: int) -> QWeights:
    assert blocks.dtype == torch.uint8 and blocks.is_cuda
    blocks = blocks.contiguous()
    out = empty_qweights(qtype, n, k, blocks.device)
    _check(lib.eb_qweights_from_canonical(QTYPES[qtype], blocks.data_ptr(), n, k,
                                          out.buf.data_ptr(), _stream(blocks.device)),
           "eb_qweights_from_canonical")
    return out


class _Scratch(threading.local):
    """Workspaces of direct calls, by device and stream.  A thread has its own: a call is
    several launches, and those of two threads on one stream (torch's default for every
    thread) may fall between each other's, since ctypes lets go of the interpreter."""

    def __init__(self):
        self.bufs = {}


_SCRATCH = _Scratch()


_get_device = torch._C._cuda_getDevice
_capturing = torch._C._cuda_isCurrentStreamCapturing


def _capturing_on(dev: int) -> bool:
    """Whether GPU `dev`'s current stream is being captured."""
    was = _get_device()
    if was == dev:
        return _capturing()
    torch.cuda.set_device(dev)
    try:
        return _capturing()
    finally:
        torch.cuda.set_device(was)


def _workspace(device, dev: int, stream: int, nbytes: int) -> torch.Tensor:
    """scratch() of GPU `dev`'s current stream."""
    if _capturing() if _get_device() == dev else _capturing_on(dev):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    bufs = _SCRATCH.bufs
    buf = bufs.get((dev, stream))
    if buf is None or buf.numel() < nbytes:
        buf = bufs[dev, stream] = torch.empty(max(nbytes, 4 << 20), dtype=torch.uint8, device=device)
    return buf


def scratch(device, nbytes: int):
    """A caller-owned workspace of at least nbytes on `device` for direct calls
    on the current stream (one growing torch buffer per thread, device and stream;
    a thread's calls on one stream run in order, so they may share it).  Under graph
    capture a fresh one, of the graph's memory: graphs may run at the same time."""
    if nbytes <= 0:
        return None
    device = torch.device(device)
    dev = device.index if device.index is not None else torch.cuda.current_device()
    return _workspace(device, dev, _stream(device), nbytes)


def _run_tuned(op: eb_qlinear_op, device, tile: int, splits: int) -> None:
    nbytes = int(lib.eb_qlinear_workspace_bytes(ctypes.byref(op), EB_PATH_MFMA))
    nbytes += 64 << 20  # room for any forced split (also where the automatic plan needs none)
    ws = scratch(device, nbytes)
    _check(lib.eb_qlinear_tuned(ctypes.byref(op), tile, splits, ws.data_ptr(), ws.numel(),
                                _stream(device)), "eb_qlinear_tuned")


# One projection called directly: at one token the kernel takes about 4 us, so
# the call's host time counts.  The op is packed into bytes of eb_qlinear_op's
# layout (0.2 us; building the two nested structures takes 1.1), and the size
# of its workspace, which depends on the shape, types, steps, path and device alone,
# is asked for once and kept after a call that succeeded.  Measured at m = 1,
# 2048 -> 2048 (kernel 4 us): 10.1 us per call before, 7.2 now.
_PACK_OP = struct.Struct("iiqqPPPqiiiiPPfi")
assert _PACK_OP.size == ctypes.sizeof(eb_qlinear_op)
_raw = ctypes.CDLL(LIB_PATH)  # the same library, taking ops as bytes
_fused_ws, _ws_bytes = _raw.eb_qlinear_fused_ws, _raw.eb_qlinear_workspace_bytes
_fused_ws.restype, _fused_ws.argtypes = _i32, [ctypes.c_char_p, _i32, _vp, ctypes.c_size_t, _vp]
_ws_bytes.restype, _ws_bytes.argtypes = ctypes.c_size_t, [ctypes.c_char_p, _i32]
_raw_stream = torch._C._cuda_getCurrentRawStream
_WS_BYTES = {}  # at most 4096 entries


def _run_op(qw: QWeights, x: torch.Tensor, out: torch.Tensor, x_type: int, path: int, prologue=0,
            norm_weight=None, eps: float = 0.0, epilogue=0, residual=None) -> None:
    m = x.shape[0]
    dev = x.get_device()
    stream = _raw_stream(dev)
    qtype = QTYPES[qw.qtype]
    op = _PACK_OP.pack(qtype, 0, qw.n, qw.k, qw.buf.data_ptr(), x.data_ptr(), out.data_ptr(), m,
                       x_type, DTYPES[out.dtype], prologue, epilogue,
                       norm_weight.data_ptr() if norm_weight is not None else 0,
                       residual.data_ptr() if residual is not None else 0, eps, 0)
    key = (qtype, m, qw.n, qw.k, x_type, prologue, epilogue, path, dev)
    nbytes = _WS_BYTES.get(key)
    known = nbytes is not None
    if not known:
        nbytes = _ws_bytes(op, path)
    if nbytes:
        ws = _workspace(x.device, dev, stream, nbytes)
        st = _fused_ws(op, path, ws.data_ptr(), ws.numel(), stream)
    else:
        st = _fused_ws(op, path, None, 0, stream)
    if st != EB_OK:
        raise EBError(st, "eb_qlinear_fused_ws")
    if not known:
        if len(_WS_BYTES) >= 4096:
            _WS_BYTES.clear()
        _WS_BYTES[key] = nbytes


def qlinear(qw: QWeights, x: torch.Tensor, out_dtype=torch.float32, path: str = "auto",
            out: torch.Tensor | None = None) -> torch.Tensor:
    """y[m, n] = x[m, k] . w_hat^T on the GPU (fp32 accumulation), with a
    workspace from scratch() so that the MFMA path may split k."""
    assert x.is_cuda and x.dim() == 2 and x.shape[1] == qw.k
    x = x.contiguous()
    if out is None:
        out = torch.empty((x.shape[0], qw.n), dtype=out_dtype, device=x.device)
    _run_op(qw, x, out, EB_BF16 if x.dtype == torch.float32 else DTYPES[x.dtype], PATHS[path])
    return out


def qlinear_tuned(qw: QWeights, x: torch.Tensor, tile: int = -1, splits: int = 0,
                  out_dtype=torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
    """qlinear on the MFMA path with a forced tile configuration / split of k
    (-1 / 0: automatic), for tuning and tests (eb_qlinear_tuned)."""
    assert x.is_cuda and x.dim() == 2 and x.shape[1] == qw.k
    x = x.contiguous()
    if out is None:
        out = torch.empty((x.shape[0], qw.n), dtype=out_dtype, device=x.device)
    _run_tuned(make_op(qw, x, out), x.device, tile, splits)
    return out


def auto_path(qtype: str, x_dtype, m: int, n: int, k: int) -> str:
    p = lib.eb_qlinear_auto_path(QTYPES[qtype], DTYPES[x_dtype], m, n, k)
    return {EB_PATH_GEMV: "gemv", EB_PATH_MFMA: "mfma"}.get(p, "invalid")


def make_op(qw: QWeights, x: torch.Tensor, y: torch.Tensor, x_dtype=None, prologue=None,
            norm_weight: torch.Tensor | None = None, eps: float = 0.0, epilogue=None,
            residual: torch.Tensor | None = None) -> eb_qlinear_op:
    """One eb_qlinear_op.  With prologue="rmsnorm", x is the fp32 residual
    stream and x_dtype the 16-bit type the product consumes (default bf16)."""
    if x_dtype is None:
        x_dtype = torch.bfloat16 if x.dtype == torch.float32 else x.dtype
    return eb_qlinear_op(qw.c, x.data_ptr(), y.data_ptr(), x.shape[0], DTYPES[x_dtype],
                         DTYPES[y.dtype], PROLOGUES[prologue], EPILOGUES[epilogue],
                         norm_weight.data_ptr() if norm_weight is not None else None,
                         residual.data_ptr() if residual is not None else None, float(eps), 0)


def make_ops(entries) -> ctypes.Array:
    """entries: iterable of (QWeights, x, y) or (QWeights, x, y, {make_op keywords}).
    Returns a ctypes eb_qlinear_op array."""
    entries = list(entries)
    arr = (eb_qlinear_op * len(entries))()
    for i, e in enumerate(entries):
        arr[i] = make_op(*e[:3], **(e[3] if len(e) > 3 else {}))
    return arr


def qlinear_fused(qw: QWeights, x: torch.Tensor, out_dtype=torch.float32, x_dtype=None,
                  prologue=None, norm_weight=None, eps: float = 0.0, epilogue=None,
                  residual=None, path: str = "auto", out: torch.Tensor | None = None,
                  tile: int | None = None, splits: int = 0) -> torch.Tensor:
    """One projection with fused steps (eb_qlinear_fused): optional RMS
    normalisation of x before the product, residual addition ("add") or the
    SiLU-gated product of interleaved gate/up rows ("glu", output n / 2).
    tile / splits force the MFMA path's tile configuration / split of k
    (eb_qlinear_tuned; -1 / 0: automatic)."""
    assert x.is_cuda and x.dim() == 2 and x.shape[1] == qw.k
    x = x.contiguous()
    m = x.shape[0]
    if out is None:
        n_out = qw.n // 2 if epilogue == "glu" else qw.n
        out = torch.empty((m, n_out), dtype=out_dtype, device=x.device)
    if tile is None and not splits:
        if x_dtype is None:
            x_dtype = torch.bfloat16 if x.dtype == torch.float32 else x.dtype
        _run_op(qw, x, out, DTYPES[x_dtype], PATHS[path], PROLOGUES[prologue], norm_weight,
                float(eps), EPILOGUES[epilogue], residual)
    else:
        op = make_op(qw, x, out, x_dtype, prologue, norm_weight, eps, epilogue, residual)
        _run_tuned(op, x.device, -1 if tile is None else tile, splits)
    return out


def stack_workspace_bytes(ops: ctypes.Array) -> int:
    return int(lib.eb_qlinear_stack_workspace_bytes(ops, len(ops)))


def _array_workspace(arr: ctypes.Array, nbytes: int, device) -> torch.Tensor:
    """The workspace kept on an op or module array, of at least nbytes.  One that
    it has outgrown stays on the array too: a cached plan may have its tables there."""
    ws = getattr(arr, "_eb_workspace", None)
    if ws is None or ws.numel() < nbytes:
        if ws is not None:
            arr._eb_outgrown = getattr(arr, "_eb_outgrown", ()) + (ws,)
        ws = torch.empty(nbytes, dtype=torch.uint8,
                         device=device if device is not None else torch.cuda.current_device())
        arr._eb_workspace = ws
    return ws


def qlinear_stack(ops: ctypes.Array, device=None) -> None:
    """eb_qlinear_stack with a workspace that belongs to this op array (kept
    on it: the cached plan keeps its tables there while it is cached).  Its size
    takes a plan on the host to tell, so it is asked for when the array's
    contents have changed since the last call (0.8 us to see for 128 ops), and
    when the library finds the workspace too small (EB_STACK_* changed since)."""
    stream = _stream(device)
    seen = bytes(ops)
    sized, nbytes = getattr(ops, "_eb_sized", (None, 0))
    if sized == seen:
        ws = ops._eb_workspace if nbytes else None
        wp, wb = (ws.data_ptr(), ws.numel()) if nbytes else (None, 0)
        st = lib.eb_qlinear_stack(ops, len(ops), wp, wb, stream)
        if st != EB_ERR_INVALID:
            return _check(st, "eb_qlinear_stack")
    nbytes = stack_workspace_bytes(ops)  # (0 too for a list that will be refused)
    ws = _array_workspace(ops, nbytes, device) if nbytes else None
    wp, wb = (ws.data_ptr(), ws.numel()) if nbytes else (None, 0)
    _check(lib.eb_qlinear_stack(ops, len(ops), wp, wb, stream), "eb_qlinear_stack")
    ops._eb_sized = (seen, nbytes)


def stack_launches(ops: ctypes.Array) -> int:
    """Kernel launches eb_qlinear_stack makes for this op list (host-only)."""
    n = lib.eb_qlinear_stack_launches(ops, len(ops))
    if n < 0:
        raise EBError(n, "eb_qlinear_stack_launches")
    return n


def stack_cache_clear() -> None:
    _check(lib.eb_stack_cache_clear(), "eb_stack_cache_clear")


def mfma_tile_count() -> int:
    return int(lib.eb_mfma_tile_count())


def make_modules(specs) -> ctypes.Array:
    """specs: iterable of (ops array from make_ops, period, phase, repeats).
    The op arrays are kept on the result (the modules point into them)."""
    specs = list(specs)
    arr = (eb_module * len(specs))()
    for i, (ops, period, phase, repeats) in enumerate(specs):
        arr[i] = eb_module(ctypes.cast(ops, ctypes.POINTER(eb_qlinear_op)), len(ops), period, phase,
                           repeats)
    arr._eb_ops = [s[0] for s in specs]
    return arr


def multirate_tick(mods: ctypes.Array, tick: int, device=None) -> None:
    """eb_multirate_tick with a workspace that belongs to this module array."""
    nbytes = int(lib.eb_multirate_workspace_bytes(mods, len(mods)))
    ws = _array_workspace(mods, nbytes, device) if nbytes else getattr(mods, "_eb_workspace", None)
    dev = ws.device if ws is not None else torch.device("cuda")
    _check(lib.eb_multirate_tick(mods, len(mods), tick, ws.data_ptr() if nbytes else None, nbytes,
                                 _stream(dev)), "eb_multirate_tick")


def multirate_launches(mods: ctypes.Array, tick: int) -> int:
    n = lib.eb_multirate_launches(mods, len(mods), tick)
    if n < 0:
        raise EBError(n, "eb_multirate_launches")
    return n


# ---------------------------------------------------------------------------
# The steps between a layer's QKV and O projections (include/eb_attention.h).
# Their ops are packed into bytes, as those of single projections are.
# ---------------------------------------------------------------------------

EB_ROT_HALF = 0
EB_ROT_ADJACENT = 1
EB_MASK_CAUSAL = 0
EB_MASK_FULL = 1
STYLES = {"half": EB_ROT_HALF, "adjacent": EB_ROT_ADJACENT}
MASKS = {"causal": EB_MASK_CAUSAL, "full": EB_MASK_FULL}


class eb_kv_cache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("type", _i32), ("heads", _i32), ("dim", _i32),
                ("page", _i32), ("pages", _i32), ("reserved", _i32)]


class eb_kv_extend_op(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("cached", "added", "table", "free_pages", "n_free", "n_free_out",
                                   "q_start", "kv_len", "slots", "positions", "short_rows")] + \
               [(n, _i32) for n in ("batch", "rows", "page", "pages", "table_stride", "free_capacity")]


class eb_rope_append_op(ctypes.Structure):
    _fields_ = [("cache", eb_kv_cache)] + \
               [(n, _vp) for n in ("qkv", "q_out", "slots", "positions", "freqs", "q_norm", "k_norm")] + \
               [(n, _i64) for n in ("qkv_stride", "q_stride", "pos_stride")] + \
               [(n, _i32) for n in ("qkv_type", "q_heads", "rows", "rot", "style", "n_axes")] + \
               [("sections", _i32 * 3), ("norm_eps", ctypes.c_float)]


class eb_attention_op(ctypes.Structure):
    _fields_ = [("cache", eb_kv_cache)] + \
               [(n, _vp) for n in ("q", "out", "table", "q_start", "kv_len", "prefix")] + \
               [("q_stride", _i64), ("out_stride", _i64)] + \
               [(n, _i32) for n in ("rows", "batch", "q_heads", "table_stride", "max_new", "max_kv",
                                    "mask", "window")] + \
               [("scale", ctypes.c_float), ("softcap", ctypes.c_float)]


_CACHE = "PPiiiiii"
_PACK_EXTEND = struct.Struct("11P6i")
_PACK_ROPE = struct.Struct(_CACHE + "7P3q6i3if")
_PACK_ATTN = struct.Struct(_CACHE + "6P2q8i2f")
for _s, _c in ((_PACK_EXTEND, eb_kv_extend_op), (_PACK_ROPE, eb_rope_append_op),
               (_PACK_ATTN, eb_attention_op)):
    assert _s.size == ctypes.sizeof(_c)

lib.eb_kv_extend.restype = _i32
lib.eb_kv_extend.argtypes = [ctypes.POINTER(eb_kv_extend_op), _vp]
lib.eb_rope_append.restype = _i32
lib.eb_rope_append.argtypes = [ctypes.POINTER(eb_rope_append_op), _vp]
lib.eb_attention_workspace_bytes.restype = ctypes.c_size_t
lib.eb_attention_workspace_bytes.argtypes = [ctypes.POINTER(eb_attention_op)]
lib.eb_attention.restype = _i32
lib.eb_attention.argtypes = [ctypes.POINTER(eb_attention_op), _vp, ctypes.c_size_t, _vp]
lib.eb_attention_plan.restype = _i32
lib.eb_attention_plan.argtypes = [_vp, ctypes.POINTER(_i32), ctypes.POINTER(_i32)]
_kv_extend, _rope_append, _attention = _raw.eb_kv_extend, _raw.eb_rope_append, _raw.eb_attention
for _f in (_kv_extend, _rope_append):
    _f.restype, _f.argtypes = _i32, [ctypes.c_char_p, _vp]
_attention.restype, _attention.argtypes = _i32, [ctypes.c_char_p, _vp, ctypes.c_size_t, _vp]
_raw.eb_attention_workspace_bytes.restype = ctypes.c_size_t
_raw.eb_attention_workspace_bytes.argtypes = [ctypes.c_char_p]
_ATTN_WS_BYTES = {}  # at most 4096 entries


def _need(ok: bool, what: str) -> None:
    """Checks of what only the binding can see: types, shapes and devices of tensors."""
    if not ok:
        raise ValueError(what)


# At one token these kernels take 3 to 10 us, so the host's part of a call counts:
# the checks below are a few attribute reads each (0.3 us a tensor).

def _ints(name: str, t: torch.Tensor, dev: int, n: int) -> int:
    """The address of n contiguous int32 values on GPU `dev`."""
    if t.dtype is not torch.int32 or t.get_device() != dev or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous int32 values on cuda:{dev}")
    return t.data_ptr()


def _floats(name: str, t: torch.Tensor | None, dev: int, n: int) -> int:
    if t is None:
        return 0
    if t.dtype is not torch.float32 or t.get_device() != dev or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous float32 values on cuda:{dev}")
    return t.data_ptr()


def _heads(name: str, t: torch.Tensor, dev: int, dtype, rows: int, heads: int, dim: int) -> int:
    """Stride between the rows of t [rows, heads, dim], whose rows are contiguous."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != (rows, heads, dim):
        raise ValueError(f"{name}: {dtype} values of shape {(rows, heads, dim)} on cuda:{dev}")
    if t.is_contiguous():
        return heads * dim
    stride, head, elem = t.stride()
    if elem != 1 or (head != dim and heads != 1):
        raise ValueError(f"{name}: rows of contiguous heads")
    return stride if rows > 1 else heads * dim


def _launch(fn, op: bytes, dev: int, *more) -> int:
    """fn(op, *more, stream) with GPU `dev` current, on its current stream."""
    was = _get_device()
    if was == dev:
        return fn(op, *more, _raw_stream(dev))
    torch.cuda.set_device(dev)
    try:
        return fn(op, *more, _raw_stream(dev))
    finally:
        torch.cuda.set_device(was)


def _attention_ws(op: bytes, stream: int) -> int:
    return _raw.eb_attention_workspace_bytes(op)


class KVCache:
    """The keys and values of one layer: k, v [pages, heads, page, dim] of
    binary16 or bfloat16, caller-owned."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        _need(k.is_cuda and k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype
              and k.device == v.device and k.is_contiguous() and v.is_contiguous()
              and k.dtype in (torch.float16, torch.bfloat16),
              "k and v: contiguous [pages, heads, page, dim] of float16 or bfloat16 on one GPU")
        self.k, self.v = k, v
        self.pages, self.heads, self.page, self.dim = k.shape
        self.device, self.dtype, self.index = k.device, k.dtype, k.get_device()
        self.shape = (DTYPES[k.dtype], self.heads, self.dim, self.page, self.pages, 0)


def empty_kv_cache(pages: int, page: int, heads: int, dim: int, dtype=torch.bfloat16,
                   device="cuda") -> KVCache:
    shape = (pages, heads, page, dim)
    return KVCache(torch.empty(shape, dtype=dtype, device=device),
                   torch.empty(shape, dtype=dtype, device=device))


class KVBatch:
    """What eb_kv_extend writes beside the block table (int32, on the GPU): one buffer
    of q_start, kv_len, slots, positions, the pages left and the tokens that did not join
    or have no page."""

    def __init__(self, batch: int, rows: int, device):
        self.batch, self.rows = batch, rows
        sizes = (batch + 1, batch, rows, rows, 1, 1)
        self.buf = torch.empty(2 * (batch + rows) + 3, dtype=torch.int32, device=device)
        self.q_start, self.kv_len, self.slots, self.positions, self.n_free, self.short = \
            torch.split_with_sizes(self.buf, sizes)


def kv_extend(table: torch.Tensor, cached: torch.Tensor, added: torch.Tensor,
              free_pages: torch.Tensor, n_free: torch.Tensor, page: int, pages: int, rows: int,
              out: KVBatch | None = None) -> KVBatch:
    """New tokens join the sequences of a batch (eb_kv_extend): `table`
    [batch, stride] gets the new pages' entries in place; the lengths, slots and
    positions of a step of `rows` rows are returned.  n_free stays as it was:
    the pages left are the result's n_free.  Tokens behind the first `rows` do not
    join (kv_len is without them) and count in `short`, as do those without a page."""
    dev = table.get_device()
    _need(dev >= 0 and table.dim() == 2, "table: [batch, stride] on a GPU")
    batch, stride = table.shape
    if out is None:
        out = KVBatch(batch, rows, table.device)
    _need(out.batch == batch and out.rows == rows, "out: a KVBatch of this batch and these rows")
    free = free_pages.numel()
    at = _ints("out", out.buf, dev, 2 * (batch + rows) + 3)
    lens, slots = at + 4 * (batch + 1), at + 4 * (2 * batch + 1)
    op = _PACK_EXTEND.pack(
        _ints("cached", cached, dev, batch), _ints("added", added, dev, batch),
        _ints("table", table, dev, batch * stride), _ints("free_pages", free_pages, dev, free),
        _ints("n_free", n_free, dev, 1), slots + 8 * rows, at, lens, slots if rows else 0,
        slots + 4 * rows if rows else 0, slots + 8 * rows + 4, batch, rows, page, pages, stride, free)
    _check(_launch(_kv_extend, op, dev), "eb_kv_extend")
    return out


def rope_append(qkv: torch.Tensor, cache: KVCache, slots: torch.Tensor, positions: torch.Tensor | None,
                freqs: torch.Tensor | None, q_heads: int, q_norm: torch.Tensor | None = None,
                k_norm: torch.Tensor | None = None, eps: float = 0.0, style: str = "half",
                sections=None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Head norms, rotation and the cache write of one layer (eb_rope_append):
    qkv [rows, (q_heads + 2 heads) * dim] -> queries [rows, q_heads, dim]; keys
    and values go to `cache` at `slots`.  positions: [rows], or [axes, rows] with
    `sections` (rotated pairs along each axis); freqs: radians per position of
    each rotated pair, 2 * len(freqs) elements of a head being rotated."""
    dev, dim = cache.index, cache.dim
    width = (q_heads + 2 * cache.heads) * dim
    qkv_type = DTYPES.get(qkv.dtype)
    if qkv.dim() != 2 or qkv_type is None or qkv.get_device() != dev or qkv.stride(1) != 1 \
            or qkv.shape[1] != width:
        raise ValueError(f"qkv: rows of {width} float32, float16 or bfloat16 values on cuda:{dev}")
    rows = qkv.shape[0]
    if out is None:
        out = torch.empty((rows, q_heads, dim), dtype=cache.dtype, device=cache.device)
    q_stride = _heads("out", out, dev, cache.dtype, rows, q_heads, dim)
    half = freqs.numel() if freqs is not None else 0
    axes, pos, pos_stride = 1, 0, 0
    if half:
        _need(positions is not None and positions.dim() <= 2, "positions: [rows] or [axes, rows]")
        axes = positions.shape[0] if positions.dim() == 2 else 1
        pos, pos_stride = _ints("positions", positions, dev, axes * rows), rows
    sections = tuple(sections) if sections is not None else (half,)
    _need(len(sections) == axes and axes <= 3, "sections: rotated pairs for each of up to 3 axes")
    op = _PACK_ROPE.pack(
        cache.k.data_ptr(), cache.v.data_ptr(), *cache.shape, qkv.data_ptr(), out.data_ptr(),
        _ints("slots", slots, dev, rows), pos, _floats("freqs", freqs, dev, half),
        _floats("q_norm", q_norm, dev, dim), _floats("k_norm", k_norm, dev, dim),
        qkv.stride(0) if rows > 1 else width, q_stride, pos_stride, qkv_type, q_heads, rows,
        2 * half, STYLES[style], axes, *(sections + (0, 0))[:3], eps)
    _check(_launch(_rope_append, op, dev), "eb_rope_append")
    return out


def attention(q: torch.Tensor, cache: KVCache, table: torch.Tensor, q_start: torch.Tensor,
              kv_len: torch.Tensor, max_new: int, max_kv: int, mask: str = "causal",
              prefix: torch.Tensor | None = None, window: int = 0, softcap: float = 0.0,
              scale: float | None = None, out: torch.Tensor | None = None,
              workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of a batch's new tokens over the paged cache (eb_attention):
    q [rows, q_heads, dim] -> the same shape.  scale: dim ** -0.5 where not
    given.  workspace: a uint8 tensor of attention_workspace_bytes bytes; without
    one the call takes one from scratch()."""
    dev, dim = cache.index, cache.dim
    if q.dim() != 3 or table.dim() != 2:
        raise ValueError("q: [rows, q_heads, dim]; table: [batch, stride]")
    rows, q_heads, _ = q.shape
    batch, stride = table.shape
    q_stride = _heads("q", q, dev, cache.dtype, rows, q_heads, dim)
    if out is None:
        out_stride = q_heads * dim
        out = torch.empty_like(q) if q_stride == out_stride else q.new_empty((rows, q_heads, dim))
    else:
        out_stride = _heads("out", out, dev, cache.dtype, rows, q_heads, dim)
    op = _PACK_ATTN.pack(
        cache.k.data_ptr(), cache.v.data_ptr(), *cache.shape, q.data_ptr(), out.data_ptr(),
        _ints("table", table, dev, batch * stride), _ints("q_start", q_start, dev, batch + 1),
        _ints("kv_len", kv_len, dev, batch), _ints("prefix", prefix, dev, batch) if prefix is not None else 0,
        q_stride, out_stride, rows, batch, q_heads, stride, max_new, max_kv, MASKS[mask], window,
        dim ** -0.5 if scale is None else scale, softcap)
    if workspace is not None:
        _need(workspace.dtype is torch.uint8 and workspace.get_device() == dev and workspace.is_contiguous(),
              "workspace: contiguous uint8 on the cache's GPU")
        _check(_launch(_attention, op, dev, workspace.data_ptr(), workspace.numel()), "eb_attention")
        return out
    # its size, by what it depends on, is kept after a call that succeeded
    key = (rows, batch, q_heads, cache.heads, dim, max_new, max_kv, mask, prefix is None, window, dev)
    nbytes = _ATTN_WS_BYTES.get(key)
    known = nbytes is not None
    if not known:
        nbytes = _launch(_attention_ws, op, dev)  # 0 too for a call that will be refused
    if not nbytes:
        st = _launch(_attention, op, dev, None, 0)
    else:
        ws = _workspace(cache.device, dev, _raw_stream(dev), nbytes)
        st = _launch(_attention, op, dev, ws.data_ptr(), ws.numel())
    _check(st, "eb_attention")
    if not known:
        if len(_ATTN_WS_BYTES) >= 4096:
            _ATTN_WS_BYTES.clear()
        _ATTN_WS_BYTES[key] = nbytes
    return out


def _attention_sizes(q_shape, cache, batch, table_stride, max_new, max_kv, mask, prefix, window) -> bytes:
    rows, q_heads, dim = q_shape
    w, stand_in = q_heads * dim, cache.k.data_ptr()  # pointers are only checked for alignment
    return _PACK_ATTN.pack(stand_in, stand_in, *cache.shape, stand_in, stand_in, stand_in, stand_in,
                           stand_in, stand_in if prefix else 0, w, w, rows, batch, q_heads, table_stride,
                           max_new, max_kv, MASKS[mask], window, 1.0, 0.0)


def attention_workspace_bytes(q_shape, cache: KVCache, batch: int, table_stride: int, max_new: int,
                              max_kv: int, mask: str = "causal", prefix: bool = False,
                              window: int = 0) -> int:
    """Bytes of workspace that attention() needs for queries of q_shape, with or
    without a prefix, under this mask and window."""
    op = _attention_sizes(q_shape, cache, batch, table_stride, max_new, max_kv, mask, prefix, window)
    return int(_launch(_attention_ws, op, cache.index))


def attention_plan(q_shape, cache: KVCache, batch: int, table_stride: int, max_new: int, max_kv: int,
                   mask: str = "causal", prefix: bool = False, window: int = 0) -> tuple:
    """(rows of a tile, workgroups that splits may add) of attention() on these sizes, for
    tuning and tests (eb_attention_plan)."""
    op = _attention_sizes(q_shape, cache, batch, table_stride, max_new, max_kv, mask, prefix, window)
    tile_rows, splits = _i32(), _i32()
    _check(_launch(lambda op, stream: lib.eb_attention_plan(op, tile_rows, splits), op, cache.index),
           "eb_attention_plan")
    return tile_rows.value, splits.value
