"""Python binding of libspdp: the MI355X Tiled-CBC spMspV library.

Argument marshalling only. Every step of the decode path (activity test,
column selection, bitmap decode, accumulation, split-K reduction) runs in
the HIP kernel behind ``spdp_spmspv``; the encoder, pruning and threshold
calibration run in the library's host C++. PyTorch supplies device memory
and streams. There is no fallback: if ``libspdp.so`` is not built, every
entry point raises.

    import paper_2607_21985_amd as spdp
    w_sp = spdp.prune_magnitude(w16, 0.5)          # numpy fp16, host
    m = spdp.encode(w_sp, tile=(256, 16))          # device copy on cuda:current
    t = spdp.calibrate_threshold(x16_calib, 0.5)   # TEAL-style quantile
    y = m(x_cuda_fp16, t)                          # torch fp16 [batch, rows]
"""

from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

__all__ = [
    "SpdpError",
    "Matrix",
    "lib",
    "lib_path",
    "encode",
    "encode_host",
    "encode_rtn",
    "encode_rtn_host",
    "spmspv_many",
    "Adapters",
    "adapters_many",
    "rotate_heads",
    "rotate_heads_grad",
    "MASKS",
    "Chain",
    "prune_magnitude",
    "calibrate_threshold",
    "threshold_code",
    "EXPORTED_SYMBOLS",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libspdp.so"

EXPORTED_SYMBOLS = (
    "spdp_encode", "spdp_encode_host", "spdp_spmspv", "spdp_spmspv_many", "spdp_spmspv_many_mask",
    "spdp_reserve", "spdp_split_plan", "spdp_free",
    "spdp_format", "spdp_prune_magnitude", "spdp_calibrate_threshold",
    "spdp_threshold_code", "spdp_strerror", "spdp_last_error",
    "spdp_encode_rtn", "spdp_encode_rtn_host", "spdp_spmspv_noalloc", "spdp_spmm",
    "spdp_spmm_grad_workspace", "spdp_spmm_grad", "spdp_adapt_workspace", "spdp_adapt",
    "spdp_adapt_grad_workspace", "spdp_adapt_grad",
    "spdp_rotate_heads", "spdp_rotate_heads_grad_workspace", "spdp_rotate_heads_grad",
)

SPDP_OK = 0
_STATUS = {0: "SPDP_OK", -1: "SPDP_ERR_INVALID_ARG", -2: "SPDP_ERR_UNSUPPORTED",
           -3: "SPDP_ERR_OOM", -4: "SPDP_ERR_HIP"}


class SpdpError(RuntimeError):
    """A libspdp call returned an error status."""

    def __init__(self, status: int, detail: str):
        super().__init__(f"{_STATUS.get(status, status)}: {detail}")
        self.status = status


class _Format(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
        ("tile_m", ctypes.c_int32), ("tile_k", ctypes.c_int32),
        ("n_stripes", ctypes.c_int64), ("n_colblocks", ctypes.c_int64),
        ("n_gtiles", ctypes.c_int64), ("n_values", ctypes.c_int64),
        ("tile_offset", ctypes.POINTER(ctypes.c_uint32)),
        ("col_info", ctypes.POINTER(ctypes.c_uint32)),
        ("bitmap", ctypes.POINTER(ctypes.c_uint64)),
        ("values", ctypes.POINTER(ctypes.c_uint16)),
        ("d_tile_offset", ctypes.c_void_p), ("d_col_info", ctypes.c_void_p),
        ("d_bitmap", ctypes.c_void_p), ("d_values", ctypes.c_void_p),
        ("device", ctypes.c_int32),
        ("value_bits", ctypes.c_int32),
        ("codes", ctypes.POINTER(ctypes.c_int8)),
        ("scales", ctypes.POINTER(ctypes.c_float)),
        ("d_scales", ctypes.c_void_p),
    ]


class _Bank(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("scale", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("count", ctypes.c_int32), ("rank", ctypes.c_int32)]


class _Rotation(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("cosine", ctypes.c_void_p), ("sine", ctypes.c_void_p),
                ("table", ctypes.c_int64), ("dim", ctypes.c_int32), ("rot", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("eps", ctypes.c_float)]


class _Heads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("dy", ctypes.c_void_p),
                ("y", ctypes.c_void_p), ("dweight", ctypes.c_void_p), ("heads", ctypes.c_int32)]


# the same layouts as bytes, which small calls build in a fraction of the time
_PACK_BANK = struct.Struct("PPPqqii")
_PACK_ROTATION = struct.Struct("PPPqiiif")
_PACK_HEADS = struct.Struct("PPPPPi4x")
_PACK_POINTERS = [struct.Struct(f"{_k}P").pack for _k in range(9)]
for _a, _b in ((_PACK_BANK, _Bank), (_PACK_ROTATION, _Rotation), (_PACK_HEADS, _Heads)):
    assert _a.size == ctypes.sizeof(_b)


_lib = None


def lib_path() -> str:
    return os.path.join(_HERE, _LIB_NAME)


def lib() -> ctypes.CDLL:
    """Load libspdp.so (built in-tree by ``build.py``); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built; run `python -m paper_2607_21985_amd.build`")
    L = ctypes.CDLL(path)
    u16p, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    H = ctypes.c_void_p
    L.spdp_encode.argtypes = [u16p, i64, i64, i32, i32, ctypes.POINTER(H)]
    L.spdp_encode_host.argtypes = [u16p, i64, i64, i32, i32, ctypes.POINTER(H)]
    L.spdp_encode_rtn.argtypes = [u16p, i64, i64, i32, i32, i32, ctypes.POINTER(H)]
    L.spdp_encode_rtn_host.argtypes = [u16p, i64, i64, i32, i32, i32, ctypes.POINTER(H)]
    L.spdp_spmspv.argtypes = [H, ctypes.c_void_p, i32, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p]
    L.spdp_spmspv_noalloc.argtypes = [H, ctypes.c_void_p, i32, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p]
    L.spdp_spmm.argtypes = [H, ctypes.c_void_p, i64, ctypes.c_void_p, ctypes.c_void_p]
    L.spdp_spmspv_many.argtypes = [ctypes.POINTER(H), i32, ctypes.POINTER(ctypes.c_void_p), i32,
                                   ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_void_p),
                                   ctypes.c_void_p]
    L.spdp_spmspv_many_mask.argtypes = [ctypes.POINTER(H), i32, ctypes.POINTER(ctypes.c_void_p), i32,
                                        ctypes.POINTER(ctypes.c_float), i32, ctypes.POINTER(ctypes.c_void_p),
                                        ctypes.c_void_p]
    P, size = ctypes.c_void_p, ctypes.c_size_t
    L.spdp_spmm_grad_workspace.argtypes = [H, i64, ctypes.POINTER(size)]
    L.spdp_spmm_grad.argtypes = [H, P, i64, P, P, size, P]
    L.spdp_adapt_workspace.argtypes = [P, i32, i64, i32, ctypes.POINTER(size)]
    L.spdp_adapt.argtypes = [P, i32, P, P, P, P, P, i64, P, size, P]
    L.spdp_adapt_grad_workspace.argtypes = [P, i64, i32, ctypes.POINTER(size)]
    L.spdp_adapt_grad.argtypes = [P, P, P, P, P, P, P, P, P, i64, P, size, P]
    L.spdp_rotate_heads.argtypes = [P, i32, P, i64, P]
    L.spdp_rotate_heads_grad_workspace.argtypes = [P, i32, P, i64, ctypes.POINTER(size)]
    L.spdp_rotate_heads_grad.argtypes = [P, i32, P, i64, P, size, P]
    L.spdp_reserve.argtypes = [H, i32]
    L.spdp_split_plan.argtypes = [H, i32, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.spdp_free.argtypes = [H]
    L.spdp_free.restype = None
    L.spdp_format.argtypes = [H, ctypes.POINTER(_Format)]
    L.spdp_prune_magnitude.argtypes = [u16p, i64, ctypes.c_double, u16p]
    L.spdp_calibrate_threshold.argtypes = [u16p, i64, ctypes.c_double, ctypes.POINTER(ctypes.c_float)]
    L.spdp_threshold_code.argtypes = [ctypes.c_float, ctypes.POINTER(i32)]
    L.spdp_strerror.argtypes = [ctypes.c_int]
    L.spdp_strerror.restype = ctypes.c_char_p
    L.spdp_last_error.argtypes = []
    L.spdp_last_error.restype = ctypes.c_char_p
    for name in ("spdp_encode", "spdp_encode_host", "spdp_spmspv", "spdp_spmspv_noalloc", "spdp_spmm",
                 "spdp_spmspv_many",
                 "spdp_spmspv_many_mask",
                 "spdp_spmm_grad_workspace", "spdp_spmm_grad", "spdp_adapt_workspace", "spdp_adapt",
                 "spdp_adapt_grad_workspace", "spdp_adapt_grad",
                 "spdp_rotate_heads", "spdp_rotate_heads_grad_workspace", "spdp_rotate_heads_grad",
                 "spdp_reserve", "spdp_split_plan",
                 "spdp_format",
                 "spdp_prune_magnitude", "spdp_calibrate_threshold", "spdp_threshold_code"):
        getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def _check(status: int) -> None:
    if status != SPDP_OK:
        raise SpdpError(status, lib().spdp_last_error().decode())


def _u16(a: np.ndarray) -> np.ndarray:
    a = np.ascontiguousarray(a)
    if a.dtype == np.float16:
        return a.view(np.uint16)
    if a.dtype == np.uint16:
        return a
    raise TypeError(f"expected fp16 (or its uint16 bits), got {a.dtype}")


def _ptr(a: np.ndarray) -> ctypes.c_void_p:
    return ctypes.c_void_p(a.ctypes.data)


def _tensor(t, name: str, dtype, shape) -> None:
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} tensor")


_raw_stream = None  # a device's current stream


def _stream(stream, tensors) -> int:
    """The HIP stream to enqueue on, after a check of the tensors' device."""
    global _raw_stream
    import torch
    dev = tensors[0].get_device()  # -1: not on a GPU
    for t in tensors:
        if t.get_device() != dev:
            dev = -1
    if dev < 0:
        raise ValueError("all tensors must be on one GPU")
    if torch.cuda.current_device() != dev:
        raise ValueError("the tensors are not on the current device")
    if stream is None:
        if _raw_stream is None:
            # (the stream's number alone: an object of it takes longer than a launch)
            _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
                (lambda d: torch.cuda.current_stream(d).cuda_stream)
        return _raw_stream(dev)
    if stream.device.index != dev:
        raise ValueError("the stream is not on the tensors' device")
    return stream.cuda_stream


def _workspace(size: int, device, stream):
    """Device memory for one call. It belongs to the call's stream (or to the
    graph that the stream is captured into), so that torch hands it out again
    only to work behind the call."""
    import torch
    if stream is None:
        return torch.empty(size or 1, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(size or 1, dtype=torch.uint8, device=device)


def _output(shape, device, stream):
    """An fp16 array that a call writes and the caller gets. It is taken, like a
    workspace, as the call's stream's own (what else is queued on the caller's
    may still use a block of that one's), and kept from reuse until what the
    caller's stream does with it is done, too."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=torch.float16, device=device)
    with torch.cuda.stream(stream):
        out = torch.empty(shape, dtype=torch.float16, device=device)
    out.record_stream(torch.cuda.current_stream(device))
    return out


class Matrix:
    """An encoded weight matrix (owns the library handle)."""

    def __init__(self, handle: ctypes.c_void_p):
        self._h = handle
        f = _Format()
        _check(lib().spdp_format(self._h, ctypes.byref(f)))
        self.rows, self.cols = int(f.rows), int(f.cols)
        self.tile = (int(f.tile_m), int(f.tile_k))
        self.device = int(f.device)

    def _fmt(self) -> _Format:
        f = _Format()
        _check(lib().spdp_format(self._h, ctypes.byref(f)))
        return f

    def format(self) -> dict:
        """Copies of the four Tiled-CBC arrays (host) plus shape fields."""
        f = self._fmt()
        ngt, tk, tm = int(f.n_gtiles), int(f.tile_k), int(f.tile_m)

        def arr(p, n, dt):
            if n == 0:
                return np.zeros(0, dtype=dt)
            return np.ctypeslib.as_array(p, shape=(n,)).astype(dt, copy=True)

        out = {
            "rows": int(f.rows), "cols": int(f.cols), "tile_m": tm, "tile_k": tk,
            "n_stripes": int(f.n_stripes), "n_colblocks": int(f.n_colblocks), "n_gtiles": ngt,
            "tile_offset": arr(f.tile_offset, ngt + 1, np.uint32),
            "col_info": arr(f.col_info, ngt * tk, np.uint32),
            "bitmap": arr(f.bitmap, ngt * tk * tm // 64, np.uint64),
            "value_bits": int(f.value_bits),
        }
        if f.value_bits < 16:
            # one byte per code; "values" holds the codes' bytes
            out["codes"] = arr(f.codes, int(f.n_values), np.int8)
            out["values"] = out["codes"].view(np.uint8)
            out["scales"] = arr(f.scales, int(f.rows), np.float32)
        else:
            out["values"] = arr(f.values, int(f.n_values), np.uint16)
        return out

    def device_pointers(self) -> dict:
        f = self._fmt()
        return {"tile_offset": f.d_tile_offset, "col_info": f.d_col_info,
                "bitmap": f.d_bitmap, "values": f.d_values}

    def reserve(self, max_batch: int) -> None:
        _check(lib().spdp_reserve(self._h, int(max_batch)))

    def split_plan(self, batch: int) -> tuple:
        """(segments, wave_cols, passes) of a call with ``batch`` tokens (``spdp_split_plan``)."""
        sg, wc, ps = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
        _check(lib().spdp_split_plan(self._h, int(batch), ctypes.byref(sg), ctypes.byref(wc), ctypes.byref(ps)))
        return sg.value, wc.value, ps.value

    def spmspv_into(self, x, threshold: float, y, stream=None, mask: str = "token") -> None:
        """Enqueue ``y = W_sp . mask(x)`` on ``stream`` (torch stream, or the current one).

        ``mask``: "token" (each token's own columns) or "batch" (one column
        set for the batch, by its fp32 sum of magnitudes; see
        ``spmspv_many``)."""
        import torch
        if x.dtype != torch.float16 or y.dtype != torch.float16:
            raise TypeError("x and y must be torch.float16")
        if x.dim() != 2 or x.shape[1] != self.cols or not x.is_contiguous():
            raise ValueError(f"x must be a contiguous [batch, {self.cols}] tensor")
        b = x.shape[0]
        if tuple(y.shape) != (b, self.rows) or not y.is_contiguous():
            raise ValueError(f"y must be a contiguous [{b}, {self.rows}] tensor")
        if not (x.is_cuda and y.is_cuda):
            raise ValueError("x and y must be device tensors")
        s = stream if stream is not None else torch.cuda.current_stream(x.device)
        if mask == "token":
            _check(lib().spdp_spmspv(self._h, ctypes.c_void_p(x.data_ptr()), int(b),
                                     ctypes.c_float(threshold), ctypes.c_void_p(y.data_ptr()),
                                     ctypes.c_void_p(s.cuda_stream)))
        else:
            hs = (ctypes.c_void_p * 1)(self._h)
            xp = (ctypes.c_void_p * 1)(x.data_ptr())
            yp = (ctypes.c_void_p * 1)(y.data_ptr())
            ts = (ctypes.c_float * 1)(float(threshold))
            _check(lib().spdp_spmspv_many_mask(hs, 1, xp, int(b), ts, _mask_code(mask), yp,
                                               ctypes.c_void_p(s.cuda_stream)))

    def spmspv_noalloc_into(self, x, threshold: float, y, stream=None) -> None:
        """``spmspv_into`` through ``spdp_spmspv_noalloc``: the split-K partials
        go to the library's static workspace, so the call allocates nothing
        (per-token mask; calls on one GPU must not overlap)."""
        import torch
        if x.dtype != torch.float16 or y.dtype != torch.float16:
            raise TypeError("x and y must be torch.float16")
        if x.dim() != 2 or x.shape[1] != self.cols or not x.is_contiguous():
            raise ValueError(f"x must be a contiguous [batch, {self.cols}] tensor")
        b = x.shape[0]
        if tuple(y.shape) != (b, self.rows) or not y.is_contiguous():
            raise ValueError(f"y must be a contiguous [{b}, {self.rows}] tensor")
        if not (x.is_cuda and y.is_cuda):
            raise ValueError("x and y must be device tensors")
        s = stream if stream is not None else torch.cuda.current_stream(x.device)
        _check(lib().spdp_spmspv_noalloc(self._h, ctypes.c_void_p(x.data_ptr()), int(b),
                                         ctypes.c_float(threshold), ctypes.c_void_p(y.data_ptr()),
                                         ctypes.c_void_p(s.cuda_stream)))

    def spmm_into(self, x, y, stream=None) -> None:
        """Enqueue the prefill product ``y = x W_sp^T`` (every column, no
        threshold) for ``x`` [tokens, cols] into ``y`` [tokens, rows]."""
        import torch
        if x.dtype != torch.float16 or y.dtype != torch.float16:
            raise TypeError("x and y must be torch.float16")
        if x.dim() != 2 or x.shape[1] != self.cols or not x.is_contiguous():
            raise ValueError(f"x must be a contiguous [tokens, {self.cols}] tensor")
        n = x.shape[0]
        if tuple(y.shape) != (n, self.rows) or not y.is_contiguous():
            raise ValueError(f"y must be a contiguous [{n}, {self.rows}] tensor")
        if not (x.is_cuda and y.is_cuda):
            raise ValueError("x and y must be device tensors")
        s = stream if stream is not None else torch.cuda.current_stream(x.device)
        _check(lib().spdp_spmm(self._h, ctypes.c_void_p(x.data_ptr()), int(n), ctypes.c_void_p(y.data_ptr()),
                               ctypes.c_void_p(s.cuda_stream)))

    def spmm(self, x, stream=None):
        """The prefill product ``x W_sp^T`` as a new fp16 tensor (which belongs to ``stream``)."""
        y = _output((x.shape[0], self.rows), x.device, stream)
        self.spmm_into(x, y, stream)
        return y

    def spmm_grad_into(self, dy, dx, stream=None) -> None:
        """Enqueue the gradient of ``spmm`` with respect to its input,
        ``dx = dy W_sp``, for ``dy`` [tokens, rows] into ``dx`` [tokens, cols].
        (torch's autograd does not know of it: ``spmm``'s result has no graph.)"""
        import torch
        n = dy.shape[0]
        _tensor(dy, "dy", torch.float16, (n, self.rows))
        _tensor(dx, "dx", torch.float16, (n, self.cols))
        s = _stream(stream, (dy, dx))
        need = ctypes.c_size_t()
        _check(lib().spdp_spmm_grad_workspace(self._h, n, ctypes.byref(need)))
        ws = _workspace(need.value, dy.device, stream)
        _check(lib().spdp_spmm_grad(self._h, dy.data_ptr(), n, dx.data_ptr(), ws.data_ptr(), need.value, s))

    def spmm_grad(self, dy, stream=None):
        """The gradient ``dy W_sp`` as a new fp16 tensor (which belongs to ``stream``)."""
        dx = _output((dy.shape[0], self.cols), dy.device, stream)
        self.spmm_grad_into(dy, dx, stream)
        return dx

    def __call__(self, x, threshold: float, stream=None, mask: str = "token"):
        y = _output((x.shape[0], self.rows), x.device, stream)
        self.spmspv_into(x, threshold, y, stream, mask)
        return y

    def close(self) -> None:
        """Free the handle (synchronizes the device; never while a stream capture runs)."""
        if getattr(self, "_h", None):
            lib().spdp_free(self._h)
            self._h = None
        _free_deferred()

    def __del__(self):
        # spdp_free synchronizes the device, which would invalidate a HIP
        # graph capture in progress: a handle that becomes garbage during a
        # capture is freed at the next close() or encode() instead.
        try:
            h = getattr(self, "_h", None)
            if not h:
                return
            self._h = None
            if _capturing():
                _DEFERRED.append(h)
            else:
                lib().spdp_free(h)
        except Exception:
            pass


_DEFERRED: list = []


def _capturing() -> bool:
    try:
        import torch
        return bool(torch.cuda.is_available() and torch.cuda.is_current_stream_capturing())
    except Exception:
        return False


def _free_deferred() -> None:
    while _DEFERRED and not _capturing():
        lib().spdp_free(_DEFERRED.pop())


def encode(w: np.ndarray, tile=(256, 16)) -> Matrix:
    """Encode a pruned fp16 matrix (host numpy) and upload it to the current HIP device."""
    wb = _u16(w)
    if wb.ndim != 2:
        raise ValueError("w must be 2-D")
    _free_deferred()
    h = ctypes.c_void_p()
    _check(lib().spdp_encode(_ptr(wb), wb.shape[0], wb.shape[1], int(tile[0]), int(tile[1]),
                             ctypes.byref(h)))
    return Matrix(h)


MASKS = {"token": 0, "batch": 1}  # SPDP_MASK_TOKEN, SPDP_MASK_BATCH


def _mask_code(mask: str) -> int:
    if mask not in MASKS:
        raise ValueError(f"mask must be one of {sorted(MASKS)}")
    return MASKS[mask]


def spmspv_many(mats, xs, thresholds, ys, stream=None, mask: str = "token") -> None:
    """Enqueue ``ys[i] = W_i . mask(xs[i])`` for every i in one launch.

    ``mats`` are encoded matrices with one tile height, ``xs``/``ys`` torch
    fp16 device tensors ``[batch, cols_i]`` / ``[batch, rows_i]`` (one batch
    for all), ``thresholds`` one float per product. Inputs may be shared.
    ``mask="token"``: column k takes part for token b iff |x[b, k]| > t;
    ``mask="batch"``: one column set for the batch, column k taking part for
    every token iff the fp32 running sum of |x[b, k]| over the tokens exceeds
    fp32(batch * t) (the batch's mean magnitude exceeds t).
    """
    import torch
    n = len(mats)
    if not (len(xs) == len(ys) == len(thresholds) == n):
        raise ValueError("mats, xs, thresholds and ys must have one entry per product")
    for m, x, y in zip(mats, xs, ys):
        if x.dtype != torch.float16 or y.dtype != torch.float16:
            raise TypeError("x and y must be torch.float16")
        if x.dim() != 2 or x.shape[1] != m.cols or not x.is_contiguous():
            raise ValueError(f"x must be a contiguous [batch, {m.cols}] tensor")
        if tuple(y.shape) != (x.shape[0], m.rows) or not y.is_contiguous():
            raise ValueError(f"y must be a contiguous [{x.shape[0]}, {m.rows}] tensor")
        if x.shape[0] != xs[0].shape[0]:
            raise ValueError("every product of one call takes the same batch")
        if not (x.is_cuda and y.is_cuda):
            raise ValueError("x and y must be device tensors")
    s = stream if stream is not None else torch.cuda.current_stream(xs[0].device)
    hs = (ctypes.c_void_p * n)(*[m._h for m in mats])
    xp = (ctypes.c_void_p * n)(*[x.data_ptr() for x in xs])
    yp = (ctypes.c_void_p * n)(*[y.data_ptr() for y in ys])
    ts = (ctypes.c_float * n)(*[float(t) for t in thresholds])
    _check(lib().spdp_spmspv_many_mask(hs, n, xp, int(xs[0].shape[0]), ts, _mask_code(mask), yp,
                                       ctypes.c_void_p(s.cuda_stream)))


class Adapters:
    """The low-rank adapters of one projection (rows x cols), of one rank.

    ``a`` is fp16 [count, rank, cols], ``b`` fp16 [count, rank, rows] (the
    second factor rank by rank), ``scale`` fp32 [count], all contiguous on one
    GPU. Nothing is copied: weights that are changed in place, or replaced by
    others of the same shape, count from the next call on. Every call looks at
    the weights anew, and refuses those of another shape, type or layout.

        y = fp16(base + scale[id] * (x a[id]^T) b[id])

    with the adapter ``id`` of each token. ``base`` is the shared projection's
    output (``Matrix``, ``spmspv_many``, ``Matrix.spmm``).

    torch's autograd records none of the calls: a result has no graph, whether or
    not its inputs require gradients, and the gradients are ``grad_into``'s.
    """

    def __init__(self, a, b, scale):
        import torch
        if a.dim() != 3 or b.dim() != 3:
            raise ValueError("a and b must be [count, rank, features]")
        self.a, self.b, self.scale = a, b, scale
        self.count, self.rank, self.cols = a.shape
        self.rows = b.shape[2]
        self._form = (torch.float16, torch.float32, a.shape, torch.Size((self.count, self.rank, self.rows)),
                      torch.Size((self.count,)))
        self._key = (self.rows, self.cols, self.rank, self.count)
        self._pointers = None
        self._sizes = {}  # workspaces of calls, by their sizes
        need = ctypes.c_size_t()  # checks the sizes
        _check(lib().spdp_adapt_workspace(self._struct(), 1, 1, 0, ctypes.byref(need)))

    def _struct(self) -> bytes:
        # the tensors may have been replaced since the last call, or given other
        # memory (``p.data = ...``), by ones of another shape, type or layout, too,
        # and at the same address: a view of the old ones, or what the allocator
        # has put in their place
        a, b, scale = self.a, self.b, self.scale
        half, single, of_a, of_b, of_scale = self._form
        if not (a.dtype is half and b.dtype is half and scale.dtype is single and a.shape == of_a and b.shape == of_b
                and scale.shape == of_scale and a.is_contiguous() and b.is_contiguous() and scale.is_contiguous()):
            _tensor(a, "a", half, of_a)
            _tensor(b, "b", half, of_b)
            _tensor(scale, "scale", single, of_scale)
        at = (a.data_ptr(), b.data_ptr(), scale.data_ptr())
        if at != self._pointers:
            _stream(None, (a, b, scale))
            self._bank = _PACK_BANK.pack(*at, self.rows, self.cols, self.count, self.rank)
            self._pointers = at
        return self._bank

    def add_into(self, x, ids, base, y, h=None, stream=None) -> None:
        """Enqueue ``y = base + the adapters' products of x`` for ``x`` [tokens,
        cols], ``base`` and ``y`` [tokens, rows], fp16 (``y`` may be ``base``).

        ``ids``: int32 [tokens], each token's adapter, one outside [0, count)
        for none; or None, adapter 0 for all. ``h``: fp32 [tokens, rank] that
        receives ``x a[id]^T``, which ``grad_into`` reads."""
        adapters_many([self], [x], ids, [base], [y], None if h is None else [h], stream)

    def __call__(self, x, ids, base, stream=None):
        """``add_into`` a new tensor (which belongs to ``stream``)."""
        y = _output(base.shape, base.device, stream)
        self.add_into(x, ids, base, y, stream=stream)
        return y

    def grad_into(self, x, ids, h, dy, base, dx, da, db, stream=None) -> None:
        """Enqueue the gradients for ``dy`` [tokens, rows] of ``add_into``'s
        ``y``: ``dx = base + the adapters' part`` fp16 [tokens, cols] (``base``:
        the shared projection's gradient, ``Matrix.spmm_grad``; ``dx`` may be
        ``base``), ``da`` and ``db`` fp32 like ``a`` and ``b`` (overwritten).
        ``x``, ``ids`` and ``h`` are the forward call's."""
        import torch
        n = x.shape[0]
        _tensor(x, "x", torch.float16, (n, self.cols))
        _tensor(h, "h", torch.float32, (n, self.rank))
        _tensor(dy, "dy", torch.float16, (n, self.rows))
        _tensor(base, "base", torch.float16, (n, self.cols))
        _tensor(dx, "dx", torch.float16, (n, self.cols))
        _tensor(da, "da", torch.float32, self._form[2])
        _tensor(db, "db", torch.float32, self._form[3])
        some = (x, h, dy, base, dx, da, db, self.a)
        if ids is not None:
            _tensor(ids, "ids", torch.int32, (n,))
            some += (ids,)
        s = _stream(stream, some)
        need = ctypes.c_size_t()
        bank = self._struct()
        _check(lib().spdp_adapt_grad_workspace(bank, n, ids is not None, ctypes.byref(need)))
        ws = _workspace(need.value, x.device, stream)
        _check(lib().spdp_adapt_grad(bank, x.data_ptr(), None if ids is None else ids.data_ptr(), h.data_ptr(),
                                     dy.data_ptr(), base.data_ptr(), dx.data_ptr(), da.data_ptr(), db.data_ptr(), n,
                                     ws.data_ptr(), need.value, s))


def adapters_many(banks, xs, ids, bases, ys, hs=None, stream=None) -> None:
    """Enqueue ``Adapters.add_into`` of several projections (q, k and v; gate
    and up) as one call. The banks have one rank and one count; ``ids`` goes for
    all. Inputs may be shared."""
    import torch
    k = len(banks)
    if not (len(xs) == len(bases) == len(ys) == k) or (hs is not None and len(hs) != k) or k == 0:
        raise ValueError("banks, xs, bases, ys and hs must have one entry per projection")
    f16, n, L = torch.float16, xs[0].shape[0], lib()
    some = [*xs, *bases, *ys]
    bk, key, seen, cols = [], [n, ids is not None], None, 0
    for m, x, base, y in zip(banks, xs, bases, ys):
        bk.append(m._struct())
        some.append(m.a)
        key.append(m._key)
        if x is not seen or m.cols != cols:  # (mostly one input for all)
            seen, cols = x, m.cols
            _tensor(x, "x", f16, (n, cols))
        out = (n, m.rows)
        if not (base.dtype is f16 and y.dtype is f16 and base.shape == out and y.shape == out and base.is_contiguous()
                and y.is_contiguous()):
            _tensor(base, "base", f16, out)
            _tensor(y, "y", f16, out)
    if hs is not None:
        for m, h in zip(banks, hs):
            _tensor(h, "h", torch.float32, (n, m.rank))
        some += hs
    if ids is not None:
        _tensor(ids, "ids", torch.int32, (n,))
        some.append(ids)
    s = _stream(stream, some)
    bk = b"".join(bk)
    # the size of a workspace depends on nothing but the call's sizes
    sizes, key = banks[0]._sizes, tuple(key)
    size = sizes.get(key)
    if size is None:
        need = ctypes.c_size_t()
        _check(L.spdp_adapt_workspace(bk, k, n, ids is not None, ctypes.byref(need)))
        if len(sizes) >= 256:
            sizes.clear()
        sizes[key] = size = need.value
    ws = _workspace(size, xs[0].device, stream) if size else None
    P = _PACK_POINTERS[k] if k < len(_PACK_POINTERS) else struct.Struct(f"{k}P").pack
    _check(L.spdp_adapt(bk, k, P(*[x.data_ptr() for x in xs]), None if ids is None else ids.data_ptr(),
                        P(*[b.data_ptr() for b in bases]), P(*[y.data_ptr() for y in ys]),
                        None if hs is None else P(*[h.data_ptr() for h in hs]), n, ws.data_ptr() if size else None, size, s))


def _heads(xs, dim, pos, cos, sin, ys, weights, eps, interleaved, stream, dys=None, dweights=None):
    import torch
    k = len(xs)
    if k == 0 or len(ys) != k or (weights is not None and len(weights) != k) or (dys is not None and len(dys) != k) or \
            (dweights is not None and len(dweights) != k):
        raise ValueError("every list must have one entry per input")
    if dim < 1:
        raise ValueError("dim must be at least 1")
    f16, f32, n = torch.float16, torch.float32, xs[0].shape[0]
    _tensor(pos, "pos", torch.int32, (n,))
    angles = cos.shape
    if len(angles) != 2:
        raise ValueError("cos and sin must be [positions, rot / 2]")
    _tensor(cos, "cos", f32, angles)
    _tensor(sin, "sin", f32, angles)
    some = [pos, cos, sin, *xs, *ys]
    inputs = []
    for i in range(k):
        x, y = xs[i], ys[i]
        shape = x.shape
        if len(shape) != 2 or shape[0] != n or shape[1] % dim or shape[1] == 0:
            raise ValueError(f"x must be [{n}, heads * {dim}]")
        _tensor(x, "x", f16, shape)
        _tensor(y, "the output", f16, shape)
        w = d = dw = 0
        if weights is not None and weights[i] is not None:
            _tensor(weights[i], "a weight", f16, (dim,))
            some.append(weights[i])
            w = weights[i].data_ptr()
        if dys is not None:
            _tensor(dys[i], "dy", f16, shape)
            some.append(dys[i])
            d = dys[i].data_ptr()
        if dweights is not None and dweights[i] is not None:
            _tensor(dweights[i], "a weight's gradient", f32, (dim,))
            some.append(dweights[i])
            dw = dweights[i].data_ptr()
        inputs.append(_PACK_HEADS.pack(x.data_ptr(), w, d, y.data_ptr(), dw, shape[1] // dim))
    s = _stream(stream, some)
    r = _PACK_ROTATION.pack(pos.data_ptr(), cos.data_ptr(), sin.data_ptr(), angles[0], dim, 2 * angles[1],
                            1 if interleaved else 0, eps)
    return b"".join(inputs), k, r, n, s


def rotate_heads(xs, dim, pos, cos, sin, ys, weights=None, eps=1e-6, interleaved=False, stream=None) -> None:
    """Enqueue the norm and position rotation of the heads of ``xs`` (queries,
    keys; fp16 [tokens, heads * dim] as the projections write them) into ``ys``
    (which may be ``xs``), one launch.

    ``pos``: int32 [tokens], rows of ``cos`` and ``sin``, fp32 [positions,
    rot / 2]; a token whose position is none of them is padding, and its outputs
    are left as they were. ``weights``: per input the norm's fp16 [dim] weight,
    or None for no norm. ``interleaved``: pairs are neighbours, else (i, i +
    rot / 2). torch's autograd does not record it: the gradients are
    ``rotate_heads_grad``'s."""
    inputs, k, r, n, s = _heads(xs, dim, pos, cos, sin, ys, weights, eps, interleaved, stream)
    _check(lib().spdp_rotate_heads(inputs, k, r, n, s))


def rotate_heads_grad(xs, dim, pos, cos, sin, dys, dxs, weights=None, dweights=None, eps=1e-6, interleaved=False,
                      stream=None) -> None:
    """Enqueue ``rotate_heads``'s gradients for ``dys``: ``dxs`` (0 for padding;
    each may be its x or dy) and, for inputs with a weight, ``dweights`` (fp32
    [dim], overwritten)."""
    inputs, k, r, n, s = _heads(xs, dim, pos, cos, sin, dxs, weights, eps, interleaved, stream, dys, dweights)
    need = ctypes.c_size_t()
    _check(lib().spdp_rotate_heads_grad_workspace(inputs, k, r, n, ctypes.byref(need)))
    ws = _workspace(need.value, xs[0].device, stream)
    _check(lib().spdp_rotate_heads_grad(inputs, k, r, n, ws.data_ptr(), need.value, s))


def encode_rtn(w: np.ndarray, tile=(256, 16), bits: int = 4) -> Matrix:
    """Quantize a pruned fp16 matrix to ``bits``-bit round-to-nearest codes
    (one scale per row), encode it with one byte per code and upload it."""
    wb = _u16(w)
    if wb.ndim != 2:
        raise ValueError("w must be 2-D")
    _free_deferred()
    h = ctypes.c_void_p()
    _check(lib().spdp_encode_rtn(_ptr(wb), wb.shape[0], wb.shape[1], int(tile[0]), int(tile[1]),
                                 int(bits), ctypes.byref(h)))
    return Matrix(h)


def encode_rtn_host(w: np.ndarray, tile=(256, 16), bits: int = 4) -> Matrix:
    """``encode_rtn`` without touching any device."""
    wb = _u16(w)
    if wb.ndim != 2:
        raise ValueError("w must be 2-D")
    h = ctypes.c_void_p()
    _check(lib().spdp_encode_rtn_host(_ptr(wb), wb.shape[0], wb.shape[1], int(tile[0]), int(tile[1]),
                                      int(bits), ctypes.byref(h)))
    return Matrix(h)


def encode_host(w: np.ndarray, tile=(256, 16)) -> Matrix:
    """Encode without touching any device (inspection, CPU-only machines)."""
    wb = _u16(w)
    if wb.ndim != 2:
        raise ValueError("w must be 2-D")
    h = ctypes.c_void_p()
    _check(lib().spdp_encode_host(_ptr(wb), wb.shape[0], wb.shape[1], int(tile[0]),
                                  int(tile[1]), ctypes.byref(h)))
    return Matrix(h)


def prune_magnitude(w: np.ndarray, sparsity: float) -> np.ndarray:
    """Global magnitude pruning (host C++); returns a new fp16 array."""
    wb = _u16(w)
    out = np.empty_like(wb)
    _check(lib().spdp_prune_magnitude(_ptr(wb), wb.size, float(sparsity), _ptr(out)))
    return out.view(np.float16)


def calibrate_threshold(x: np.ndarray, p: float) -> float:
    """Threshold that drops a fraction p of |x| under the strict rule |x| > t."""
    xb = _u16(x)
    t = ctypes.c_float()
    _check(lib().spdp_calibrate_threshold(_ptr(xb), xb.size, float(p), ctypes.byref(t)))
    return float(t.value)


def threshold_code(t: float) -> int:
    """Integer magnitude bound the kernels compare fp16 bits against."""
    c = ctypes.c_int32()
    _check(lib().spdp_threshold_code(ctypes.c_float(t), ctypes.byref(c)))
    return int(c.value)


class Chain:
    """A decoder layer's projections issued as one HIP graph.

    ``add`` records one launch: a list of products that read one input
    (q, k and v; gate and up) goes out as one grouped launch, a single
    product as a plain call. ``add_adapters`` and ``add_heads`` record what
    stands between them: the requests' adapters, and the norm and rotation of
    the heads. ``capture`` sizes every matrix's workspace for
    the batches recorded, issues the launches once eagerly (what works in place
    changes its tensors then, too) and records them into a graph on a side stream; ``replay`` re-issues the whole chain on
    the current stream with one host call. Between replays the caller
    rewrites the input tensors in place (and the thresholds are fixed at
    capture); the calls keep no host-side state, so every replay computes on
    the tensors' current contents, those of the adapters' and heads' weights,
    too. The graph has the addresses that the weights had at capture: where one
    has been replaced since (another tensor, or ``p.data = ...``), ``replay``
    raises, and the chain has to be captured again.
    """

    def __init__(self):
        self._calls = []
        self._graph = None
        self._weights = []   # of the recorded calls: Adapters, and the heads' tensors
        self._captured = []  # where the graph reads them
        self._alive = ()     # and that memory, which a replaced tensor would give back

    def add(self, mats, xs, thresholds, ys, mask: str = "token") -> "Chain":
        if self._graph is not None:
            raise RuntimeError("the chain is captured already")
        if isinstance(mats, Matrix):
            mats, xs, thresholds, ys = [mats], [xs], [thresholds], [ys]
        _mask_code(mask)
        self._calls.append((list(mats), list(xs), [float(t) for t in thresholds], list(ys), mask))
        return self

    def add_adapters(self, banks, xs, ids, bases, ys) -> "Chain":
        """Record an ``adapters_many`` call, behind the launch that wrote ``bases``."""
        if self._graph is not None:
            raise RuntimeError("the chain is captured already")
        if isinstance(banks, Adapters):
            banks, xs, bases, ys = [banks], [xs], [bases], [ys]
        args = (list(banks), list(xs), ids, list(bases), list(ys))
        self._weights += args[0]
        self._calls.append((None, args[1], None, lambda: adapters_many(*args), None))
        return self

    def add_heads(self, xs, dim, pos, cos, sin, ys, weights=None, eps=1e-6, interleaved=False) -> "Chain":
        """Record a ``rotate_heads`` call, behind the launch that wrote ``xs``."""
        if self._graph is not None:
            raise RuntimeError("the chain is captured already")
        args = (list(xs), dim, pos, cos, sin, list(ys), None if weights is None else list(weights), eps, interleaved)
        self._weights += [w for w in weights or [] if w is not None]
        self._calls.append((None, args[0], None, lambda: rotate_heads(*args), None))
        return self

    def _issue(self):
        for mats, xs, ts, ys, mask in self._calls:
            if mats is None:
                ys()
            elif len(mats) == 1:
                mats[0].spmspv_into(xs[0], ts[0], ys[0], mask=mask)
            else:
                spmspv_many(mats, xs, ts, ys, mask=mask)

    def _addresses(self) -> list:
        return [w._struct() if isinstance(w, Adapters) else w.data_ptr() for w in self._weights]

    def capture(self) -> "Chain":
        import torch
        if not self._calls:
            raise RuntimeError("nothing to capture")
        for mats, xs, _, _, _ in self._calls:
            for m, x in zip(mats or [], xs):
                m.reserve(int(x.shape[0]))
        dev = self._calls[0][1][0].device
        self._issue()  # eager once: every workspace and phase in place
        torch.cuda.synchronize(dev)
        s = torch.cuda.Stream(device=dev)
        s.wait_stream(torch.cuda.current_stream(dev))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            self._issue()
        torch.cuda.current_stream(dev).wait_stream(s)
        self._captured = self._addresses()
        self._alive = [t.detach() for w in self._weights
                       for t in ((w.a, w.b, w.scale) if isinstance(w, Adapters) else (w,))]
        self._graph = g
        return self

    def replay(self) -> None:
        if self._graph is None:
            raise RuntimeError("capture() first")
        if self._weights and self._addresses() != self._captured:
            raise RuntimeError("weights of adapters or heads were replaced since capture(): capture the chain again")
        self._graph.replay()
