"""Python binding of libflock (the C ABI in include/flock.h).

Argument marshalling only: torch tensors provide device memory and the
current HIP stream; every step of the computation runs in the library's HIP
kernels.  There is no CPU fallback: if libflock.so is missing or the device is
not a gfx950 GPU, calls raise.
"""

from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libflock.so")

FLOCK_OK = 0
FLOCK_EINVAL = -1
FLOCK_ENOMEM = -2
FLOCK_EDEVICE = -3
FLOCK_EUNSUPPORTED = -4

QUANTA_PER_PX = 16

_lib = None


class FlockError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"flock status {status}: {message}")
        self.status = status


def lib() -> ctypes.CDLL:
    """The loaded libflock.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2512_07009_amd.build` (there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        p, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        L.cluster_frames.argtypes = [p, p, i32, i32, i32, i32, i32, p, p, p, p, sz, p]
        L.cluster_frames.restype = i32
        L.density_frames.argtypes = [p, p, i32, i32, i32, i32, i32, i32, i32, ctypes.c_float, p, p, sz, p]
        L.density_frames.restype = i32
        L.cluster_frames_workspace.argtypes = [i32, i32, i32]
        L.cluster_frames_workspace.restype = sz
        L.density_frames_noalloc.argtypes = [p, p, i32, i32, i32, i32, i32, i32, i32, ctypes.c_float, p, p]
        L.density_frames_noalloc.restype = i32
        L.density_frames_workspace.argtypes = [i32, i32, i32, i32]
        L.density_frames_workspace.restype = sz
        L.heatmap_frames.argtypes = [p, i32, i32, i32, ctypes.c_double, ctypes.c_float, i32,
                                     p, p, p, p, p, p, p, sz, p]
        L.heatmap_frames.restype = i32
        L.heatmap_frames_workspace.argtypes = [i32, i32, i32]
        L.heatmap_frames_workspace.restype = sz
        L.roi_filter_frames.argtypes = [p, p, i32, i32, p, i32, p, p, p, p, p, sz, p]
        L.roi_filter_frames.restype = i32
        L.roi_filter_frames_workspace.argtypes = [i32, i32]
        L.roi_filter_frames_workspace.restype = sz
        L.drinker_proximity_frames.argtypes = [p, p, i32, i32, p, i32, i32, p, p, p, p, sz, p]
        L.drinker_proximity_frames.restype = i32
        L.drinker_proximity_frames_workspace.argtypes = [i32, i32]
        L.drinker_proximity_frames_workspace.restype = sz
        L.mask_components_frames.argtypes = [p, i32, i32, i32, ctypes.c_float, i32, p, p, p, i32,
                                             p, p, p, p, p, p, p, sz, p]
        L.mask_components_frames.restype = i32
        L.mask_components_frames_workspace.argtypes = [i32, i32, i32, i32]
        L.mask_components_frames_workspace.restype = sz
        i64, f32 = ctypes.c_int64, ctypes.c_float
        L.layer_norm_rows.argtypes = [i32, p, i64, p, i64, i32, i32, p, p, f32, p, i64, p, i64, p, p, p]
        L.layer_norm_rows.restype = i32
        L.layer_norm_rows_backward.argtypes = [i32, p, i64, p, i64, p, i64, i32, i32, p, p, p, p, i64, p, p, p, sz, p]
        L.layer_norm_rows_backward.restype = i32
        L.layer_norm_rows_backward_workspace.argtypes = [i32, i32]
        L.layer_norm_rows_backward_workspace.restype = sz
        L.rotary_frames.argtypes = [i32, p, i64, p, i64, i32, i32, i32, i32, p, p, p, i32, i32, i32, i32, i32,
                                    p, i64, p, i64, p]
        L.rotary_frames.restype = i32
        L.attention_frames.argtypes = [i32, p, i64, p, i64, p, i64, p, p, i32, i32, i32, i32, i32, i32, p, p, p, p, i32,
                                       p, f32, f32, p, i64, p, p, sz, p]
        L.attention_frames.restype = i32
        L.attention_frames_workspace.argtypes = [i32, i32, i32, i32, i32, i32]
        L.attention_frames_workspace.restype = sz
        L.attention_frames_backward.argtypes = [i32, p, i64, p, i64, p, i64, p, i64, p, i64, p, p, p, i32, i32, i32, i32,
                                                i32, i32, p, p, p, p, i32, p, f32, f32, p, i64, p, i64, p, i64, p, p,
                                                sz, p]
        L.attention_frames_backward.restype = i32
        L.attention_frames_backward_workspace.argtypes = [i32, i32, i32, i32, i32, i32]
        L.attention_frames_backward_workspace.restype = sz
        L.flock_last_error.argtypes = []
        L.flock_last_error.restype = ctypes.c_char_p
        L.flock_version.argtypes = []
        L.flock_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(status: int):
    if status != FLOCK_OK:
        msg = lib().flock_last_error().decode()
        if status == FLOCK_EINVAL:
            raise ValueError(f"flock: {msg}")
        raise FlockError(status, msg)


def _ptr(t):
    return t.data_ptr() if t is not None else None


# The current device and a device's current stream, without the objects that
# torch.cuda.current_device() and current_stream() make (about 1 us each; a
# call with one small kernel takes about 10 us in all).
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _workspace(nbytes: int, dev, stream):
    """Scratch for one call, allocated on the stream the kernels run on.
    torch's caching allocator hands a freed block out again only to work
    ordered after it on that stream, so the block is not reused before the
    kernels finish, with no cross-stream bookkeeping (and none under graph
    capture, where the block comes from the graph's own pool)."""
    if not nbytes:
        return None
    if stream is None or stream.cuda_stream == _raw_stream(dev.index):
        return torch.empty(nbytes, dtype=torch.uint8, device=dev)  # on dev's current stream
    with torch.cuda.device(dev), torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=dev)


def _new(shape, dtype, dev, stream):
    """An output of a call, in memory of the stream the kernels run on: a block
    that the current stream freed may still be in use there.  The current stream
    is recorded in turn, since the caller goes on with the output there."""
    if stream is None or stream.cuda_stream == _raw_stream(dev.index):
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.device(dev):
        here = torch.cuda.current_stream()
        with torch.cuda.stream(stream):
            t = torch.empty(shape, dtype=dtype, device=dev)
        t.record_stream(here)
    return t


def _call(fn, dev, stream, *args):
    """fn(*args, stream) with dev as the current device."""
    if _current_device() == dev.index:
        st = fn(*args, _raw_stream(dev.index) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(dev):
            st = fn(*args, _raw_stream(dev.index) if stream is None else stream.cuda_stream)
    _check(st)


def _batch(xy: torch.Tensor, offsets: torch.Tensor):
    if not (xy.is_cuda and offsets.is_cuda):
        raise ValueError("xy and offsets must be device tensors")
    if xy.dtype != torch.int32 or offsets.dtype != torch.int32:
        raise ValueError("xy and offsets must be int32")
    if xy.dim() != 2 or xy.shape[1] != 2 or not xy.is_contiguous():
        raise ValueError("xy must be a contiguous [T, 2] tensor")
    if offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous [F + 1] tensor")
    return offsets.numel() - 1, xy.shape[0]


def eps_to_quanta(eps_px: float) -> int:
    q = eps_px * QUANTA_PER_PX
    if abs(q - round(q)) > 1e-9:
        raise ValueError(f"eps_px = {eps_px} is not a multiple of 1/16 px")
    return int(round(q))


def cluster_frames(xy: torch.Tensor, offsets: torch.Tensor, eps_px: float, min_pts: int,
                   max_frame_points: int = 0, out=None, stream=None):
    """Cluster every frame; returns (labels int32[T], kind uint8[T], n_clusters int32[F]).

    max_frame_points: an upper bound on birds per frame (0 = unknown); it
    sizes on-chip storage and is not checked against the data.
    out: optional (labels, kind, n_clusters) tensors to write into.
    """
    F, T = _batch(xy, offsets)
    dev = xy.device
    if out is None:
        labels = _new(T, torch.int32, dev, stream)
        kind = _new(T, torch.uint8, dev, stream)
        ncl = _new(max(F, 0), torch.int32, dev, stream)
    else:
        labels, kind, ncl = out
    L = lib()
    ws_bytes = L.cluster_frames_workspace(F, T, int(max_frame_points))
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.cluster_frames, dev, stream, _ptr(xy), _ptr(offsets), F, T, int(max_frame_points),
          eps_to_quanta(eps_px), int(min_pts), _ptr(labels), _ptr(kind), _ptr(ncl), _ptr(ws), ws_bytes)
    return labels, kind, ncl


def density_frames(xy: torch.Tensor, offsets: torch.Tensor, width_px: int, height_px: int,
                   grid_w: int, grid_h: int, sigma_px: float, max_frame_points: int = 0, out=None,
                   stream=None):
    """Gaussian density grid of every frame: float32[F, grid_h, grid_w] (birds / px^2).

    max_frame_points: an upper bound on birds per frame, or 0 (a planning hint).
    """
    F, T = _batch(xy, offsets)
    dev = xy.device
    dens = out if out is not None else _new((max(F, 0), grid_h, grid_w), torch.float32, dev, stream)
    L = lib()
    ws_bytes = L.density_frames_workspace(F, T, int(grid_w), int(grid_h))
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.density_frames, dev, stream, _ptr(xy), _ptr(offsets), F, T, int(max_frame_points), int(width_px),
          int(height_px), int(grid_w), int(grid_h), float(sigma_px), _ptr(dens), _ptr(ws), ws_bytes)
    return dens


def heatmap_frames(density: torch.Tensor, cell_area_px2: float, threshold: float, connectivity: int = 8,
                   out=None, stream=None):
    """Heatmap analytics of float32 density grids [F, grid_h, grid_w] on the device.

    Returns a dict of device tensors: labels int32[F, h, w] (smallest cell
    index of the component, -1 for cold cells), n_components int32[F],
    entropy float64[F], degree float64[F], comp_cells int32[F, h, w] and
    comp_mass float64[F, h, w] (at label cells, 0 elsewhere).
    out: optional dict of such tensors to write into.
    """
    if not density.is_cuda or density.dtype != torch.float32 or density.dim() != 3 \
            or not density.is_contiguous():
        raise ValueError("density must be a contiguous float32 device tensor [F, grid_h, grid_w]")
    F, gh, gw = density.shape
    dev = density.device
    if out is None:
        out = {"labels": _new((F, gh, gw), torch.int32, dev, stream),
               "n_components": _new(F, torch.int32, dev, stream),
               "entropy": _new(F, torch.float64, dev, stream),
               "degree": _new(F, torch.float64, dev, stream),
               "comp_cells": _new((F, gh, gw), torch.int32, dev, stream),
               "comp_mass": _new((F, gh, gw), torch.float64, dev, stream)}
    L = lib()
    ws_bytes = L.heatmap_frames_workspace(F, gw, gh)
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.heatmap_frames, dev, stream, _ptr(density), F, gw, gh, float(cell_area_px2), float(threshold),
          int(connectivity), _ptr(out["labels"]), _ptr(out["n_components"]), _ptr(out["entropy"]),
          _ptr(out["degree"]), _ptr(out["comp_cells"]), _ptr(out["comp_mass"]), _ptr(ws), ws_bytes)
    return out


def roi_filter_frames(xy: torch.Tensor, offsets: torch.Tensor, roi_xy, with_index: bool = True, out=None,
                      stream=None):
    """Birds inside the closed ROI polygon roi_xy (host, [V, 2] int quanta).

    Returns a dict of device tensors: counts int32[F], xy int32[T, 2]
    (capacity; the first offsets[F] rows are the kept birds, frame after
    frame), offsets int32[F + 1], index int32[T] (capacity; input index of
    each kept bird) or None.
    """
    import numpy as np
    F, T = _batch(xy, offsets)
    poly = np.ascontiguousarray(np.asarray(roi_xy, dtype=np.int32).reshape(-1, 2))
    dev = xy.device
    if out is None:
        out = {"counts": _new(max(F, 0), torch.int32, dev, stream),
               "xy": _new((T, 2), torch.int32, dev, stream),
               "offsets": _new(F + 1, torch.int32, dev, stream),
               "index": _new(T, torch.int32, dev, stream) if with_index else None}
    L = lib()
    ws_bytes = L.roi_filter_frames_workspace(F, T)
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.roi_filter_frames, dev, stream, _ptr(xy), _ptr(offsets), F, T, poly.ctypes.data, poly.shape[0],
          _ptr(out["counts"]), _ptr(out["xy"]), _ptr(out["offsets"]), _ptr(out.get("index")), _ptr(ws),
          ws_bytes)
    return out


def drinker_proximity_frames(xy: torch.Tensor, offsets: torch.Tensor, lines, threshold_q: int,
                             with_line: bool = True, out=None, stream=None):
    """Birds strictly closer than threshold_q (1/16 px) to some drinker-line
    segment; lines: host [L, 4] int (ax, ay, bx, by) in 1/16 px.

    Returns a dict of device tensors: drinking uint8[T], line int32[T]
    (smallest index of such a segment, -1 if none) or None, counts int32[F].
    """
    import numpy as np
    F, T = _batch(xy, offsets)
    ln = np.ascontiguousarray(np.asarray(lines, dtype=np.int32).reshape(-1, 4))
    dev = xy.device
    if out is None:
        out = {"drinking": _new(T, torch.uint8, dev, stream),
               "line": _new(T, torch.int32, dev, stream) if with_line else None,
               "counts": _new(max(F, 0), torch.int32, dev, stream)}
    L = lib()
    ws_bytes = L.drinker_proximity_frames_workspace(F, T)
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.drinker_proximity_frames, dev, stream, _ptr(xy), _ptr(offsets), F, T, ln.ctypes.data, ln.shape[0],
          int(threshold_q), _ptr(out["drinking"]), _ptr(out.get("line")), _ptr(out["counts"]), _ptr(ws),
          ws_bytes)
    return out


def mask_capacity(n_frames: int, height: int, width: int, connectivity: int = 8) -> int:
    """Most components a batch of this shape can hold (isolated pixels on
    every other row and column with 8 neighbours, a checkerboard with 4)."""
    if connectivity == 8:
        return n_frames * ((height + 1) // 2) * ((width + 1) // 2)
    return n_frames * ((height * width + 1) // 2)


def mask_components_frames(prob: torch.Tensor, threshold: float, connectivity: int = 8, with_labels: bool = True,
                           capacity: int | None = None, out=None, stream=None):
    """Connected components of prob > threshold in float32 device masks
    [F, H, W], with statistics (the detection post-processing).

    Returns a dict of device tensors: labels int32[F, H, W] (first pixel of
    the component in raster order, -1 background) or None, n_components
    int32[F], offsets int32[F + 1] (offsets[F] = number of components K),
    and per component, in rows 0 .. min(K, capacity) - 1: label int32[C],
    area int32[C], box int32[C, 4] (x, y, width, height), centroid
    float64[C, 2], xy int32[C, 2] (1/16 px), score float32[C].  capacity
    defaults to the most components the shape can hold.
    """
    if not prob.is_cuda or prob.dtype != torch.float32 or prob.dim() != 3 or not prob.is_contiguous():
        raise ValueError("prob must be a contiguous float32 device tensor [F, H, W]")
    F, H, W = prob.shape
    dev = prob.device
    if capacity is None:
        capacity = mask_capacity(F, H, W, connectivity)
    C = int(capacity)
    if out is None:
        out = {"labels": _new((F, H, W), torch.int32, dev, stream) if with_labels else None,
               "n_components": _new(F, torch.int32, dev, stream),
               "offsets": _new(F + 1, torch.int32, dev, stream),
               "label": _new(C, torch.int32, dev, stream),
               "area": _new(C, torch.int32, dev, stream),
               "box": _new((C, 4), torch.int32, dev, stream),
               "centroid": _new((C, 2), torch.float64, dev, stream),
               "xy": _new((C, 2), torch.int32, dev, stream),
               "score": _new(C, torch.float32, dev, stream)}
    L = lib()
    ws_bytes = L.mask_components_frames_workspace(F, W, H, int(connectivity))
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.mask_components_frames, dev, stream, _ptr(prob), F, W, H, float(threshold), int(connectivity),
          _ptr(out.get("labels")), _ptr(out["n_components"]), _ptr(out["offsets"]), C, _ptr(out.get("label")),
          _ptr(out.get("area")), _ptr(out.get("box")), _ptr(out.get("centroid")), _ptr(out.get("xy")),
          _ptr(out.get("score")), _ptr(ws), ws_bytes)
    return out


# ---------------------------------------------------------------------------
# Per-bird encoder
# ---------------------------------------------------------------------------

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _dtype(t):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"features of {t.dtype}: expected float32, float16 or bfloat16")
    return code


# The checks below read each attribute once and compare device numbers: a call
# on few birds is bound by the host.

def _like(t, stream):
    """A contiguous output of t's shape, type and device (0.9 us on the current
    stream; torch.empty of them takes 1.4)."""
    if stream is None:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    return _new(t.shape, t.dtype, t.device, stream)


_MOST = 2 ** 31 - 1  # rows, birds and frames are numbered in 32 bits; ctypes would cut what is more


def _rows(t, name, like=None):
    """Stride of a device matrix [rows, width] whose rows are contiguous."""
    shape = t.shape
    if max(shape, default=0) > _MOST:
        raise ValueError(f"{name} has more than 2^31 - 1 rows or columns")
    if len(shape) != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a device matrix with contiguous rows")
    stride = t.stride()
    if stride[1] != 1 and shape[1] > 1 and shape[0] > 0:  # (an empty matrix may have any strides)
        raise ValueError(f"{name} must be a device matrix with contiguous rows")
    if like is not None and (shape != like.shape or t.dtype != like.dtype or t.get_device() != like.get_device()):
        raise ValueError(f"{name} must have the shape, type and device of its counterpart")
    return stride[0] if shape[0] > 1 else shape[1]


def _heads(t, name, like=None):
    """Stride of a device tensor [birds, heads, head_dim] whose rows are
    contiguous, of the type and on the device of `like`."""
    shape = t.shape
    if len(shape) != 3 or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor [birds, heads, head_dim] with contiguous rows")
    if max(shape) > _MOST:
        raise ValueError(f"{name} has more than 2^31 - 1 birds, heads or dimensions")
    n, heads, dim = shape
    stride = t.stride()
    if n > 0 and ((stride[2] != 1 and dim > 1) or (stride[1] != dim and heads > 1)):
        raise ValueError(f"{name} must be a device tensor [birds, heads, head_dim] with contiguous rows")
    if like is not None and (t.dtype != like.dtype or t.get_device() != like.get_device()):
        raise ValueError(f"{name} must have the type and device of the queries")
    return stride[0] if n > 1 else heads * dim


def _vector(t, name, dtype, numel, index):
    """Pointer of `numel` contiguous values on device number `index`."""
    if t.dtype != dtype or t.numel() != numel or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be {numel} contiguous {dtype} values on the features' device")
    return t.data_ptr()


def _matrix(t, name, dtype, rows, columns, index):
    """Pointer of [rows, columns] contiguous values on device number `index`."""
    if t.dtype != dtype or t.shape != (rows, columns) or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} [{rows}, {columns}] tensor on the features' device")
    return t.data_ptr()


def layer_norm_rows(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                    eps: float = 1e-5, residual: torch.Tensor | None = None, out=None, stream=None):
    """Layer norm of every row of x [N, width] (float32, float16 or bfloat16),
    or of x + residual, with float32 weight and bias.

    Returns (y, h, mean, rstd): h is what was normalised (x itself, or the sum
    in x's type), and h, mean and rstd (float32 [N]) are what
    layer_norm_rows_backward takes.
    out: optional (y, h, mean, rstd) tensors to write into (h only with residual).
    """
    code, xs = _dtype(x), _rows(x, "x")
    n, width = x.shape
    dev = x.device
    index = dev.index
    wp = _vector(weight, "weight", torch.float32, width, index) if weight is not None else None
    bp = _vector(bias, "bias", torch.float32, width, index) if bias is not None else None
    rs = _rows(residual, "residual", x) if residual is not None else 0
    if out is None:
        y = _like(x, stream)
        h = _like(x, stream) if residual is not None else x
        mean, rstd = _new((2, n), torch.float32, dev, stream).unbind()
        ys = hs = width
    else:
        y, h, mean, rstd = out
        ys = _rows(y, "y", x)
        hs = _rows(h, "h", x) if residual is not None else 0
        _vector(mean, "mean", torch.float32, n, index)
        _vector(rstd, "rstd", torch.float32, n, index)
        if residual is None:
            h = x
    _call(lib().layer_norm_rows, dev, stream, code, x.data_ptr(), xs, _ptr(residual), rs, n, width, wp,
          bp, eps, y.data_ptr(), ys, h.data_ptr() if residual is not None else None, hs, mean.data_ptr(),
          rstd.data_ptr())
    return y, h, mean, rstd


def layer_norm_rows_backward(grad_y: torch.Tensor, h: torch.Tensor, weight: torch.Tensor | None, mean: torch.Tensor,
                             rstd: torch.Tensor, grad_sum: torch.Tensor | None = None, stream=None):
    """Gradients of layer_norm_rows from its h, mean and rstd; grad_sum is the
    gradient that h got elsewhere.

    Returns (grad_x in h's type, also the residual's gradient; grad_weight and
    grad_bias float32 [width]).
    """
    code, xs = _dtype(h), _rows(h, "h")
    n, width = h.shape
    dev = h.device
    gs = _rows(grad_y, "grad_y", h)
    ss = _rows(grad_sum, "grad_sum", h) if grad_sum is not None else 0
    index = dev.index
    wp = _vector(weight, "weight", torch.float32, width, index) if weight is not None else None
    mp = _vector(mean, "mean", torch.float32, n, index)
    rp = _vector(rstd, "rstd", torch.float32, n, index)
    dx = _like(h, stream)
    dw, db = _new((2, width), torch.float32, dev, stream).unbind()
    L = lib()
    ws_bytes = L.layer_norm_rows_backward_workspace(n, width)
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.layer_norm_rows_backward, dev, stream, code, grad_y.data_ptr(), gs, _ptr(grad_sum), ss, h.data_ptr(), xs, n,
          width, wp, mp, rp, dx.data_ptr(), width, dw.data_ptr(), db.data_ptr(),
          _ptr(ws), ws_bytes)
    return dx, dw, db


class RotaryAxes:
    """The frequencies of rotary_frames: radians per unit of time for the first
    pairs of dimensions, per px of y for the next, per px of x for the last."""

    def __init__(self, time=(), y=(), x=()):
        freq = [float(f) for f in (*time, *y, *x)]
        self.counts = (len(time), len(y), len(x))
        self.pairs = len(freq)
        self.freq = (ctypes.c_double * max(len(freq), 1))(*freq)


def rotary_frames(q: torch.Tensor | None, k: torch.Tensor | None, xy: torch.Tensor | None, axes: RotaryAxes,
                  time: torch.Tensor | None = None, interleaved: bool = False, inverse: bool = False, out=None,
                  stream=None):
    """Rotary positions from time (int32 [T]), y and x (xy, 1/16 px) of queries
    [T, Hq, D] and keys [T, Hk, D] (either may be None); returns (q, k) turned.

    Pair p of the axes' pairs is dimensions (p, p + pairs), or (2p, 2p + 1)
    where interleaved; the rest is copied.  inverse turns back: with the
    gradients of the turned tensors it gives the gradients of q and k.
    out: optional (q, k) to write into, which may be q and k themselves.
    """
    first = q if q is not None else k
    if first is None:
        raise ValueError("q or k must be given")
    code, dev, n = _dtype(first), first.device, first.shape[0]
    dim = first.shape[-1]
    qs = _heads(q, "q") if q is not None else 0
    ks = _heads(k, "k", first) if k is not None else 0
    if k is not None and (k.shape[0] != n or k.shape[2] != dim):
        raise ValueError("q and k must have the same birds and head_dim")
    nt, ny, nx = axes.counts
    if ny or nx:
        if xy is None or xy.dtype != torch.int32 or xy.get_device() != dev.index or xy.shape != (n, 2) \
                or not xy.is_contiguous():
            raise ValueError("xy must be a contiguous int32 [T, 2] tensor on the features' device")
    if nt:
        if time is None:
            raise ValueError("time is needed by the axes' time pairs")
        _vector(time, "time", torch.int32, n, dev.index)
    qo, ko = out if out is not None else (None, None)
    qos = kos = 0
    if q is not None:
        if qo is None:
            qo, qos = _like(q, stream), q.shape[1] * dim
        else:
            qos = _heads(qo, "out's q", first)
            if qo.shape != q.shape:
                raise ValueError("out's q must have the shape of q")
    if k is not None:
        if ko is None:
            ko, kos = _like(k, stream), k.shape[1] * dim
        else:
            kos = _heads(ko, "out's k", first)
            if ko.shape != k.shape:
                raise ValueError("out's k must have the shape of k")
    _call(lib().rotary_frames, dev, stream, code, _ptr(q), qs, _ptr(k), ks, n, q.shape[1] if q is not None else 0,
          k.shape[1] if k is not None else 0, dim, _ptr(xy) if ny or nx else None, _ptr(time) if nt else None,
          axes.freq, nt, ny, nx, int(interleaved), int(inverse), _ptr(qo), qos, _ptr(ko), kos)
    return qo, ko


def _attention(q, k, v, q_offsets, k_offsets, q_xy, k_xy, slopes, keep, prefix, causal):
    """The checked arguments that the forward and the backward call share."""
    code = _dtype(q)
    qs, ks, vs = _heads(q, "q"), _heads(k, "k", q), _heads(v, "v", q)
    tq, hq, dim = q.shape
    tk, hk, k_dim = k.shape
    if v.shape != k.shape or k_dim != dim:
        raise ValueError("k and v must have one shape, with the head_dim of q")
    index = q.get_device()
    frames = q_offsets.numel() - 1
    if not 0 <= frames <= _MOST or q_offsets.dim() != 1:
        raise ValueError("q_offsets must be a contiguous [F + 1] tensor")
    qo = _vector(q_offsets, "q_offsets", torch.int32, frames + 1, index)
    ko = qo
    if k_offsets is not None and k_offsets is not q_offsets:
        ko = _vector(k_offsets, "k_offsets", torch.int32, frames + 1, index)
    sp = qp = kp = None
    if slopes is not None:
        sp = _vector(slopes, "slopes", torch.float32, hq, index)
        if q_xy is None:
            raise ValueError("q_xy is needed with slopes")
        qp = _matrix(q_xy, "q_xy", torch.int32, tq, 2, index)
        kp = _matrix(q_xy if k_xy is None else k_xy, "k_xy", torch.int32, tk, 2, index)
    keep_p = _vector(keep, "keep", torch.uint8, tk, index) if keep is not None else None
    prefix_p = _vector(prefix, "prefix", torch.int32, frames, index) if prefix is not None else None
    return (code, q.device, (frames, tq, tk, hq, hk, dim), (q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs),
            (qo, ko, frames, tq, tk, hq, hk, dim, qp, kp, sp, keep_p, int(causal), prefix_p if causal else None))


def attention_frames(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor,
                     k_offsets: torch.Tensor | None = None, q_xy: torch.Tensor | None = None,
                     k_xy: torch.Tensor | None = None, slopes: torch.Tensor | None = None,
                     scale: float | None = None, cap: float = 0.0, keep: torch.Tensor | None = None,
                     causal: bool = False, prefix: torch.Tensor | None = None, return_lse: bool = False, out=None,
                     stream=None):
    """Attention of queries [Tq, Hq, D] over the keys and values [Tk, Hkv, D] of
    their frame (float16 or bfloat16), frames given by CSR offsets.

    k_offsets: the keys' offsets (None: the queries').  slopes: float32 [Hq],
    with places q_xy and k_xy (None: q_xy) in 1/16 px: slopes[h] times the
    squared distance in px is taken off the scores.  scale: 1 / sqrt(D) if None.
    cap: scores become cap * tanh(score / cap).  keep: uint8 [Tk], 0 hides a
    key.  causal: key j of a frame is seen by query i if j < prefix[frame]
    (int32 [F], None: 0) or j <= i + keys - queries.
    Returns out [Tq, Hq, D], or (out, lse float64 [Tq, Hq]) with return_lse.
    out: optional tensor to write into.
    """
    code, dev, shape, head, tail = _attention(q, k, v, q_offsets, k_offsets, q_xy, k_xy, slopes, keep, prefix, causal)
    if out is None:
        out = _like(q, stream)
        out_stride = shape[3] * shape[5]
    else:
        out_stride = _heads(out, "out", q)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    lse = _new((shape[1], shape[3]), torch.float64, dev, stream) if return_lse else None
    L = lib()
    ws_bytes = L.attention_frames_workspace(*shape)
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.attention_frames, dev, stream, code, *head, *tail, shape[5] ** -0.5 if scale is None else scale, cap,
          out.data_ptr(), out_stride, _ptr(lse), _ptr(ws), ws_bytes)
    return (out, lse) if return_lse else out


def attention_frames_backward(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                              out: torch.Tensor, lse: torch.Tensor, q_offsets: torch.Tensor,
                              k_offsets: torch.Tensor | None = None, q_xy: torch.Tensor | None = None,
                              k_xy: torch.Tensor | None = None, slopes: torch.Tensor | None = None,
                              scale: float | None = None, cap: float = 0.0, keep: torch.Tensor | None = None,
                              causal: bool = False, prefix: torch.Tensor | None = None, stream=None):
    """Gradients of attention_frames: its arguments with its out and lse, and
    grad_out.  Returns (grad_q, grad_k, grad_v, grad_slopes float32 [Hq], or
    None without slopes)."""
    code, dev, shape, head, tail = _attention(q, k, v, q_offsets, k_offsets, q_xy, k_xy, slopes, keep, prefix, causal)
    gs = _heads(grad_out, "grad_out", q)
    out_stride = _heads(out, "out", q)
    if grad_out.shape != q.shape or out.shape != q.shape:
        raise ValueError("grad_out and out must have the shape of q")
    lp = _matrix(lse, "lse", torch.float64, shape[1], shape[3], dev.index)
    dq, dk, dv = _like(q, stream), _like(k, stream), _like(k, stream)
    ds = _new(shape[3], torch.float32, dev, stream) if slopes is not None else None
    q_row, k_row = shape[3] * shape[5], shape[4] * shape[5]
    L = lib()
    ws_bytes = L.attention_frames_backward_workspace(*shape)
    ws = _workspace(ws_bytes, dev, stream)
    _call(L.attention_frames_backward, dev, stream, code, grad_out.data_ptr(), gs, *head, out.data_ptr(), out_stride,
          lp, *tail, shape[5] ** -0.5 if scale is None else scale, cap, dq.data_ptr(), q_row,
          dk.data_ptr(), k_row, dv.data_ptr(), k_row, _ptr(ds), _ptr(ws), ws_bytes)
    return dq, dk, dv, ds


def version() -> str:
    return lib().flock_version().decode()
