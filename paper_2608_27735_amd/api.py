"""Python binding of the ABCD C ABI (include/abcd.h) for torch tensors on the GPU.

Argument marshalling only: tensors are checked for device, dtype and layout,
their device pointers and the current HIP stream are passed to libabcd.so,
and every step runs in the library's kernels. There is no CPU fallback.
"""
import ctypes as C

import torch

from . import _lib
from ._lib import AbcdError, check

_lib.load()  # no fallback: the binding is unusable without the built library


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    """The current stream's handle (torch.cuda.current_stream makes an object of it
    first, which takes 2.7 us of a call)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


_dummies = {}


def _ptr_nz(t, device):
    """Device pointer of t; for a missing or empty tensor (whose pointer may be
    NULL) a small placeholder buffer on the device that no kernel reads (the
    library requires these input pointers to be non-NULL)."""
    if t is not None and t.numel() > 0:
        return t.data_ptr()
    d = _dummies.get(device)
    if d is None:
        d = _dummies[device] = torch.zeros(64, dtype=torch.float32, device=device)
    return d.data_ptr()


def _need(t, name, dtype, shape=None):
    if t is None:
        raise ValueError(f"{name} is required")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t


def _opt(t, name, dtype, shape=None):
    return None if t is None else _need(t, name, dtype, shape)


def n_tiles(width, height):
    return ((width + 15) // 16) * ((height + 15) // 16)


def _empty(shape, dtype, device):
    return torch.empty(shape, dtype=dtype, device=device)


def version():
    return _lib.load().abcd_version().decode()


# ------------------------------------------------------------------ project

def project(cam, prm, means, log_scales, quats, opacity_logits, sh, out=None):
    """EWA projection; returns dict(means2d, conic_opacity, depth, extent
    (n, 2: half extents of the binning box), tiles_touched (int32 view of
    uint32), rgb)."""
    n = means.shape[0]
    nc = (prm.sh_degree + 1) ** 2
    f32 = torch.float32
    _need(means, "means", f32, (n, 3))
    _need(log_scales, "log_scales", f32, (n, 3))
    _need(quats, "quats", f32, (n, 4))
    _need(opacity_logits, "opacity_logits", f32, (n,))
    _need(sh, "sh", f32, (n, nc, 3))
    dev = means.device
    if out is None:
        out = dict(means2d=_empty((n, 2), f32, dev), conic_opacity=_empty((n, 4), f32, dev),
                   depth=_empty((n,), f32, dev), extent=_empty((n, 2), f32, dev),
                   tiles_touched=_empty((n,), torch.int32, dev), rgb=_empty((n, 3), f32, dev))
    lib = _lib.load()
    check(lib.abcd_project(C.byref(_lib.camera_struct(cam)), C.byref(_lib.params_struct(prm)), n,
                           _ptr(means), _ptr(log_scales), _ptr(quats), _ptr(opacity_logits),
                           _ptr(sh), _ptr(out["means2d"]), _ptr(out["conic_opacity"]),
                           _ptr(out["depth"]), _ptr(out["extent"]), _ptr(out["tiles_touched"]),
                           _ptr(out["rgb"]), _stream()))
    return out


# ------------------------------------------------------------------ binning

def bin_sort_workspace_size(n, width, height, capacity=0):
    sz = C.c_size_t(0)
    check(_lib.load().abcd_bin_sort_workspace_size(n, capacity, width, height, C.byref(sz)))
    return sz.value


def bin_sort(width, height, proj, capacity=None, workspace=None, values=None, keys=None,
             tile_ranges=None, tile_order=None, want_keys=False, sync=True):
    """Per-tile depth-sorted lists. Returns dict(values, tile_ranges, tile_order,
    keys, n_isect); tile_order is the forward's schedule (heaviest lists first).

    With sync=True (default) M is read back (one stream synchronisation) and
    the buffers are grown to fit it; with sync=False the call never
    synchronises and `capacity`/`values` must already be large enough: an
    overflow leaves values unwritten and every tile range empty, and
    intersections(workspace) > capacity tells it afterwards."""
    means2d, extent = proj["means2d"], proj["extent"]
    depth, tiles = proj["depth"], proj["tiles_touched"]
    n = means2d.shape[0]
    dev = means2d.device
    _need(means2d, "means2d", torch.float32, (n, 2))
    _need(extent, "extent", torch.float32, (n, 2))
    _need(depth, "depth", torch.float32, (n,))
    _need(tiles, "tiles_touched", torch.int32, (n,))
    if tile_ranges is None:
        tile_ranges = _empty((n_tiles(width, height), 2), torch.int32, dev)
    if tile_order is None:
        tile_order = _empty((n_tiles(width, height),), torch.int32, dev)
    if capacity is None:
        capacity = 0 if values is None else values.numel()
    ws_bytes = bin_sort_workspace_size(n, width, height, capacity)
    if workspace is None or workspace.numel() < ws_bytes:
        workspace = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=dev)
    if values is None and capacity > 0:
        values = _empty((capacity,), torch.int32, dev)
    if want_keys and (keys is None or keys.numel() < capacity):
        keys = _empty((max(capacity, 1),), torch.int64, dev)
    lib = _lib.load()
    m = C.c_int64(0)
    st = lib.abcd_bin_sort(width, height, n, _ptr(means2d), _ptr(extent), _ptr(depth), _ptr(tiles),
                           capacity, _ptr(workspace), workspace.numel(),
                           _ptr(keys) if want_keys else None, _ptr(values), _ptr(tile_ranges),
                           _ptr(tile_order), C.byref(m) if sync else None, _stream())
    if st == _lib.ABCD_E_CAPACITY and sync:
        capacity = int(m.value)
        values = _empty((max(capacity, 1),), torch.int32, dev)
        if want_keys:
            keys = _empty((max(capacity, 1),), torch.int64, dev)
        ws_bytes = bin_sort_workspace_size(n, width, height, capacity)
        if workspace.numel() < ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        st = lib.abcd_bin_sort(width, height, n, _ptr(means2d), _ptr(extent), _ptr(depth),
                               _ptr(tiles), capacity, _ptr(workspace), workspace.numel(),
                               _ptr(keys) if want_keys else None, _ptr(values), _ptr(tile_ranges),
                               _ptr(tile_order), C.byref(m), _stream())
    check(st)
    return dict(values=values, tile_ranges=tile_ranges, tile_order=tile_order,
                keys=keys if want_keys else None,
                n_isect=int(m.value) if sync else None, workspace=workspace, capacity=capacity)


def intersections(workspace):
    """The intersection count M the last abcd_bin_sort on this workspace found
    (the uint64 at the workspace's start; reading it synchronises with the
    stream). M > capacity means that call overflowed and rendered nothing."""
    return int(workspace[:8].cpu().view(torch.int64).item())


# -------------------------------------------------------------- rasterise

def split_workspace_size(n_slots):
    sz = C.c_size_t(0)
    check(_lib.load().abcd_split_workspace_size(int(n_slots), C.byref(sz)))
    return sz.value


def make_split(n_slots, chunk=2048, device=None):
    """A split workspace (see abcd_split) with n_slots checkpoint slots; give
    the same one to a forward and its backward."""
    dev = device or torch.device("cuda", torch.cuda.current_device())
    ws = torch.empty(split_workspace_size(n_slots), dtype=torch.uint8, device=dev)
    return dict(workspace=ws, chunk=int(chunk))


def _split_struct(split):
    if split is None:
        return None
    ws = split["workspace"]
    if not ws.is_cuda or ws.dtype != torch.uint8:
        raise ValueError("split workspace must be a uint8 GPU tensor")
    return C.byref(_lib.abcd_split(ws.data_ptr(), ws.numel(), int(split["chunk"]), 0))


def render_fwd(cam, prm, bins, proj, F=None, B=None, n_blends=None, out=None, split=None):
    """out = F over A over B; returns dict(out, final_T, last). split: see
    make_split (the backward must get the same one)."""
    H, W = cam.height, cam.width
    dev = proj["means2d"].device
    _opt(F, "F", torch.float32, (H, W, 4))
    _opt(B, "B", torch.float32, (H, W, 4))
    _opt(n_blends, "n_blends", torch.int64, (1,))
    if out is None:
        out = dict(out=_empty((H, W, 4), torch.float32, dev),
                   final_T=_empty((H, W), torch.float32, dev),
                   last=_empty((H, W), torch.int32, dev))
    lib = _lib.load()
    check(lib.abcd_render_fwd(C.byref(_lib.camera_struct(cam)), C.byref(_lib.params_struct(prm)),
                              _ptr(bins["tile_ranges"]), _ptr(bins.get("tile_order")),
                              _ptr_nz(bins["values"], dev), _ptr_nz(proj["means2d"], dev),
                              _ptr_nz(proj["conic_opacity"], dev), _ptr_nz(proj["rgb"], dev),
                              _ptr(F), _ptr(B), _ptr(out["out"]), _ptr(out["final_T"]),
                              _ptr(out["last"]), _ptr(n_blends), _split_struct(split), _stream()))
    return out


def render_cache(cam, prm, bins, proj, image=None, rect=None):
    """The partition rendered alone (F = B = transparent) as premultiplied fp16
    RGBA [H, W, 4] (torch.float16), the form abcd_composite_cache consumes.
    rect: optional int32 [4] GPU tensor that receives the coverage box."""
    H, W = cam.height, cam.width
    if image is None:
        image = _empty((H, W, 4), torch.float16, proj["means2d"].device)
    _need(image, "image", torch.float16, (H, W, 4))
    _opt(rect, "rect", torch.int32, (4,))
    dev = proj["means2d"].device
    check(_lib.load().abcd_render_cache(
        C.byref(_lib.camera_struct(cam)), C.byref(_lib.params_struct(prm)),
        _ptr(bins["tile_ranges"]), _ptr(bins.get("tile_order")), _ptr_nz(bins["values"], dev),
        _ptr_nz(proj["means2d"], dev), _ptr_nz(proj["conic_opacity"], dev),
        _ptr_nz(proj["rgb"], dev), _ptr(image),
        _ptr(rect), _stream()))
    return image


def render_bwd_workspace_size(n):
    sz = C.c_size_t(0)
    check(_lib.load().abcd_render_bwd_workspace_size(n, C.byref(sz)))
    return sz.value


def render_bwd(cam, prm, params, proj, bins, fwd, dL_dout, F=None, B=None, workspace=None,
               grads=None, accumulate=False, want_means2d=False, split=None):
    """Gradients of the active parameters; returns dict(means, log_scales, quats,
    opacity_logits, sh[, means2d])."""
    n = params["means"].shape[0]
    H, W = cam.height, cam.width
    dev = params["means"].device
    _need(dL_dout, "dL_dout", torch.float32, (H, W, 4))
    _opt(F, "F", torch.float32, (H, W, 4))
    _opt(B, "B", torch.float32, (H, W, 4))
    ws_bytes = render_bwd_workspace_size(n)
    if workspace is None or workspace.numel() < ws_bytes:
        workspace = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=dev)
    if grads is None:
        grads = {k: torch.zeros_like(params[k]) for k in
                 ("means", "log_scales", "quats", "opacity_logits", "sh")}
        if want_means2d:
            grads["means2d"] = torch.zeros((n, 2), dtype=torch.float32, device=dev)
    lib = _lib.load()
    check(lib.abcd_render_bwd(
        C.byref(_lib.camera_struct(cam)), C.byref(_lib.params_struct(prm)), n,
        _ptr(params["means"]), _ptr(params["log_scales"]), _ptr(params["quats"]),
        _ptr(params["opacity_logits"]), _ptr(params["sh"]), _ptr(proj["means2d"]),
        _ptr(proj["conic_opacity"]), _ptr(proj["rgb"]), _ptr(proj["extent"]),
        _ptr(bins["tile_ranges"]), _ptr_nz(bins["values"], dev), _ptr(F), _ptr(B),
        _ptr(fwd["final_T"]),
        _ptr(fwd["last"]), _ptr(dL_dout), _ptr(workspace), workspace.numel(), _ptr(grads["means"]),
        _ptr(grads["log_scales"]), _ptr(grads["quats"]), _ptr(grads["opacity_logits"]),
        _ptr(grads["sh"]), _ptr(grads.get("means2d")), 1 if accumulate else 0,
        _split_struct(split), _stream()))
    return grads


def render_bwd_noalloc(cam, prm, params, proj, bins, fwd, dL_dout, F=None, B=None, grads=None,
                       accumulate=False, want_means2d=False, split=None):
    """render_bwd through abcd_render_bwd_noalloc: no workspace, the library's
    static per-GPU scratch instead (n <= NOALLOC_MAX_GAUSSIANS; calls that
    overlap on one GPU race). `grads` should be preallocated by callers that
    must not allocate."""
    n = params["means"].shape[0]
    H, W = cam.height, cam.width
    dev = params["means"].device
    _need(dL_dout, "dL_dout", torch.float32, (H, W, 4))
    _opt(F, "F", torch.float32, (H, W, 4))
    _opt(B, "B", torch.float32, (H, W, 4))
    if grads is None:
        grads = {k: torch.zeros_like(params[k]) for k in
                 ("means", "log_scales", "quats", "opacity_logits", "sh")}
        if want_means2d:
            grads["means2d"] = torch.zeros((n, 2), dtype=torch.float32, device=dev)
    check(_lib.load().abcd_render_bwd_noalloc(
        C.byref(_lib.camera_struct(cam)), C.byref(_lib.params_struct(prm)), n,
        _ptr(params["means"]), _ptr(params["log_scales"]), _ptr(params["quats"]),
        _ptr(params["opacity_logits"]), _ptr(params["sh"]), _ptr(proj["means2d"]),
        _ptr(proj["conic_opacity"]), _ptr(proj["rgb"]), _ptr(proj["extent"]),
        _ptr(bins["tile_ranges"]), _ptr_nz(bins["values"], dev), _ptr(F), _ptr(B),
        _ptr(fwd["final_T"]), _ptr(fwd["last"]), _ptr(dL_dout), _ptr(grads["means"]),
        _ptr(grads["log_scales"]), _ptr(grads["quats"]), _ptr(grads["opacity_logits"]),
        _ptr(grads["sh"]), _ptr(grads.get("means2d")), 1 if accumulate else 0,
        _split_struct(split), _stream()))
    return grads


# --------------------------------------------------------------- optimizer

PARAM_GROUPS = ("means", "log_scales", "quats", "opacity_logits", "sh")


def adam_step(params, grads, exp_avg, exp_avg_sq, lr, step, beta1=0.9, beta2=0.999, eps=1e-15):
    """One Adam update of the parameter groups (dicts of fp32 GPU tensors, in
    place); lr is a dict (one rate per group) or a float."""
    names = [k for k in params if params[k].numel() > 0]
    if len(names) > _lib.ADAM_MAX_GROUPS:
        raise ValueError("too many parameter groups")
    arr = (_lib.abcd_adam_group * max(len(names), 1))()
    for i, k in enumerate(names):
        for t, nm in ((params[k], "param"), (grads[k], "grad"), (exp_avg[k], "exp_avg"),
                      (exp_avg_sq[k], "exp_avg_sq")):
            _need(t, f"{nm}[{k}]", torch.float32, tuple(params[k].shape))
        arr[i].param, arr[i].grad = _ptr(params[k]), _ptr(grads[k])
        arr[i].exp_avg, arr[i].exp_avg_sq = _ptr(exp_avg[k]), _ptr(exp_avg_sq[k])
        arr[i].count = params[k].numel()
        arr[i].lr = float(lr[k] if isinstance(lr, dict) else lr)
    check(_lib.load().abcd_adam_step(arr, len(names), float(beta1), float(beta2), float(eps),
                                     int(step), _stream()))


# ------------------------------------------------------------ decoder: rows

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}  # abcd_dtype


def _dtype_of(t, name):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a tensor")
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, got {t.dtype}")
    return code


def _rows(t, name, like=None, shape=None):
    """Checks a matrix of rows with unit stride along a row; returns the distance
    between its rows. like: a tensor whose dtype and device it shares."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{name} must be {like.dtype} on {like.device}, "
                         f"got {t.dtype} on {t.device}")
    size = t.shape
    if len(size) != 2 or (shape is not None and size != shape):
        raise ValueError(f"{name} has shape {tuple(size)}, expected "
                         f"{'(rows, width)' if shape is None else tuple(shape)}")
    n, d = size
    if d == 0:
        raise ValueError(f"{name} has rows of width 0")
    if n <= 1 and d <= 1:
        return d
    s0, s1 = t.stride()
    if n <= 1:
        s0 = d
    if (d > 1 and s1 != 1) or s0 < d:
        raise ValueError(f"{name} must have unit stride along a row and rows that do not overlap, "
                         f"got strides {t.stride()}")
    return s0


def _vector(t, name, d, dtype, device):
    if t is None:
        return
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} on {device}, got {t.dtype} on {t.device}")
    if t.shape != (d,) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with shape ({d},), got {tuple(t.shape)}")


def _param_dtype(x, weight, bias):
    """The common type of weight and bias: x's or float32."""
    wt = weight.dtype if weight is not None else bias.dtype if bias is not None else x.dtype
    if wt != x.dtype and wt != torch.float32:
        raise ValueError(f"weight and bias must be {x.dtype} or float32, got {wt}")
    return wt


def _new(x, size):
    """An array of x's type beside x (empty_like is half of what torch.empty takes)."""
    return torch.empty_like(x) if x.shape == size and x.is_contiguous() else x.new_empty(size)


def _workspace(workspace, need, device):
    if workspace is None:
        return torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    if not workspace.is_cuda or workspace.device != device or workspace.dtype != torch.uint8 \
            or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {device}")
    return workspace  # its size is checked by the library


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, mean=None, rstd=None):
    """Layer norm of the rows of x [n, d] (float32, float16 or bfloat16; any row
    stride): dict(y, mean, rstd), mean and rstd in float32, which
    layer_norm_bwd takes. weight, bias [d]: of x's type or float32. out, mean,
    rstd: where to write (out may be x)."""
    code = _dtype_of(x, "x")
    ldx = _rows(x, "x")
    size, dev = x.shape, x.device
    n, d = size
    wt = _param_dtype(x, weight, bias)
    _vector(weight, "weight", d, wt, dev)
    _vector(bias, "bias", d, wt, dev)
    if out is None:
        out, ldy = _new(x, size), d
    else:
        ldy = _rows(out, "out", x, size)
    _vector(mean, "mean", n, torch.float32, dev)
    _vector(rstd, "rstd", n, torch.float32, dev)
    if mean is None:
        mean = torch.empty(n, dtype=torch.float32, device=dev)
    if rstd is None:
        rstd = torch.empty(n, dtype=torch.float32, device=dev)
    check(_lib.load().abcd_layer_norm(code, n, d, x.data_ptr(), ldx, _DTYPES[wt], _ptr(weight),
                                      _ptr(bias), eps, out.data_ptr(), ldy,
                                      mean.data_ptr(), rstd.data_ptr(), _stream()))
    return dict(y=out, mean=mean, rstd=rstd)


def layer_norm_bwd_workspace_size(n, d, dtype):
    sz = C.c_size_t(0)
    check(_lib.load().abcd_layer_norm_bwd_workspace_size(_DTYPES[dtype], n, d, C.byref(sz)))
    return sz.value


def layer_norm_bwd(dy, x, mean, rstd, weight=None, add=None, wdtype=None, workspace=None,
                   grads=None):
    """Gradients of layer_norm: dict(x, weight, bias). mean and rstd are the
    forward's; add [n, d] is added to x's gradient (a residual path's). weight
    and bias gradients have weight's type (wdtype without a weight). grads: a
    dict of tensors to write into, where a None leaves that gradient out; x's may be
    dy or add itself."""
    code = _dtype_of(x, "x")
    ldx = _rows(x, "x")
    size, dev = x.shape, x.device
    n, d = size
    lddy = _rows(dy, "dy", x, size)
    ldadd = 0 if add is None else _rows(add, "add", x, size)
    _vector(mean, "mean", n, torch.float32, dev)
    _vector(rstd, "rstd", n, torch.float32, dev)
    if weight is not None or wdtype is None:
        wdtype = _param_dtype(x, weight, None)
    elif wdtype != x.dtype and wdtype != torch.float32:
        raise ValueError(f"wdtype must be {x.dtype} or float32, got {wdtype}")
    _vector(weight, "weight", d, wdtype, dev)
    if grads is None:
        dx, lddx = _new(x, size), d
        if weight is not None:
            dw, db = torch.empty_like(weight), torch.empty_like(weight)
        else:
            dw, db = torch.empty((2, d), dtype=wdtype, device=dev).unbind(0)
        grads = dict(x=dx, weight=dw, bias=db)
    else:
        dx, dw, db = grads.get("x"), grads.get("weight"), grads.get("bias")
        lddx = 0 if dx is None else _rows(dx, "grads[x]", x, size)
        _vector(dw, "grads[weight]", d, wdtype, dev)
        _vector(db, "grads[bias]", d, wdtype, dev)
    if dw is not None or db is not None:
        workspace = _workspace(workspace, layer_norm_bwd_workspace_size(n, d, x.dtype), dev)
    check(_lib.load().abcd_layer_norm_bwd(
        code, n, d, dy.data_ptr(), lddy, x.data_ptr(), ldx, _ptr(mean), _ptr(rstd),
        _DTYPES[wdtype], _ptr(weight), _ptr(add), ldadd, _ptr(dx), lddx, _ptr(dw), _ptr(db),
        _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream()))
    return grads


def _drop_args(p, seed, offset):
    p, seed, offset = float(p), int(seed), int(offset)
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"p must be in [0, 1], got {p}")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must be in [0, 2^64)")
    return p, seed, offset


def dropout(x, p, seed, offset=0, residual=None, out=None):
    """residual + dropout(x) for x [n, d] (any row stride): an element is kept
    with probability 1 - p and divided by it. The mask is a function of seed,
    offset and the element's row and column (see abcd_dropout) and is never
    stored; calls whose masks are to be independent differ in offset. out may be
    x or residual."""
    code = _dtype_of(x, "x")
    ldx = _rows(x, "x")
    size = x.shape
    p, seed, offset = _drop_args(p, seed, offset)
    ldr = 0 if residual is None else _rows(residual, "residual", x, size)
    if out is None:
        out, ldy = _new(x, size), size[1]
    else:
        ldy = _rows(out, "out", x, size)
    check(_lib.load().abcd_dropout(code, size[0], size[1], x.data_ptr(), ldx, _ptr(residual), ldr,
                                   out.data_ptr(), ldy, p, seed, offset, _stream()))
    return out


def dropout_bwd(dy, p, seed, offset=0, out=None):
    """Gradient of dropout's x: the forward's p, seed and offset make its mask
    again (the residual's gradient is dy itself)."""
    return dropout(dy, p, seed, offset, out=out)


_ACTS = {"silu": 0, "gelu": 1, "relu": 2}  # ABCD_ACT_*
FFN_WEIGHTS = ("w_gate", "w_up", "w_down")
FFN_BIASES = ("b_gate", "b_up", "b_down")
FFN_SAVED = ("by_gate", "by_up", "hidden")
_FFN_PARAMS = frozenset(FFN_WEIGHTS + FFN_BIASES)


def _ffn(x, params, act, p, seed, offset):
    """The block's description for the library, checked against x [n, d]."""
    code = _dtype_of(x, "x")
    ldx = _rows(x, "x")
    d, dtype, dev = x.shape[1], x.dtype, x.device
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}, got {act!r}")
    if not params.keys() <= _FFN_PARAMS:
        raise ValueError(f"unknown parameters {sorted(params.keys() - _FFN_PARAMS)}")
    get = params.get
    for k in FFN_WEIGHTS:
        t = get(k)
        if t is None:
            raise ValueError(f"{k} is required")
        if t.dim() != 2 or t.shape[0] == 0:
            raise ValueError(f"{k} must be a matrix with rows, got {tuple(t.shape)}")
    h, o = params["w_gate"].shape[0], params["w_down"].shape[0]
    ptrs = []
    for k, shape in (("w_gate", (h, d)), ("w_up", (h, d)), ("w_down", (o, h)),
                     ("b_gate", (h,)), ("b_up", (h,)), ("b_down", (o,))):
        t = get(k)
        if t is None:
            ptrs.append(None)
            continue
        if t.dtype != dtype or t.device != dev:
            raise ValueError(f"{k} must be {dtype} on {dev}, got {t.dtype} on {t.device}")
        if t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{k} must be contiguous with shape {shape}, got {tuple(t.shape)}")
        ptrs.append(t.data_ptr())
    p, seed, offset = _drop_args(p, seed, offset)
    return _lib.abcd_ffn(code, _ACTS[act], d, h, o, *ptrs, p, seed, offset), ldx


def _saved_ptrs(saved, n, h, like):
    """What a forward kept: h's derivatives by the pre-activations, and h."""
    if saved is None:
        return [None] * 3
    out = []
    for k in FFN_SAVED:
        t = saved[k]
        if t.dtype != like.dtype or t.device != like.device or not t.is_contiguous() \
                or tuple(t.shape) != (n, (h + 7) // 8 * 8):
            raise ValueError(f"saved[{k}] must be a contiguous {like.dtype} tensor of shape "
                             f"({n}, {(h + 7) // 8 * 8}) on {like.device}")
        out.append(t.data_ptr() if n > 0 else None)
    return out


def gated_ffn(x, params, act="silu", residual=None, p=0.0, seed=0, offset=0, save=False, out=None,
              workspace=None):
    """Gated feed-forward block of x [n, d] (float32, float16 or bfloat16; any
    row stride): residual + dropout(h w_down' + b_down) with
    h = act(x w_gate' + b_gate) * (x w_up' + b_up). params: dict(w_gate [h, d],
    w_up [h, d], w_down [o, h][, b_gate [h], b_up [h], b_down [o]]) of x's type.
    act: "silu", "gelu" or "relu". Dropout as in dropout(). h, and in the backward the
    gradients that reach it, are rounded to x's type between products: in float16
    they overflow beyond 65,504 and vanish below 2^-25.

    Returns dict(y [n, o], saved): with save=True what gated_ffn_bwd takes of
    this pass, else None; None too where the backward makes it again faster than
    it would read it (narrow blocks). out may be residual."""
    f, ldx = _ffn(x, params, act, p, seed, offset)
    n, dev = x.shape[0], x.device
    ldr = 0 if residual is None else _rows(residual, "residual", x, (n, f.o))
    if out is None:
        out, ldy = _new(x, (n, f.o)), f.o
    else:
        ldy = _rows(out, "out", x, (n, f.o))
    lib = _lib.load()
    saved = None
    if save:
        keeps = C.c_int32(0)
        check(lib.abcd_gated_ffn_keeps(C.byref(f), n, C.byref(keeps)))
        save = keeps.value != 0
    if save:
        hp = (f.h + 7) // 8 * 8
        kept = _new(x, (n, hp))
        saved = dict(zip(FFN_SAVED, (kept, torch.empty_like(kept), torch.empty_like(kept))))
    sz = C.c_size_t(0)
    check(lib.abcd_gated_ffn_workspace_size(C.byref(f), n, 1 if save else 0, C.byref(sz)))
    workspace = _workspace(workspace, sz.value, dev)
    check(lib.abcd_gated_ffn(C.byref(f), n, x.data_ptr(), ldx, _ptr(residual), ldr, out.data_ptr(),
                             ldy, *_saved_ptrs(saved, n, f.h, x), workspace.data_ptr(),
                             workspace.numel(), _stream()))
    return dict(y=out, saved=saved)


def gated_ffn_bwd(dy, x, params, act="silu", saved=None, p=0.0, seed=0, offset=0, grads=None,
                  workspace=None):
    """Gradients of gated_ffn for dy [n, o]: dict(x, w_gate, w_up, w_down[, and
    the biases that params has]); the residual's is dy itself. saved: the
    forward's, or None to compute it again. p, seed and offset are the forward's.
    grads: a dict of tensors to write into, where a missing one is left out; none may
    overlap an input."""
    f, ldx = _ffn(x, params, act, p, seed, offset)
    n, d = x.shape
    dev = x.device
    lddy = _rows(dy, "dy", x, (n, f.o))
    if grads is None:  # laid out as the parameters, which _ffn has checked
        grads = {k: torch.empty_like(params[k]) for k in FFN_WEIGHTS + FFN_BIASES
                 if params.get(k) is not None}
        dx, lddx = _new(x, (n, d)), d
        grads["x"] = dx
    else:
        for k, shape in (("w_gate", (f.h, d)), ("w_up", (f.h, d)), ("w_down", (f.o, f.h)),
                         ("b_gate", (f.h,)), ("b_up", (f.h,)), ("b_down", (f.o,))):
            t = grads.get(k)
            if t is not None and (t.dtype != x.dtype or t.device != dev or t.shape != shape
                                  or not t.is_contiguous()):
                raise ValueError(f"grads[{k}] must be contiguous {x.dtype} on {dev} with shape {shape}")
        dx = grads.get("x")
        lddx = 0 if dx is None else _rows(dx, "grads[x]", x, (n, d))
    lib = _lib.load()
    sz = C.c_size_t(0)
    check(lib.abcd_gated_ffn_bwd_workspace_size(C.byref(f), n, 0 if saved is None else 1,
                                                C.byref(sz)))
    workspace = _workspace(workspace, sz.value, dev)
    check(lib.abcd_gated_ffn_bwd(
        C.byref(f), n, dy.data_ptr(), lddy, x.data_ptr(), ldx, *_saved_ptrs(saved, n, f.h, x),
        _ptr(dx), lddx, *[_ptr(grads.get(k)) for k in FFN_WEIGHTS + FFN_BIASES],
        workspace.data_ptr(), workspace.numel(), _stream()))
    return grads


# ---------------------------------------------------------------- collapse

def composite_cache(images, order, n_front, F=None, B=None, accumulate=False, rects=None,
                    stop_t=0.0, beside=False):
    """Collapse cached fp16 renders [K, H, W, 4] (torch.float16, or int16
    holding binary16 bits) into F and B (fp32 [H, W, 4]). rects: optional
    int32 [K, 4] GPU tensor of per-image coverage boxes (x0, y0, x1, y1);
    stop_t > 0 skips layers that can no longer be seen. beside: at most two
    workgroups per CU, for a collapse that runs beside other work on another
    stream (slower alone)."""
    if images.dtype not in (torch.float16, torch.int16):
        raise ValueError("images must be float16 (or int16 bit patterns)")
    if not images.is_cuda or not images.is_contiguous() or images.dim() != 4:
        raise ValueError("images must be a contiguous GPU tensor [K, H, W, 4]")
    k, H, W, c = images.shape
    if c != 4:
        raise ValueError("images must be RGBA")
    dev = images.device
    if F is None:
        F = _empty((H, W, 4), torch.float32, dev)
    if B is None:
        B = _empty((H, W, 4), torch.float32, dev)
    _need(F, "F", torch.float32, (H, W, 4))
    _need(B, "B", torch.float32, (H, W, 4))
    _opt(rects, "rects", torch.int32, (k, 4))
    order_arr = (C.c_int32 * max(k, 1))(*[int(x) for x in order])
    check(_lib.load().abcd_composite_cache(W, H, k, _ptr(images), order_arr, int(n_front),
                                           _ptr(rects), float(stop_t), _ptr(F), _ptr(B),
                                           (1 if accumulate else 0) | (2 if beside else 0),
                                           _stream()))
    return F, B


def stage_cached(host_images, dst, rects=None):
    """Copy pinned host fp16 images (a list of [H, W, 4] tensors) into the
    device chunk dst [>= k, H, W, 4], only inside each image's coverage box
    (rects: host int32 array [k, 4], or None for whole images), on the
    current stream."""
    k = len(host_images)
    if k == 0:
        return dst
    H, W = dst.shape[1], dst.shape[2]
    if dst.dtype not in (torch.float16, torch.int16) or not dst.is_cuda or \
            not dst.is_contiguous() or dst.shape[0] < k or dst.shape[3] != 4:
        raise ValueError("dst must be a contiguous fp16 GPU tensor [>= k, H, W, 4]")
    for h in host_images:
        if h.is_cuda or not h.is_pinned() or h.dtype not in (torch.float16, torch.int16) or \
                tuple(h.shape) != (H, W, 4) or not h.is_contiguous():
            raise ValueError("host images must be pinned contiguous fp16 [H, W, 4] tensors")
    ptrs = (C.c_void_p * k)(*[h.data_ptr() for h in host_images])
    r = None
    if rects is not None:
        import numpy as np
        ra = np.ascontiguousarray(np.asarray(rects, dtype=np.int32).reshape(-1, 4)[:k])
        r = ra.ctypes.data_as(C.POINTER(C.c_int32))
    check(_lib.load().abcd_stage_cached(W, H, k, ptrs, r, _ptr(dst), _stream()))
    return dst


def loss_l1_grad(out, target, bg=None, dL_dout=None, loss=None):
    H, W = out.shape[:2]
    _need(out, "out", torch.float32, (H, W, 4))
    _need(target, "target", torch.float32, (H, W, 3))
    _opt(loss, "loss", torch.float32, (1,))
    if dL_dout is None:
        dL_dout = torch.empty_like(out)
    bg_arr = None if bg is None else (C.c_float * 3)(*[float(x) for x in bg])
    check(_lib.load().abcd_loss_l1_grad(W, H, _ptr(out), _ptr(target), bg_arr, _ptr(dL_dout),
                                        _ptr(loss), _stream()))
    return dL_dout


# ------------------------------------------------------------------ timing

def timing_enable(flag=True):
    check(_lib.load().abcd_timing_enable(1 if flag else 0))


def timing_reset():
    check(_lib.load().abcd_timing_reset())


def timing_read(kernel):
    ms = C.c_double(0)
    cnt = C.c_int64(0)
    check(_lib.load().abcd_timing_read(kernel.encode(), C.byref(ms), C.byref(cnt)))
    return ms.value, cnt.value


__all__ = ["AbcdError", "project", "bin_sort", "bin_sort_workspace_size", "render_fwd",
           "render_bwd", "render_bwd_workspace_size", "composite_cache", "loss_l1_grad",
           "timing_enable", "timing_reset", "timing_read", "version", "n_tiles", "adam_step",
           "render_cache", "stage_cached", "make_split", "split_workspace_size", "intersections",
           "render_bwd_noalloc", "layer_norm", "layer_norm_bwd", "layer_norm_bwd_workspace_size",
           "dropout", "dropout_bwd", "gated_ffn", "gated_ffn_bwd"]
