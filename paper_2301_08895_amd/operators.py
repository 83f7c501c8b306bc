"""Operators of a network's hidden layers on torch tensors: a layer's product with bias, activation and
residual, group normalisation (channels last) with an activation, dropout whose mask is a function of a
counter, and their gradients (abs_linear_*, abs_group_norm_*, abs_dropout_* in include/abs.h).

Tensors are on one GPU; a matrix is the last dimension times the others flattened, its rows a common
distance apart (a slice of columns is fine, a transposed or expanded view is refused).  Operands are all
float32 or all bfloat16; biases, gamma, beta, saved statistics and their gradients are float32.  The
work goes to torch's current stream of the tensors' device; outputs and workspaces come from torch's
allocator on that stream, so calls can be captured into a graph.  Nothing here records gradients, also
where a tensor requires one (what comes back is cut off from its graph): a backward pass is a call of
its own.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import AbsError, AbsLinear, AbsGroupNorm, AbsDropout, _lib, _check

ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3
ABS_E_ARG = -1
_DTYPE = {torch.float32: 0, torch.bfloat16: 1}
_byref = C.byref

# A small call is bound by its host part, so the tensors' checks are few and flat, and the current stream and device are
# asked for as numbers (torch.cuda.current_stream builds an object: 1.9 us of a call's 11).
_empty, _empty_like = torch.empty, torch.empty_like
_stream_of = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _bad(text: str):
    raise AbsError(ABS_E_ARG, text)


def _first(t, what: str, least_dim: int):
    """(dtype code, device number) of the tensor that the others are held against."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _bad(f"{what} must be a tensor on a GPU")
    code = _DTYPE.get(t.dtype)
    if code is None:
        _bad(f"{what} must be float32 or bfloat16, not {t.dtype}")
    if t.dim() < least_dim:
        _bad(f"{what} needs {least_dim} dimensions at least")
    return code, t.get_device()


def _whole(v, lo: int, hi: int, what: str) -> int:
    """v as a whole number in [lo, hi] (a C struct would cut it to its field)."""
    if type(v) is not int or not lo <= v <= hi:
        _bad(f"{what} must be a whole number in [{lo}, {hi}]")
    return v


def _pitch(t, what: str, shape, dtype, dev: int) -> int:
    """Elements between the rows of t, whose last dimension is a row; the rows a common distance apart."""
    if not isinstance(t, torch.Tensor) or t.get_device() != dev or t.dtype != dtype:
        _bad(f"{what} must be a tensor of x's device and dtype")
    if t.shape != shape:
        _bad(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.is_contiguous():
        return shape[-1]
    cols = shape[-1]
    stride = t.stride()
    if cols > 1 and stride[-1] != 1:
        _bad(f"{what}: the elements of a row must be neighbours")
    pitch, rows = None, 1
    for d in range(t.dim() - 2, -1, -1):
        if t.shape[d] == 1:
            continue
        if pitch is None:
            pitch = stride[d]
        elif stride[d] != pitch * rows:
            _bad(f"{what}: rows must be a common distance apart")
        rows *= t.shape[d]
    if pitch is None or t.numel() == 0:
        return cols
    if pitch < cols:
        _bad(f"{what}: rows overlap")
    return pitch


def _vector(t, what: str, shape, dev: int):
    """Address of a dense float32 tensor (None: None)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.get_device() != dev or t.dtype != torch.float32:
        _bad(f"{what} must be a float32 tensor on x's device")
    if t.shape != shape:
        _bad(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        _bad(f"{what} must be contiguous")
    return t.data_ptr()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _like(x, shape):
    """A dense tensor of that shape, of x's dtype and device."""
    return _empty_like(x) if x.is_contiguous() and x.shape == shape else x.new_empty(shape)


def _workspace(n: int, device):
    """(tensor that holds the bytes, 256-byte aligned address)."""
    if n == 0:
        return None, None
    ws = _empty(n + 256, dtype=torch.uint8, device=device)
    return ws, (ws.data_ptr() + 255) // 256 * 256


def _run(dev: int, fn, *args):
    """fn(*args, stream) with the tensors' device current (the library launches on the current one)."""
    if _current_device() == dev:
        _check(fn(*args, _stream_of(dev)))
    else:
        with torch.cuda.device(dev):
            _check(fn(*args, _stream_of(dev)))


def _layer(x, w, act):
    """What both passes of a layer say about x and w: (struct, device, d_in, d_out, shape of y)."""
    code, dev = _first(x, "x", 1)
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        _bad("linear: w must be [d_in, d_out] and x [..., d_in]")
    xs, ws = x.shape, w.shape
    d_in, d_out = ws
    if xs[-1] != d_in:
        _bad("linear: w must be [d_in, d_out] and x [..., d_in]")
    if not 1 <= d_in <= 1 << 20 or not 1 <= d_out <= 1 << 20:
        _bad("linear: d_in and d_out must be in [1, 2^20]")
    shape = (xs[0], d_out) if len(xs) == 2 else tuple(xs[:-1]) + (d_out,)
    return AbsLinear(code, _whole(act, 0, 3, "act"), x.numel() // d_in, d_in, d_out, _pitch(x, "x", xs, x.dtype, dev),
                     _pitch(w, "w", ws, x.dtype, dev)), dev, d_in, d_out, shape


def linear_forward(x, w, b=None, *, act=ACT_NONE, residual=None, keep_z=False, out=None):
    """y = act(x w + b) + residual; with keep_z (y, z), z = x w + b for the backward pass.
    x [..., d_in], w [d_in, d_out], b float32 [d_out]; residual, out (may be residual) [..., d_out]."""
    p, dev, d_in, d_out, shape = _layer(x, w, act)
    bias = _vector(b, "b", (d_out,), dev)
    if residual is not None:
        p.ldr = _pitch(residual, "residual", shape, x.dtype, dev)
    if out is None:
        y, p.ldy = _like(x, shape), d_out
    else:
        y, p.ldy = out, _pitch(out, "out", shape, x.dtype, dev)
    z = _like(x, shape) if keep_z else None
    p.ldz = d_out
    xp, wp, ref = x.data_ptr(), w.data_ptr(), _byref(p)
    n = _lib.abs_linear_workspace_size(ref, 0, (xp | wp) & 15 == 0)
    ws, at = _workspace(n, x.device)
    _run(dev, _lib.abs_linear_forward, ref, xp, wp, bias, _ptr(residual), y.data_ptr(), _ptr(z), at, n)
    return (y, z) if keep_z else y


def linear_backward(x, w, dy, *, act=ACT_NONE, z=None, need_dx=True, need_dw=True, need_db=True):
    """(dx, dw, db) for a gradient dy of linear_forward's y; z as it returned it (not needed without an
    activation).  What is not needed comes back as None.  The residual's gradient is dy."""
    p, dev, d_in, d_out, shape = _layer(x, w, act)
    p.lddy = _pitch(dy, "dy", shape, x.dtype, dev)
    if act == ACT_NONE:
        z = None
    elif z is None:
        _bad("linear: the backward pass of an activation needs z")
    else:
        p.ldz = _pitch(z, "z", shape, x.dtype, dev)
    dx = _like(x, x.shape) if need_dx else None
    dw = _like(w, w.shape) if need_dw else None
    db = _empty((d_out,), dtype=torch.float32, device=x.device) if need_db else None
    p.lddx, p.lddw = d_in, d_out
    xp, wp, dp, ref = x.data_ptr(), w.data_ptr(), dy.data_ptr(), _byref(p)
    n = _lib.abs_linear_workspace_size(ref, 1, (xp | wp | dp) & 15 == 0)
    ws, at = _workspace(n, x.device)
    _run(dev, _lib.abs_linear_backward, ref, xp, wp, _ptr(z), dp, _ptr(dx), _ptr(dw), _ptr(db), at, n)
    return dx, dw, db


def _normed(x, gamma, beta, groups, eps, act):
    """What both passes of a normalisation say: (struct, device, gamma's and beta's address)."""
    code, dev = _first(x, "x", 2)
    shape = x.shape
    n, channels = shape[0], _whole(shape[-1], 1, 1 << 20, "channels")
    spatial = shape[1] if len(shape) == 3 else 1
    if len(shape) > 3:
        for d in shape[1:-1]:
            spatial *= d
    if (gamma is None) != (beta is None):
        _bad("group norm: gamma and beta come together")
    p = AbsGroupNorm(code, _whole(act, 0, 3, "act"), n, spatial, channels, _whole(groups, 0, 1 << 20, "groups"), eps, 0,
                     _pitch(x, "x", shape, x.dtype, dev))
    return p, dev, _vector(gamma, "gamma", (channels,), dev), _vector(beta, "beta", (channels,), dev)


def group_norm_forward(x, gamma, beta, groups, *, eps=1e-5, act=ACT_NONE, out=None):
    """(y, mean, rstd): y = act((x - mean) rstd gamma + beta), mean and rstd per sample and group, float32
    [n, groups].  x [n, ..., channels]; gamma, beta float32 [channels] or both None; out may be x."""
    p, dev, gp, bp = _normed(x, gamma, beta, groups, eps, act)
    if out is None:
        y, p.ldy = _like(x, x.shape), p.channels
    else:
        y, p.ldy = out, _pitch(out, "out", x.shape, x.dtype, dev)
    ref = _byref(p)
    n = _lib.abs_group_norm_workspace_size(ref, 0)
    ws, at = _workspace(n, x.device)
    mean = _empty((p.n, groups), dtype=torch.float32, device=x.device)
    rstd = _empty_like(mean)
    _run(dev, _lib.abs_group_norm_forward, ref, x.data_ptr(), gp, bp, y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), at, n)
    return y, mean, rstd


def group_norm_backward(x, gamma, beta, mean, rstd, dy, *, act=ACT_NONE, residual=None, need_dgamma=True, out=None):
    """(dx, dgamma, dbeta) for a gradient dy of group_norm_forward's y, with the mean and rstd it returned;
    `residual`: a gradient that reaches x past the normalised branch, added to dx; out (may be residual): dx."""
    if not isinstance(mean, torch.Tensor) or mean.dim() != 2 or rstd is None:
        _bad("group norm: mean and rstd must be float32 [n, groups]")
    p, dev, gp, bp = _normed(x, gamma, beta, mean.shape[1], 0.0, act)
    saved = (p.n, p.groups)
    mp, rp = _vector(mean, "mean", saved, dev), _vector(rstd, "rstd", saved, dev)
    p.lddy = _pitch(dy, "dy", x.shape, x.dtype, dev)
    if residual is not None:
        p.lddres = _pitch(residual, "residual", x.shape, x.dtype, dev)
    if out is None:
        dx, p.lddx = _like(x, x.shape), p.channels
    else:
        dx, p.lddx = out, _pitch(out, "out", x.shape, x.dtype, dev)
    dgamma = dbeta = None
    if need_dgamma:
        dgamma = _empty_like(gamma) if gamma is not None else _empty((p.channels,), dtype=torch.float32, device=x.device)
        dbeta = _empty_like(dgamma)
    ref = _byref(p)
    n = _lib.abs_group_norm_workspace_size(ref, 1)
    ws, at = _workspace(n, x.device)
    _run(dev, _lib.abs_group_norm_backward, ref, x.data_ptr(), gp, bp, mp, rp, dy.data_ptr(), _ptr(residual), dx.data_ptr(),
         _ptr(dgamma), _ptr(dbeta), at, n)
    return dx, dgamma, dbeta


_WORD = 2 ** 64 - 1


def _dropped(x, drop, seed, offset):
    code, dev = _first(x, "x", 1)
    shape = x.shape
    cols = shape[-1]
    if cols < 1:
        _bad("dropout: x must be [..., cols]")
    pitch = _pitch(x, "x", shape, x.dtype, dev)
    return AbsDropout(code, _whole(drop, 0, 65535, "drop"), x.numel() // cols, cols, pitch, cols, cols, seed & _WORD, offset & _WORD), dev


def dropout_forward(x, drop, seed, offset, *, residual=None, out=None):
    """y = (kept ? x 65536 / (65536 - drop) : 0) + residual.  drop: the probability in 65536ths, in
    [0, 65535]; which elements stay depends on seed, offset and the element's row-major index alone.
    out may be x or residual."""
    p, dev = _dropped(x, drop, seed, offset)
    rp = None
    if residual is not None:
        p.ldr, rp = _pitch(residual, "residual", x.shape, x.dtype, dev), residual.data_ptr()
    if out is None:
        out = _like(x, x.shape)
    else:
        p.ldy = _pitch(out, "out", x.shape, x.dtype, dev)
    _run(dev, _lib.abs_dropout_forward, _byref(p), x.data_ptr(), rp, out.data_ptr())
    return out


def dropout_backward(dy, drop, seed, offset, *, out=None):
    """dx for a gradient dy of dropout_forward's y (the residual's gradient is dy); out may be dy."""
    p, dev = _dropped(dy, drop, seed, offset)
    if out is None:
        out = _like(dy, dy.shape)
    else:
        p.ldy = _pitch(out, "out", dy.shape, dy.dtype, dev)
    _run(dev, _lib.abs_dropout_backward, _byref(p), dy.data_ptr(), out.data_ptr())
    return out


def dropout_kept(rows, cols, drop, seed, offset):
    """The mask of a rows x cols matrix as the library draws it, on the host: uint8 [rows, cols], 1 = stays."""
    p = AbsDropout(dtype=0, drop=_whole(drop, 0, 65535, "drop"), rows=rows, cols=cols, seed=seed & _WORD, offset=offset & _WORD)
    kept = _empty((rows, cols), dtype=torch.uint8)
    _check(_lib.abs_dropout_kept(C.byref(p), 0, rows * cols, kept.data_ptr()))
    return kept
