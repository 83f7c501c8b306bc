"""Operators of a network's hidden layers on torch tensors: a layer's product with bias, activation and
residual, group normalisation (channels last) with an activation, dropout whose mask is a function of a
counter, and their gradients (abs_linear_*, abs_group_norm_*, abs_dropout_* in include/abs.h).

Tensors are on one GPU; a matrix is the last dimension times the others flattened, its rows a common
distance apart (a slice of columns is fine, a transposed or expanded view is refused).  Operands are all
float32 or all bfloat16; biases, gamma, beta, saved statistics and their gradients are float32.  The
work goes to torch's current stream of the tensors' device; outputs and workspaces come from torch's
allocator on that stream, so calls can be captured into a graph.  Nothing here records gradients: a
backward pass is a call of its own.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import AbsError, AbsLinear, AbsGroupNorm, AbsDropout, _lib, _check

ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3
ABS_E_ARG = -1
_DTYPE = {torch.float32: 0, torch.bfloat16: 1}


def _bad(text: str):
    raise AbsError(ABS_E_ARG, text)


def _dtype(t: torch.Tensor, what: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _bad(f"{what} must be a tensor on a GPU")
    if t.dtype not in _DTYPE:
        _bad(f"{what} must be float32 or bfloat16, not {t.dtype}")
    return _DTYPE[t.dtype]


def _whole(v, lo: int, hi: int, what: str) -> int:
    """v as a whole number in [lo, hi] (a C struct would cut it to its field)."""
    if isinstance(v, bool) or not isinstance(v, int) or not lo <= v <= hi:
        _bad(f"{what} must be a whole number in [{lo}, {hi}]")
    return v


def _pitch(t: torch.Tensor, what: str, shape, like: torch.Tensor) -> int:
    """Elements between the rows of t, whose last dimension is a row; the rows a common distance apart."""
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dtype != like.dtype:
        _bad(f"{what} must be a tensor of x's device and dtype")
    if tuple(t.shape) != tuple(shape):
        _bad(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    cols = t.shape[-1]
    if t.is_contiguous():
        return cols
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


def _vector(t, what: str, shape, like: torch.Tensor):
    """Address of a dense float32 tensor (None: 0)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dtype != torch.float32:
        _bad(f"{what} must be a float32 tensor on x's device")
    if tuple(t.shape) != tuple(shape):
        _bad(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        _bad(f"{what} must be contiguous")
    return t.data_ptr()


def _ptr(t):
    return None if t is None else t.data_ptr()


class _on:
    """The tensors' device made current, where it is not, for a launch."""

    def __init__(self, t):
        self.index = t.device.index
        self.back = None

    def __enter__(self):
        now = torch.cuda.current_device()
        if now != self.index:
            self.back = now
            torch.cuda.set_device(self.index)

    def __exit__(self, *exc):
        if self.back is not None:
            torch.cuda.set_device(self.back)


def _stream(t):
    return torch.cuda.current_stream(t.device).cuda_stream


def _workspace(n: int, like: torch.Tensor):
    """(tensor that holds the bytes, 256-byte aligned address)."""
    if n == 0:
        return None, None
    ws = torch.empty(n + 256, dtype=torch.uint8, device=like.device)
    return ws, (ws.data_ptr() + 255) // 256 * 256


def _out(out, shape, like):
    if out is None:
        return torch.empty(shape, dtype=like.dtype, device=like.device)
    return out


def linear_forward(x, w, b=None, *, act=ACT_NONE, residual=None, keep_z=False, out=None):
    """y = act(x w + b) + residual; with keep_z (y, z), z = x w + b for the backward pass.
    x [..., d_in], w [d_in, d_out], b float32 [d_out]; residual, out (may be residual) [..., d_out]."""
    p = AbsLinear(dtype=_dtype(x, "x"), act=_whole(act, 0, 3, "act"))
    if x.dim() < 1 or not isinstance(w, torch.Tensor) or w.dim() != 2 or w.shape[0] != x.shape[-1]:
        _bad("linear: w must be [d_in, d_out] and x [..., d_in]")
    d_in, d_out = w.shape
    shape = tuple(x.shape[:-1]) + (d_out,)
    p.rows, p.d_in, p.d_out = (x.numel() // d_in if d_in else 0), d_in, d_out
    p.ldx, p.ldw = _pitch(x, "x", x.shape, x), _pitch(w, "w", (d_in, d_out), x)
    bias = _vector(b, "b", (d_out,), x)
    if residual is not None:
        p.ldr = _pitch(residual, "residual", shape, x)
    y = _out(out, shape, x)
    p.ldy = _pitch(y, "out", shape, x)
    z = torch.empty(shape, dtype=x.dtype, device=x.device) if keep_z else None
    p.ldz = d_out
    xp, wp = x.data_ptr(), w.data_ptr()
    with _on(x):
        n = _lib.abs_linear_workspace_size(C.byref(p), 0, int((xp | wp) % 16 == 0))
        ws, at = _workspace(n, x)
        _check(_lib.abs_linear_forward(C.byref(p), xp, wp, bias, _ptr(residual), y.data_ptr(), _ptr(z), at, n, _stream(x)))
    return (y, z) if keep_z else y


def linear_backward(x, w, dy, *, act=ACT_NONE, z=None, need_dx=True, need_dw=True, need_db=True):
    """(dx, dw, db) for a gradient dy of linear_forward's y; z as it returned it (not needed without an
    activation).  What is not needed comes back as None.  The residual's gradient is dy."""
    p = AbsLinear(dtype=_dtype(x, "x"), act=_whole(act, 0, 3, "act"))
    if x.dim() < 1 or not isinstance(w, torch.Tensor) or w.dim() != 2 or w.shape[0] != x.shape[-1]:
        _bad("linear: w must be [d_in, d_out] and x [..., d_in]")
    d_in, d_out = w.shape
    shape = tuple(x.shape[:-1]) + (d_out,)
    p.rows, p.d_in, p.d_out = (x.numel() // d_in if d_in else 0), d_in, d_out
    p.ldx, p.ldw = _pitch(x, "x", x.shape, x), _pitch(w, "w", (d_in, d_out), x)
    p.lddy = _pitch(dy, "dy", shape, x)
    if act != ACT_NONE:
        if z is None:
            _bad("linear: the backward pass of an activation needs z")
        p.ldz = _pitch(z, "z", shape, x)
    else:
        z = None
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need_dx else None
    dw = torch.empty((d_in, d_out), dtype=x.dtype, device=x.device) if need_dw else None
    db = torch.empty(d_out, dtype=torch.float32, device=x.device) if need_db else None
    p.lddx, p.lddw = d_in, d_out
    xp, wp, dp = x.data_ptr(), w.data_ptr(), dy.data_ptr()
    with _on(x):
        n = _lib.abs_linear_workspace_size(C.byref(p), 1, int((xp | wp | dp) % 16 == 0))
        ws, at = _workspace(n, x)
        _check(_lib.abs_linear_backward(C.byref(p), xp, wp, _ptr(z), dp, _ptr(dx), _ptr(dw), _ptr(db), at, n, _stream(x)))
    return dx, dw, db


def _norm_params(x, gamma, beta, groups, eps, act):
    p = AbsGroupNorm(dtype=_dtype(x, "x"), act=_whole(act, 0, 3, "act"), groups=_whole(groups, 0, 1 << 20, "groups"), eps=eps)
    if x.dim() < 2:
        _bad("group norm: x must be [n, ..., channels]")
    p.n, p.channels = x.shape[0], x.shape[-1]
    p.spatial = 1
    for d in x.shape[1:-1]:
        p.spatial *= d
    p.ldx = _pitch(x, "x", x.shape, x)
    if (gamma is None) != (beta is None):
        _bad("group norm: gamma and beta come together")
    return p, _vector(gamma, "gamma", (p.channels,), x), _vector(beta, "beta", (p.channels,), x)


def group_norm_forward(x, gamma, beta, groups, *, eps=1e-5, act=ACT_NONE, out=None):
    """(y, mean, rstd): y = act((x - mean) rstd gamma + beta), mean and rstd per sample and group, float32
    [n, groups].  x [n, ..., channels]; gamma, beta float32 [channels] or both None; out may be x."""
    p, gp, bp = _norm_params(x, gamma, beta, groups, eps, act)
    y = _out(out, x.shape, x)
    p.ldy = _pitch(y, "out", x.shape, x)
    mean = torch.empty((p.n, groups), dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    with _on(x):
        n = _lib.abs_group_norm_workspace_size(C.byref(p), 0)
        ws, at = _workspace(n, x)
        _check(_lib.abs_group_norm_forward(C.byref(p), x.data_ptr(), gp, bp, y.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                           at, n, _stream(x)))
    return y, mean, rstd


def group_norm_backward(x, gamma, beta, mean, rstd, dy, *, act=ACT_NONE, residual=None, need_dgamma=True, out=None):
    """(dx, dgamma, dbeta) for a gradient dy of group_norm_forward's y, with the mean and rstd it returned;
    `residual`: a gradient that reaches x past the normalised branch, added to dx; out (may be residual): dx."""
    if not isinstance(mean, torch.Tensor) or mean.dim() != 2:
        _bad("group norm: mean must be float32 [n, groups]")
    p, gp, bp = _norm_params(x, gamma, beta, mean.shape[1], 0.0, act)
    saved = (x.shape[0], mean.shape[1])
    mp, rp = _vector(mean, "mean", saved, x), _vector(rstd, "rstd", saved, x)
    if rp is None:
        _bad("group norm: rstd must be float32 [n, groups]")
    p.lddy = _pitch(dy, "dy", x.shape, x)
    if residual is not None:
        p.lddres = _pitch(residual, "residual", x.shape, x)
    dx = _out(out, x.shape, x)
    p.lddx = _pitch(dx, "out", x.shape, x)
    dgamma = dbeta = None
    if need_dgamma:
        dgamma = torch.empty(p.channels, dtype=torch.float32, device=x.device)
        dbeta = torch.empty_like(dgamma)
    with _on(x):
        n = _lib.abs_group_norm_workspace_size(C.byref(p), 1)
        ws, at = _workspace(n, x)
        _check(_lib.abs_group_norm_backward(C.byref(p), x.data_ptr(), gp, bp, mp, rp, dy.data_ptr(), _ptr(residual),
                                            dx.data_ptr(), _ptr(dgamma), _ptr(dbeta), at, n, _stream(x)))
    return dx, dgamma, dbeta


def _dropout_params(x, drop, seed, offset):
    p = AbsDropout(dtype=_dtype(x, "x"), drop=_whole(drop, 0, 65535, "drop"))
    if x.dim() < 1:
        _bad("dropout: x must be [..., cols]")
    p.seed, p.offset = seed & (2 ** 64 - 1), offset & (2 ** 64 - 1)
    p.cols = x.shape[-1]
    p.rows = x.numel() // p.cols if p.cols else 0
    p.ldx = _pitch(x, "x", x.shape, x)
    return p


def dropout_forward(x, drop, seed, offset, *, residual=None, out=None):
    """y = (kept ? x 65536 / (65536 - drop) : 0) + residual.  drop: the probability in 65536ths, in
    [0, 65535]; which elements stay depends on seed, offset and the element's row-major index alone.
    out may be x or residual."""
    p = _dropout_params(x, drop, seed, offset)
    if residual is not None:
        p.ldr = _pitch(residual, "residual", x.shape, x)
    y = _out(out, x.shape, x)
    p.ldy = _pitch(y, "out", x.shape, x)
    with _on(x):
        _check(_lib.abs_dropout_forward(C.byref(p), x.data_ptr(), _ptr(residual), y.data_ptr(), _stream(x)))
    return y


def dropout_backward(dy, drop, seed, offset, *, out=None):
    """dx for a gradient dy of dropout_forward's y (the residual's gradient is dy); out may be dy."""
    p = _dropout_params(dy, drop, seed, offset)
    dx = _out(out, dy.shape, dy)
    p.ldy = _pitch(dx, "out", dy.shape, dy)
    with _on(dy):
        _check(_lib.abs_dropout_backward(C.byref(p), dy.data_ptr(), dx.data_ptr(), _stream(dy)))
    return dx


def dropout_kept(rows, cols, drop, seed, offset):
    """The mask of a rows x cols matrix as the library draws it, on the host: uint8 [rows, cols], 1 = stays."""
    p = AbsDropout(dtype=0, drop=_whole(drop, 0, 65535, "drop"), rows=rows, cols=cols, seed=seed & (2 ** 64 - 1), offset=offset & (2 ** 64 - 1))
    kept = torch.empty((rows, cols), dtype=torch.uint8)
    _check(_lib.abs_dropout_kept(C.byref(p), 0, rows * cols, kept.data_ptr()))
    return kept
