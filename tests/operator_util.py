"""Plain 64-bit forms of the operators of a network's hidden layers, and how far a result may be from them.

u = 2^-24 is half a step of fp32, eps / 2 half a step of the output's dtype (bf16 2^-8, fp32 2^-24).  A sum of K
products in fp32 is off by at most (K + 2) u times the sum of their sizes; the matrix instructions may round their
partial sums down instead of to the nearest, which doubles it.
"""
import math

import torch

U = 2.0 ** -24
NONE, RELU, SILU, GELU = 0, 1, 2, 3


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def act(z, a):
    if a == RELU:
        return torch.where(z < 0, torch.zeros_like(z), z)
    if a == SILU:
        return z * torch.sigmoid(z)
    if a == GELU:
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z


def slope(z, a):
    if a == RELU:
        return (z > 0).to(z.dtype)
    if a == SILU:
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    if a == GELU:
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def close(got, want, slack, what=""):
    """Every element of got within half a step of its dtype, and `slack` (a tensor or number, for what happened in fp32
    before that rounding), of want; infinities and NaN where want has them."""
    got64 = got.double().cpu()
    want = want.double().cpu()
    slack = slack.double().cpu() if isinstance(slack, torch.Tensor) else slack
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got64), torch.isnan(want)), what
    assert torch.equal(got64[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    # (bf16's and fp32's least normal number: below it a step no longer shrinks)
    tol = (slack + half_step(got.dtype) * (want.abs() + slack) + 2.0 ** -126) * torch.ones_like(want)
    off = (got64 - want).abs() - tol
    worst = off[fine].max().item() if fine.any() else -1.0
    assert worst <= 0, f"{what}: beyond its tolerance by {worst:.3g} (tolerance there {tol[fine][off[fine].argmax()].item():.3g})"


def linear(x, w, b, a, r):
    """(y, z, slack of y, slack of z)."""
    x, w = x.double(), w.double()
    z = x @ w
    size = x.abs() @ w.abs()
    if b is not None:
        z, size = z + b.double(), size + b.double().abs()
    slack = 2 * (x.shape[-1] + 4) * U * size
    y = act(z, a)
    # an activation's slope is at most 1.13; its own evaluation: a few roundings of numbers up to |z| + 1
    sy = 1.13 * slack + (16 * U * (z.abs() + 1) if a in (SILU, GELU) else 0)
    if r is not None:
        y, sy = y + r.double(), sy + U * (y.abs() + r.double().abs())
    return y, z, sy, slack


def linear_gradient(x, w, z, dy, a):
    """(dx, dw, db) and their slacks; dz is rounded once to the operands' dtype."""
    dt = x.dtype
    x, w, dy = x.double(), w.double(), dy.double()
    s = slope(z.double(), a) if a != NONE else torch.ones_like(dy)
    dz = dy * s
    # slopes are evaluated with a few roundings of numbers up to 1 + |z|
    raw = U * dy.abs() * (24 * (1 + z.double().abs()) if a in (SILU, GELU) else 2)
    off = raw + (half_step(dt) * dz.abs() if a != NONE else 0)
    dx, dw, db = dz @ w.t().contiguous(), x.t().contiguous() @ dz, dz.sum(0)
    rows, d_out = dz.shape
    sx = off @ w.abs().t().contiguous() + 2 * (d_out + 4) * U * (dz.abs() @ w.abs().t().contiguous())
    sw = x.abs().t().contiguous() @ off + 2 * (rows + 4) * U * (x.abs().t().contiguous() @ dz.abs())
    sb = raw.sum(0) + (rows + 4) * U * dz.abs().sum(0)
    return (dx, dw, db), (sx, sw, sb)


def norm(x, gamma, beta, groups, eps, a):
    """y, mean, rstd with their slacks.  x [n, spatial, channels]."""
    n, S, C = x.shape
    v = x.double().reshape(n, S, groups, C // groups)
    m = S * (C // groups)
    mean = v.mean(dim=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(dim=(1, 3))
    rstd = 1 / torch.sqrt(var + eps)
    depth = min(m, 128) + 40                      # additions in a row: a lane's own values, then trees and parts
    s_mean = depth * U * v.abs().mean(dim=(1, 3))
    # a mean that is off by d adds d^2 to the variance, and each difference is rounded once
    s_var = (depth + 4) * U * var + s_mean ** 2 + 2 * U * s_mean * torch.sqrt(var)
    s_rstd = rstd * (s_var / (2 * (var + eps)) + 4 * U)
    g = gamma.double() if gamma is not None else torch.ones(C, dtype=torch.float64, device=x.device)
    b = beta.double() if beta is not None else torch.zeros(C, dtype=torch.float64, device=x.device)
    d = v - mean[:, None, :, None]
    xh = d * rstd[:, None, :, None]
    s_xh = (s_mean[:, None, :, None] + U * d.abs()) * rstd[:, None, :, None] + d.abs() * s_rstd[:, None, :, None] + U * xh.abs()
    xh, s_xh = xh.reshape(n, S, C), s_xh.reshape(n, S, C)
    h = xh * g + b
    s_h = s_xh * g.abs() + 2 * U * ((xh * g).abs() + b.abs())
    y = act(h, a)
    return (y, mean, rstd), (1.13 * s_h + (16 * U * (h.abs() + 1) if a in (SILU, GELU) else 0), s_mean, s_rstd)


def norm_gradient(x, gamma, beta, mean, rstd, dy, res, a):
    """(dx, dgamma, dbeta) for given mean and rstd, with their slacks."""
    n, S, C = x.shape
    groups = mean.shape[1]
    per = C // groups
    wide = lambda t: t.double().repeat_interleave(per, 1)[:, None, :]
    g = gamma.double() if gamma is not None else torch.ones(C, dtype=torch.float64, device=x.device)
    b = beta.double() if beta is not None else torch.zeros(C, dtype=torch.float64, device=x.device)
    xh = (x.double() - wide(mean)) * wide(rstd)
    s_xh = 2 * U * xh.abs()
    h = xh * g + b
    dh = dy.double() * slope(h, a)
    # slope' is at most 1 (silu 0.5, gelu 0.8); relu's corner is on the side that the fp32 value of h is on
    s_dh = dy.double().abs() * (U * 24 * (1 + h.abs()) + (s_xh * g.abs() + 2 * U * ((xh * g).abs() + b.abs())) if a in (SILU, GELU) else 2 * U)
    q = dh * g
    s_q = s_dh * g.abs() + U * q.abs()
    means = lambda t: t.reshape(n, S, groups, per).mean(dim=(1, 3)).repeat_interleave(per, 1)[:, None, :]
    depth = min(S * per, 128) + 40
    m1, m2 = means(q), means(q * xh)
    s_m1 = means(s_q) + depth * U * means(q.abs())
    s_m2 = means(s_q * xh.abs() + q.abs() * s_xh) + (depth + 2) * U * means((q * xh).abs())
    r = wide(rstd)
    dx = r * (q - m1 - xh * m2)
    s_dx = r * (s_q + s_m1 + s_xh * m2.abs() + xh.abs() * s_m2 + 4 * U * (q.abs() + m1.abs() + (xh * m2).abs()))
    if res is not None:
        dx = dx + res.double()
        s_dx = s_dx + U * (dx.abs() + res.double().abs())
    rows = n * S
    dgamma, dbeta = (dh * xh).sum((0, 1)), dh.sum((0, 1))
    s_g = (s_dh * xh.abs() + dh.abs() * s_xh).sum((0, 1)) + (rows + 4) * U * (dh * xh).abs().sum((0, 1))
    s_b = s_dh.sum((0, 1)) + (rows + 4) * U * dh.abs().sum((0, 1))
    return (dx, dgamma, dbeta), (s_dx, s_g, s_b)
