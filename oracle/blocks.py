"""One round of the MLP whose hidden layers are residual blocks (oracle side; test infrastructure only).

  a_1 = x W_0 + b_0,  u_l = dropout(act(group norm(a_l))),  a_{l+1} = u_l W_l + b_l (+ a_l where the widths agree),
softmax cross-entropy on a_L.  Parameter vector: W_0, b_0, then per layer l >= 1 gamma_l, beta_l, W_l, b_l.
Rounding points of the bf16 path: matrices; a_l of the hidden layers; the normalised and activated value; after dropout; the logits'
gradient; every gradient that is handed on (of u_l, after dropout, of a_l).  The logits, matrix gradients and sums are wide.
"""
from __future__ import annotations

import numpy as np

from . import counter_rng as crng
from .bf16 import round_bf16


def unpack(dims, w):
    """[(gamma, beta or None, None; W, b)] views of the parameter vector."""
    out, o = [], 0
    for l in range(len(dims) - 1):
        g = b = None
        if l:
            g, b = w[o:o + dims[l]], w[o + dims[l]:o + 2 * dims[l]]
            o += 2 * dims[l]
        W = w[o:o + dims[l] * dims[l + 1]].reshape(dims[l], dims[l + 1])
        o += dims[l] * dims[l + 1]
        out.append((g, b, W, w[o:o + dims[l + 1]]))
        o += dims[l + 1]
    assert o == w.size
    return out


def kept(rows, cols, drop, seed, offset):
    """The dropout mask: 16-bit part e % 4 of draw e / 4 of stream 2 of the seed's counters at `offset`."""
    key = crng.mix64(crng.mix64(seed + 3 * crng.GOLDEN_GAMMA) ^ offset)
    with np.errstate(over="ignore"):
        z = np.uint64(key) + np.uint64(crng.GOLDEN_GAMMA) * np.arange(1, rows * cols // 4 + 2, dtype=np.uint64)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    parts = (z[:, None] >> np.array([0, 16, 32, 48], dtype=np.uint64)) & np.uint64(0xFFFF)
    return (parts.reshape(-1)[:rows * cols] >= drop).reshape(rows, cols)


def _act(h, a):
    if a == 1:
        return np.maximum(h, 0), (h > 0).astype(float)
    if a == 2:
        p = 1 / (1 + np.exp(-h))
        return h * p, p * (1 + h * (1 - p))
    if a == 3:
        from math import erf, pi, sqrt
        phi = 0.5 * (1 + np.vectorize(erf)(h / sqrt(2)))
        return h * phi, phi + h * np.exp(-h * h / 2) / sqrt(2 * pi)
    return h, np.ones_like(h)


def forward(dims, opt, w, X, masks=None, rnd=round_bf16):
    """Everything the backward pass needs, for rows X at parameters w; masks: per layer the kept elements, or None."""
    a, st = X, []
    layers = unpack(dims, np.asarray(w, dtype=np.float64))
    L = len(layers)
    for l, (gamma, beta, W, b) in enumerate(layers):
        rec = dict(a=a)
        u = a
        if l:
            n, d = a.shape
            v = a.reshape(n, opt["groups"], -1)
            mean = v.mean(2, keepdims=True)
            rec["rstd"] = 1 / np.sqrt(((v - mean) ** 2).mean(2, keepdims=True) + opt["eps"])
            rec["xhat"] = ((v - mean) * rec["rstd"]).reshape(n, d)
            y, rec["slope"] = _act(rec["xhat"] * gamma + beta, opt["act"])
            u = rnd(y)
            if masks is not None and opt["drop"]:
                u = rnd(np.where(masks[l], u * (65536 / (65536 - opt["drop"])), 0.0))
        rec["u"], rec["W"] = u, rnd(W)
        z = u @ rec["W"] + b
        rec["adds"] = bool(opt["residual"] and 1 <= l < L - 1 and dims[l] == dims[l + 1])
        a = z if l == L - 1 else rnd(z + rec["a"]) if rec["adds"] else rnd(z)
        st.append(rec)
    return a, st


def loss_of(z, y):
    top = z.max(1, keepdims=True)
    e = np.exp(z - top)
    return np.log(e.sum(1)) + top[:, 0] - z[np.arange(len(y)), y], e / e.sum(1, keepdims=True)


def gradient(dims, opt, w, X, y, coef, masks=None, rnd=round_bf16):
    """(sum over rows of coef grad f, per-row losses)."""
    z, st = forward(dims, opt, w, X, masks, rnd)
    per_row, P = loss_of(z, y)
    P[np.arange(len(y)), y] -= 1
    da = rnd(coef[:, None] * P)
    out = np.zeros(np.asarray(w).size)
    grads = unpack(dims, out)
    params = unpack(dims, np.asarray(w, dtype=np.float64))
    for l in range(len(st) - 1, -1, -1):
        r, (gg, gb, gW, gbias) = st[l], grads[l]
        gW[:] = r["u"].T @ da
        gbias[:] = da.sum(0)
        if not l:
            break
        du = rnd(da @ r["W"].T)
        if masks is not None and opt["drop"]:
            du = rnd(np.where(masks[l], du * (65536 / (65536 - opt["drop"])), 0.0))
        dh = du * r["slope"]
        gg[:], gb[:] = (dh * r["xhat"]).sum(0), dh.sum(0)
        q = (dh * params[l][0]).reshape(len(y), opt["groups"], -1)
        xh = r["xhat"].reshape(q.shape)
        dx = (r["rstd"] * (q - q.mean(2, keepdims=True) - xh * (q * xh).mean(2, keepdims=True))).reshape(len(y), -1)
        da = rnd(dx + da) if r["adds"] else rnd(dx)
    return out, per_row
