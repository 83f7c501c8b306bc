"""The operators of a network's hidden layers, as cases that can be timed and compared.

Three operators, each with its gradient: the product of a layer (rows times weights, with bias, activation and
residual in one pass), group normalisation over channels-last positions with an activation behind it, and dropout
whose mask is a function of a counter and never stored.  Together they are a residual block of the networks that the
parameter-server rounds train; a case here is one operator, one direction, one type, at one size.

Where `own` is false `run` computes them from elementary torch operations in 32 bits, rounded once at the end; where
it is true it makes the package's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
device = "cuda"

NONE, RELU, SILU, GELU = 0, 1, 2, 3
BF16, FP32 = "bf16", "fp32"
TYPE = {BF16: torch.bfloat16, FP32: torch.float32}
EPS = 1e-5


def _linear(name, dtype, rows, d_in, d_out, act, *, backward=False, residual=False, keep=False, pad=0):
    """rows x d_in times d_in x d_out.  keep: the forward pass also returns the pre-activations (training).
    pad: the rows of x are that many elements longer than d_in (a slice of a wider matrix)."""
    return dict(name=name, op="linear", backward=backward, dtype=dtype, rows=rows, d_in=d_in, d_out=d_out, act=act,
                residual=residual, keep=keep, pad=pad)


def _norm(name, dtype, n, spatial, channels, groups, act, *, backward=False, residual=False):
    """n samples of `spatial` positions of `channels` channels in `groups` groups.
    residual (backward): the gradient that reaches x past the block is added."""
    return dict(name=name, op="norm", backward=backward, dtype=dtype, n=n, spatial=spatial, channels=channels,
                groups=groups, act=act, residual=residual)


def _drop(name, dtype, rows, cols, drop, *, backward=False, residual=False, pad=0):
    """drop: of 65536 equal parts of the draws, how many are dropped."""
    return dict(name=name, op="dropout", backward=backward, dtype=dtype, rows=rows, cols=cols, drop=drop,
                residual=residual, pad=pad)


def listed():
    return [
        # one row through a hidden layer, as a model answers a single request: the weights' bytes and launches
        _linear("linear one row", BF16, 1, 2048, 2048, GELU, residual=True),
        # a minibatch of 9 uploads of 90 rows through the ragged network's second layer: nothing a multiple of a tile
        _linear("linear ragged", BF16, 810, 520, 300, RELU, keep=True),
        # every worker's minibatch stacked, a hidden layer of the widest network: the largest product
        _linear("linear wide", BF16, 32768, 2048, 2048, SILU, residual=True, keep=True),
        # the first dense layer behind the convolutions, fp32, 20 workers of 32 images
        _linear("linear fp32", FP32, 640, 400, 120, RELU, keep=True),
        # gradients of a hidden layer, the first rounds of a run (32 uploads of 256 rows)
        _linear("linear gradient", BF16, 8192, 2048, 2048, SILU, backward=True),
        # gradients of an fp32 layer
        _linear("linear gradient fp32", FP32, 4096, 1024, 1000, GELU, backward=True),
        # the maps behind the first convolution of an image model: a batch of 640 maps of 14 x 14
        _norm("norm images", FP32, 640, 196, 24, 6, RELU),
        # deeper maps of a large image model, the whole forward pass bound by memory
        _norm("norm maps", BF16, 64, 4096, 256, 32, SILU),
        # hidden activations of a dense network, every row normalised in 32 groups, gradient with the residual's
        _norm("norm rows gradient", BF16, 8192, 1, 2048, 32, SILU, backward=True, residual=True),
        # gradient over maps of 32 x 32
        _norm("norm maps gradient", BF16, 32, 1024, 512, 32, SILU, backward=True),
        # hidden activations of every worker, a tenth dropped, added to the residual
        _drop("dropout wide", BF16, 32768, 2048, 6554, residual=True),
        # the gradient of half-dropped activations of the ragged network: an odd width
        _drop("dropout gradient ragged", FP32, 810, 300, 32768, backward=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths are multiples of 8, as networks have them, the others whatever comes."""
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.5 else max(8, w // 8 * 8)


def draw(rng):
    """One more case: any operator, direction and type, with sizes spread over the range of the listed ones."""
    op = rng.choice(["linear", "norm", "dropout"])
    backward = rng.random() < 0.5
    dtype = rng.choice([BF16, BF16, FP32])
    act = rng.choice([NONE, RELU, SILU, GELU])
    if op == "linear":
        d_in, d_out = _width(rng, 16, 4096), _width(rng, 8, 4096)
        most = 32768 * 2048 * 2048 // (16 if dtype == FP32 else 2 if backward else 1)
        rows = _log(rng, 1, max(1, min(32768, most // (d_in * d_out))))
        c = _linear("", dtype, rows, d_in, d_out, act, backward=backward, residual=not backward and rng.random() < 0.5,
                    keep=not backward and rng.random() < 0.5, pad=rng.choice([0, 0, 8, 3]))
    elif op == "norm":
        groups = rng.choice([1, 2, 4, 8, 16, 32, 32, rng.randint(1, 40)])
        channels = groups * max(1, _log(rng, 1, max(1, 2048 // groups)))
        spatial = rng.choice([1, _log(rng, 2, 64) ** 2, _log(rng, 2, 64) ** 2, _log(rng, 2, 4096)])
        most = 64 * 4096 * 256 // (2 if dtype == FP32 else 1) // (2 if backward else 1)
        n = _log(rng, 1, max(1, min(8192, most // (spatial * channels))))
        if n * spatial * channels > most:
            spatial = max(1, most // channels)
        spatial = max(spatial, -(-8 * groups // channels))      # a group of a value or two has nothing left but its rounding
        c = _norm("", dtype, n, spatial, channels, groups, act, backward=backward, residual=backward and rng.random() < 0.5)
    else:
        cols = _width(rng, 1, 4096)
        rows = _log(rng, 1, min(32768, 32768 * 1024 // cols))
        c = _drop("", dtype, rows, cols, rng.choice([0, 3277, 6554, 13107, 32768, rng.randint(1, 65535)]), backward=backward,
                  residual=not backward and rng.random() < 0.5, pad=rng.choice([0, 0, 8, 1]))
    del c["name"]
    return c


class _State:
    pass


def _rows(g, rows, cols, pad, dtype, scale=1.0):
    """rows x cols normal values, as the first columns of rows that are `pad` longer."""
    t = torch.randn(rows, cols + pad, generator=g, device=device).mul_(scale).to(TYPE[dtype])
    return t[:, :cols] if pad else t


def _saved(x, groups):
    """Mean and reciprocal standard deviation that a forward pass leaves for the backward one, fp32 [n, groups]."""
    n, spatial, channels = x.shape
    v = x.float().view(n, spatial, groups, channels // groups)
    mean = v.mean(dim=(1, 3))
    var = (v - mean.view(n, 1, groups, 1)).square_().mean(dim=(1, 3))
    return mean, torch.rsqrt(var + EPS)


def prepare(case, seed):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    s = _State()
    s.case = case
    dt = case["dtype"]
    if case["op"] == "linear":
        rows, d_in, d_out = case["rows"], case["d_in"], case["d_out"]
        s.x = _rows(g, rows, d_in, case["pad"], dt)
        s.w = _rows(g, d_in, d_out, 0, dt, 1.0 / math.sqrt(d_in))
        s.b = torch.randn(d_out, generator=g, device=device) * 0.1
        s.r = _rows(g, rows, d_out, 0, dt) if case["residual"] else None
        if case["backward"]:
            s.z = (s.x.float() @ s.w.float() + s.b).to(TYPE[dt]) if case["act"] != NONE else None
            s.dy = _rows(g, rows, d_out, 0, dt, 1e-2)
    elif case["op"] == "norm":
        n, spatial, channels, groups = case["n"], case["spatial"], case["channels"], case["groups"]
        # channels have means and spreads of their own, as a layer's outputs do
        spread = 0.5 + torch.rand(channels, generator=g, device=device)
        shift = torch.randn(channels, generator=g, device=device) * 0.5
        s.x = torch.randn(n * spatial, channels, generator=g, device=device).mul_(spread).add_(shift).to(TYPE[dt])
        s.x = s.x.view(n, spatial, channels)
        s.gamma = 1.0 + 0.2 * torch.randn(channels, generator=g, device=device)
        s.beta = 0.2 * torch.randn(channels, generator=g, device=device)
        if case["backward"]:
            s.mean, s.rstd = _saved(s.x, groups)
            s.dy = _rows(g, n * spatial, channels, 0, dt).view(n, spatial, channels)
            s.r = _rows(g, n * spatial, channels, 0, dt).view(n, spatial, channels) if case["residual"] else None
    else:
        s.x = _rows(g, case["rows"], case["cols"], case["pad"], dt)
        s.r = _rows(g, case["rows"], case["cols"], 0, dt) if case["residual"] else None
        s.seed, s.offset = 1_000_003 * seed + 17, 5 * seed + 2
    return s


# ---- plain forms ----------------------------------------------------------------------------------

def _act(z, act):
    if act == RELU:
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == SILU:
        return z * torch.sigmoid(z)
    if act == GELU:
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_gradient(z, act):
    """The activation's derivative at z (relu: 0 at 0)."""
    if act == RELU:
        return (z > 0).to(z.dtype)
    if act == SILU:
        p = torch.sigmoid(z)
        return p * (1.0 + z * (1.0 - p))
    if act == GELU:
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _plain_linear(s):
    case, dt = s.case, TYPE[s.case["dtype"]]
    if not case["backward"]:
        z = s.x.float() @ s.w.float() + s.b
        y = _act(z, case["act"])
        if s.r is not None:
            y = y + s.r.float()
        return {"y": y.to(dt), "z": z.to(dt)} if case["keep"] else {"y": y.to(dt)}
    d = s.dy.float()
    if s.z is not None:
        d = d * _act_gradient(s.z.float(), case["act"])
    return {"dx": (d @ s.w.float().t()).to(dt), "dw": (s.x.float().t() @ d).to(dt), "db": d.sum(dim=0)}


def _plain_norm(s):
    case, dt = s.case, TYPE[s.case["dtype"]]
    n, spatial, channels, groups = case["n"], case["spatial"], case["channels"], case["groups"]
    v = s.x.float().view(n, spatial, groups, channels // groups)
    if not case["backward"]:
        mean, rstd = _saved(s.x, groups)
        h = ((v - mean.view(n, 1, groups, 1)) * rstd.view(n, 1, groups, 1)).view(n, spatial, channels) * s.gamma + s.beta
        return {"y": _act(h, case["act"]).to(dt), "mean": mean, "rstd": rstd}
    xh = (v - s.mean.view(n, 1, groups, 1)) * s.rstd.view(n, 1, groups, 1)
    dh = s.dy.float()
    if case["act"] != NONE:
        dh = dh * _act_gradient(xh.view(n, spatial, channels) * s.gamma + s.beta, case["act"])
    dgamma = (dh * xh.view(n, spatial, channels)).sum(dim=(0, 1))
    dbeta = dh.sum(dim=(0, 1))
    q = (dh * s.gamma).view(n, spatial, groups, channels // groups)
    first = q.mean(dim=(1, 3), keepdim=True)
    second = (q * xh).mean(dim=(1, 3), keepdim=True)
    dx = ((q - first - xh * second) * s.rstd.view(n, 1, groups, 1)).view(n, spatial, channels)
    if s.r is not None:
        dx = dx + s.r.float()
    return {"dx": dx.to(dt), "dgamma": dgamma, "dbeta": dbeta}


def _signed(v):
    """A 64-bit word as the signed number torch holds it in."""
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


GAMMA, MUL1, MUL2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


def _mix_word(z):
    z &= (1 << 64) - 1
    z = (z ^ (z >> 30)) * MUL1 & ((1 << 64) - 1)
    z = (z ^ (z >> 27)) * MUL2 & ((1 << 64) - 1)
    return z ^ (z >> 31)


def _key(seed, offset):
    """The draws of one call: stream 2 of the seed's counters, at `offset`."""
    return _mix_word(_mix_word(seed + 3 * GAMMA) ^ offset)


def _shifted(z, by):
    return (z >> by) & ((1 << (64 - by)) - 1)        # a logical shift


def _plain_dropout(s):
    """Element e of the row-major matrix is dropped where the 16-bit part e % 4 of draw e / 4 is below `drop`."""
    case, dt = s.case, TYPE[s.case["dtype"]]
    rows, cols = s.x.shape
    total = rows * cols
    z = torch.arange(1, (total + 3) // 4 + 1, device=device, dtype=torch.int64) * _signed(GAMMA) + _signed(_key(s.seed, s.offset))
    z = (z ^ _shifted(z, 30)) * _signed(MUL1)
    z = (z ^ _shifted(z, 27)) * _signed(MUL2)
    z = z ^ _shifted(z, 31)
    parts = (z.view(-1, 1) >> torch.tensor([0, 16, 32, 48], device=device)) & 0xFFFF
    keep = (parts.view(-1)[:total] >= case["drop"]).view(rows, cols)
    x = s.x.float() * (65536.0 / (65536 - case["drop"]))
    y = torch.where(keep, x, torch.zeros_like(x))
    if s.r is not None:
        y = y + s.r.float()
    return {"dx" if case["backward"] else "y": y.to(dt)}


# ---- the package's calls --------------------------------------------------------------------------

def _own(s):
    import paper_2301_08895_amd as lib
    case = s.case
    if case["op"] == "linear":
        if case["backward"]:
            dx, dw, db = lib.linear_backward(s.x, s.w, s.dy, act=case["act"], z=s.z)
            return {"dx": dx, "dw": dw, "db": db}
        if case["keep"]:
            y, z = lib.linear_forward(s.x, s.w, s.b, act=case["act"], residual=s.r, keep_z=True)
            return {"y": y, "z": z}
        return {"y": lib.linear_forward(s.x, s.w, s.b, act=case["act"], residual=s.r)}
    if case["op"] == "norm":
        if case["backward"]:
            dx, dgamma, dbeta = lib.group_norm_backward(s.x, s.gamma, s.beta, s.mean, s.rstd, s.dy, act=case["act"],
                                                        residual=s.r)
            return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
        y, mean, rstd = lib.group_norm_forward(s.x, s.gamma, s.beta, case["groups"], eps=EPS, act=case["act"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if case["backward"]:
        return {"dx": lib.dropout_backward(s.x, case["drop"], s.seed, s.offset)}
    return {"y": lib.dropout_forward(s.x, case["drop"], s.seed, s.offset, residual=s.r)}


PLAIN = {"linear": _plain_linear, "norm": _plain_norm, "dropout": _plain_dropout}


def run(s):
    if own:
        return _own(s)
    return PLAIN[s.case["op"]](s)


# ---- the work of a pass, and its result in 64 bits ------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == BF16 else 4
    if case["op"] == "linear":
        rows, d_in, d_out = case["rows"], case["d_in"], case["d_out"]
        x, w, y = rows * d_in * size, d_in * d_out * size, rows * d_out * size
        if case["backward"]:
            read = x + w + y * (2 if case["act"] != NONE else 1)
            return {"bytes": float(read + x + w + 4 * d_out), "flops": 4.0 * rows * d_in * d_out}
        return {"bytes": float(x + w + 4 * d_out + y * (1 + int(case["residual"]) + int(case["keep"]))),
                "flops": 2.0 * rows * d_in * d_out}
    if case["op"] == "norm":
        m = case["n"] * case["spatial"] * case["channels"]
        small = 8.0 * case["n"] * case["groups"] + 8.0 * case["channels"]
        if case["backward"]:
            return {"bytes": m * size * (3.0 + int(case["residual"])) + small + 8.0 * case["channels"], "flops": 20.0 * m}
        return {"bytes": m * size * 2.0 + small, "flops": 10.0 * m}
    m = case["rows"] * case["cols"]
    return {"bytes": m * size * (2.0 + int(case["residual"])), "flops": 10.0 * m}


def _act64(z, act):
    if act == RELU:
        return z.clamp(min=0)
    if act == SILU:
        return z / (1 + torch.exp(-z))
    if act == GELU:
        return z * (1 - torch.special.erfc(z / math.sqrt(2)) / 2)
    return z


def _slope64(z, act):
    """d act / dz in 64 bits, with the formulas of _act64 differentiated."""
    if act == RELU:
        return torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
    if act == SILU:
        e = torch.exp(-z)
        return 1 / (1 + e) + z * e / (1 + e) ** 2
    if act == GELU:
        return 1 - torch.special.erfc(z / math.sqrt(2)) / 2 + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi)
    return z * 0 + 1


def _kept64(rows, cols, drop, seed, offset):
    """Which elements stay, from unsigned 64-bit arithmetic on the host."""
    def mix(v):
        v = (v ^ (v >> np.uint64(30))) * np.uint64(MUL1)
        v = (v ^ (v >> np.uint64(27))) * np.uint64(MUL2)
        return v ^ (v >> np.uint64(31))

    with np.errstate(over="ignore"):
        first = mix(np.array([(seed + 3 * GAMMA) % 2 ** 64], dtype=np.uint64))
        key = mix(first ^ np.uint64(offset))
        n = rows * cols
        words = mix(key + np.uint64(GAMMA) * np.arange(1, n // 4 + 2, dtype=np.uint64))
    return words.astype("<u8").view("<u2")[:n].reshape(rows, cols) >= drop


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        x, w = s.x.double(), s.w.double()
        if case["backward"]:
            dz = s.dy.double() * (_slope64(s.z.double(), case["act"]) if s.z is not None else 1)
            return {"dx": torch.matmul(dz, w.t().contiguous()), "dw": torch.matmul(x.t().contiguous(), dz), "db": dz.sum(0)}
        z = torch.addmm(s.b.double(), x, w)
        y = _act64(z, case["act"]) + (s.r.double() if s.r is not None else 0)
        return {"y": y, "z": z} if case["keep"] else {"y": y}
    if case["op"] == "norm":
        n, spatial, channels, groups = case["n"], case["spatial"], case["channels"], case["groups"]
        per = channels // groups

        def spread(t):                              # [n, groups] over the positions and channels
            return t.double().repeat_interleave(per, dim=1).unsqueeze(1)

        def means(t):                               # [n, spatial, channels] to [n, groups]
            return t.sum(dim=1).view(n, groups, per).sum(dim=2) / (spatial * per)

        x = s.x.double()
        if case["backward"]:
            xh = (x - spread(s.mean)) * spread(s.rstd)
            dh = s.dy.double() * _slope64(xh * s.gamma.double() + s.beta.double(), case["act"])
            dxh = dh * s.gamma.double()
            dx = spread(s.rstd) * (dxh - spread(means(dxh)) - xh * spread(means(dxh * xh)))
            return {"dx": dx + (s.r.double() if s.r is not None else 0), "dgamma": (dh * xh).flatten(0, 1).sum(0),
                    "dbeta": dh.flatten(0, 1).sum(0)}
        mean = means(x)
        rstd = 1 / torch.sqrt(means((x - spread(mean)) ** 2) + EPS)
        h = (x - spread(mean)) * spread(rstd) * s.gamma.double() + s.beta.double()
        return {"y": _act64(h, case["act"]), "mean": mean, "rstd": rstd}
    kept = torch.from_numpy(_kept64(s.x.shape[0], s.x.shape[1], case["drop"], s.seed, s.offset)).to(s.x.device)
    y = s.x.double() / (1 - case["drop"] / 65536)
    y = torch.where(kept, y, 0.0)
    return {"dx" if case["backward"] else "y": y + (s.r.double() if s.r is not None else 0)}
