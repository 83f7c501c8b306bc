"""Calls of the hidden layers' operators on the GPU that the documentation allows beside those of test_gpu_operators.py: missing
operands, values at the edges of a type, ranges of plans, different pitches of one call's matrices."""
import ctypes as C

import pytest
import torch

import paper_2301_08895_amd as lib
import operator_util as ou
from operator_util import NONE, RELU, SILU, GELU
from paper_2301_08895_amd.binding import AbsLinear, _lib

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(23)


def normal(rows, cols, dtype, scale=1.0):
    return (torch.randn(rows, cols, device="cuda") * scale).to(dtype)


def gradient_call(x, w, z, dy, act, dx, dw, db):
    """abs_linear_backward itself, any operand or output missing."""
    rows, d_out = dy.shape
    d_in = next(t for t in (x, dx) if t is not None).shape[1] if x is not None or dx is not None else 24
    p = AbsLinear(0 if dy.dtype == F32 else 1, act, rows, d_in, d_out, d_in, d_out, d_out, d_out, d_out, d_out, d_in, d_out)
    n = _lib.abs_linear_workspace_size(C.byref(p), 1, 0)
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    at = (ws.data_ptr() + 255) // 256 * 256
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = _lib.abs_linear_backward(C.byref(p), ptr(x), ptr(w), ptr(z), ptr(dy), ptr(dx), ptr(dw), ptr(db), at, n,
                                  torch.cuda.current_stream().cuda_stream)
    assert rc == 0, lib.abs_last_error(None)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d_out", [(40, 33), (5000, 40), (30000, 2100)])
@pytest.mark.parametrize("act", [NONE, GELU])
def test_bias_gradient_needs_neither_x_nor_w(rows, d_out, act, dtype):
    """One workgroup's layer, one whose rows are cut into shares, and one beyond the single launch."""
    z, dy = normal(rows, d_out, dtype), normal(rows, d_out, dtype)
    db = torch.empty(d_out, device="cuda")
    gradient_call(None, None, z, dy, act, None, None, db)
    x, w = torch.zeros(rows, 24, dtype=dtype, device="cuda"), torch.zeros(24, d_out, dtype=dtype, device="cuda")
    want, slack = ou.linear_gradient(x, w, z, dy, act)
    ou.close(db, want[2], slack[2], "db")
    assert torch.equal(lib.linear_backward(x, w, dy, act=act, z=z, need_dx=False, need_dw=False)[2], db)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d_in,d_out", [(40, 50, 33), (3000, 640, 900)])
def test_input_gradient_needs_no_x_and_weight_gradient_no_w(rows, d_in, d_out, dtype):
    x, w = normal(rows, d_in, dtype), normal(d_in, d_out, dtype, d_in ** -0.5)
    z, dy = normal(rows, d_out, dtype), normal(rows, d_out, dtype)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    gradient_call(None, w, z, dy, SILU, dx, None, None)
    gradient_call(x, None, z, dy, SILU, None, dw, None)
    want, slack = ou.linear_gradient(x, w, z, dy, SILU)
    ou.close(dx, want[0], slack[0], "dx")
    ou.close(dw, want[1], slack[1], "dw")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d_in,d_out", [(60, 40, 33), (900, 700, 904)])
def test_relu_lets_nothing_of_masked_gradients_through(rows, d_in, d_out, dtype):
    """dz is 0 where z is not positive, whatever dy holds there (one launch, and tiles behind a pass for dz)."""
    x, w = normal(rows, d_in, dtype), normal(d_in, d_out, dtype, d_in ** -0.5)
    z, dy = normal(rows, d_out, dtype), normal(rows, d_out, dtype)
    off = z <= 0
    off[0, 0], z[0, 0] = True, 0.0
    wild = dy.clone()
    wild[off] = torch.tensor([float("inf"), -float("inf"), float("nan"), 3e38], device="cuda").to(dtype).repeat(off.sum() // 4 + 1)[:off.sum()]
    got = lib.linear_backward(x, w, wild, act=RELU, z=z)
    for g, v, s, name in zip(got, *ou.linear_gradient(x, w, z, torch.where(off, 0, dy), RELU), ("dx", "dw", "db")):
        ou.close(g, v, s, name)


# one workgroup per sample, samples in parts, single positions, wide groups of those, groups of the plain kernel
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,S,C,G", [(5, 49, 32, 4), (1, 5000, 16, 2), (40, 1, 256, 8), (9, 1, 4096, 1), (2, 3, 16400, 2)])
def test_relu_behind_a_norm_lets_nothing_of_masked_gradients_through(n, S, C, G, dtype):
    x, dy = normal(n * S, C, dtype).view(n, S, C), normal(n * S, C, dtype).view(n, S, C)
    gamma, beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    _, mean, rstd = lib.group_norm_forward(x, gamma, beta, G)
    wide = lambda t: t.repeat_interleave(C // G, 1)[:, None, :]
    # on the border the sign is the distance's (gamma and rstd are positive, beta is 0)
    off = (x.float() - wide(mean)) <= 0
    wild = torch.where(off, float("inf"), dy.float()).to(dtype)
    got = lib.group_norm_backward(x, gamma, beta, mean, rstd, wild, act=RELU)
    want, slack = ou.norm_gradient(x, gamma, beta, mean, rstd, torch.where(off, 0, dy), None, NONE)
    for g, v, s, name in zip(got, want, slack, ("dx", "dgamma", "dbeta")):
        ou.close(g, v, s, name)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", [NONE, SILU, GELU])
@pytest.mark.parametrize("rows,d_in,d_out", [(40, 50, 33), (5000, 40, 24), (900, 700, 904)])
def test_infinite_operands_of_a_gradient(rows, d_in, d_out, act, dtype):
    """A single infinite factor gives an infinity of its sign, where dz has one; NaN where dz is 0."""
    x, w = normal(rows, d_in, dtype), normal(d_in, d_out, dtype, d_in ** -0.5)
    z, dy = normal(rows, d_out, dtype), normal(rows, d_out, dtype)
    x[rows // 2, 3], x[1, 20], w[7, 5], w[d_in - 1, d_out - 1] = float("inf"), -float("inf"), -float("inf"), float("inf")
    dy[1, 4] = dy[rows - 1, 5] = 0.0
    got = lib.linear_backward(x, w, dy, act=act, z=z)
    want, slack = ou.linear_gradient(x, w, z, dy, act)
    assert torch.isinf(want[0]).any() and torch.isinf(want[1]).any() and torch.isnan(want[0]).any() and torch.isnan(want[1]).any()
    for g, v, s, name in zip(got, want, slack, ("dx", "dw", "db")):
        ou.close(g, v, s, name)


def _act64(z, act):
    """act(z), act'(z), and Phi or the logistic function at z and |z| times its derivative; no cancellation for z < 0."""
    if act == SILU:
        p, q = torch.sigmoid(z), torch.sigmoid(-z)
        return z * p, p * (1 + z * q), p, z.abs() * p * q
    p = 0.5 * torch.special.erfc(-z / 2 ** 0.5)
    density = torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    return z * p, p + z * density, p, z.abs() * density


def _points(dtype):
    z = torch.cat([torch.linspace(-100, 100, 4001), torch.linspace(-6, 6, 4001), torch.randn(4000),
                   torch.tensor([0.0, -0.0, 2.0 ** -100, -2.0 ** -100, 88.7, -88.7, 1e30, -1e30])])
    return torch.cat([z, torch.zeros(-len(z) % 64)]).cuda().to(dtype).view(-1, 64)


@pytest.mark.parametrize("act", [SILU, GELU])
@pytest.mark.parametrize("wide", [64, 2048])
def test_fp32_activations_are_fp32_at_every_z(act, wide):
    """z = x I exactly, so what is seen is the activation's own error: 10 half steps in the polynomial's and exponential's roundings, two
    more for each of the two instructions that are one step off, and the product's.  Below 2^-126 (times |z|) the exponential is 0."""
    z = _points(F32).repeat(1, wide // 64)
    value, slope, p, part = _act64(z.double(), act)
    eye = torch.eye(wide, device="cuda")
    tiny = 2.0 ** -126 * (1 + z.double().abs())
    y, kept = lib.linear_forward(z, eye, act=act, keep_z=True)
    assert torch.equal(kept, z)
    assert ((y.double() - value).abs() <= 16 * ou.U * value.abs() + tiny).all()
    dx, _, _ = lib.linear_backward(z, eye, torch.ones_like(z), act=act, z=z)
    assert ((dx.double() - slope).abs() <= 20 * ou.U * (p + part) + tiny).all()


@pytest.mark.parametrize("act", [SILU, GELU])
def test_fp32_activations_behind_a_norm(act):
    """gamma = 0: the activation's argument is beta."""
    beta = _points(F32).flatten()
    value, slope, p, part = _act64(beta.double(), act)
    tiny = 2.0 ** -126 * (1 + beta.double().abs())
    x = torch.randn(1, 1, beta.numel(), device="cuda")
    gamma = torch.zeros_like(beta)
    for groups in (beta.numel() // 64, 1):
        y, mean, rstd = lib.group_norm_forward(x, gamma, beta, groups, act=act)
        assert ((y.flatten().double() - value).abs() <= 16 * ou.U * value.abs() + tiny).all()
        dbeta = lib.group_norm_backward(x, gamma, beta, mean, rstd, torch.ones_like(x), act=act)[2]
        assert ((dbeta.double() - slope).abs() <= 20 * ou.U * (p + part) + tiny).all()


@pytest.mark.parametrize("act", [SILU, GELU])
def test_bf16_activations_over_their_range(act):
    """What is evaluated behind bf16 elements is off by 2^-8 of the result for its rounding, and by 2 (|z| + 8) half steps of fp32 of it
    (silu) or by erf's 1.5e-7 and four half steps of 1 times |z| / 2 (gelu); the same of the slope's terms.  Where exp(-z) passes fp32, from
    z = -87 down, silu is 0."""
    z = _points(BF)
    value, slope, p, part = _act64(z.double(), act)
    size = z.double().abs()
    tiny = 2.0 ** -125 * (1 + size)
    if act == SILU:
        off, off_slope = 2 * (size + 8) * ou.U * value.abs(), 2 * (size + 8) * ou.U * (p + part) + 4 * ou.U * (1 + size) * p
    else:
        off = size * (0.75e-7 + 4 * ou.U)
        off_slope = 0.75e-7 + 4 * ou.U + (2 * size * size + 8) * ou.U * part
    eye = torch.eye(64, device="cuda").to(BF)
    y = lib.linear_forward(z, eye, act=act)
    ou.close(y, value, off + tiny, "value")
    dx, _, _ = lib.linear_backward(z, eye, torch.ones_like(z), act=act, z=z)
    ou.close(dx, slope, off_slope + tiny + 2.0 ** -15 * slope.abs(), "slope")


# ---- what the rounds of residual blocks hold in fp32 ----------------------------------------------------
def _blocks(dims, N=4, B=16, **over):
    import workloads
    p = workloads.scaled_preset(3, M=2000, dims=dims, n_classes=dims[-1], N=N, B=B, n_slow=1, lr=0.05, K0=N, k_mode=1, tau_cap=3, **over)
    p = workloads.with_blocks(p, groups=4, drop=0)
    return p, workloads.make_split(p, 333)


def _last_bias(w0, dims):
    return w0[w0.size - dims[-1]:]


@pytest.mark.parametrize("dims", [[16, 24, 10], [32, 64, 64, 33], [16, 520, 200]])
def test_logits_closer_than_a_bf16_step(dims):
    """W_{L-1} = 0: the logits are the biases, 16 and steps of 0.01 above it, where bf16 has steps of 0.125: losses are those of the biases,
    and a row is a hit where its label is the last class."""
    import numpy as np
    p, (train, Xe, ye) = _blocks(dims)
    C, d = dims[-1], dims[-2]
    w0 = train["w0"].copy()
    w0[w0.size - C - d * C:] = 0.0
    _last_bias(w0, dims)[:] = 16 + 0.01 * np.arange(C)
    train = dict(train, w0=w0)
    bias = _last_bias(w0, dims).astype(np.float64)
    per_class = np.log(np.exp(bias - bias[-1]).sum()) + bias[-1] - bias
    sim = lib.Simulation(p, train)
    loss, acc = sim.evaluate(Xe, ye)
    # a loss is a logarithm of a sum of C exponentials less a difference, each a few half steps of numbers up to log C + 0.01 C
    tol = 64 * ou.U * (np.log(C) + 0.01 * C + 1)
    assert abs(loss - per_class[ye].mean()) <= tol
    assert acc == (ye == C - 1).mean()
    sim.round(1)
    rows = np.concatenate([lib.abs_draw_batch_rows(sim.cfg, n, 0) for n in range(p["N"])])
    got = float(sim.trace()[0][10:11].view(np.float32)[0])
    assert abs(got - per_class[train["y"][rows]].mean()) <= tol + p["B"] * ou.U * per_class.max()
    sim.close()


@pytest.mark.parametrize("dims,B", [([16, 24, 10], 16), ([64, 128, 128, 50], 40), ([1024, 1096, 200], 128)])
def test_matrix_gradients_are_not_rounded_on_their_way_into_the_model(dims, B):
    """From W_{L-1} = 0 the first round's matrix is the gradient, coefficients and signs included: one rounded to bf16 has 16 bits of zeros."""
    import numpy as np
    p, (train, _, _) = _blocks(dims, B=B)
    w0 = train["w0"].copy()
    C, d = dims[-1], dims[-2]
    w0[w0.size - C - d * C:] = 0.0
    sim = lib.Simulation(p, dict(train, w0=w0))
    sim.round(1)
    last = sim.model()[w0.size - C - d * C:w0.size - C]
    low = last.view(np.uint32) & 0xFFFF
    assert (last != 0).mean() > 0.9 and (low != 0).mean() > 0.9
    sim.close()


# ---- several tiles of a small product in one workgroup: two, four or eight of dW (few rows, wide layers), of the forward product and of dx
# (many rows, narrow layers), in both dtypes
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d_in,d_out", [(8, 2048, 2048), (9, 2047, 2045), (60, 2000, 2050), (1, 2900, 1450), (20, 1030, 4095), (30000, 300, 20),
                                             (30000, 24, 20), (100_000, 64, 64), (70_000, 17, 9), (12_000, 9, 3000), (70_000, 2, 3), (40_000, 130, 33)])
def test_several_small_tiles_in_a_workgroup(rows, d_in, d_out, dtype):
    x, w = normal(rows, d_in, dtype), normal(d_in, d_out, dtype, d_in ** -0.5)
    b, r = torch.randn(d_out, device="cuda"), normal(rows, d_out, dtype)
    y, z = lib.linear_forward(x, w, b, act=SILU, residual=r, keep_z=True)
    want, wz, sy, sz = ou.linear(x, w, b, SILU, r)
    ou.close(z, wz, sz, "z")
    ou.close(y, want, sy, "y")
    dy = normal(rows, d_out, dtype)
    want, slack = ou.linear_gradient(x, w, z, dy, SILU)
    whole = lib.linear_backward(x, w, dy, act=SILU, z=z)
    for g, v, s, name in zip(whole, want, slack, ("dx", "dw", "db")):
        ou.close(g, v, s, name)
    for only in range(3):
        one = lib.linear_backward(x, w, dy, act=SILU, z=z, need_dx=only == 0, need_dw=only == 1, need_db=only == 2)
        assert [g is not None for g in one] == [i == only for i in range(3)]
        ou.close(one[only], want[only], slack[only], f"{only} alone")        # (not the same bits: without the others its contraction may be cut elsewhere)


# ---- dz of small bf16 gradients: two bf16 values
@pytest.mark.parametrize("act", [SILU, GELU])
@pytest.mark.parametrize("rows,d_in,d_out", [(64, 48, 64), (300, 200, 130), (2000, 64, 40), (9, 2047, 515)])
def test_small_bf16_gradients_round_once(rows, d_in, d_out, act):
    """dz reaches the matrix cores to 2^-15 of itself (its second bf16 value, at most 2^-7 of it, is off by 2^-8 of that), so dx and dW are off by
    their own rounding and little else; with dz rounded to bf16 once they would not be."""
    x, w = normal(rows, d_in, BF), normal(d_in, d_out, BF, d_in ** -0.5)
    z, dy = normal(rows, d_out, BF), normal(rows, d_out, BF)
    got = lib.linear_backward(x, w, dy, act=act, z=z)
    want, slack = ou.linear_gradient(x.float(), w.float(), z.float(), dy.float(), act)         # (their slacks without dz's rounding)
    dz = (dy.double() * ou.slope(z.double(), act))
    wide, tall = w.double().t().contiguous(), x.double().t().contiguous()
    sx, sw = slack[0] + 2.0 ** -15 * (dz.abs() @ wide.abs()), slack[1] + 2.0 ** -15 * (tall.abs() @ dz.abs())
    ou.close(got[0], want[0], sx, "dx")
    ou.close(got[1], want[1], sw, "dw")
    once = dz.to(BF).double()
    for coarse, v, s, length in ((once @ wide, want[0], sx, d_out), (tall @ once, want[1], sw, rows)):
        if length > 300:
            continue
        with pytest.raises(AssertionError):
            ou.close(coarse.to(BF), v, s)


# ---- group norm: pitches of its own for each array of a gradient, results and everything around them
def _padded(n, S, C, pad, lead, dtype, fill=float("nan")):
    """([n, S, C] view of normal values in rows that are pad longer, the whole memory, a mask of the rest of it)."""
    flat = torch.full((lead + n * S * (C + pad),), fill, dtype=dtype, device="cuda")
    view = flat[lead:].view(n, S, C + pad)[:, :, :C]
    view.copy_(torch.randn(n, S, C, device="cuda"))
    rest = torch.ones_like(flat, dtype=torch.bool)
    rest[lead:].view(n, S, C + pad)[:, :, :C] = False
    return view, flat, rest


# samples whole, in parts, single positions, wide ones, groups of the plain kernel; starts that are no whole piece
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,S,C,G,lead", [(3, 50, 32, 8, 0), (3, 50, 32, 8, 1), (2, 1, 32, 8, 3), (1, 9000, 32, 8, 0), (2, 20000, 12, 3, 1), (300, 1, 264, 1, 0),
                                          (5, 1, 4096, 1, 8), (40, 9, 224, 32, 0), (3, 4, 1200, 2, 2), (2, 3, 16400, 2, 1)])
def test_group_norm_gradient_at_pitches_of_its_own(n, S, C, G, lead, dtype):
    (x, *_), (dy, *_), (res, *_) = (_padded(n, S, C, pad, lead, dtype) for pad in (8, 3, 16))
    out, flat, rest = _padded(n, S, C, 5, lead, dtype, 7.0)
    gamma, beta = 1 + 0.3 * torch.randn(C, device="cuda"), 0.3 * torch.randn(C, device="cuda")
    y, mean, rstd = lib.group_norm_forward(x, gamma, beta, G, act=SILU, out=out)
    assert y is out and (flat[rest] == 7).all()
    for g, v, s, name in zip((y, mean, rstd), *ou.norm(x, gamma, beta, G, 1e-5, SILU), ("y", "mean", "rstd")):
        ou.close(g, v, s, name)
    for r in (res, None):
        want, slack = ou.norm_gradient(x, gamma, beta, mean, rstd, dy, r, SILU)
        got = lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=SILU, residual=r, out=out)
        assert got[0] is out and (flat[rest] == 7).all()
        for g, v, s, name in zip(got, want, slack, ("dx", "dgamma", "dbeta")):
            ou.close(g, v, s, name)
    over, flat, rest = _padded(n, S, C, 5, lead, dtype, 7.0)
    want, slack = ou.norm_gradient(x, gamma, beta, mean, rstd, dy, over.clone(), SILU)
    got = lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=SILU, residual=over, out=over)
    assert (flat[rest] == 7).all()
    for g, v, s, name in zip(got, want, slack, ("dx over the residual", "dgamma", "dbeta")):
        ou.close(g, v, s, name)


# ---- rounds of residual blocks whose products run on tiles: whole pieces, copied operands, several versions a round
@pytest.mark.parametrize("over", [dict(dims=[64, 1536, 1536, 100], groups=32, K0=8), dict(dims=[72, 1530, 1530, 37], groups=5, K0=8, act=1),
                                  dict(dims=[64, 1400, 1400, 1400, 10], groups=7, K0=5)])
def test_wide_blocks_follow_the_oracle(over):
    import numpy as np
    import workloads
    from test_gpu_blocks import TOL, oracle_rounds, preset, tensors
    from oracle import blocks as ob
    from oracle.bf16 import bits_to_f64
    p = preset(N=8, B=160, **over)
    d, Xe, ye = workloads.make_split(p, 1500)
    sim = lib.Simulation(p, d)
    T = 3
    got = [sim.model()]
    for _ in range(T):
        sim.round(1)
        got.append(sim.model())
    want, losses = oracle_rounds(p, d, sim, T)
    trace = sim.trace()
    for t in range(T):
        gl = float(trace[t][10:11].view(np.float32)[0])
        assert abs(gl - losses[t]) <= TOL * max(1.0, losses[t]), t
    for t in (1, T):
        for name, s in tensors(p):
            up, back = got[t][s].astype(np.float64) - got[0][s], want[t][s] - want[0][s]
            assert np.linalg.norm(up - back) <= TOL * max(np.linalg.norm(back), 1e-12), (t, name)
    loss, _ = sim.evaluate(Xe, ye)
    per_row, _ = ob.loss_of(ob.forward(p["dims"], p["blocks"], sim.model(), bits_to_f64(Xe))[0], ye)
    assert abs(loss - per_row.mean()) <= TOL * max(1.0, per_row.mean())
    sim.close()


# ---- the ends of the documented ranges
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d_in,d_out", [(1, 1 << 20, 3), (2, 3, 1 << 20), (1, 1, 1 << 20), (1, 1 << 20, 1), ((1 << 22) + 3, 1, 1), ((1 << 22) + 3, 2, 2),
                                             ((1 << 21) + 1, 3, 1)])
def test_linear_at_the_ends_of_its_range(rows, d_in, d_out, dtype):
    x, w = normal(rows, d_in, dtype), normal(d_in, d_out, dtype, d_in ** -0.5)
    b = torch.randn(d_out, device="cuda")
    y, z = lib.linear_forward(x, w, b, act=SILU, keep_z=True)
    want, wz, sy, sz = ou.linear(x, w, b, SILU, None)
    ou.close(z, wz, sz, "z")
    ou.close(y, want, sy, "y")
    dy = normal(rows, d_out, dtype)
    for g, v, s, name in zip(lib.linear_backward(x, w, dy, act=SILU, z=z), *ou.linear_gradient(x, w, z, dy, SILU), ("dx", "dw", "db")):
        ou.close(g, v, s, name)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,S,C,G", [(2, 1, 1 << 20, 1), (2, 1, 1 << 20, 1 << 20), (1, 1 << 22, 1, 1), (1 << 22, 1, 2, 1), (1 << 20, 3, 2, 2), (1, 2, 1 << 20, 1 << 10)])
def test_group_norm_at_the_ends_of_its_range(n, S, C, G, dtype):
    x, dy = normal(n * S, C, dtype).view(n, S, C), normal(n * S, C, dtype).view(n, S, C)
    gamma, beta = 1 + 0.3 * torch.randn(C, device="cuda"), 0.3 * torch.randn(C, device="cuda")
    # (groups of one or two values: eps keeps the reciprocal deviation, and with it every error, near 1)
    got = lib.group_norm_forward(x, gamma, beta, G, eps=1.0, act=SILU)
    for g, v, s, name in zip(got, *ou.norm(x, gamma, beta, G, 1.0, SILU), ("y", "mean", "rstd")):
        ou.close(g, v, s, name)
    _, mean, rstd = got
    want, slack = ou.norm_gradient(x, gamma, beta, mean, rstd, dy, None, SILU)
    for g, v, s, name in zip(lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=SILU), want, slack, ("dx", "dgamma", "dbeta")):
        ou.close(g, v, s, name)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_losses_of_blocks_that_are_not_finite_end_the_round(value):
    """A logit that is not finite in one class: the round is refused and not counted, and the model stays; held-out losses say so too."""
    import numpy as np
    p, (train, Xe, ye) = _blocks([16, 24, 10])
    w0 = train["w0"].copy()
    _last_bias(w0, p["dims"])[3] = value
    sim = lib.Simulation(p, dict(train, w0=w0))
    with pytest.raises(lib.AbsError) as e:
        sim.round(1)
    assert e.value.code == -5 and lib.abs_rounds_done(sim.handle) == 0
    assert np.array_equal(sim.model(), w0, equal_nan=True)
    loss, _ = sim.evaluate(Xe, ye)
    assert not np.isfinite(loss)
    sim.close()
