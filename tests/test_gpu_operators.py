"""The operators of a network's hidden layers on the GPU against their plain forms in 64 bits (operator_util.py, with the
tolerances' derivation), at the sizes, pitches and values where they can go wrong."""
import threading

import numpy as np
import pytest
import torch

import paper_2301_08895_amd as lib
import operator_util as ou
from operator_util import NONE, RELU, SILU, GELU

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(11)


def rows_of(rows, cols, dtype, pad=0, scale=1.0, lead=0):
    """A rows x cols matrix in rows that are `pad` longer, NaN behind their ends, starting `lead` elements into the allocation."""
    flat = torch.full((lead + rows * (cols + pad),), float("nan"), dtype=dtype, device="cuda")
    m = flat[lead:].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn(rows, cols, device="cuda") * scale)
    return m


# one element, one row, ends of pieces / k-steps / tiles on either side, few and many rows, a contraction in shares
SIZES = [(1, 1, 1), (1, 64, 8), (1, 2048, 520), (3, 65, 7), (8, 200, 33), (9, 7, 129), (17, 128, 128), (64, 72, 40), (127, 63, 127),
         (128, 64, 256), (129, 65, 257), (130, 1000, 24), (257, 520, 300), (300, 1, 5), (33, 4100, 16), (512, 264, 640),
         # either side of where one launch takes the whole pass; its contractions in shares; tile kernels on ragged operands
         (3, 9000, 40), (9001, 30, 18), (700, 1601, 1100), (1500, 1030, 1440), (6000, 515, 770), (2100, 2050, 2046), (5, 2100, 2101)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d_in,d_out", SIZES)
def test_linear_forward(rows, d_in, d_out, dtype):
    x, w = rows_of(rows, d_in, dtype), rows_of(d_in, d_out, dtype, scale=d_in ** -0.5)
    b, r = torch.randn(d_out, device="cuda"), rows_of(rows, d_out, dtype)
    for a in (NONE, RELU, SILU, GELU):
        y, z = lib.linear_forward(x, w, b, act=a, residual=r, keep_z=True)
        want, wz, sy, sz = ou.linear(x, w, b, a, r)
        ou.close(z, wz, sz, "z")
        ou.close(y, want, sy, f"y, act {a}")
    y = lib.linear_forward(x, w)
    want, _, sy, _ = ou.linear(x, w, None, NONE, None)
    ou.close(y, want, sy, "no bias")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,d_in,d_out", SIZES)
def test_linear_backward(rows, d_in, d_out, dtype):
    x, w = rows_of(rows, d_in, dtype), rows_of(d_in, d_out, dtype, scale=d_in ** -0.5)
    z, dy = rows_of(rows, d_out, dtype), rows_of(rows, d_out, dtype)
    for a in (NONE, RELU, SILU, GELU):
        got = lib.linear_backward(x, w, dy, act=a, z=z)
        want, slack = ou.linear_gradient(x, w, z, dy, a)
        for g, v, s, name in zip(got, want, slack, ("dx", "dw", "db")):
            ou.close(g, v, s, f"{name}, act {a}")
    dx, dw, db = lib.linear_backward(x, w, dy, need_dw=False, need_db=False)
    assert dw is None and db is None
    ou.close(dx, ou.linear_gradient(x, w, z, dy, NONE)[0][0], ou.linear_gradient(x, w, z, dy, NONE)[1][0], "dx alone")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [2, 200])
@pytest.mark.parametrize("pad,lead", [(8, 0), (3, 0), (8, 8), (8, 1)])
def test_linear_pitches_and_starts(rows, pad, lead, dtype):
    """Rows longer than the matrix (NaN behind their ends must not be read), starts that are and are not whole pieces; what
    lies behind the output's rows stays."""
    d_in, d_out = 136, 72
    x, w = rows_of(rows, d_in, dtype, pad, 1.0, lead), rows_of(d_in, d_out, dtype, pad, 0.1, lead)
    r, dy, z = (rows_of(rows, d_out, dtype, pad, 1.0, lead) for _ in range(3))
    b = torch.randn(d_out, device="cuda")
    flat = torch.full((lead + rows * (d_out + pad),), 7.0, dtype=dtype, device="cuda")
    out = flat[lead:].view(rows, d_out + pad)
    y = lib.linear_forward(x, w, b, act=GELU, residual=r, out=out[:, :d_out])
    want, _, sy, _ = ou.linear(x, w, b, GELU, r)
    ou.close(y, want, sy, "y")
    assert (out[:, d_out:] == 7).all() and (flat[:lead] == 7).all()
    got = lib.linear_backward(x, w, dy, act=SILU, z=z)
    for g, v, s in zip(got, *ou.linear_gradient(x, w, z, dy, SILU)):
        ou.close(g, v, s)


# results of many 256 x 256 tiles: ragged in every direction, contractions of one step and two, in shares for the gradients
@pytest.mark.parametrize("rows,d_in,d_out,act", [(3400, 1000, 3904, SILU), (3333, 777, 3901, GELU), (50_000, 24, 256, RELU),
                                                 (50_000, 70, 250, NONE), (50_000, 136, 512, SILU), (12_300, 2048, 1030, NONE)])
def test_linear_of_many_tiles(rows, d_in, d_out, act):
    x, w = rows_of(rows, d_in, BF), rows_of(d_in, d_out, BF, scale=d_in ** -0.5)
    b, r = torch.randn(d_out, device="cuda"), rows_of(rows, d_out, BF)
    y, z = lib.linear_forward(x, w, b, act=act, residual=r, keep_z=True)
    want, wz, sy, sz = ou.linear(x, w, b, act, r)
    ou.close(z, wz, sz, "z")
    ou.close(y, want, sy, "y")
    dy = rows_of(rows, d_out, BF)
    got = lib.linear_backward(x, w, dy, act=act, z=z)
    for g, v, s, name in zip(got, *ou.linear_gradient(x, w, z, dy, act), ("dx", "dw", "db")):
        ou.close(g, v, s, name)


# tiles of 128 x 128: one run, contractions in shares, dx and dW side by side
TILED = [(BF, 2048, 2048, 2048), (BF, 4096, 1024, 1024), (BF, 8192, 1024, 512), (BF, 256, 4096, 4096), (BF, 3000, 1100, 1064),
         (F32, 4096, 512, 1000), (F32, 300, 2048, 2052), (F32, 1300, 1100, 1060)]


@pytest.mark.parametrize("dtype,rows,d_in,d_out", TILED)
def test_linear_tiled(dtype, rows, d_in, d_out):
    x, w = rows_of(rows, d_in, dtype), rows_of(d_in, d_out, dtype, scale=d_in ** -0.5)
    b, r = torch.randn(d_out, device="cuda"), rows_of(rows, d_out, dtype)
    want, wz, sy, sz = ou.linear(x, w, b, SILU, r)
    y, z = lib.linear_forward(x, w, b, act=SILU, residual=r, keep_z=True, out=r)
    assert y is r
    ou.close(z, wz, sz, "z")
    ou.close(y, want, sy, "y over the residual")
    dy = rows_of(rows, d_out, dtype)
    want, slack = ou.linear_gradient(x, w, z, dy, SILU)
    got = lib.linear_backward(x, w, dy, act=SILU, z=z)
    for g, v, s, name in zip(got, want, slack, ("dx", "dw", "db")):
        ou.close(g, v, s, name)
    for needs in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 0)):
        some = lib.linear_backward(x, w, dy, act=SILU, z=z, need_dx=bool(needs[0]), need_dw=bool(needs[1]), need_db=bool(needs[2]))
        for g, v, s, need in zip(some, want, slack, needs):
            assert (g is not None) == bool(need)
            if need:
                ou.close(g, v, s, f"of {needs}")


def test_linear_of_no_rows():
    x, w = torch.empty(0, 24, device="cuda", dtype=BF), rows_of(24, 16, BF)
    assert lib.linear_forward(x, w).shape == (0, 16)
    dx, dw, db = lib.linear_backward(x, w, torch.empty(0, 16, device="cuda", dtype=BF))
    assert dx.shape == (0, 24) and (dw == 0).all() and (db == 0).all() and dw.shape == (24, 16)


@pytest.mark.parametrize("rows", [4, 140])
def test_linear_keeps_infinities_in_their_rows(rows):
    x, w = rows_of(rows, 100, BF), rows_of(100, 60, BF)
    x[1, 3], x[2, 99] = float("inf"), float("nan")
    y = lib.linear_forward(x, w, act=RELU)
    plain = x.double() @ w.double()
    assert torch.isnan(y[2]).all()
    assert torch.equal(torch.isinf(y[1]), torch.isinf(plain[1]) & (plain[1] > 0))
    keep = [i for i in range(rows) if i not in (1, 2)]
    want, _, sy, _ = ou.linear(x[keep], w, None, RELU, None)
    ou.close(y[keep], want, sy)


def test_linear_residual_in_place():
    x, w, r = rows_of(150, 64, BF), rows_of(64, 48, BF, scale=0.1), rows_of(150, 48, BF)
    want, _, sy, _ = ou.linear(x, w, None, SILU, r)
    got = lib.linear_forward(x, w, act=SILU, residual=r, out=r)
    assert got is r
    ou.close(r, want, sy)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_linear_offsets_beyond_32_bits(dtype):
    """x has more than 2^32 elements (bf16: bytes too): the last rows."""
    cols = 2048 if dtype == BF else 1024
    rows = (1 << 32) // cols + 130
    x = torch.zeros(rows, cols, dtype=dtype, device="cuda")
    x[-140:] = torch.randn(140, cols, device="cuda").to(dtype)
    w = rows_of(cols, 8, dtype, scale=0.02)
    y = lib.linear_forward(x, w)
    want, _, sy, _ = ou.linear(x[-140:], w, None, NONE, None)
    ou.close(y[-140:], want, sy)
    assert (y[:-140] == 0).all()
    dy = torch.zeros(rows, 8, dtype=dtype, device="cuda")
    dy[-140:] = torch.randn(140, 8, device="cuda").to(dtype)
    dx, dw, db = lib.linear_backward(x, w, dy)
    want, slack = ou.linear_gradient(x[-140:], w, torch.zeros_like(dy[-140:]), dy[-140:], NONE)
    ou.close(dx[-140:], want[0], slack[0])
    ou.close(dw, want[1], slack[1])
    ou.close(db, want[2], slack[2])


# n, positions, channels, groups: one value a group, odd groups, groups wider than a wavefront or a workgroup's lanes,
# one position and many, samples that fit a workgroup and that are cut into parts
NORMS = [(1, 1, 1, 1), (3, 1, 8, 8), (5, 1, 48, 4), (2, 7, 6, 2), (4, 9, 24, 6), (3, 196, 24, 6), (2, 49, 33, 11), (130, 1, 256, 32),
         (6, 1, 2048, 32), (7, 1, 2048, 1), (300, 1, 264, 1), (9, 1, 2 * 4096, 2), (2, 1, 32768, 1), (700, 1, 4096, 1), (3, 1, 2 * 5004, 2), (5, 1, 16384, 1), (2, 1, 32776, 1), (3, 1, 1143, 3), (2, 1, 1500, 1), (2, 3, 1500, 1), (1, 1, 40000, 2), (2, 64, 512, 8),
         (1, 1024, 64, 32), (2, 1000, 320, 32), (1, 5000, 8, 1), (3, 300, 130, 1), (1, 40000, 16, 4), (70, 33, 12, 3)]
# groups that are no whole number of pieces: partial pieces of one to three, one that is alone in a wavefront, samples cut into parts
PARTIAL = [(3, 50, 10, 2), (2, 300, 69, 1), (2, 40, 771, 3), (1, 3000, 85, 5), (2, 9000, 7, 1), (5, 1, 4099, 1), (9, 1, 129, 3),
           (2, 20000, 14, 2), (40, 1, 9, 3), (1, 700, 1030, 2), (70, 1, 133, 1), (6, 1, 2 * 1027, 2), (3, 1, 16381, 1)]
NORMS += PARTIAL


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,S,C,G", NORMS)
def test_group_norm_forward(n, S, C, G, dtype):
    x = (torch.randn(n, S, C, device="cuda") * (0.5 + torch.rand(C, device="cuda")) + torch.randn(C, device="cuda")).to(dtype)
    gamma, beta = 1 + 0.3 * torch.randn(C, device="cuda"), 0.3 * torch.randn(C, device="cuda")
    for a in (NONE, RELU, SILU, GELU):
        got = lib.group_norm_forward(x, gamma, beta, G, act=a)
        for g, v, s, name in zip(got, *ou.norm(x, gamma, beta, G, 1e-5, a), ("y", "mean", "rstd")):
            ou.close(g, v, s, f"{name}, act {a}")
    got = lib.group_norm_forward(x, None, None, G, eps=1e-3)
    for g, v, s in zip(got, *ou.norm(x, None, None, G, 1e-3, NONE)):
        ou.close(g, v, s)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,S,C,G", NORMS)
def test_group_norm_backward(n, S, C, G, dtype):
    x = (torch.randn(n, S, C, device="cuda") + torch.randn(C, device="cuda")).to(dtype)
    gamma, beta = 1 + 0.3 * torch.randn(C, device="cuda"), 0.3 * torch.randn(C, device="cuda")
    dy, res = torch.randn(n, S, C, device="cuda").to(dtype), torch.randn(n, S, C, device="cuda").to(dtype)
    _, mean, rstd = lib.group_norm_forward(x, gamma, beta, G)
    for a, r in ((NONE, None), (SILU, res), (GELU, None)):
        got = lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=a, residual=r)
        for g, v, s, name in zip(got, *ou.norm_gradient(x, gamma, beta, mean, rstd, dy, r, a), ("dx", "dgamma", "dbeta")):
            ou.close(g, v, s, f"{name}, act {a}")
    # relu: the side of the corner is that of fma(x - mean, gamma rstd, beta), both factors rounded to fp32 (a product of two is exact in fp64)
    got = lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=RELU)
    wide = lambda t: t.repeat_interleave(C // G, 1)[:, None, :]
    h = (x.float() - wide(mean)).double() * (wide(rstd) * gamma).double() + beta.double()
    masked = dy * (h > 0)
    for g, v, s, name in zip(got, *ou.norm_gradient(x, gamma, beta, mean, rstd, masked, None, NONE), ("dx", "dgamma", "dbeta")):
        ou.close(g, v, s, f"{name}, relu")
    dx, dgamma, dbeta = lib.group_norm_backward(x, None, None, mean, rstd, dy, need_dgamma=False)
    want, slack = ou.norm_gradient(x, None, None, mean, rstd, dy, None, NONE)
    ou.close(dx, want[0], slack[0])
    assert dgamma is None and dbeta is None


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,S,pad,lead", [(3, 50, 8, 0), (3, 50, 1, 0), (2, 1, 8, 1), (1, 9000, 4, 0)])
def test_group_norm_pitches_and_starts(n, S, pad, lead, dtype):
    C, G = 32, 8
    x, dy, res = (rows_of(n * S, C, dtype, pad, 1.0, lead).unflatten(0, (n, S)) for _ in range(3))
    gamma, beta = 1 + 0.3 * torch.randn(C, device="cuda"), 0.3 * torch.randn(C, device="cuda")
    flat = torch.full((lead + n * S * (C + pad),), 7.0, dtype=dtype, device="cuda")
    out = flat[lead:].view(n, S, C + pad)
    got = lib.group_norm_forward(x, gamma, beta, G, act=SILU, out=out[:, :, :C])
    for g, v, s in zip(got, *ou.norm(x, gamma, beta, G, 1e-5, SILU)):
        ou.close(g, v, s)
    assert (out[:, :, C:] == 7).all() and (flat[:lead] == 7).all()
    got = lib.group_norm_backward(x, gamma, beta, got[1], got[2], dy, act=SILU, residual=res, out=res)
    assert got[0] is res


def test_group_norm_in_place_and_images():
    x = torch.randn(2, 5, 7, 24, device="cuda")                       # [n, height, width, channels]
    gamma, beta = torch.randn(24, device="cuda"), torch.randn(24, device="cuda")
    y, mean, rstd = lib.group_norm_forward(x, gamma, beta, 4, act=RELU)
    same, _, _ = lib.group_norm_forward(x.view(2, 35, 24), gamma, beta, 4, act=RELU)
    assert torch.equal(y.view(2, 35, 24), same)
    dy, res = torch.randn_like(x), torch.randn_like(x)
    dx, _, _ = lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=SILU, residual=res)
    got, _, _ = lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=SILU, residual=res, out=res)
    assert torch.equal(got, dx) and got is res
    assert torch.equal(lib.group_norm_forward(x, gamma, beta, 4, act=RELU, out=x)[0], y) and torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,S,C,G", PARTIAL)
def test_group_norm_in_place_partial_pieces(n, S, C, G, dtype):
    x, dy, res = (torch.randn(n, S, C, device="cuda").to(dtype) for _ in range(3))
    gamma, beta = torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    y, mean, rstd = lib.group_norm_forward(x, gamma, beta, G, act=SILU)
    dx, dgamma, dbeta = lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=SILU, residual=res)
    got = lib.group_norm_backward(x, gamma, beta, mean, rstd, dy, act=SILU, residual=res, out=res)
    assert torch.equal(got[0], dx) and got[0] is res and torch.equal(got[1], dgamma) and torch.equal(got[2], dbeta)
    lib.group_norm_forward(x, gamma, beta, G, act=SILU, out=x)
    assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("C,G", [(10, 2), (69, 1), (771, 3), (9, 3)])
def test_group_norm_partial_pieces_stay_inside(C, G, dtype):
    """Rows in longer rows whose other columns are NaN, the first one at the start of its memory, the last one at its end."""
    n, S = 2, 37
    flat = [torch.full((n * S * (C + 5) - 5,), float("nan"), dtype=dtype, device="cuda") for _ in range(4)]
    x, dy, res, out = (f.as_strided((n, S, C), (S * (C + 5), C + 5, 1)) for f in flat)
    for v in (x, dy, res):
        v.copy_(torch.randn(n, S, C, device="cuda"))
    gamma, beta = 1 + 0.3 * torch.randn(C, device="cuda"), 0.3 * torch.randn(C, device="cuda")
    got = lib.group_norm_forward(x, gamma, beta, G, act=SILU, out=out)
    for g, v, s in zip(got, *ou.norm(x, gamma, beta, G, 1e-5, SILU)):
        ou.close(g, v, s)
    grads = lib.group_norm_backward(x, gamma, beta, got[1], got[2], dy, act=SILU, residual=res, out=out)
    for g, v, s in zip(grads, *ou.norm_gradient(x, gamma, beta, got[1], got[2], dy, res, SILU)):
        ou.close(g, v, s)
    rest = torch.ones_like(flat[3], dtype=torch.bool)
    rest.as_strided((n, S, C), (S * (C + 5), C + 5, 1)).fill_(False)
    assert torch.isnan(flat[3][rest]).all()


def test_group_norm_far_from_zero():
    """Values 1000 spreads from zero: the variance is about the mean, nothing cancels."""
    x = torch.randn(4, 333, 64, device="cuda") + 1000.0
    got = lib.group_norm_forward(x, None, None, 8)
    for g, v, s in zip(got, *ou.norm(x, None, None, 8, 1e-5, NONE)):
        ou.close(g, v, s)


def test_group_norm_constant_groups_and_infinities():
    x = torch.full((3, 10, 16), 2.5, device="cuda")
    y, mean, rstd = lib.group_norm_forward(x, None, None, 4)
    assert (y == 0).all() and (mean == 2.5).all()
    ou.close(rstd, torch.full((3, 4), 1e-5, dtype=torch.float64) ** -0.5, 1e-4)        # (2 ulp of 316, and eps' own rounding)
    x[1, 4, 5] = float("inf")
    y, _, _ = lib.group_norm_forward(x, None, None, 4)
    bad = torch.zeros(3, 4, dtype=torch.bool, device="cuda")
    bad[1, 1] = True
    assert torch.equal(torch.isnan(y.view(3, 10, 4, 4)).any(dim=3).any(dim=1), bad) and (y[0] == 0).all()


def test_group_norm_of_no_samples():
    x = torch.empty(0, 4, 8, device="cuda")
    y, mean, rstd = lib.group_norm_forward(x, None, None, 2)
    assert y.shape == x.shape and mean.shape == (0, 2)
    dx, dg, db = lib.group_norm_backward(x, None, None, mean, rstd, x)
    assert (dg == 0).all() and (db == 0).all() and dg.shape == (8,)


def test_group_norm_offsets_beyond_32_bits():
    n, S, C = 260, 64 * 64, 4096                      # 2^32 elements and some
    x = torch.zeros(n, S, C, dtype=BF, device="cuda")
    x[-1] = torch.randn(S, C, device="cuda").to(BF)
    y, mean, rstd = lib.group_norm_forward(x, None, None, 32)
    for g, v, s in zip((y[-1:], mean[-1:], rstd[-1:]), *ou.norm(x[-1:], None, None, 32, 1e-5, NONE)):
        ou.close(g, v, s)
    assert (y[:-1] == 0).all()
    del y
    dx, dg, db = lib.group_norm_backward(x, None, None, mean, rstd, x)
    want, slack = ou.norm_gradient(x[-1:], None, None, mean[-1:], rstd[-1:], x[-1:], None, NONE)
    ou.close(dx[-1:], want[0], slack[0])
    ou.close(dg, want[1], slack[1])


DROPS = [(1, 1), (1, 7), (1, 4096), (5, 3), (7, 64), (33, 130), (810, 300), (64, 8), (3, 1)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", DROPS)
@pytest.mark.parametrize("pad,lead", [(0, 0), (8, 0), (1, 0), (0, 1)])
def test_dropout(rows, cols, pad, lead, dtype):
    x, r = rows_of(rows, cols, dtype, pad, 1.0, lead), rows_of(rows, cols, dtype, pad, 1.0, lead)
    for drop, seed, offset in ((0, 1, 2), (6554, 2 ** 63 + 5, 3), (32768, 77, 2 ** 40 + 9), (65535, 3, 0)):
        keep = lib.dropout_kept(rows, cols, drop, seed, offset).cuda().bool()
        want = torch.where(keep, x.double() * 65536 / (65536 - drop), 0.0)
        y = lib.dropout_forward(x, drop, seed, offset)
        ou.close(y, want, 2 * ou.U * want.abs())
        assert torch.equal(lib.dropout_backward(x, drop, seed, offset), y)
        flat = torch.full((lead + rows * (cols + pad),), 7.0, dtype=dtype, device="cuda")
        out = flat[lead:].view(rows, cols + pad)
        y = lib.dropout_forward(x, drop, seed, offset, residual=r, out=out[:, :cols])
        ou.close(y, want + r.double(), 2 * ou.U * want.abs() + ou.U * (want.abs() + r.double().abs()))
        assert (out[:, cols:] == 7).all() and (flat[:lead] == 7).all()


def test_dropout_drops_infinities():
    x = torch.full((4, 64), float("inf"), device="cuda")
    x[1] = float("nan")
    keep = lib.dropout_kept(4, 64, 30000, 5, 6).cuda().bool()
    y = lib.dropout_forward(x, 30000, 5, 6)
    assert (y[~keep] == 0).all() and torch.isinf(y[0][keep[0]]).all() and torch.isnan(y[1][keep[1]]).all()


def test_dropout_in_place_and_pitch_free():
    x = torch.randn(40, 24, device="cuda").to(BF)
    y = lib.dropout_forward(x, 20000, 1, 1)
    wide = torch.zeros(40, 31, dtype=BF, device="cuda")
    wide[:, :24] = x
    assert torch.equal(lib.dropout_forward(wide[:, :24], 20000, 1, 1), y)           # the mask goes by the element, not the pitch
    r = torch.randn(40, 24, device="cuda").to(BF)
    s = lib.dropout_forward(x, 20000, 1, 1, residual=r)
    assert torch.equal(lib.dropout_forward(x, 20000, 1, 1, residual=r, out=r), s)
    assert torch.equal(lib.dropout_forward(x, 20000, 1, 1, out=x), y)
    assert not torch.equal(lib.dropout_forward(x, 20000, 1, 2), lib.dropout_forward(x, 20000, 1, 3))


def test_dropout_offsets_beyond_32_bits():
    rows, cols = 2 ** 20 + 3, 4096
    x = torch.ones(rows, cols, dtype=BF, device="cuda")
    y = lib.dropout_forward(x, 16384, 9, 9)
    from oracle import counter_rng as crng
    key = crng.mix64(crng.mix64(9 + 3 * crng.GOLDEN_GAMMA) ^ 9)
    want = []
    for e in range(rows * cols - 64, rows * cols):
        bits = crng.mix64(key + crng.GOLDEN_GAMMA * (e // 4 + 1)) >> (16 * (e % 4)) & 0xFFFF
        want.append(bits >= 16384)
    assert (y.view(-1)[-64:] != 0).tolist() == want
    assert abs((y != 0).float().mean(dim=1).double().mean().item() - 0.75) < 1e-4      # 4e9 draws: 6e-6 is a standard deviation
    z = lib.dropout_forward(x[:, 1:], 16384, 9, 9)                                      # unaligned: one by one
    n = rows * (cols - 1)
    key_bits = [crng.mix64(key + crng.GOLDEN_GAMMA * (e // 4 + 1)) >> (16 * (e % 4)) & 0xFFFF for e in range(n - 64, n)]
    assert (z.reshape(-1)[-64:] != 0).tolist() == [b >= 16384 for b in key_bits]


# ---- together, as a residual block uses them --------------------------------------------------------------
class Block:
    """a -> a + dropout(act(norm(a))) W + b, and the head's product; forward and backward by the package's calls."""

    def __init__(self, rows, d, groups, dtype):
        self.a = torch.randn(rows, d, device="cuda").to(dtype)
        self.gamma, self.beta = 1 + 0.2 * torch.randn(d, device="cuda"), 0.2 * torch.randn(d, device="cuda")
        self.w, self.b = (torch.randn(d, d, device="cuda") * d ** -0.5).to(dtype), 0.1 * torch.randn(d, device="cuda")
        self.dy = torch.randn(rows, d, device="cuda").to(dtype)
        self.groups = groups

    def run(self, drop=6554, seed=4, offset=9):
        n, mean, rstd = lib.group_norm_forward(self.a[:, None], self.gamma, self.beta, self.groups, act=SILU)
        u = lib.dropout_forward(n[:, 0], drop, seed, offset)
        y = lib.linear_forward(u, self.w, self.b, residual=self.a)
        du, dw, db = lib.linear_backward(u, self.w, self.dy)
        dn = lib.dropout_backward(du, drop, seed, offset)
        da, dg, dbt = lib.group_norm_backward(self.a[:, None], self.gamma, self.beta, mean, rstd, dn[:, None], act=SILU,
                                              residual=self.dy[:, None])
        return [y, da[:, 0], dw, db, dg, dbt]

    def plain(self, drop=6554, seed=4, offset=9):
        rows, d = self.a.shape
        leaves = [t.double().cpu().requires_grad_() for t in (self.a, self.w, self.b, self.gamma, self.beta)]
        a, w, b, gamma, beta = leaves
        v = a.view(rows, self.groups, -1)
        h = ((v - v.mean(2, keepdim=True)) / torch.sqrt(v.var(2, unbiased=False, keepdim=True) + 1e-5)).reshape(rows, d) * gamma + beta
        keep = lib.dropout_kept(rows, d, drop, seed, offset).bool()
        u = torch.where(keep, ou.act(h, SILU) * 65536 / (65536 - drop), 0.0)
        y = a + u @ w + b
        y.backward(self.dy.double().cpu())
        return [y.detach()] + [t.grad for t in (a, w, b, gamma, beta)]


@pytest.mark.parametrize("rows,d,groups", [(1, 64, 8), (37, 96, 4), (512, 256, 32)])
def test_block_fp32_gradients(rows, d, groups):
    """fp32: every intermediate carries a few roundings; 2^-24 times the longest sum's length (256 products, then 512 rows) stays
    below 1e-4 of a tensor's largest element."""
    blk = Block(rows, d, groups, F32)
    for got, want in zip(blk.run(), blk.plain()):
        assert (got.double().cpu() - want).abs().max() <= 1e-4 * want.abs().max()


def test_block_bf16_gradients():
    """bf16: seven roundings of 2^-9 of a value (2^-8 at most) along the way into the last gradient, in the norm of a tensor."""
    blk = Block(300, 128, 16, BF)
    for got, want in zip(blk.run(), blk.plain()):
        assert (got.double().cpu() - want).norm() <= 7 * 2.0 ** -8 * want.norm()


def test_block_gradients_against_differences():
    """Central differences of the block's own forward pass in fp32 along random directions.  With a step h of 2^-6 of a unit direction's
    elements the difference's own error is h^2 / 6 times a third derivative (a few) and 2^-24 |loss| / h."""
    blk = Block(24, 64, 8, F32)
    grads = blk.run()

    def loss():
        return (blk.run()[0].double() * blk.dy.double()).sum()

    for leaf, grad in ((blk.a, grads[1]), (blk.w, grads[2]), (blk.b, grads[3]), (blk.gamma, grads[4]), (blk.beta, grads[5])):
        way = torch.randn_like(leaf)
        way /= way.norm()
        h = 2.0 ** -6
        keep = leaf.clone()
        leaf.copy_(keep + h * way)
        up = loss()
        leaf.copy_(keep - h * way)
        down = loss()
        leaf.copy_(keep)
        want = ((up - down) / (2 * h)).item()
        got = (grad.double() * way.double()).sum().item()
        scale = grad.double().norm().item()
        assert abs(got - want) <= 2e-3 * scale + 1e-3, (got, want, scale)


@pytest.mark.parametrize("rows,d,groups,dtype", [(6, 128, 8, BF), (700, 264, 33, BF), (300, 96, 4, F32)])
def test_two_runs_give_the_same_bits_on_any_stream(rows, d, groups, dtype):
    blk = Block(rows, d, groups, dtype)
    first = blk.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = blk.run()
    torch.cuda.current_stream().wait_stream(side)
    for p, q in zip(first, second):
        assert torch.equal(p, q)


def test_two_threads_on_two_streams():
    """Calls of both at once, each with workspaces of its own: the bits of calls one after the other."""
    blocks = [Block(1500, 1032, 24, BF), Block(700, 516, 12, F32)]
    want = [blk.run() for blk in blocks]
    torch.cuda.synchronize()
    got, wrong = [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    got[i] = blocks[i].run()
                torch.cuda.current_stream().synchronize()
        except Exception as e:                                     # (reported in the test's own thread)
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not wrong, wrong
    for a, b in zip(got, want):
        for p, q in zip(a, b):
            assert torch.equal(p, q)


@pytest.mark.parametrize("rows,d,groups,dtype", [(260, 128, 16, BF), (2100, 1024, 16, BF), (1200, 1028, 4, F32)])
def test_captured_and_replayed(rows, d, groups, dtype):
    """Forward and backward of a block in a graph: every replay on new inputs gives the eager call's bits, with eager work between."""
    blk = Block(rows, d, groups, dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        blk.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = blk.run()
    for i in range(4):
        blk.a.copy_(torch.randn(rows, d, device="cuda"))
        blk.dy.copy_(torch.randn(rows, d, device="cuda"))
        want = blk.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(got, want):
            assert torch.equal(p, q), i
