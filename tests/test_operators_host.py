"""What the operators of a network's hidden layers refuse, and the dropout mask's draws: no GPU needed (a refused call
makes no HIP call, so made-up addresses do)."""
import ctypes as C

import pytest
import torch

import paper_2301_08895_amd as lib
from paper_2301_08895_amd.binding import AbsLinear, AbsGroupNorm, AbsDropout, _lib
from oracle import counter_rng as crng

P = 1 << 20                 # an address that nothing reads


def _linear(**over):
    p = AbsLinear(dtype=1, act=0, rows=4, d_in=16, d_out=8, ldx=16, ldw=8, ldy=8, ldz=8, ldr=8, lddy=8, lddx=16, lddw=8)
    for k, v in over.items():
        setattr(p, k, v)
    return p


def _norm(**over):
    p = AbsGroupNorm(dtype=1, act=0, n=2, spatial=3, channels=8, groups=2, eps=1e-5, ldx=8, ldy=8, lddy=8, lddx=8, lddres=8)
    for k, v in over.items():
        setattr(p, k, v)
    return p


def _drop(**over):
    p = AbsDropout(dtype=0, drop=100, rows=4, cols=8, ldx=8, ldy=8, ldr=8, seed=1, offset=2)
    for k, v in over.items():
        setattr(p, k, v)
    return p


def _text():
    return lib.abs_last_error(None)


@pytest.mark.parametrize("over", [dict(dtype=2), dict(dtype=-1), dict(act=4), dict(act=-1), dict(rows=-1), dict(rows=1 << 31),
                                  dict(d_in=0), dict(d_out=0), dict(d_in=(1 << 20) + 1, ldx=1 << 21), dict(ldx=15), dict(ldw=7),
                                  dict(ldx=1 << 32), dict(rows=1 << 30, d_out=1 << 20, ldw=1 << 20)])
def test_linear_refuses(over):
    p = _linear(**over)
    assert _lib.abs_linear_workspace_size(C.byref(p), 0, 1) == 0 and "linear" in _text()
    assert _lib.abs_linear_forward(C.byref(p), P, P, None, None, P, None, P, 1 << 40, None) == -1
    assert _lib.abs_linear_backward(C.byref(p), P, P, P, P, P, P, P, P, 1 << 40, None) == -1


def test_linear_refuses_pointers_and_pitches():
    ok = _linear()
    f, b = _lib.abs_linear_forward, _lib.abs_linear_backward
    big = 1 << 40
    assert f(None, P, P, None, None, P, None, P, big, None) == -1
    assert f(C.byref(ok), None, P, None, None, P, None, P, big, None) == -1
    assert f(C.byref(ok), P, None, None, None, P, None, P, big, None) == -1
    assert f(C.byref(ok), P, P, None, None, None, None, P, big, None) == -1
    assert f(C.byref(ok), P + 1, P, None, None, P, None, P, big, None) == -1          # half an element
    assert f(C.byref(ok), P, P, P + 2, None, P, None, P, big, None) == -1             # the bias is fp32
    assert f(C.byref(_linear(ldy=7)), P, P, None, None, P, None, P, big, None) == -1
    assert f(C.byref(_linear(ldz=7)), P, P, None, None, P, P, P, big, None) == -1
    assert f(C.byref(_linear(ldr=7)), P, P, None, P, P, None, P, big, None) == -1
    wide = _linear(rows=40000, d_in=511, d_out=512, ldx=512, ldw=512, ldy=512)
    need = _lib.abs_linear_workspace_size(C.byref(wide), 0, 1)
    assert f(C.byref(wide), P, P, None, None, P, None, P, need - 1, None) == -2
    assert f(C.byref(wide), P, P, None, None, P, None, None, need, None) == -1
    assert f(C.byref(wide), P, P, None, None, P, None, P + 16, need, None) == -1
    assert b(C.byref(_linear(act=2)), P, P, None, P, P, P, P, P, big, None) == -1      # an activation without z
    assert b(C.byref(ok), P, P, None, None, P, P, P, P, big, None) == -1
    assert b(C.byref(ok), None, P, None, P, P, P, P, P, big, None) == -1               # dW needs x
    assert b(C.byref(ok), P, None, None, P, P, P, P, P, big, None) == -1               # dx needs W
    for name in ("lddy", "lddx", "lddw"):
        assert b(C.byref(_linear(**{name: 7})), P, P, None, P, P, P, P, P, big, None) == -1
    wide = _linear(rows=40000, d_in=512, d_out=512, ldx=512, ldw=512, lddy=512, lddx=512, lddw=512)
    need = _lib.abs_linear_workspace_size(C.byref(wide), 1, 1)
    assert need > 0 and b(C.byref(wide), P, P, None, P, P, P, P, P, need - 1, None) == -2


def test_linear_workspace_counts_copies_of_ragged_rows():
    size = lambda back, aligned, **over: _lib.abs_linear_workspace_size(C.byref(_linear(**over)), back, aligned)
    big = dict(rows=40000, d_in=512, d_out=512, ldx=512, ldw=512)
    assert size(0, 1, **big) == 0                                 # read in place
    assert size(0, 0, **big) >= 40000 * 512 * 2                   # a start that is not a whole piece: a copy
    assert size(0, 1, **dict(big, d_in=511)) >= 40000 * 512 * 2   # nor is a row's length
    assert size(0, 1) == 0 and size(1, 0, d_in=15) == 0           # small products: operands at any alignment, one launch
    assert size(0, 1, rows=0) == 0 and size(1, 1, rows=0) == 0


@pytest.mark.parametrize("over", [dict(dtype=2), dict(act=9), dict(n=-1), dict(spatial=0), dict(n=1 << 20, spatial=1 << 12), dict(channels=0),
                                  dict(groups=0), dict(groups=3), dict(groups=16), dict(eps=-1.0), dict(eps=float("nan")),
                                  dict(eps=float("inf")), dict(ldx=7), dict(reserved=1), dict(channels=1 << 21, ldx=1 << 21)])
def test_group_norm_refuses(over):
    p = _norm(**over)
    assert _lib.abs_group_norm_workspace_size(C.byref(p), 0) == 0 and "group norm" in _text()
    assert _lib.abs_group_norm_forward(C.byref(p), P, P, P, P, P, P, P, 1 << 40, None) == -1
    assert _lib.abs_group_norm_backward(C.byref(p), P, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == -1


def test_group_norm_refuses_pointers_and_pitches():
    f, b, big = _lib.abs_group_norm_forward, _lib.abs_group_norm_backward, 1 << 40
    ok = _norm()
    assert f(C.byref(ok), None, P, P, P, P, P, P, big, None) == -1
    assert f(C.byref(ok), P, P, None, P, P, P, P, big, None) == -1
    assert f(C.byref(ok), P, P, P, P, P, None, P, big, None) == -1
    assert f(C.byref(ok), P, P, P, P + 1, P, P, P, big, None) == -1
    assert f(C.byref(ok), P, P + 2, P, P, P, P, P, big, None) == -1
    assert f(C.byref(_norm(ldy=7)), P, P, P, P, P, P, P, big, None) == -1
    many = _norm(n=5000)
    need = _lib.abs_group_norm_workspace_size(C.byref(many), 1)
    assert need > 0
    args = lambda p, at, n, dres=None: (C.byref(p), P, P, P, P, P, P, dres, P, P, P, at, n, None)
    assert b(*args(many, P, need - 1)) == -2
    assert b(*args(many, None, need)) == -1
    assert b(*args(_norm(lddres=7), P, big, P)) == -1
    assert b(*args(_norm(lddy=7), P, big)) == -1
    assert b(*args(_norm(lddx=7), P, big)) == -1
    assert b(C.byref(ok), P, P, P, P, P, P, None, P, P, None, P, big, None) == -1
    assert b(C.byref(ok), P, P, P, None, P, P, None, P, P, P, P, big, None) == -1


@pytest.mark.parametrize("over", [dict(dtype=2), dict(drop=-1), dict(drop=65536), dict(rows=-1), dict(cols=0), dict(ldx=7), dict(ldy=7),
                                  dict(rows=1 << 39), dict(rows=1 << 20, cols=1 << 20, ldx=1 << 20, ldy=1 << 20)])
def test_dropout_refuses(over):
    p = _drop(**over)
    assert _lib.abs_dropout_forward(C.byref(p), P, None, P, None) == -1 and "dropout" in _text()
    assert _lib.abs_dropout_backward(C.byref(p), P, P, None) == -1


def test_dropout_refuses_pointers():
    assert _lib.abs_dropout_forward(None, P, None, P, None) == -1
    assert _lib.abs_dropout_forward(C.byref(_drop()), None, None, P, None) == -1
    assert _lib.abs_dropout_forward(C.byref(_drop()), P, None, None, None) == -1
    assert _lib.abs_dropout_forward(C.byref(_drop()), P + 2, None, P, None) == -1
    assert _lib.abs_dropout_forward(C.byref(_drop(ldr=7)), P, P, P, None) == -1


def test_dropout_mask_is_the_oracles_draws():
    for rows, cols, drop, seed, offset in ((3, 7, 20000, 5, 9), (1, 130, 6554, 2 ** 64 - 1, 2 ** 63), (4, 1, 65535, 0, 0), (2, 9, 0, 1, 1)):
        key = crng.mix64(crng.mix64(seed + 3 * crng.GOLDEN_GAMMA) ^ offset)
        want = [int((crng.mix64(key + crng.GOLDEN_GAMMA * (e // 4 + 1)) >> (16 * (e % 4)) & 0xFFFF) >= drop) for e in range(rows * cols)]
        assert lib.dropout_kept(rows, cols, drop, seed, offset).flatten().tolist() == want


def test_dropout_rate_and_independence():
    a, b = (lib.dropout_kept(1000, 1000, 19661, 3, o).double() for o in (0, 1))
    # a million draws: a standard deviation of the rate is 4.6e-4, of the products' mean the same
    assert abs(a.mean() - (1 - 19661 / 65536)) < 3e-3
    assert abs(((a - a.mean()) * (b - b.mean())).mean()) < 1.5e-3
    assert abs(((a[:, :-1] - a.mean()) * (a[:, 1:] - a.mean())).mean()) < 1.5e-3


def test_tensors_off_the_gpu_and_wrong_numbers_are_refused():
    x, w = torch.zeros(2, 8), torch.zeros(8, 4)
    for call in (lambda: lib.linear_forward(x, w), lambda: lib.linear_backward(x, w, torch.zeros(2, 4)),
                 lambda: lib.group_norm_forward(x, None, None, 2), lambda: lib.dropout_forward(x, 1, 1, 1),
                 lambda: lib.dropout_backward(x, 1, 1, 1), lambda: lib.dropout_kept(2, 2, 65536, 1, 1),
                 lambda: lib.dropout_kept(2, 2, 2 ** 32, 1, 1), lambda: lib.dropout_kept(2, 2, 0.5, 1, 1)):
        with pytest.raises(lib.AbsError) as e:
            call()
        assert e.value.code == -1


def test_structs_match_the_library():
    # (abs_linear: two 32-bit and ten 64-bit words and two more; the sizes the header's layouts give)
    assert C.sizeof(AbsLinear) == 8 + 8 + 8 + 8 * 8 and C.sizeof(AbsGroupNorm) == 8 + 16 + 16 + 40 and C.sizeof(AbsDropout) == 8 + 7 * 8


def _blocks_preset(**over):
    import workloads
    p = workloads.scaled_preset(3, M=400, dims=[16, 24, 24, 4], N=4, B=8, n_slow=1, k_mode=1)
    q = workloads.with_blocks(p, groups=8)
    q["blocks"].update({k: v for k, v in over.items() if k in q["blocks"]})
    q.update({k: v for k, v in over.items() if k not in q["blocks"]})
    return q


@pytest.mark.parametrize("over", [dict(groups=0), dict(groups=7), dict(act=4), dict(residual=2), dict(drop=65536), dict(drop=-1),
                                  dict(eps=0.0), dict(eps=float("nan")), dict(U=2), dict(N=0)])
def test_blocks_refuse(over):
    p = _blocks_preset(**over)
    with pytest.raises(lib.AbsError) as e:
        lib.Simulation(p, None, device_mode=0)
    assert e.value.code == -1
    with pytest.raises(lib.AbsError):
        lib.abs_blocks_workspace_size(lib.make_config(p), lib.make_blocks(p["blocks"]))


def test_blocks_follow_the_same_schedule_and_count_their_parameters():
    import numpy as np
    import workloads
    p = _blocks_preset()
    sim = lib.Simulation(p, None, device_mode=0)
    plain = lib.Simulation({k: v for k, v in p.items() if k != "blocks"}, None, device_mode=0)
    for s in (sim, plain):
        s.round(20)
    a, b = sim.trace(), plain.trace()
    a[:, 10] = b[:, 10] = 0                    # the loss word: there are no losses without a device
    assert np.array_equal(a, b)
    assert workloads.param_count(p) == workloads.make_inputs(p)["w0"].size == 16 * 24 + 24 + 48 + 24 * 24 + 24 + 48 + 24 * 4 + 4
    size = lambda q: lib.abs_blocks_workspace_size(lib.make_config(q), lib.make_blocks(q["blocks"]))
    assert 0 < size(p) < size(dict(p, N=8)) < size(dict(p, N=8, tau_cap=12))
    for s in (sim, plain):
        s.close()
