"""The oracle's residual-block MLP: its gradient against differences of its loss (no rounding), its mask against the plain
counter draws."""
import numpy as np
import pytest

from oracle import blocks as ob
from oracle import counter_rng as crng


@pytest.mark.parametrize("act,residual,drop", [(2, 1, 20000), (3, 0, 0), (0, 1, 6554)])
def test_gradient_is_the_derivative(act, residual, drop):
    rng = np.random.default_rng(5)
    dims, opt = [6, 8, 8, 4], dict(groups=2, act=act, residual=residual, drop=drop, eps=1e-5)
    n = sum(dims[l] * dims[l + 1] + dims[l + 1] + (2 * dims[l] if l else 0) for l in range(3))
    w, X, y = rng.standard_normal(n) * 0.5, rng.standard_normal((5, 6)), rng.integers(0, 4, 5)
    coef = rng.uniform(0.1, 1, 5)
    masks = [None] + [ob.kept(5, dims[l], drop, 3, l) for l in (1, 2)]
    same = lambda v: v
    g, _ = ob.gradient(dims, opt, w, X, y, coef, masks, same)

    def f(v):
        return (coef * ob.loss_of(ob.forward(dims, opt, v, X, masks, same)[0], y)[0]).sum()

    for i in rng.integers(0, n, 25):
        h = 1e-5
        e = np.zeros(n)
        e[i] = h
        assert abs((f(w + e) - f(w - e)) / (2 * h) - g[i]) <= 1e-6 * max(1, abs(g[i]))


def test_mask_is_the_counter_draws():
    got = ob.kept(3, 7, 30000, 9, 4)
    key = crng.mix64(crng.mix64(9 + 3 * crng.GOLDEN_GAMMA) ^ 4)
    for e in range(21):
        bits = crng.mix64(key + crng.GOLDEN_GAMMA * (e // 4 + 1)) >> (16 * (e % 4)) & 0xFFFF
        assert got[e // 7, e % 7] == (bits >= 30000)
