"""The element-wise bounds of the distillation's gradient reject what a broken kernel would leave: zeros, rows moved by a vector, another row's gradient, a class left without
its teacher's entry."""
import numpy as np
import pytest

import distill_bounds as B


def row_inputs(rows, classes, k, seed):
    g = np.random.default_rng(seed)
    z = (g.standard_normal((rows, classes)) * 3).astype(np.float32).astype(float)
    ids = np.stack([g.choice(classes, k, replace=False) for _ in range(rows)])
    t = (g.standard_normal((rows, k)) * 3).astype(np.float32).astype(float)
    return z, t, ids, g.random(rows) + 0.5


@pytest.mark.parametrize("half_step", [2.0 ** -8, 2.0 ** -24])
@pytest.mark.parametrize("classes,k", [(100, 7), (2049, 129), (50304, 64), (160001, 8)])
@pytest.mark.parametrize("from_lse", [False, True])
def test_wrong_gradients_are_outside(classes, k, half_step, from_lse):
    z, t, ids, weight = row_inputs(2, classes, k, 1)
    want, bound = B.gradient(z, t, ids, weight, 2.0, 0.5, half_step, from_lse)
    assert (bound < 0.02 * np.abs(want).clip(1e-12) + 1e-3 * bound.max()).all()

    def outside(wrong):
        return (np.abs(wrong - want) > bound).mean()
    assert outside(np.zeros_like(want)) == 1.0
    assert outside(want * 0.98) > 0.999
    assert outside(np.roll(want, 8, axis=1)) > 0.95                 # neighbours a few steps of the type apart may look alike
    assert outside(want[::-1]) > 0.95
    without = want.copy()
    without[0, ids[0, 0]] = weight[0] * B.parts(z, t, ids, 2.0)[0][0, ids[0, 0]]
    assert (np.abs(without - want) > bound).sum() == 1


def test_the_formula_in_fp32_is_inside():
    """The kernel's arithmetic, one rounding after the other, in numpy's fp32."""
    f = np.float32
    z, t, ids, weight = row_inputs(3, 5000, 20, 2)
    for temp in (0.5, 1.0, 2.0):
        want, bound = B.gradient(z, t, ids, weight, temp, 0.25, 2.0 ** -24, False)
        c2 = f(1.44269504) / f(temp)
        for r in range(3):
            x, v = z[r].astype(f), t[r].astype(f)
            m = x.max()
            e = np.exp2((x - m) * c2)
            total = np.add.reduce(e.reshape(-1, 8).cumsum(0, dtype=f)[-1], dtype=f)
            q = np.exp2((x - m) * c2 - np.log2(total))
            p = np.exp2((v - v.max()) * c2)
            p = p * (f(1) / p.sum(dtype=f))
            coef = f(0.25) * f(weight[r]) * f(temp)
            got = coef * q
            got[ids[r]] = coef * (q[ids[r]] - p)
            # (5000 / 8 additions in a row here, for the 104 + 45 of the bound: weights of fp32 beside them)
            assert (np.abs(got - want[r]) <= bound[r] + 2.0 ** -24 * 1200 * np.abs(want[r])).all()
