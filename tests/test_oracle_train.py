"""Pins of the 64-bit operators of a policy update: gradients against differences of the forward value, codes against a search over all of them."""
import numpy as np
import pytest

from oracle import train


def slope(f, x, d, h=1e-5):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


@pytest.mark.parametrize("lq,lk", [((3, 1, 5), (4, 0, 2)), ((2,), (7,))])
def test_attention_gradients_are_the_slopes_of_the_output(lq, lk):
    r = np.random.default_rng(0)
    q_off, k_off = np.cumsum((0,) + lq), np.cumsum((0,) + lk)
    q, w = r.standard_normal((2, q_off[-1], 4, 8))
    k, v = r.standard_normal((2, k_off[-1], 2, 8))
    grads, _ = train.attention_grad(w, q, k, v, q_off, k_off, 0.4)
    f = lambda *t: (train.attention(*t, q_off, k_off, 0.4)[0] * w).sum()
    for i, g in enumerate(grads):
        x = [q, k, v]
        d = r.standard_normal(x[i].shape)
        got = slope(lambda y: f(*x[:i], y, *x[i + 1:]), x[i], d)
        assert abs(got - (g * d).sum()) < 1e-7 * max(1, np.abs(g * d).sum())
    assert np.isinf(train.attention(q, k, v, q_off, k_off, 0.4)[1]).any() == (0 in lk)


def test_layer_norm_gradients_are_the_slopes_of_the_output():
    r = np.random.default_rng(1)
    off, group, H = [1, 4, 4, 6], [1, 0, 1], 12
    x, w, res = r.standard_normal((3, 7, H))
    mods = r.standard_normal((2, 3 * H))
    f = lambda xx, mm: np.nansum(train.layer_norm(xx, mm, 0, 2 * H, off, group)[0] * w) + (xx * res)[1:6].sum()
    _, mean, rstd = train.layer_norm(x, mods, 0, 2 * H, off, group)
    dx, dshift, dscale = train.layer_norm_grad(w, x, mean, rstd, mods, 0, 2 * H, off, group, res)
    assert np.isnan(dx[[0, 6]]).all() and np.all(dshift[0] == 0)
    d = r.standard_normal(x.shape)
    d[[0, 6]] = 0
    assert abs(slope(lambda y: f(y, mods), x, d) - np.nansum(dx * d)) < 1e-7 * np.nansum(np.abs(dx * d))
    d = r.standard_normal(mods.shape)
    assert abs(slope(lambda y: f(x, y), mods, d) - (dshift * d[:, :H]).sum() - (dscale * d[:, 2 * H:]).sum()) < 1e-7 * np.abs(dscale).sum()


def test_objective_gradient_is_the_slope_of_its_value():
    r = np.random.default_rng(2)
    z, v = r.standard_normal((6, 8)), r.standard_normal((2, 8))
    ids, parent, first, coef = [2, 3, 5], [0, 1], [0, 2, 3], [(0.9, -0.2, 0.05, 0.1), (0.95, -0.1, 0.03, 0.2)]
    logp = train.objective_grad(z, v, ids, parent, first, coef, np.zeros(6), np.ones(6), 0.1, 3)[1]
    old, adv = np.zeros(6), r.standard_normal(6)
    old[ids] = logp - [0.02, 0.5, -0.05]
    adv[ids] = [1.3, 2.0, -0.7]
    J, _, grad, clipped = train.objective_grad(z, v, ids, parent, first, coef, old, adv, 0.1, 3)
    assert list(clipped) == [False, True, False]
    d = r.standard_normal(v.shape)
    f = lambda y: -train.objective_grad(z, y, ids, parent, first, coef, old, adv, 0.1, 3)[0]
    assert abs(slope(f, v, d) - (grad * d).sum()) < 1e-8


@pytest.mark.parametrize("bits", [3, 4])
def test_codes_are_neighbours_and_keep_the_mean(bits):
    table = train.code_values(bits)
    assert np.all(np.diff(table) > 0) and len(table) == 16 << bits
    r = np.random.default_rng(3)
    x = np.concatenate([[1.0], np.exp(r.uniform(-14, 0, 254)), [0.0]]).astype(np.float32)
    seen = np.zeros(256)
    for k in range(64):  # fractions (2 k + 1) / 128 of the way up
        code, scale = train.encode(x, bits, np.full(256, 1024 * k + 512), False)
        value = table[code] * np.float64(scale[0])
        y = x.astype(np.float64) / scale[0]
        below = np.searchsorted(table, y * (1 + 1e-6), side="right") - 1
        assert np.all((code == below) | (code == below + 1) | (np.abs(table[code] - y) <= 1e-6 * y))
        seen += value / 64
    gap = np.diff(np.append(table, table[-1]))[np.searchsorted(table, x / scale[0], side="right") - 1] * scale[0]
    assert np.all(np.abs(seen - x) <= gap / 64 + 1e-6 * x)
    assert np.array_equal(train.decode(*train.encode(-x, bits, np.zeros(256), True)[:2], bits, True) < 0, x > scale[0]) if bits == 3 else True
