"""The 64-bit losses that the GPU tests compare with, against differences of themselves and worked values."""
import math

import numpy as np
import pytest

import losses64 as L


def problem(seed, rows, n):
    g = np.random.RandomState(seed)
    z = g.randn(rows, n) * 2
    t = g.randint(0, n, rows)
    lp = np.array([q["lp"] for q in L.rows64(z, t)])
    return g, z, t, lp


def test_log_probabilities_of_a_worked_row():
    q, = L.rows64([[math.log(1), math.log(2), math.log(5), -math.inf]], [2])
    assert abs(q["lp"] - math.log(5 / 8)) < 1e-15 and np.allclose(q["p"], [1 / 8, 2 / 8, 5 / 8, 0])
    assert L.rows64([[0.0, -math.inf]], [1])[0]["lp"] == -math.inf and L.rows64([[]], [0])[0]["lp"] == -math.inf
    assert L.rows64([[3.0, 4.0]], [9], ids=[[5, 9]])[0]["col"] == 1 and L.rows64([[3.0, 4.0]], [7], ids=[[5, 9]])[0]["col"] == -1


@pytest.mark.parametrize("seed,beta", [(0, 0.0), (1, 0.3)])
def test_the_policy_gradient_is_the_slope_of_the_policy_loss(seed, beta):
    g, z, t, lp = problem(seed, 12, 9)
    old, ref, adv, w = lp + g.randn(12) * 0.4, lp + g.randn(12) * 0.5, g.randn(12), g.rand(12) * (g.rand(12) > 0.3)
    loss = lambda x: L.policy(L.rows64(x, t, weight=w), old, ref, adv, w, 0.2, 0.3, beta)[0]
    _, _, _, _, dlp, slack = L.policy(L.rows64(z, t, weight=w), old, ref, adv, w, 0.2, 0.3, beta)
    assert (np.abs(dlp) > 0).sum() >= 4
    check(z, t, w, loss, dlp, slack)


@pytest.mark.parametrize("seed,smoothing", [(2, 0.0), (3, 0.2)])
def test_the_preference_gradient_is_the_slope_of_the_preference_loss(seed, smoothing):
    g, z, t, lp = problem(seed, 12, 9)
    ref, w, off = lp + g.randn(12), g.rand(12) * (g.rand(12) > 0.2), np.array([1, 4, 4, 9, 11])
    inside = (np.arange(12) >= 1) & (np.arange(12) < 11)
    loss = lambda x: L.preference(L.rows64(x, t, weight=w, inside=inside), off, ref, w, 0.7, smoothing)[0]
    dlp, slack = L.preference(L.rows64(z, t, weight=w, inside=inside), off, ref, w, 0.7, smoothing)[4:]
    check(z, t, np.where(inside, w, 0), loss, dlp, slack)


def check(z, t, w, loss, dlp, slack):
    h = 1e-5
    grads = L.gradient(L.rows64(z, t, weight=w), [z.shape[1]] * len(z), dlp, slack)
    for r in range(len(z)):
        for c in range(z.shape[1]):
            up, down = z.copy(), z.copy()
            up[r, c] += h
            down[r, c] -= h
            slope = (loss(up) - loss(down)) / (2 * h)
            assert abs(slope - grads[r][0][c]) < 1e-8, (r, c)         # h^2 of a third derivative and 2^-53 / h of the losses


def test_worked_preference():
    z = np.log(np.array([[0.5, 0.5], [0.25, 0.75]]))
    loss, _, margin, _, dlp, _ = L.preference(L.rows64(z, [0, 0]), [0, 1, 2], None, None, 1.0, 0.0)
    assert abs(margin[0] - math.log(2)) < 1e-12 and abs(loss - math.log(1.5)) < 1e-12 and np.allclose(dlp, [-1 / 3, 1 / 3])
