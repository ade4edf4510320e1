"""Pins of the fp64 oracle of the dense operators (oracle/dense.py) on the CPU:
gradients against central differences, identities, and planted mistakes that
have to fail."""

import numpy as np
import pytest

from oracle import dense as od

RNG = np.random.default_rng(11)
EPS = 1e-6
# central differences in fp64: truncation eps^2 times third derivatives of order 1 (1e-12), cancellation 1e-16 / eps
# times values of order 10 (1e-9)
TOL = 1e-7


def _diff(f, a, da):
    return (f(a + EPS * da) - f(a - EPS * da)) / (2 * EPS)


@pytest.mark.parametrize("name", ["none", "silu", "gelu"])
def test_linear_gradients_match_differences(name):
    x, w, b = RNG.normal(size=(5, 4)), RNG.normal(size=(3, 4)), RNG.normal(size=3)
    r, dy = RNG.normal(size=(5, 3)), RNG.normal(size=(5, 3))
    _, pre = od.linear_forward(x, w, b, r, name)
    g = od.linear_backward(x, w, pre, dy, name)
    fs = (lambda v: (od.linear_forward(v, w, b, r, name)[0] * dy).sum(),
          lambda v: (od.linear_forward(x, v, b, r, name)[0] * dy).sum(),
          lambda v: (od.linear_forward(x, w, v, r, name)[0] * dy).sum())
    for f, a, ga in zip(fs, (x, w, b), g):
        for _ in range(4):
            d = RNG.normal(size=a.shape)
            assert abs(_diff(f, a, d) - (ga * d).sum()) < TOL * max(1.0, abs((ga * d).sum()))


def test_activations():
    z = np.linspace(-12, 12, 101)
    for name in ("silu", "gelu"):
        y = od.act(name, z)
        assert np.allclose(y - od.act(name, -z), z, atol=1e-12)  # z sigmoid(u) with an odd u
        d = (od.act(name, z + EPS) - od.act(name, z - EPS)) / (2 * EPS)
        assert np.max(np.abs(d - od.act_grad(name, z))) < 1e-8
    assert od.act("gelu", np.array([1.0]))[0] == pytest.approx(0.8411919906082768, abs=1e-12)
    assert od.act("silu", np.array([1.0]))[0] == pytest.approx(0.7310585786300049, abs=1e-12)


def _case(t=6, k=4, v=7, excluded=-1):
    h, w = RNG.normal(size=(t, k)), RNG.normal(size=(v, k))
    target = RNG.integers(0, v - 1, size=t)
    weight = RNG.uniform(0.2, 2.0, size=t)
    weight[1] = 0.0
    target[2] = -1
    target[3] = v
    return h, w, target, weight, RNG.uniform(0.5, 1.5, size=t), excluded


@pytest.mark.parametrize("excluded", [-1, 6])
def test_loss_gradients_match_differences(excluded):
    h, w, target, weight, dloss, ex = _case(excluded=excluded)
    dh, dw = od.lm_loss_backward(h, w, target, weight, dloss, ex)
    fh = lambda a: (od.lm_loss_forward(a, w, target, weight, ex)[0] * dloss).sum()
    fw = lambda a: (od.lm_loss_forward(h, a, target, weight, ex)[0] * dloss).sum()
    for f, a, g in ((fh, h, dh), (fw, w, dw)):
        for _ in range(4):
            d = RNG.normal(size=a.shape)
            assert abs(_diff(f, a, d) - (g * d).sum()) < TOL * max(1.0, abs((g * d).sum()))
    assert np.all(dh[[1, 2, 3]] == 0.0)
    if excluded >= 0:
        assert np.all(dw[excluded] == 0.0)


def test_loss_identities():
    h, w, target, weight, dloss, _ = _case()
    loss, lse = od.lm_loss_forward(h, w, target, weight)
    assert np.all(loss[[1, 2, 3]] == 0.0) and np.all(lse[[1, 2, 3]] == 0.0)
    # a shift of every logit of a row leaves the loss: w + outer(1, c) adds h . c to each
    loss2, _ = od.lm_loss_forward(h, w + RNG.normal(size=4)[None, :], target, weight)
    assert np.allclose(loss, loss2, atol=1e-12)
    # so the gradient of w sums to zero over the vocabulary
    assert np.allclose(od.lm_loss_backward(h, w, target, weight, dloss)[1].sum(0), 0.0, atol=1e-12)
    # equal logits: log of the number of entries, one less with an excluded one
    z = np.zeros_like(h)
    assert np.allclose(od.lm_loss_forward(z, w, target, np.ones(6))[0][[0, 4, 5]], np.log(7.0))
    assert np.allclose(od.lm_loss_forward(z, w, target, np.ones(6), 6)[0][[0, 4, 5]], np.log(6.0))
    # the excluded entry as the target; nothing left at all
    assert od.lm_loss_forward(h[:1], w, np.array([6]), np.ones(1), 6)[0][0] == np.inf
    assert od.lm_loss_forward(h[:1], w[:1], np.array([0]), np.ones(1), 0)[1][0] == -np.inf


def test_planted_mistakes_fail():
    """The pins see a wrong target, a dropped weight and a dropped derivative term."""
    h, w, target, weight, dloss, _ = _case()
    dh, dw = od.lm_loss_backward(h, w, target, weight, dloss)
    d = RNG.normal(size=h.shape)
    true = _diff(lambda a: (od.lm_loss_forward(a, w, target, weight)[0] * dloss).sum(), h, d)
    for bad in (od.lm_loss_backward(h, w, (target + 1) % 7, weight, dloss)[0],
                od.lm_loss_backward(h, w, target, np.where(weight != 0, 1.0, 0.0), dloss)[0]):
        assert abs((bad * d).sum() - true) > 100 * TOL
    x, z = RNG.normal(size=(5, 4)), RNG.normal(size=(5, 3))
    dy, ww = RNG.normal(size=(5, 3)), RNG.normal(size=(3, 4))
    good = od.linear_backward(x, ww, z, dy, "silu")[0]
    s = 1.0 / (1.0 + np.exp(-z))
    assert np.max(np.abs((dy * s) @ ww - good)) > 100 * TOL
