"""fp64 oracle of the dense operators either side of the mixers: the linear
layer with bias, activation and residual, and the weighted softmax cross
entropy over the vocabulary of the masked objective (Sec. 3; Sec. 4.1;
Appendix C: MLP ratio 4).

TEST INFRASTRUCTURE, like the rest of ``oracle/``: only ``tests/``,
``__graft_entry__.smoke()`` and the CPU baseline of ``bench.py`` may use it.

Readings (the paper names these layers without writing them out):
  * y = residual + act(x w^T + b), act none, SiLU or GELU in its tanh form.
  * loss_t = weight_t (log sum_v exp z_tv - z_t,target), z = h w^T. A row counts
    where its target is in the vocabulary and its weight is not zero; the
    others have loss and log sum 0 and no gradient. The excluded entry (the
    mask token) has logit minus infinity.

Every function takes and returns fp64 numpy arrays. Pins:
tests/test_dense_oracle_pins.py.
"""

from __future__ import annotations

import numpy as np

GELU_A = np.sqrt(2.0 / np.pi)
GELU_B = 0.044715


def act(name, z):
    if name == "none":
        return z
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    return 0.5 * z * (1.0 + np.tanh(GELU_A * (z + GELU_B * z ** 3)))


def act_grad(name, z):
    if name == "none":
        return np.ones_like(z)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1.0 - s)
    t = np.tanh(GELU_A * (z + GELU_B * z ** 3))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * GELU_A * (1.0 + 3.0 * GELU_B * z * z)


def linear_forward(x, w, bias=None, residual=None, name="none"):
    """y and the pre-activation."""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    y = act(name, z)
    return (y if residual is None else y + residual), z


def linear_backward(x, w, pre, dy, name="none"):
    """dx, dw, dbias."""
    dz = dy * act_grad(name, pre)
    return dz @ w, dz.T @ x, dz.sum(0)


def _rows(target, weight, vocab):
    return (target >= 0) & (target < vocab) & (weight != 0)


def lm_loss_forward(h, w, target, weight, excluded=-1):
    """loss and log sum per row."""
    loss = np.zeros(h.shape[0])
    lse = np.zeros(h.shape[0])
    for t in np.nonzero(_rows(target, weight, w.shape[0]))[0]:
        z = w @ h[t]
        if excluded >= 0:
            z[excluded] = -np.inf
        m = z.max()
        lse[t] = m + np.log(np.exp(z - m).sum()) if np.isfinite(m) else m
        loss[t] = weight[t] * (np.inf if z[target[t]] == -np.inf else lse[t] - z[target[t]])
    return loss, lse


def lm_loss_backward(h, w, target, weight, dloss, excluded=-1):
    """dh, dw."""
    dh, dw = np.zeros_like(h), np.zeros_like(w)
    _, lse = lm_loss_forward(h, w, target, weight, excluded)
    for t in np.nonzero(_rows(target, weight, w.shape[0]) & (dloss != 0))[0]:
        z = w @ h[t]
        dz = np.exp(z - lse[t])
        dz[target[t]] -= 1.0
        if excluded >= 0:
            dz[excluded] = 0.0
        dz *= weight[t] * dloss[t]
        dh[t] = dz @ w
        dw += np.outer(dz, h[t])
    return dh, dw
