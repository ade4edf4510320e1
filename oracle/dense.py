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


def gated_linear_forward(x, w, bias=None, name="silu"):
    """y = act(gate) * up; w holds the rows of the gate's weights, then the others."""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    gate, up = np.split(z, 2, axis=1)
    return act(name, gate) * up


def gated_linear_backward(x, w, bias, dy, name="silu"):
    """dx, dw, dbias."""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    gate, up = np.split(z, 2, axis=1)
    dz = np.concatenate((dy * up * act_grad(name, gate), dy * act(name, gate)), axis=1)
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


def _teacher(ids, logits, vocab, excluded, temperature):
    """Known entries of a row, and their q."""
    known = (ids >= 0) & (ids < vocab) & (ids != excluded) & (logits != -np.inf)
    q = np.zeros(len(ids))
    if known.any():
        t = logits[known] / temperature
        e = np.exp(t - t.max())
        q[known] = e / e.sum()
    return known, q


def distill_loss_forward(h, w, ids, teacher, weight, excluded=-1, temperature=1.0):
    """loss, log sum and the student's logits at the known entries, per row."""
    loss, lse, at = np.zeros(h.shape[0]), np.zeros(h.shape[0]), np.zeros(ids.shape)
    for t in range(h.shape[0]):
        known, q = _teacher(ids[t], teacher[t], w.shape[0], excluded, temperature)
        if weight[t] == 0 or not known.any():
            continue
        raw = w @ h[t]
        z = raw / temperature
        if excluded >= 0:
            z[excluded] = -np.inf
        lse[t] = z.max() + np.log(np.exp(z - z.max()).sum())
        at[t, known] = raw[ids[t, known]]
        full = np.zeros(w.shape[0])
        np.add.at(full, ids[t, known], q[known])
        some = full > 0
        loss[t] = weight[t] * (full[some] * (np.log(full[some]) - z[some] + lse[t])).sum()
    return loss, lse, at


def distill_loss_backward(h, w, ids, teacher, weight, dloss, excluded=-1, temperature=1.0):
    """dh, dw."""
    dh, dw = np.zeros_like(h), np.zeros_like(w)
    _, lse, _ = distill_loss_forward(h, w, ids, teacher, weight, excluded, temperature)
    for t in range(h.shape[0]):
        known, q = _teacher(ids[t], teacher[t], w.shape[0], excluded, temperature)
        if weight[t] == 0 or dloss[t] == 0 or not known.any():
            continue
        dz = np.exp(w @ h[t] / temperature - lse[t])
        if excluded >= 0:
            dz[excluded] = 0.0
        np.subtract.at(dz, ids[t, known], q[known])
        dz *= weight[t] * dloss[t] / temperature
        dh[t] = dz @ w
        dw += np.outer(dz, h[t])
    return dh, dw


def token_scores_forward(z, token=None, top=0, excluded=-1, temperature=1.0):
    """logp (None without token), entropy, ids and log probabilities of the likeliest entries of rows of logits."""
    rows, vocab = z.shape
    logp, entropy = np.zeros(rows), np.zeros(rows)
    ids, best = np.full((rows, top), -1), np.full((rows, top), -np.inf)
    for t in range(rows):
        if token is not None and not 0 <= token[t] < vocab:
            continue
        v = z[t].astype(np.float64) / temperature
        if excluded >= 0:
            v[excluded] = -np.inf
        if np.isnan(v).any() or (v == np.inf).any():
            logp[t] = entropy[t] = best[t] = np.nan
            continue
        if (v == -np.inf).all():
            logp[t] = -np.inf
            continue
        v -= v.max()
        v -= np.log(np.exp(v).sum())
        there = v > -np.inf
        entropy[t] = -(np.exp(v[there]) * v[there]).sum()
        if token is not None:
            logp[t] = v[token[t]]
        # the logits themselves decide the order; a stable sort keeps the lower index first
        order = np.argsort(-np.where(there, z[t].astype(np.float64), -np.inf), kind="stable")[:top]
        order = order[there[order]]
        ids[t, :len(order)], best[t, :len(order)] = order, v[order]
    return (None if token is None else logp), entropy, ids, best


def token_scores_backward(z, token, dlogp, dentropy, excluded=-1, temperature=1.0):
    """Gradient at the logits; token, dlogp and dentropy may be None."""
    rows, vocab = z.shape
    dz = np.zeros(z.shape)
    for t in range(rows):
        if token is not None and not 0 <= token[t] < vocab:
            continue
        v = z[t].astype(np.float64) / temperature
        if excluded >= 0:
            v[excluded] = -np.inf
        if (v == -np.inf).all():
            continue
        v = v - v.max()
        v = v - np.log(np.exp(v).sum())
        p = np.exp(v)
        there = p > 0
        plogp = np.where(there, p * np.where(there, v, 0.0), 0.0)
        if dentropy is not None:
            dz[t] -= dentropy[t] * (plogp + p * -plogp.sum())
        if dlogp is not None:
            dz[t] -= dlogp[t] * p
            dz[t, token[t]] += dlogp[t]
        dz[t] /= temperature
        if excluded >= 0:
            dz[t, excluded] = 0.0
    return dz
