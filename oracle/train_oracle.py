"""The training operators in 64 bits, from their definitions (numpy; CPU).

Shares no code with the library and imports neither it nor torch.
"""
from __future__ import annotations

import numpy as np


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """y, mean, rstd of each row."""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(np.mean((x - mean) ** 2, axis=1, keepdims=True) + eps)
    y = (x - mean) * rstd
    if weight is not None:
        y = y * np.asarray(weight, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, mean[:, 0], rstd[:, 0]


def layer_norm_backward(dy, x, weight, mean, rstd):
    """dx, dweight, dbias for given statistics."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    mean, rstd = np.asarray(mean, np.float64)[:, None], np.asarray(rstd, np.float64)[:, None]
    xhat = (x - mean) * rstd
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    d = x.shape[1]
    dx = rstd * (g - g.sum(axis=1, keepdims=True) / d - xhat * (g * xhat).sum(axis=1, keepdims=True) / d)
    return dx, (dy * xhat).sum(axis=0), dy.sum(axis=0)


def linear_cross_entropy(hidden, weight, targets, ignore_index=-100):
    """loss and log-sum-exp of each token."""
    z = np.asarray(hidden, np.float64) @ np.asarray(weight, np.float64).T
    top = z.max(axis=1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    loss = np.zeros(len(z))
    for i, t in enumerate(targets):
        if t == ignore_index:
            continue
        loss[i] = lse[i] - z[i, t] if 0 <= t < z.shape[1] else np.nan
    return loss, lse


def linear_cross_entropy_backward(dloss, hidden, weight, targets, ignore_index=-100):
    """dhidden, dweight and the gradient of the logits."""
    h, w = np.asarray(hidden, np.float64), np.asarray(weight, np.float64)
    z = h @ w.T
    p = np.exp(z - z.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    for i, t in enumerate(targets):
        if t == ignore_index:
            p[i] = 0.0
        else:
            p[i, t] -= 1.0
            p[i] *= float(dloss[i])
    return p @ w, p.T @ h, p


def newton_schulz(u, coefficients, eps=1e-7):
    """The polynomial of a matrix's singular values that `coefficients`, one (a, b, c) a step, make."""
    x = np.asarray(u, np.float64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    for a, b, c in coefficients:
        gram = x @ x.T
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.T if tall else x


def muon_step(grads, params, momentum, matrices, lr, mu, weight_decay, nesterov, coefficients, eps=1e-7):
    """x' and m' of a flat buffer; matrices are (start, rows, cols, scale)."""
    x, m = np.array(params, np.float64), np.array(momentum, np.float64)
    gbar = np.sum([np.asarray(g, np.float64) for g in grads], axis=0) / len(grads)
    for start, rows, cols, scale in matrices:
        cut = slice(start, start + rows * cols)
        m[cut] = mu * m[cut] + gbar[cut]
        u = gbar[cut] + mu * m[cut] if nesterov else m[cut]
        o = newton_schulz(u.reshape(rows, cols), coefficients, eps).ravel()
        x[cut] = x[cut] * (1.0 - lr * weight_decay) - lr * scale * o
    return x, m
