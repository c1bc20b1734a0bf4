"""The transformer block's operators in 64 bits, from their definitions (numpy; CPU).

Shares no code with the library and imports neither it nor torch.
"""
from __future__ import annotations

import numpy as np


def _pair_indexes(rotated, interleaved):
    j = np.arange(rotated // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rotated // 2)


def _turn(x, positions, frequencies, interleaved, sign):
    """Pairs of the last axis of x [tokens, heads, dim] turned by the tokens' angles."""
    angle = np.asarray(positions, np.float64)[:, None, None] * np.asarray(frequencies, np.float64)
    a, b = _pair_indexes(2 * len(frequencies), interleaved)
    y = np.array(x, np.float64)
    y[..., a] = x[..., a] * np.cos(angle) - sign * x[..., b] * np.sin(angle)
    y[..., b] = x[..., b] * np.cos(angle) + sign * x[..., a] * np.sin(angle)
    return y


def head_norm_rotary(x, positions, frequencies, weight=None, eps=1e-6, interleaved=False):
    x = np.asarray(x, np.float64)
    n = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    if weight is not None:
        n = n * np.asarray(weight, np.float64)
    return _turn(n, positions, frequencies, interleaved, 1.0)


def head_norm_rotary_backward(dy, x, positions, frequencies, weight=None, eps=1e-6, interleaved=False):
    """dx and dweight."""
    x = np.asarray(x, np.float64)
    dn = _turn(np.asarray(dy, np.float64), positions, frequencies, interleaved, -1.0)
    rstd = 1 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    xhat = x * rstd
    g = dn if weight is None else dn * np.asarray(weight, np.float64)
    dx = rstd * (g - xhat * (g * xhat).mean(axis=-1, keepdims=True))
    return dx, (dn * xhat).sum(axis=(0, 1))


def _rows(offsets, tokens):
    return [range(0, tokens)] if offsets is None else [range(a, b) for a, b in zip(offsets[:-1], offsets[1:])]


def attention(q, k, v, offsets=None, causal=True, scale=None):
    """out [tokens, heads, dim], lse [heads, tokens] and, by (head, sequence), the probabilities; NaN in rows of no sequence.
    Sums run over the tokens seen alone."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    n, heads, dim = q.shape
    share = heads // k.shape[1]
    c = 1 / np.sqrt(dim) if scale is None else scale
    out, lse, probs = np.full(q.shape, np.nan), np.full((heads, n), np.nan), {}
    for s, rows in enumerate(_rows(offsets, n)):
        if len(rows) == 0:
            continue
        at = slice(rows.start, rows.stop)
        for h in range(heads):
            kk, vv = k[at, h // share], v[at, h // share]
            z = c * (q[at, h] @ kk.T)
            p = np.zeros_like(z)
            for i in range(len(rows)):
                seen = i + 1 if causal else len(rows)
                top = z[i, :seen].max()
                e = np.exp(z[i, :seen] - top)
                lse[h, rows.start + i] = top + np.log(e.sum())
                p[i, :seen] = e / e.sum()
                out[rows.start + i, h] = p[i, :seen] @ vv[:seen]
            probs[h, s] = p
    return out, lse, probs


def attention_backward(dout, q, k, v, offsets=None, causal=True, scale=None):
    """dq, dk, dv; zero in rows of no sequence."""
    dout, q, k, v = (np.asarray(t, np.float64) for t in (dout, q, k, v))
    n, heads, dim = q.shape
    share = heads // k.shape[1]
    c = 1 / np.sqrt(dim) if scale is None else scale
    _, _, probs = attention(q, k, v, offsets, causal, scale)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for s, rows in enumerate(_rows(offsets, n)):
        if len(rows) == 0:
            continue
        at = slice(rows.start, rows.stop)
        for h in range(heads):
            p, kk, vv, g = probs[h, s], k[at, h // share], v[at, h // share], dout[at, h]
            dv[at, h // share] += p.T @ g
            dp = g @ vv.T
            ds = p * (dp - (p * dp).sum(axis=1, keepdims=True))
            dq[at, h] = c * (ds @ kk)
            dk[at, h // share] += c * (ds.T @ q[at, h])
    return dq, dk, dv


def clip_gradients(grads, max_norm, tensors, eps=1e-6):
    """The scaled mean, the norm and the tensors' norms."""
    mean = np.sum([np.asarray(g, np.float64) for g in grads], axis=0) / len(grads)
    norms = np.array([np.sqrt((mean[a:a + k] ** 2).sum()) for a, k in tensors])
    norm = np.sqrt((norms ** 2).sum())
    return mean * min(1.0, max_norm / (norm + eps)), norm, norms
