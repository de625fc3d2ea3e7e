"""Oracle of layer norm, log probabilities and distillation (numpy, fp64), from their definitions."""
from __future__ import annotations

import numpy as np


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """(y, stats): stats holds the mean and 1 / sqrt(variance + eps) of every row."""
    x = np.asarray(x, dtype=np.float64)
    m = x.mean(1, keepdims=True)
    r = 1 / np.sqrt(((x - m) ** 2).mean(1, keepdims=True) + eps)
    y = (x - m) * r * (1 if weight is None else weight) + (0 if bias is None else bias)
    return y, np.hstack([m, r])


def layer_norm_grad(grad, x, stats, weight=None):
    """(x_grad, weight_grad, bias_grad)"""
    grad, x, stats = (np.asarray(a, dtype=np.float64) for a in (grad, x, stats))
    h = (x - stats[:, :1]) * stats[:, 1:]
    u = grad * (1 if weight is None else weight)
    x_grad = stats[:, 1:] * (u - u.mean(1, keepdims=True) - h * (u * h).mean(1, keepdims=True))
    return x_grad, (grad * h).sum(0), grad.sum(0)


def log_softmax(z):
    """log p of every row; -inf throughout where a row holds nothing else."""
    z = np.asarray(z, dtype=np.float64)
    m = z.max(1, keepdims=True)
    m = np.where(np.isneginf(m), 0.0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        total = np.exp(z - m).sum(1, keepdims=True)
        return np.where(total == 0, -np.inf, z - m - np.log(total))


def log_probs(logits, tokens=None, scale=1.0, k=0):
    """(logp, entropy, top_index, top_logp)"""
    x = np.asarray(logits, dtype=np.float64)
    N, C = x.shape
    lp = log_softmax(x * float(np.float32(scale)))
    p = np.exp(lp)
    with np.errstate(invalid="ignore"):
        entropy = -np.where(p == 0, 0.0, p * lp).sum(1)
    logp = np.zeros(N)
    if tokens is not None:
        for i, t in enumerate(tokens):
            if 0 <= t < C:
                logp[i] = lp[i, t]
    index, top = np.full((N, k), -1, dtype=np.int32), np.full((N, k), -np.inf)
    for i in range(N if k else 0):
        value = np.where(np.isnan(x[i]), np.inf, x[i])
        order = np.lexsort((np.arange(C), -value, ~np.isnan(x[i])))[:k]
        order = order[~np.isneginf(x[i][order])]
        index[i, :len(order)], top[i, :len(order)] = order, lp[i][order]
    return logp, entropy, index, top


def log_probs_grad(logits, tokens, scale=1.0, grad_logp=None, grad_entropy=None):
    x = np.asarray(logits, dtype=np.float64)
    N, C = x.shape
    s = float(np.float32(scale))
    lp = log_softmax(x * s)
    p = np.exp(lp)
    grad = np.zeros((N, C))
    if grad_logp is not None:
        g = np.broadcast_to(np.asarray(grad_logp, dtype=np.float64), (N,))
        for i, t in enumerate(tokens):
            if 0 <= t < C:
                grad[i] -= g[i] * p[i]
                grad[i, t] += g[i]
    if grad_entropy is not None:
        with np.errstate(invalid="ignore"):
            plp = np.where(p == 0, 0.0, p * lp)
        grad -= np.broadcast_to(np.asarray(grad_entropy, dtype=np.float64), (N,))[:, None] * (plp - p * plp.sum(1, keepdims=True))
    return s * grad


def distill(logits, index, teacher, T=1.0, grad_loss=None):
    """(loss, gradient or None)"""
    x, v = np.asarray(logits, dtype=np.float64), np.asarray(teacher, dtype=np.float64)
    T = float(np.float32(T))
    N, C = x.shape
    lp = log_softmax(x / T)
    loss, q_of = np.zeros(N), np.zeros((N, C))
    some = np.zeros(N, dtype=bool)
    for i in range(N):
        named = [k for k in range(v.shape[1]) if 0 <= index[i, k] < C and not np.isneginf(v[i, k])]
        if not named:
            continue
        some[i] = True
        z = v[i, named] / T
        lq = z - z.max() - np.log(np.exp(z - z.max()).sum())
        for j, k in enumerate(named):
            loss[i] += T * T * np.exp(lq[j]) * (lq[j] - lp[i, index[i, k]])
            q_of[i, index[i, k]] += np.exp(lq[j])
    if grad_loss is None:
        return loss, None
    g = np.broadcast_to(np.asarray(grad_loss, dtype=np.float64), (N,))[:, None]
    return loss, np.where(some[:, None], g * T * (np.exp(lp) - q_of), 0.0)
