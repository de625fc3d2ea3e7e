"""Oracle of the training operators (numpy, fp64): embedding rows, their gradient, Newton-Schulz directions and the step of a
weight matrix around them, from their definitions."""
from __future__ import annotations

import numpy as np

COEFF = (3.4445, -4.7750, 2.0315)


def embedding(table, tokens, scale=1.0):
    out = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < table.shape[0]:
            out[i] = scale * table[t].astype(np.float64)
    return out


def embedding_grad(tokens, grad, V, scale=1.0):
    """The gradient, and the sum of the magnitudes and the number of terms of every row (what rounding errors are in proportion to)."""
    out, size, terms = np.zeros((V, grad.shape[1])), np.zeros((V, grad.shape[1])), np.zeros(V, dtype=np.int64)
    known = np.flatnonzero((tokens >= 0) & (tokens < V))
    g = grad[known].astype(np.float64)
    np.add.at(out, tokens[known], scale * g)
    np.add.at(size, tokens[known], np.abs(scale * g))
    np.add.at(terms, tokens[known], 1)
    return out, size, terms


def newton_schulz(G, steps=5, coeff=COEFF, eps=1e-7):
    """Every iterate, the first included, in G's orientation."""
    coeff = np.broadcast_to(np.asarray(coeff, dtype=np.float64), (steps, 3))
    G = np.asarray(G, dtype=np.float64)
    X = G / (np.sqrt((G * G).sum()) + eps)
    tall = X.shape[0] > X.shape[1]
    if tall:
        X = X.T
    seen = [X]
    for a, b, c in coeff:
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
        seen.append(X)
    return [x.T if tall else x for x in seen]


def muon_step(W, M, G, lr, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, coeff=COEFF, eps=1e-7):
    W, M, G = (np.asarray(x, dtype=np.float64) for x in (W, M, G))
    M = momentum * M + G
    U = G + momentum * M if nesterov else M
    return (1 - lr * weight_decay) * W - lr * newton_schulz(U, steps, coeff, eps)[-1], M
