"""Newton-Schulz steps as the kernels take them, in numpy: operands in f16 parts, each of a product's part products summed by itself.

steps_in_parts(G, lost=...) leaves one of them out, which is what a kernel with a mistake in its products does.  Sums are exact here: what the parts
and the products that are left out cost is what the emulation is for.
"""
from __future__ import annotations

import math

import numpy as np

from oracle import training

A, B, C = (float(np.float32(x)) for x in training.COEFF)
F32, F64 = np.float32, np.float64


def relative_errors(X, exact):
    """Of every matrix, in the Frobenius norm."""
    X, exact = np.asarray(X, dtype=F64), np.asarray(exact, dtype=F64)
    return np.linalg.norm(X - exact, axis=(1, 2)) / np.linalg.norm(exact, axis=(1, 2))


def in_64_bits(G):
    return np.stack([training.newton_schulz(g, 5, (A, B, C))[-1] for g in np.asarray(G, dtype=F64)])


def in_fp32(G):
    """The steps in fp32 throughout."""
    X = np.asarray(G, dtype=F32)
    tall = X.shape[1] > X.shape[2]
    X = X.transpose(0, 2, 1) if tall else X
    X = X / (np.sqrt((X * X).sum((1, 2), keepdims=True, dtype=F32)) + F32(1e-7))
    for _ in range(5):
        S = X @ X.transpose(0, 2, 1)
        X = F32(A) * X + (F32(B) * S + F32(C) * (S @ S)) @ X
    return X.transpose(0, 2, 1) if tall else X


def _split(v, parts):
    rest, out = v.astype(F32), []
    for _ in range(parts):
        out.append(rest.astype(np.float16))
        rest = rest - out[-1].astype(F32)
    return [x.astype(F64) for x in out]


def _product(P, Q, lost):
    """P Q of matrices in two parts: hi hi + hi lo + lo hi without those that are lost; rounded to fp32."""
    total = P[0] @ Q[0]
    if len(P) > 1:
        for i, j in ((1, 0), (0, 1)):
            if (i, j) not in lost:
                total = total + P[i] @ Q[j]
    return total.astype(F32)


def _turned(parts):
    return [x.transpose(0, 2, 1) for x in parts]


def _power(bound):
    return 15 - math.frexp(bound * 1.01)[1]


def _largest(polynomial, top):
    s = np.linspace(0.0, top, 20_001)
    return float(np.abs(polynomial(s)).max())


# lost: (product, (part of the left operand, part of the right one)); products: "A" = X X^T, then "Y" = A X and "Z" = A Y (the step's last two in one
# launch), or "square" = A A and "update" = B X (in one each)
def mistakes(panel):
    return [(which, pair) for which in (("A", "Y", "Z") if panel else ("A", "square", "update")) for pair in ((1, 0), (0, 1))]


def steps_in_parts(G, panel, lost=None, parts=2):
    def without(which):
        return {lost[1]} if lost and lost[0] == which else set()
    X = np.asarray(G, dtype=F64)
    tall = X.shape[1] > X.shape[2]
    X = X.transpose(0, 2, 1) if tall else X
    top = 1.0
    ex = _power(top)
    v = (X * (2.0 ** ex / (np.sqrt((X * X).sum((1, 2), keepdims=True)) + 1e-7))).astype(F32)
    for k in range(5):
        ea, ey = _power(top ** 2), _power(top ** 3)
        eb = _power(_largest(lambda t: B * t + C * t * t, top * top))
        top = _largest(lambda s: A * s + B * s ** 3 + C * s ** 5, top)
        after = _power(top) if k < 4 else 0
        x = _split(v, parts)
        a = _split(_product(x, _turned(x), without("A")) * F32(2.0 ** (ea - 2 * ex)), parts)
        if panel:
            y = _product(a, x, without("Y"))
            z = _product(a, _split(y * F32(2.0 ** (ey - ea - ex)), parts), without("Z"))
            v = F32(A * 2.0 ** (after - ex)) * v + (F32(B * 2.0 ** (after - ea - ex)) * y + F32(C * 2.0 ** (after - ea - ey)) * z)
        else:
            held = sum(p.astype(F32) for p in a)
            b = _split(F32(C * 2.0 ** (eb - 2 * ea)) * _product(a, a, without("square")) + F32(B * 2.0 ** (eb - ea)) * held, parts)
            held = sum(p.astype(F32) for p in x)
            v = F32(2.0 ** (after - ex - eb + ex)) * _product(b, x, without("update")) * F32(2.0 ** -ex) + F32(A * 2.0 ** (after - ex)) * held
        ex = after
    return v.transpose(0, 2, 1) if tall else v
