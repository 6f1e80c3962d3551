"""Orthogonalised updates from their definition, in 64 bits, and how far a computation with pairs of fp16
numbers may be from it.  Shares no code with the library."""
from __future__ import annotations

import numpy as np

DEFAULT = ((3.4445, -4.7750, 2.0315),) * 5


def orthogonalize(G: np.ndarray, coefficients=DEFAULT) -> np.ndarray:
    G = np.asarray(G, dtype=np.float64)
    if not np.isfinite(G).all():
        return np.full(G.shape, np.nan)
    norm = np.sqrt((G * G).sum())
    if norm == 0:
        return np.zeros(G.shape)
    X = G / norm
    X = X.T if G.shape[0] > G.shape[1] else X
    for a, b, c in coefficients:
        S = X @ X.T
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.T if G.shape[0] > G.shape[1] else X


def limit(G: np.ndarray, coefficients=DEFAULT) -> float:
    """A bound for the Frobenius norm of the error of an fp32 result.

    A value is held to 2^-22 of itself, a product of two pairs leaves out 2^-22 of it, and the fp32 sum of n products
    rounds n times by at most 2^-24 of what it has reached, which add up like sqrt(n).  So with u(n) = 2^-21 + sqrt(n) 2^-24
    a product A B of inner length k is off by u(3 k) |A| |B| (Frobenius norms).  What one step is off by grows on the way through the
    others by no more than the steepest slope of their polynomials: a function of the singular values alone changes a
    matrix by no more, in the Frobenius norm, than its slope times the change.
    """
    X = np.asarray(G, dtype=np.float64)
    X = X / np.sqrt((X * X).sum())
    X = X.T if X.shape[0] > X.shape[1] else X
    s, l = X.shape

    def u(n):
        return 2.0 ** -21 + np.sqrt(n) * 2.0 ** -24

    fro = np.linalg.norm
    # slopes of the steps from step j on, over all singular values that X_j can have
    tops, sigma = [], np.linspace(0.0, 1.0, 20001)
    values = sigma
    for a, b, c in coefficients:
        tops.append(values.max())
        values = np.abs(a * values + b * values ** 3 + c * values ** 5)
    slopes = []
    for j in range(len(coefficients)):
        v, d = np.linspace(0.0, tops[j] * 1.001, 20001), np.ones(20001)
        for a, b, c in coefficients[j:]:
            d = d * (a + 3 * b * v ** 2 + 5 * c * v ** 4)
            v = a * v + b * v ** 3 + c * v ** 5
        slopes.append(np.abs(d).max())
    slopes.append(1.0)
    total = slopes[0] * 2.0 ** -22
    for j, (a, b, c) in enumerate(coefficients):
        S = X @ X.T
        P = b * S + c * (S @ S)
        new = a * X + P @ X
        x2 = np.sqrt(np.abs(np.linalg.eigvalsh(S)).max())
        e_s = u(3 * l) * fro(X) ** 2 + 2.0 ** -22 * fro(S)
        e_p = abs(b) * e_s + abs(c) * (2 * x2 ** 2 * e_s + u(3 * s) * fro(S) ** 2) + 2.0 ** -22 * (abs(b) * fro(S) + fro(P))
        e_x = x2 * e_p + u(3 * s) * fro(P) * fro(X) + 2.0 ** -22 * (abs(a) * fro(X) + fro(new))
        total += slopes[j + 1] * e_x
        X = new
    return float(total)


def pair(x: np.ndarray) -> np.ndarray:
    """Values as pairs of fp16 numbers hold them: x 2^12 = high + low.  22 bits, and no finer than steps of 2^-36."""
    high = (x * 4096).astype(np.float16).astype(np.float64)
    return (high + (x * 4096 - high).astype(np.float16)) / 4096


def held(G: np.ndarray, hold, coefficients=DEFAULT) -> np.ndarray:
    """The steps in 64 bits with every matrix on the way as `hold` leaves it: what that rounding by itself does to the result."""
    X = np.asarray(G, dtype=np.float64)
    X = hold(X / np.sqrt((X * X).sum()))
    X = X.T if G.shape[0] > G.shape[1] else X
    for a, b, c in coefficients:
        S = hold(X @ X.T)
        X = hold(a * X + hold(b * S + c * (S @ S)) @ X)
    return X.T if G.shape[0] > G.shape[1] else X


def in_fp32(G: np.ndarray, coefficients=DEFAULT) -> np.ndarray:
    """The steps in fp32 throughout."""
    X = np.asarray(G, dtype=np.float64)
    X = (X / np.sqrt((X * X).sum())).astype(np.float32)
    X = X.T if G.shape[0] > G.shape[1] else X
    for a, b, c in np.asarray(coefficients, dtype=np.float32):
        S = X @ X.T
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.T if G.shape[0] > G.shape[1] else X
