"""4-bit microscaled matrices from their definition, in 64 bits: what `dmm_mx_quantize` has to write and what it
stands for.  Shares no code with the library."""
from __future__ import annotations

import numpy as np

BLOCK, CHUNK = 32, 128
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x: np.ndarray):
    """Codes (one an element) and scale bytes of an h x w matrix of doubles in blocks along its rows, both filled up to whole
    chunks with zeros."""
    h, w = x.shape
    chunks = -(-w // CHUNK)
    padded = np.zeros((h, chunks * CHUNK))
    padded[:, :w] = x
    blocks = padded.reshape(h, chunks * CHUNK // BLOCK, BLOCK)
    bad = ~np.isfinite(blocks).all(axis=2)
    blocks = np.where(bad[:, :, None], 0.0, blocks)
    top = np.abs(blocks).max(axis=2)
    _, e = np.frexp(top)                                  # top = f 2^e with f in [0.5, 1)
    e = np.where(top > 0, np.clip(e - 1 - 2, -127, 127), -127)
    y = np.abs(blocks) / np.ldexp(1.0, e)[:, :, None]
    # distance to every value; of two that are equally near the one whose code is even
    d = np.abs(y[..., None] - VALUES)
    best = d.min(axis=-1, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(near.sum(axis=-1) > 1, even.argmax(axis=-1), near.argmax(axis=-1)).astype(np.uint8)
    code = np.where(y > 6, 7, code).astype(np.uint8)
    code |= (np.signbit(blocks) & True).astype(np.uint8) << 3
    scale = np.where(bad, 255, e + 127).astype(np.uint8)
    scale[:, -(-w // BLOCK):] = 0
    return code.reshape(h, -1), scale


def pack(code: np.ndarray) -> np.ndarray:
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)


def unpack(packed: np.ndarray) -> np.ndarray:
    out = np.empty((packed.shape[0], packed.shape[1] * 2), dtype=np.uint8)
    out[:, 0::2] = packed & 15
    out[:, 1::2] = packed >> 4
    return out


def values(code: np.ndarray, scale: np.ndarray, w: int) -> np.ndarray:
    """The w values of every row that codes (one an element) and scale bytes stand for."""
    v = VALUES[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.ldexp(1.0, scale.astype(np.int64) - 127)
    s = np.where(scale == 255, np.nan, s)
    return (v.reshape(*scale.shape, BLOCK) * s[:, :, None]).reshape(v.shape)[:, :w]


def sum_limit(A: np.ndarray, B: np.ndarray) -> float:
    """A bound for the Frobenius norm of the error of A B where every term is exact and sums are fp32: adding term t rounds by
    at most half a step, 2^-24, of the sum so far.  Roundings of different additions are independent, so that their squares
    add up.  Sums over ranges of k that are added up afterwards are differences of two sums from k = 0 on: at most
    twice the largest so far; within a chunk these grow by no more than the magnitudes of its terms."""
    total, top, S = 0.0, 0.0, np.zeros((A.shape[0], B.shape[1]))
    for c in range(0, A.shape[1], CHUNK):
        a, b = A[:, c:c + CHUNK], B[c:c + CHUNK]
        inside = top + np.linalg.norm(np.abs(a) @ np.abs(b))
        total += a.shape[1] * (2 * inside) ** 2
        S = S + a @ b
        top = max(top, np.linalg.norm(S))
    return float(2.0 ** -24 * np.sqrt(total))
