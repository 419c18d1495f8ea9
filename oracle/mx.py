"""MXFP4 quantizer and product, routing to experts and the weighted sum behind them -- CPU oracle (test infrastructure only; see
formats.py).

OCP microscaling formats, version 1.0: 32 channels share the scale 2^(floor(log2 amax) - 2), 2 being the exponent of the largest
E2M1 magnitude; the exponent is held to -127 .. 127 (zeros: -127) and stored plus 127; elements are x / scale rounded to the nearest
E2M1 value, ties to the even code, saturating at 6.  Everything here is exact in fp64.  A group with a value that is not finite is NaN.
"""
from __future__ import annotations

from typing import NamedTuple

import numpy as np

from . import formats as F

BLOCK = 32
MIDPOINTS = (F.E2M1_VALUES[1:] + F.E2M1_VALUES[:-1]) / 2


class MxQuant(NamedTuple):
    code: np.ndarray     # [rows, K] uint8 nibbles: sign << 3 | E2M1 index
    scale: np.ndarray    # [rows, K / 32] uint8: exponent + 127, 255 = NaN


def quantize(x) -> MxQuant:
    x = np.asarray(x, dtype=np.float64)
    rows, K = x.shape
    g = x.reshape(rows, K // BLOCK, BLOCK)
    amax = np.abs(g).max(axis=2)
    finite = np.isfinite(amax)
    e = np.clip(np.frexp(np.where(finite, amax, 1.0))[1] - 1 - 2, -127, 127)
    e = np.where(amax == 0, -127, e)
    a = np.abs(np.where(finite[:, :, None], g, 0.0)) / np.ldexp(1.0, e)[:, :, None]
    code = np.zeros(a.shape, dtype=np.uint8)
    for i, mid in enumerate(MIDPOINTS):                 # a midpoint goes to the even one of its two codes
        code += (a > mid) if i % 2 == 0 else (a >= mid)
    code |= np.signbit(g).astype(np.uint8) << 3
    return MxQuant(code.reshape(rows, K), np.where(finite, e + 127, 255).astype(np.uint8))


def dequantize(q: MxQuant) -> np.ndarray:
    v = F.E2M1_VALUES[q.code & 7] * np.where(q.code & 8, -1.0, 1.0)
    s = np.where(q.scale == 255, np.nan, np.ldexp(1.0, q.scale.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, axis=1)


def packed_codes(q: MxQuant) -> np.ndarray:
    return (q.code[:, 0::2] | q.code[:, 1::2] << 4).astype(np.uint8)


def unpacked(codes, scales) -> MxQuant:
    code = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1)
    return MxQuant(code, np.asarray(scales))


class Routed(NamedTuple):
    ids: np.ndarray
    weights: np.ndarray
    offsets: np.ndarray
    rows: np.ndarray
    positions: np.ndarray


def route(logits, k: int, renormalize: bool) -> Routed:
    """Token by token; an expert whose logit is -inf or NaN is not chosen, -1 stands where none is left."""
    x = np.asarray(logits, dtype=np.float64)
    T, E = x.shape
    x = np.where(np.isnan(x), -np.inf, x)
    ids, weights = np.full((T, k), -1, dtype=np.int32), np.zeros((T, k))
    chosen = [[] for _ in range(E)]
    for t in range(T):
        order = [e for e in sorted(range(E), key=lambda e: (-x[t, e], e)) if x[t, e] > -np.inf][:k]
        if not order:
            continue
        p = np.exp(x[t] - x[t, order[0]])
        total = p[order].sum() if renormalize else p.sum()
        for j, e in enumerate(order):
            ids[t, j], weights[t, j] = e, p[e] / total
            chosen[e].append((t, j))
    offsets = np.concatenate([[0], np.cumsum([len(c) for c in chosen])]).astype(np.int32)
    rows, positions = np.full(T * k, -1, dtype=np.int32), np.full((T, k), -1, dtype=np.int32)
    for at, (t, j) in enumerate(pair for c in chosen for pair in c):
        rows[at], positions[t, j] = t, at
    return Routed(ids, weights, offsets, rows, positions)


def combine(y, positions, weights, addend=None):
    """(sum, sum of the magnitudes of its terms)."""
    T, k = positions.shape
    out = np.zeros((T, y.shape[1])) if addend is None else np.array(addend, dtype=np.float64)
    mag = np.abs(out)
    for t in range(T):
        for j in range(k):
            if 0 <= positions[t, j] < y.shape[0]:
                term = np.float64(weights[t, j]) * y[positions[t, j]]
                out[t] += term
                mag[t] += np.abs(term)
    return out, mag
