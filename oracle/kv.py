"""Key-value cache and the attention of one new token over it -- CPU oracle (test infrastructure only; see formats.py).

What the cache holds of a (token, head) row is the per-group quantizer's output of that row (quantize.py), groups along the head's
channels.  Attention: out = sum_t p_t v_t, p the softmax over the attended tokens of scale * q . k_t; nothing attended gives
zeros and ln 0 = -inf.
"""
from __future__ import annotations

import numpy as np

from . import formats as F
from . import quantize as Q

BF16 = 3


def stored(fmt: int, group: int, x, tensor_scale=None) -> np.ndarray:
    """The exact values that a cache holds of x [..., head_dim] (float64 of bf16 values)."""
    x = np.asarray(x, dtype=np.float64)
    if fmt == BF16:
        return x.copy()
    rows = x.reshape(-1, x.shape[-1])
    if fmt == F.FMT_NVFP4:
        return Q.dequantize_nvfp4(Q.quantize_nvfp4(rows, tensor_scale)).reshape(x.shape)
    return Q.dequantize_int(Q.quantize_int(rows, group, fmt), group).reshape(x.shape)


def read_back(fmt: int, group: int, x, tensor_scale=None) -> np.ndarray:
    """The bf16 bits that reading gives: the stored value by binary32 operations, rounded to nearest even."""
    return F.f64_to_bf16_bits_rne(F.fl32(stored(fmt, group, x, tensor_scale)))


def attended(length: int, window: int = 0) -> range:
    length = max(0, length)
    return range(max(0, length - window) if window else 0, length)


def attention(q, k, v, scale: float):
    """q [q_heads, dim], k, v [tokens, kv_heads, dim] -> (out [q_heads, dim], lse [q_heads], sum_t p |v| like out, and the
    largest sum of |scale q_d k_d| over a row and token, [q_heads])."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    per = q.shape[0] // k.shape[1]
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, top = np.full(q.shape[0], -np.inf), np.zeros(q.shape[0])
    if k.shape[0] == 0:
        return out, lse, mag, top
    for h in range(q.shape[0]):
        kk, vv = k[:, h // per], v[:, h // per]
        s = scale * (kk @ q[h])
        m = s.max()
        p = np.exp(s - m)
        total = p.sum()
        out[h], mag[h] = (p / total) @ vv, (p / total) @ np.abs(vv)
        lse[h], top[h] = m + np.log(total), abs(scale) * (np.abs(kk) @ np.abs(q[h])).max()
    return out, lse, mag, top
