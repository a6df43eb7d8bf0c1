"""fp64 oracle of the operators on a cache in 8 bits (test infrastructure).

A cache in 8 bits holds OCP E4M3 codes and, for each block of entries of one (sequence, layer,
KV head), a power-of-two scale as its exponent byte x (2^(x-127)).  Everything here works on one
such plane: codes [entries][d], scales [entries / block].  Written from the definitions of the
operators; it shares no code with the library.
"""
from __future__ import annotations

import numpy as np

from .cc_oracle import e4m3_decode, e4m3_encode

LOW = 27   # exponent byte of the smallest scale given to a block, 2^-100


def scale_value(x) -> np.ndarray:
    return np.exp2(np.asarray(x, dtype=np.float64) - 127.0)


def scale_byte(amax: float) -> int:
    """The smallest 2^e, e >= -100, with amax <= 448 * 2^e, as its exponent byte."""
    x = LOW
    while amax > 448.0 * 2.0 ** (x - 127):
        x += 1
    return x


def top(x) -> float:
    """Largest finite magnitude (0 without one)."""
    a = np.abs(x)[np.isfinite(x)]
    return float(a.max()) if a.size else 0.0


def encode(x, byte: int) -> np.ndarray:
    y = np.where(np.isfinite(x), x, np.nan) / scale_value(byte)
    return e4m3_encode(y)


def values(codes, scales, block: int) -> np.ndarray:
    """The numbers that the entries stand for."""
    s = np.repeat(scale_value(scales), block)[: len(codes)]
    return e4m3_decode(codes) * s[:, None]


def rotate(x, pos, theta: float) -> np.ndarray:
    """Elements e and e + d/2 of rows x [n][..][d] turned by pos * theta^(-2e/d)."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    a = np.asarray(pos, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(d // 2) / d)
    a = a.reshape(a.shape[0], *([1] * (x.ndim - 2)), d // 2)
    lo, hi = x[..., : d // 2], x[..., d // 2:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)


def append(codes, scales, cached: int, new, block: int, capacity: int):
    """New rows behind `cached` entries; codes and scales are changed in place."""
    end = min(cached + len(new), capacity)
    for b0 in range(cached // block * block, end, block):
        t0, t1 = max(b0, cached), min(b0 + block, end)
        x = np.asarray(new[t0 - cached: t1 - cached], dtype=np.float64)
        byte = scale_byte(top(x))
        if t0 > b0:
            old = int(scales[b0 // block])
            byte = max(byte, old)
            if byte > old:
                codes[b0:t0] = encode(e4m3_decode(codes[b0:t0]) * scale_value(old), byte)
        codes[t0:t1] = encode(x, byte)
        scales[b0 // block] = byte


def compact(codes, scales, keep, block: int):
    """(codes, scales) of the kept entries, len(keep) and ceil(len / block) of them."""
    x = values(codes, scales, block)[np.asarray(keep, dtype=np.int64)]
    out = np.empty(x.shape, np.uint8)
    bytes_ = []
    for b0 in range(0, len(x), block):
        byte = scale_byte(top(x[b0:b0 + block]))
        out[b0:b0 + block] = encode(x[b0:b0 + block], byte)
        bytes_.append(byte)
    return out, np.array(bytes_, dtype=np.uint8)


def attention(q, k, v, mask: str, inclusive: bool = False, scale=None) -> np.ndarray:
    """Rows q [m][d] standing at the last m of the n entries k, v [n][d]."""
    m, d = q.shape
    n = len(k)
    out = np.zeros((m, d))
    tau = d ** -0.5 if scale is None else scale
    for i in range(m):
        at = n - m + i
        if mask == "causal":
            js = np.arange(0, max(0, at + 1))
        else:
            js = np.arange(max(0, at + (0 if inclusive else 1)), n)
        if len(js) == 0:
            continue
        z = tau * (k[js] @ q[i])
        w = np.exp(z - np.nanmax(z)) if not np.isnan(z).all() else z
        out[i] = (w / w.sum()) @ v[js]
    return out
