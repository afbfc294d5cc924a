"""Definitions in 64 bits of the normed and quantised append and of attention with formed scores, written from the formulas in
include/ecoserve.h, one row or token at a time.  Test infrastructure only; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

BS = 16
BAD = 255
MOST = {"int8": 127.0, "e4m3": 448.0}


def norm(x: np.ndarray, eps: float, weight):
    """x [D] -> fp64."""
    x = x.astype(np.float64)
    with np.errstate(all="ignore"):
        y = x / math.sqrt(float((x * x).mean()) + eps) if np.isfinite(x).all() else x * np.where(np.isnan(x).any(), np.nan, 0.0)
    return y if weight is None else y * weight.astype(np.float64)


def e4m3_number(byte: int) -> float:
    sign, up, low = -1.0 if byte & 128 else 1.0, byte >> 3 & 15, byte & 7
    if up == 15 and low == 7:
        return math.nan
    return sign * (low * 2.0 ** -9 if up == 0 else (8 + low) * 2.0 ** (up - 10))


E4M3 = np.array([e4m3_number(b) for b in range(256)])
_POSITIVE = E4M3[:127]  # 0 .. 448, ascending


def to_e4m3(x: float) -> int:
    """The nearest e4m3 number's byte, the even one of two; |x| <= 448."""
    a = abs(x)
    i = int(np.searchsorted(_POSITIVE, a))
    if i > 0 and (i == 127 or a - _POSITIVE[i - 1] < _POSITIVE[i] - a or (a - _POSITIVE[i - 1] == _POSITIVE[i] - a and (i - 1) % 2 == 0)):
        i -= 1
    return i | (128 if math.copysign(1.0, x) < 0 else 0)


def scale_byte(size: float, fmt: str) -> int:
    e = -126
    while size > MOST[fmt] * 2.0 ** e:
        e += 1
    return e + 127


def code(x: np.ndarray, fmt: str):
    """A row [D] -> (bytes uint8 [D], scale byte)."""
    x = x.astype(np.float64)
    if not np.isfinite(x).all():
        return np.zeros(len(x), dtype=np.uint8), BAD
    b = scale_byte(float(np.abs(x).max()), fmt)
    y = x / 2.0 ** (b - 127)
    if fmt == "int8":
        return np.array([round(float(v)) & 255 for v in y], dtype=np.uint8), b
    return np.array([to_e4m3(float(v)) for v in y], dtype=np.uint8), b


def number(codes: np.ndarray, fmt: str) -> np.ndarray:
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else E4M3[codes]


def value(codes: np.ndarray, b, fmt: str) -> np.ndarray:
    """codes [..., D], scale bytes [...] -> what they stand for."""
    b = np.asarray(b)
    return np.where(b[..., None] == BAD, np.nan, number(codes, fmt) * 2.0 ** (b[..., None].astype(np.float64) - 127))


def attend(q: np.ndarray, keys: np.ndarray, values: np.ndarray, at: np.ndarray, position: int, scale: float, cap: float = 0.0, slopes=None):
    """One token's group of heads q [G, D] over keys, values [n, D] at places `at`: (out [G, D], lse [G], sum of weights times |value| [G, D], how far
    fp32 may be off the scores, [G])."""
    G, D = q.shape
    if len(keys) == 0:
        return np.zeros((G, D)), np.full(G, -np.inf), np.zeros((G, D)), np.zeros(G)
    q, keys, values = (t.astype(np.float64) for t in (q, keys, values))
    with np.errstate(all="ignore"):
        s = q @ keys.T * scale
        # products of 8-bit significands are exact in fp32; D of them are added, then a handful of roundings
        off = (D + 8) * 2.0 ** -24 * (np.abs(q) @ np.abs(keys).T).max(1) * scale
        if cap:
            s = cap * np.tanh(s / cap)
            # (up to 64 of the cap, beyond that of the score: what is small beside a cap is not to feel it)
            off = off + np.minimum(cap, np.maximum(np.abs(s).max(1), 64.0)) * 2.0 ** -21
        if slopes is not None:
            bias = slopes[:, None] * (at - position)[None]
            s = s + bias
            off = off + np.abs(bias).max(1) * 2.0 ** -22
        off = off + np.abs(s).max(1) * 2.0 ** -22
        m = s.max(1, keepdims=True)
        w = np.exp(s - m)
        l = w.sum(1, keepdims=True)
        return (w / l) @ values, (m + np.log(l))[:, 0], (w / l) @ np.abs(values), off
