"""Definitions in 64 bits of the rotated append, the block summaries, block selection and attention over listed blocks, written from
the formulas in include/ecoserve.h, one token, block or head at a time.  Test infrastructure only; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

BS = 16
NOT_FINITE = 127


def rotate(x: np.ndarray, where: np.ndarray, freq: np.ndarray, adjacent: bool):
    """x [..., D] turned by `where` [pairs] (the coordinate of each pair's axis): (turned, |a| + |b| of each element's pair, 0 where nothing is turned)."""
    out, size = x.astype(np.float64).copy(), np.zeros(x.shape)
    pairs = len(freq)
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + pairs)
        c, s = math.cos(float(where[i]) * freq[i]), math.sin(float(where[i]) * freq[i])
        p, q = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
        out[..., a], out[..., b] = p * c - q * s, p * s + q * c
        size[..., a] = size[..., b] = np.abs(p) + np.abs(q)
    return out, size


def code_exponent(size: float) -> int:
    e = -126
    while size > 127.0 * 2.0 ** e:
        e += 1
    return e


def summarise(keys: np.ndarray):
    """keys [16, D] -> (codes int [2, D], exponent)."""
    if not np.isfinite(keys).all():
        return np.zeros((2, keys.shape[1]), dtype=np.int64), NOT_FINITE
    k = keys.astype(np.float64)
    e = code_exponent(float(np.abs(k).max()))
    return np.stack([np.ceil(k.max(0) / 2.0 ** e), np.floor(k.min(0) / 2.0 ** e)]).astype(np.int64), e


def query_codes(q: np.ndarray):
    """q [D] -> (codes int [D], exponent); Python's round is to even."""
    if not (np.abs(q.astype(np.float64)) <= 127.0 * 2.0 ** 100).all():
        return np.zeros(len(q), dtype=np.int64), 0
    e = code_exponent(float(np.abs(q.astype(np.float64)).max()))
    return np.array([round(float(x) / 2.0 ** e) for x in q], dtype=np.int64), e


def scores(q: np.ndarray, codes: np.ndarray, exps: np.ndarray):
    """q [G, D], codes int [n, 2, D], exps [n] -> fp64 [n]."""
    best = np.full(len(exps), -np.inf)
    for head in q:
        qc, eq = query_codes(head)
        bound = np.maximum(codes[:, 0] * qc, codes[:, 1] * qc).sum(1)
        best = np.maximum(best, bound.astype(np.float64) * 2.0 ** (eq + exps.astype(np.float64)))
    return np.where(exps == NOT_FINITE, np.inf, best)


def choose(score: np.ndarray, n: int, K: int, keep_first: int, keep_last: int):
    """The blocks of a token that sees n of them; score[j] for the full ones."""
    if n <= K:
        return list(range(n))
    kept = [j for j in range(n) if j < keep_first or j >= n - keep_last]
    others = sorted((j for j in range(n) if keep_first <= j < n - keep_last), key=lambda j: (-score[j], j))
    return sorted(kept + others[:K - len(kept)])


def attend(q: np.ndarray, keys: np.ndarray, values: np.ndarray, scale: float):
    """One token's group of heads q [G, D] over keys, values [n, D]: (out [G, D], lse [G], sum of weights times |value| [G, D], the largest
    sum of |q k| over the keys, scaled, [G])."""
    G, D = q.shape
    if len(keys) == 0:
        return np.zeros((G, D)), np.full(G, -np.inf), np.zeros((G, D)), np.zeros(G)
    s = (q.astype(np.float64) @ keys.astype(np.float64).T) * scale
    m = s.max(1, keepdims=True)
    w = np.exp(s - m)
    l = w.sum(1, keepdims=True)
    v = values.astype(np.float64)
    return (w / l) @ v, (m + np.log(l))[:, 0], (w / l) @ np.abs(v), (np.abs(q.astype(np.float64)) @ np.abs(keys.astype(np.float64)).T).max(1) * scale
