"""CPU oracle of the 8-bit pruned cache and of eviction by collected attention weight: NumPy, 64 bits,
written from the definitions in include/gvote.h.  Shares no code with the CUDA library.

Caches are lists: `codes[r][h]` holds the e4m3 values (as float64, before the scale) of the rows head h of
request r has, `scales[r][h]` one scale per 64 rows."""
from __future__ import annotations

import math
from typing import Optional, Tuple

import numpy as np

BLOCK = 64
E4M3_MAX = 448.0
MIN_EXP = -126


def e4m3_round(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value (|x| <= 448; ties to the even code; not finite -> NaN): 3 fraction bits, exponents -6 .. 8,
    multiples of 2^-9 below 2^-6."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))          # |x| in [2^(e-1), 2^e)
        step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
        return np.where(np.isfinite(x), np.rint(x / step) * step, np.nan)


def block_scale(rows: np.ndarray) -> float:
    """The smallest 2^e, e >= -126, with max |x| <= 448 * 2^e over the finite entries."""
    a = np.abs(rows[np.isfinite(rows)])
    top = float(a.max()) if a.size else 0.0
    e = MIN_EXP
    if top > 0:
        e = max(MIN_EXP, math.frexp(top)[1] - 10)
        while top > math.ldexp(E4M3_MAX, e):
            e += 1
    return math.ldexp(1.0, e)


def quantise(rows: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """Rows [n, d] -> (code values [n, d], scales [ceil(n / 64)])."""
    rows = np.asarray(rows, dtype=np.float64)
    codes = np.empty_like(rows)
    scales = np.empty((rows.shape[0] + BLOCK - 1) // BLOCK)
    for b in range(scales.size):
        s = slice(b * BLOCK, (b + 1) * BLOCK)
        scales[b] = block_scale(rows[s])
        codes[s] = e4m3_round(rows[s] / scales[b])
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    return codes * np.repeat(scales, BLOCK)[:codes.shape[0], None]


def append(codes: np.ndarray, scales: np.ndarray, new: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """One call's new rows [m, d] behind the rows held."""
    codes, scales, new = codes.copy(), list(scales), np.asarray(new, dtype=np.float64)
    n, m = codes.shape[0], new.shape[0]
    codes = np.concatenate([codes, np.zeros_like(new)])
    for first in range(n - n % BLOCK, n + m, BLOCK):
        b, last = first // BLOCK, min(first + BLOCK, n + m)
        lo = max(first, n)
        x = new[lo - n:last - n]
        s = block_scale(x)
        if lo > first:                                             # the block holds rows already
            s = max(s, scales[b])
            if x.shape[0]:
                codes[first:lo] = e4m3_round(codes[first:lo] * (scales[b] / s))
                scales[b] = s
        else:
            scales.append(s)
        codes[lo:last] = e4m3_round(x / s)
    return codes, np.asarray(scales)


def softmax_rows(q: np.ndarray, k: np.ndarray, n_q: int) -> Tuple[np.ndarray, np.ndarray]:
    """Weights [n_q, g, n] and log denominators [n_q, g] of q [n_q, g, d] over k [n, d], the query tokens being the
    last n_q rows: token i sees rows < n - (n_q - 1 - i)."""
    n, d = k.shape
    logit = np.einsum("igd,nd->ign", q, k) / math.sqrt(d)
    sees = np.arange(n)[None, :] < (n - (n_q - 1 - np.arange(n_q)))[:, None]
    logit = np.where(sees[:, None, :], logit, -np.inf)
    top = logit.max(axis=2, keepdims=True) if n else np.full(logit.shape[:2] + (1,), -np.inf)
    e = np.exp(logit - np.where(np.isinf(top), 0.0, top))
    z = e.sum(axis=2, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (np.where(np.isinf(top), 0.0, top) + np.log(z))[:, :, 0]
    return e / np.where(z == 0, 1.0, z), lse


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray):
    """q [n_q, g, d] over the rows k, v [n, d] of one KV head: out [n_q, g, d], lse [n_q, g], and the weight each row
    collects [n]."""
    w, lse = softmax_rows(q, k, q.shape[0])
    return np.einsum("ign,nd->igd", w, v), lse, w.sum(axis=(0, 1))


def collected(q: np.ndarray, k: np.ndarray) -> np.ndarray:
    """Weight each key of one KV head collects from q [n_q, g, d], the last n_q rows' queries."""
    return softmax_rows(q, k, q.shape[0])[0].sum(axis=(0, 1))


def evict(acc: np.ndarray, keep: int, n_recent: int, n_sink: int) -> np.ndarray:
    """Keep flags of one head's n rows: the last n_recent, the first n_sink, then by weight (ties: lower slot; a NaN
    is the lowest weight), keep in all."""
    n = acc.shape[0]
    k = min(max(keep, 0), n)
    recent = min(n_recent, k)
    sink = min(n_sink, k - recent)
    out = np.zeros(n, dtype=bool)
    out[n - recent:] = True
    out[:sink] = True
    mid = np.arange(sink, n - recent)
    w = acc[mid].astype(np.float64)
    order = np.lexsort((mid, -np.where(np.isnan(w), 0.0, w), np.isnan(w)))
    out[mid[order[:k - recent - sink]]] = True
    return out


def rows_of(mask: Optional[np.ndarray], n: int) -> np.ndarray:
    """Source slots a head keeps among its n rows, ascending (mask None: all)."""
    return np.arange(n) if mask is None else np.flatnonzero(mask[:n])
