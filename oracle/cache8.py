"""Plain numpy form of the 8-bit cache: what its codes are, attention over it in fp64, and block selection.

A block of 64 rows x of one head is held as
    a = max(max |x|, 2^-100),  scale = fl(a fl(1/127)),  c = rint(fl(x fl(127 / a)))
in 32-bit arithmetic, and stands for c * scale.  These roundings are part of the definition (codes are compared
exactly); everything computed from the codes is in 64 bits.
"""
from __future__ import annotations

import numpy as np

BLOCK = 64
FLOOR = np.float32(2.0 ** -100)


def quantise_block(x: np.ndarray):
    """Codes int8 [r, d] and scale of the rows x [r, d] (fp32 values)."""
    x = np.asarray(x, np.float32)
    a = max(np.float32(np.max(np.abs(x))), FLOOR)
    codes = np.rint(x * (np.float32(127.0) / a)).astype(np.int8)
    return codes, np.float32(a * (np.float32(1.0) / np.float32(127.0)))


def quantise(x: np.ndarray):
    """Codes [T, d], scales [blocks] and per-block (least, largest) codes [blocks, 2, d] of one head's rows."""
    T, d = x.shape
    nb = -(-T // BLOCK)
    codes, scale, bounds = np.zeros((T, d), np.int8), np.zeros(nb, np.float32), np.zeros((nb, 2, d), np.int8)
    for b in range(nb):
        sl = slice(b * BLOCK, min(T, (b + 1) * BLOCK))
        codes[sl], scale[b] = quantise_block(x[sl])
        bounds[b, 0], bounds[b, 1] = codes[sl].min(0), codes[sl].max(0)
    return codes, scale, bounds


def values(codes: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """What the codes of one head stand for, in 64 bits."""
    return codes.astype(np.float64) * np.repeat(scale.astype(np.float64), BLOCK)[:len(codes), None]


def visible(T: int, n_pos: int, p: int, causal: bool) -> int:
    return max(0, T - n_pos + 1 + p) if causal else T


def attend(q, k, v, scale: float, bias=None, causal: bool = False, blocks=None) -> np.ndarray:
    """O [n_pos, G, d] of one head for q [n_pos, G, d] over values k, v [T, d]; blocks [n_pos, m] (-1: none)
    restricts what each position reads; rows that see nothing are zero."""
    n_pos, G, d = q.shape
    T = len(k)
    out = np.zeros((n_pos, G, d))
    for p in range(n_pos):
        seen = np.arange(T) < visible(T, n_pos, p, causal)
        if blocks is not None:
            seen &= np.isin(np.arange(T) // BLOCK, [b for b in blocks[p] if b >= 0])
        if bias is not None:
            seen &= bias != -np.inf
        if not seen.any():
            continue
        a = scale * (q[p].astype(np.float64) @ k[seen].T)
        if bias is not None:
            a = a + bias[seen].astype(np.float64)
        e = np.exp(a - a.max(1, keepdims=True))
        out[p] = (e / e.sum(1, keepdims=True)) @ v[seen]
    return out


def block_scores(q, bounds, k_scale) -> np.ndarray:
    """Scores [blocks] (fp32 as defined) of one position's rows q [G, d]: the largest over the rows of
    fl(fl(s_q I) scale), I the exact integer sum_e max(c lo_e, c hi_e)."""
    best = np.full(len(k_scale), -np.inf, np.float32)
    for row in np.asarray(q, np.float32):
        c, s = quantise_block(row[None])
        c = c[0].astype(np.int64)
        whole = np.maximum(c * bounds[:, 0].astype(np.int64), c * bounds[:, 1].astype(np.int64)).sum(1)
        best = np.maximum(best, (s * whole.astype(np.float32)) * k_scale)
    return best


def select(q, bounds, k_scale, T: int, m: int, keep_first: int, keep_last: int, causal: bool) -> np.ndarray:
    """Blocks [n_pos, m] of one head, ascending, -1 after the last."""
    n_pos = q.shape[0]
    out = np.full((n_pos, m), -1, np.int64)
    for p in range(n_pos):
        cand = -(-visible(T, n_pos, p, causal) // BLOCK)
        s = block_scores(q[p], bounds[:cand], k_scale[:cand]).astype(np.float64)
        forced = [b for b in range(cand) if b < keep_first or b >= cand - keep_last]
        s[forced] = np.inf
        order = np.lexsort((np.arange(cand), -s))[:m]
        out[p, :len(order)] = np.sort(order)
    return out
