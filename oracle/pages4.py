"""Plain numpy form of the paged 4-bit cache and of rotary positions.

A group of elements x of one row (32 dims of K, 128 of V) is held as
    m = bf16(min x),  s = max(bf16(fl(fl(max x - m) fl(1/15))), 2^-100),  c = clamp(rint(fl(fl(x - m) fl(1/s))), 0, 15)
in 32-bit arithmetic, and stands for m + c s.  These roundings are part of the definition; everything computed from the
values is in 64 bits, and tables and slots are integers.
"""
from __future__ import annotations

import numpy as np

PAGE = 64
MOST = np.float32(2.0 ** 64)


def as_bf16(x: np.ndarray) -> np.ndarray:
    """fp32 values rounded to bf16 (nearest, ties to even)."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


def held(x: np.ndarray, group: int) -> np.ndarray:
    """What rows x [..., d] stand for once held in groups of `group` dims, in 64 bits."""
    x = np.asarray(x, np.float32)
    x = np.where(np.isfinite(x), np.clip(x, -MOST, MOST), np.float32(0))
    y = x.reshape(*x.shape[:-1], x.shape[-1] // group, group)
    m = as_bf16(y.min(-1, keepdims=True))
    s = as_bf16((y.max(-1, keepdims=True) - m) * np.float32(1.0 / 15.0))
    s = np.maximum(s, np.float32(2.0 ** -100))
    c = np.clip(np.rint((y - m) * (np.float32(1.0) / s)), 0, 15)
    return (m.astype(np.float64) + c.astype(np.float64) * s.astype(np.float64)).reshape(x.shape)


def held_rows(k: np.ndarray, v: np.ndarray):
    """Keys and values [..., 128] as the pages hold them."""
    return held(k, 32), held(v, 128)


def attend(q, k, v, scale: float, sees, bias=None):
    """softmax(scale q k^T + bias) v for rows q [n, d] over k, v [T, d], row i over the first sees[i] tokens; and the same
    sum over |v|, which what a weight's rounding costs is proportional to.  Rows that see nothing are zero."""
    out, size = np.zeros((len(q), v.shape[1])), np.zeros((len(q), v.shape[1]))
    for i, row in enumerate(np.asarray(q, np.float64)):
        a = scale * (k[:sees[i]] @ row)
        if bias is not None:
            with np.errstate(invalid="ignore"):
                a = a + bias[:sees[i]].astype(np.float64)
        if not len(a) or a.max() == -np.inf:
            continue
        e = np.exp(a - a.max())
        out[i], size[i] = e @ v[:sees[i]] / e.sum(), e @ np.abs(v[:sees[i]]) / e.sum()
    return out, size


class Tables:
    """Page tables as the definition has them: one request after the other."""

    def __init__(self, S: int, M: int, P: int):
        self.M, self.P = M, P
        self.table, self.len = np.full((S, M), -1), np.zeros(S, np.int64)
        self.free = list(range(P - 1, -1, -1))

    def extend(self, counts, n_rows: int):
        S = len(self.len)
        starts, slots, positions = [0], np.full(n_rows, -1), np.full(n_rows, -1)
        need, total, left = [], 0, len(self.free)
        for s in range(S):
            c = max(0, int(counts[s]))
            ok = starts[s] + c <= n_rows and self.len[s] + c <= self.M * PAGE
            need.append(-(-(self.len[s] + c) // PAGE) - -(-self.len[s] // PAGE) if ok else 0)
            total += need[s]
            if ok and (need[s] == 0 or total <= left):
                for j in range(int(need[s])):
                    self.table[s, -(-self.len[s] // PAGE) + j] = self.free.pop()
                pos = self.len[s] + np.arange(c)
                rows = slice(starts[s], starts[s] + c)
                slots[rows], positions[rows] = self.table[s, pos // PAGE] * PAGE + pos % PAGE, pos
                self.len[s] += c
            starts.append(starts[s] + c)
        return np.minimum(starts, n_rows), slots, positions

    def truncate(self, lens):
        back = []
        for s, to in enumerate(lens):
            if not 0 <= to <= self.len[s]:
                continue
            for j in range(-(-int(to) // PAGE), -(-int(self.len[s]) // PAGE)):
                if 0 <= self.table[s, j] < self.P:           # (a page that is missing is not given back)
                    back.append(int(self.table[s, j]))
                self.table[s, j] = -1
            self.len[s] = to
        self.free += back[::-1]


def rotate(x, positions, turns, factor: float = 1.0, interleaved: bool = False, transpose: bool = False) -> np.ndarray:
    """Rows x [N, heads, d] turned by 2 pi positions[n] turns[i] / 2^64 (whole numbers; reduced exactly)."""
    x = np.asarray(x, np.float64)
    r = 2 * len(turns)
    angle = np.array([[(int(p) * int(t)) % 2 ** 64 / 2.0 ** 64 for t in turns] for p in positions]).reshape(len(positions), r // 2)
    c, s = factor * np.cos(2 * np.pi * angle)[:, None], factor * np.sin(2 * np.pi * angle)[:, None] * (-1 if transpose else 1)
    y = x.copy()
    one, two = (np.s_[..., 0:r:2], np.s_[..., 1:r:2]) if interleaved else (np.s_[..., :r // 2], np.s_[..., r // 2:r])
    y[one], y[two] = x[one] * c - x[two] * s, x[two] * c + x[one] * s
    skip = np.asarray(positions) < 0
    y[skip] = x[skip]
    return y
