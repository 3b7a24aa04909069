"""CPU reference of the 4-bit cache and of the eviction by attention weight, in float64 numpy from their definitions.  Test infrastructure only."""
from __future__ import annotations

import math
from typing import List, Sequence, Tuple

import numpy as np

D = 128
ROW = 68
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


def scale_byte(block: np.ndarray) -> int:
    """The e8m0 byte of a block of 32 values: the smallest power of two at which the largest needs at most half a step, not below 2^-127."""
    top = float(np.max(np.abs(block))) if np.all(np.isfinite(block)) else math.nan
    if math.isnan(top):
        return 255
    if top == 0.0:
        return 0
    m, e = math.frexp(top)                                  # top = m 2^e, m in [.5, 1); 7 2^(s - 127) = .875 2^(s - 124)
    return max(0, e + 124 + (1 if m > 0.875 else 0))


def code_of(x: float) -> int:
    """The code of |x| times 1: nearest of the grid, ties to the even code, at most 6."""
    d = np.abs(GRID - abs(x))
    best = np.flatnonzero(d == d.min())
    return int(best[0]) if len(best) == 1 or best[0] % 2 == 0 else int(best[1])


def pack(rows: np.ndarray) -> np.ndarray:
    """float64 [n, 128] of bfloat16 values -> uint8 [n, 68]."""
    out = np.zeros((len(rows), ROW), dtype=np.uint8)
    for r, row in enumerate(np.asarray(rows, dtype=np.float64)):
        for k in range(4):
            block = row[32 * k:32 * k + 32]
            s = scale_byte(block)
            out[r, 64 + k] = s
            if s == 255:
                continue
            for i, x in enumerate(block):
                c = code_of(x * 2.0 ** (127 - s))
                if s == 253:
                    c = min(c, 5)
                c |= 8 if math.copysign(1.0, x) < 0 else 0
                out[r, 16 * k + i // 2] |= c << (4 * (i % 2))
    return out


def unpack(rows: np.ndarray) -> np.ndarray:
    """uint8 [n, 68] -> float64 [n, 128]."""
    rows = np.asarray(rows, dtype=np.uint8)
    codes = np.stack([rows[:, :64] & 15, rows[:, :64] >> 4], -1).reshape(-1, D)
    s = rows[:, 64:].astype(np.float64)
    unit = np.where(s == 255, np.nan, 2.0 ** (s - 127)).repeat(32, axis=1)
    return np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7] * unit


def active_rows(bounds: np.ndarray, T: int, ids: Sequence[int], tail: bool = True) -> np.ndarray:
    M = len(bounds) - 1
    parts = [np.arange(bounds[j], bounds[j + 1]) for j in ids if 0 <= j < M]
    if tail:
        parts.append(np.arange(bounds[M], T))
    return np.concatenate(parts).astype(np.int64) if parts else np.zeros(0, dtype=np.int64)


def attend(q: np.ndarray, K: np.ndarray, V: np.ndarray, rows: np.ndarray) -> Tuple[np.ndarray, np.ndarray, np.ndarray, float]:
    """(out [G, d], lse [G], sum of p |v| [G, d], largest sum of |q_i k_i| / sqrt(d)) over cache rows `rows`."""
    G = len(q)
    if len(rows) == 0:
        return np.zeros((G, D)), np.full(G, -math.inf), np.zeros((G, D)), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        x = q @ K[rows].T / math.sqrt(D)
        m = x.max(axis=1, keepdims=True)
        p = np.exp(x - m)
        l = p.sum(axis=1, keepdims=True)
        p /= l
        return p @ V[rows], (m + np.log(l))[:, 0], p @ np.abs(V[rows]), float((np.abs(q) @ np.abs(K[rows]).T).max() / math.sqrt(D))


def chunk_weights(q: np.ndarray, K: np.ndarray, lse: np.ndarray, bounds: np.ndarray, ids: Sequence[int]) -> dict:
    """{chunk: sum over its tokens and the heads of exp(logit - lse)}."""
    out = {}
    for j in ids:
        x = q @ K[bounds[j]:bounds[j + 1]].T / math.sqrt(D)
        out[int(j)] = math.fsum(np.exp(x - lse[:, None]).ravel())
    return out


def keep(weights: np.ndarray, bounds: np.ndarray, keep_tokens: int, recent: int, sink: int) -> List[int]:
    """weights [H, M] -> ids of the chunks that stay, ascending."""
    M, end = len(bounds) - 1, int(bounds[-1])
    size = np.diff(bounds)
    pinned = [j for j in range(M) if bounds[j] < sink or bounds[j + 1] > end - recent]
    left = max(0, keep_tokens - int(size[pinned].sum()))
    total = {}
    for j in range(M):
        t = math.fsum(float(w) for w in weights[:, j]) if np.all(np.isfinite(weights[:, j])) else float(np.sum(weights[:, j], dtype=np.float64))
        total[j] = (1, 0.0) if math.isnan(t) else (0, -t)   # sort key: numbers first, largest first
    kept = list(pinned)
    for j in sorted(set(range(M)) - set(pinned), key=lambda j: (total[j], j)):
        left -= int(size[j])
        if left < 0:
            break
        kept.append(j)
    return sorted(kept)
