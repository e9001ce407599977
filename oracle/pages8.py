"""Plain definitions behind the paged 8-bit KV cache (pipo_kv8_pages): codes and
scales of a sequence's blocks as rows are added, and attention with the scores
that pipo_attn_scores describes."""
from __future__ import annotations

from typing import Optional

import numpy as np

BLOCK = 16
CLAMP = 57344.0
TOP = {"e4m3": 448.0, "int8": 127.0}
EXPONENTS = {"e4m3": (-15, 7), "int8": (-24, 9)}


def nearest(x: np.ndarray, fmt: str) -> np.ndarray:
    """The numbers that have a code nearest to x (in units of the scale), half to even."""
    if fmt == "int8":
        return np.rint(x)
    exp = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -40)))
    step = 2.0 ** (np.maximum(exp, -6) - 3)
    return np.rint(x / step) * step


def least_exponent(amax: float, fmt: str) -> int:
    lo, hi = EXPONENTS[fmt]
    e = lo
    while amax > TOP[fmt] * 2.0 ** e and e < hi:
        e += 1
    return e


class Blocks:
    """One sequence's keys (or values): numbers in units of their block's scale."""

    def __init__(self, heads: int, dim: int, fmt: str):
        self.fmt = fmt
        self.units = np.zeros((0, heads, dim))
        self.exps = np.zeros((0, heads), np.int64)

    def append(self, rows: np.ndarray, length: int) -> None:
        """rows [n][heads][dim] become the positions length - n .. length - 1; those
        below stay, whatever was behind them goes"""
        rows = np.nan_to_num(np.asarray(rows, np.float16).astype(np.float64), nan=0.0)
        rows = np.clip(rows, -CLAMP, CLAMP)
        n, heads = len(rows), self.units.shape[1]
        first = length - n
        assert first <= len(self.units)
        units = np.zeros((length,) + self.units.shape[1:])
        units[:first] = self.units[:first]
        tiles = -(-length // BLOCK)
        exps = np.full((tiles, heads), EXPONENTS[self.fmt][0])
        kept = min(len(self.exps), tiles)
        exps[:kept] = self.exps[:kept]
        for t in range(first // BLOCK, tiles):
            lo, hi = max(first, BLOCK * t), min(length, BLOCK * (t + 1))
            if lo >= hi:
                continue
            for h in range(heads):
                e = least_exponent(np.abs(rows[lo - first:hi - first, h]).max(), self.fmt)
                if lo > BLOCK * t:
                    e = max(e, exps[t, h])
                    units[BLOCK * t:lo, h] = nearest(
                        units[BLOCK * t:lo, h] * 2.0 ** (exps[t, h] - e), self.fmt)
                units[lo:hi, h] = nearest(rows[lo - first:hi - first, h] * 2.0 ** -float(e), self.fmt)
                exps[t, h] = e
        self.units, self.exps = units, exps

    def values(self) -> np.ndarray:
        """float64 [length][heads][dim]"""
        e = np.repeat(self.exps, BLOCK, axis=0)[:len(self.units)]
        return self.units * 2.0 ** e[..., None].astype(np.float64)


def seen(n_rows: int, length: int, window: int = 0, prefix: int = 0) -> np.ndarray:
    """[rows][keys] that a sequence's last rows see"""
    pos, key = length - n_rows + np.arange(n_rows)[:, None], np.arange(length)[None]
    out = key <= pos
    if window:
        out &= pos - key < window
    return out | (key < prefix)


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, cap: float = 0.0,
              slopes: Optional[np.ndarray] = None, window: int = 0, prefix: int = 0) -> np.ndarray:
    """q [n][H][D], k and v [T][Hkv][D] -> [n][H][D] in float64: the last n of T positions;
    a row that sees nothing is 0."""
    n, H, D = q.shape
    G, T = H // k.shape[1], len(k)
    mask, out = seen(n, T, window, prefix), np.zeros((n, H, D))
    far = np.abs(T - n + np.arange(n)[:, None] - np.arange(T)[None])
    for h in range(H):
        s = q[:, h].astype(np.float64) @ k[:, h // G].astype(np.float64).T
        if cap:
            s = cap * np.tanh(s / cap)
        if slopes is not None:
            s = s - float(slopes[h]) * far
        s = np.where(mask, s, -np.inf)
        for j in np.nonzero(mask.any(axis=1))[0]:
            p = np.exp(s[j] - s[j].max())
            out[j, h] = p @ v[:, h // G] / p.sum()
    return out
