"""Plain definitions behind the paged 4-bit KV cache (pipo_kv_pages): what a
cached row stands for, attention of sequences of different lengths, and what
the calls on page tables do, one sequence and page after the other."""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import numpy as np

from .opt import dequant_int4_g64, quant_kv_int4_g64

CLAMP = 57344.0


def page_rows(x: np.ndarray) -> np.ndarray:
    """float64 values that fp16 rows x [R][d] have in the cache: elements are
    clamped to +-57344 (NaN: 0), then quantized as quant_kv_int4_g64 does."""
    x = np.nan_to_num(np.asarray(x, np.float16).astype(np.float32), nan=0.0, posinf=CLAMP,
                      neginf=-CLAMP)
    q, sm = quant_kv_int4_g64(np.clip(x, -CLAMP, CLAMP).astype(np.float16))
    return dequant_int4_g64(q, sm, np.float64)


def page_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, seen: np.ndarray) -> np.ndarray:
    """q [n][H][D], k and v [T][Hkv][D], seen [n][T] -> [n][H][D] in float64;
    head h reads key/value head h // (H // Hkv), a row that sees nothing is 0."""
    n, H, D = q.shape
    G = H // k.shape[1]
    out = np.zeros((n, H, D))
    for h in range(H):
        s = q[:, h].astype(np.float64) @ k[:, h // G].astype(np.float64).T
        s = np.where(seen, s, -np.inf)
        for j in np.nonzero(seen.any(axis=1))[0]:
            p = np.exp(s[j] - s[j].max())
            out[j, h] = p @ v[:, h // G] / p.sum()
    return out


def norm_rope(x: np.ndarray, gamma: Optional[np.ndarray], cos_sin: np.ndarray, eps: float,
              scale: float) -> np.ndarray:
    """x [M][heads][D], cos_sin [M][D/2][2] -> float64 [M][heads][D]"""
    x = x.astype(np.float64)
    if gamma is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * gamma.astype(np.float64)
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    c, s = (cos_sin[:, None, :, i].astype(np.float64) for i in (0, 1))
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1) * scale


# ---------------------------------------------------------------------------
def _pages(n: int, ps: int) -> int:
    return -(-max(n, 0) // ps)


def _held(table, lens, ps) -> List[List[int]]:
    return [[int(p) for p in row[:_pages(n, ps)]] for row, n in zip(table, lens)]


def _as_table(rows: Sequence[Sequence[int]], width: int) -> np.ndarray:
    out = np.full((len(rows), width), -1, np.int32)
    for i, r in enumerate(rows):
        out[i, :len(r)] = r
    return out


def _free(rows, n_pages) -> List[int]:
    return sorted(set(range(n_pages)) - {p for r in rows for p in r})


def resize(table, lens, want, n_pages: int, ps: int) -> Tuple[np.ndarray, np.ndarray, int]:
    """(table, lengths, pages lacking)"""
    width, held = table.shape[1], _held(table, lens, ps)
    rows = [r if w < 0 else r[:_pages(w, ps)] for r, w in zip(held, want)]
    free = _free(rows, n_pages)
    need = [0 if w < 0 else max(0, _pages(w, ps) - len(r)) for r, w in zip(rows, want)]
    excess = [0 if w < 0 else max(0, _pages(w, ps) - width) for w in want]
    lacking = max(0, sum(need) - sum(excess) - len(free)) + sum(excess)
    if lacking:
        return _as_table(held, width), np.array(lens, np.int32), lacking
    for r, n in zip(rows, need):
        r += free[:n]
        free = free[n:]
    return (_as_table(rows, width),
            np.array([n if w < 0 else w for n, w in zip(lens, want)], np.int32), 0)


def fork(table, lens, parent, n_pages: int, ps: int):
    """(table, lengths, pairs, 0), or (None, None, [], pages lacking)"""
    held = _held(table, lens, ps)
    ok = [0 <= p < len(held) for p in parent]
    rows = [list(held[p]) if k else [] for p, k in zip(parent, ok)]
    out_len = np.array([max(lens[p], 0) if k else 0 for p, k in zip(parent, ok)], np.int32)
    copies = [i for i, (p, k) in enumerate(zip(parent, ok))
              if k and out_len[i] % ps and p in parent[:i]]
    free = _free([r[:-1] if i in copies else r for i, r in enumerate(rows)], n_pages)
    if len(copies) > len(free):
        return None, None, [], len(copies) - len(free)
    pairs = []
    for i, p in zip(copies, free):
        pairs.append((rows[i][-1], p))
        rows[i][-1] = p
    return _as_table(rows, table.shape[1]), out_len, pairs, 0


def compact(table, lens, n_pages: int, ps: int):
    """(table, pairs)"""
    rows = _held(table, lens, ps)
    used = {p for r in rows for p in r}
    U = len(used)
    pairs = list(zip(sorted(p for p in used if p >= U), [p for p in range(U) if p not in used]))
    to = dict(pairs)
    return _as_table([[to.get(p, p) for p in r] for r in rows], table.shape[1]), pairs
