"""CPU oracle (fp64, NumPy) of the serving operators: rotary positions, the paged cache, attention over it.

Written from the definitions in include/prism.h's serving section; shares no code with the GPU path.  Values held in 8
bits are handled as the numbers they stand for.
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import numpy as np

E4M3_MAX = 448.0
MIN_SCALE_EXPONENT = -120


# ---- rotary positions ------------------------------------------------------------------------------
def frequencies(base: float, rot_dim: int, yarn: Optional[Tuple[float, float, float, float]] = None) -> np.ndarray:
    """theta'_j of the rot_dim / 2 pairs; yarn = (native length, scale, alpha, beta)."""
    theta = np.array([base ** (-2.0 * j / rot_dim) for j in range(rot_dim // 2)])
    if yarn is None:
        return theta
    native, s, alpha, beta = yarn
    gamma = np.clip((native * theta / (2 * math.pi) - alpha) / (beta - alpha), 0.0, 1.0)
    return (1 - gamma) * theta / s + gamma * theta


def pairs(rot_dim: int, half: bool) -> Tuple[np.ndarray, np.ndarray]:
    """Dims of the first and of the second members of the pairs."""
    j = np.arange(rot_dim // 2)
    return (j, j + rot_dim // 2) if half else (2 * j, 2 * j + 1)


def rotate(x: np.ndarray, positions: np.ndarray, theta: np.ndarray, half: bool, magnitude: float = 1.0,
           backward: bool = False) -> np.ndarray:
    """x [heads, tokens, d] in fp64."""
    a, b = pairs(2 * len(theta), half)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * theta
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
    if backward:
        s = -s
    y = np.array(x, dtype=np.float64)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def pair_magnitude(x: np.ndarray, rot_dim: int, half: bool) -> np.ndarray:
    """hypot of the pair that each element belongs to; |x| behind the pairs."""
    a, b = pairs(rot_dim, half)
    m = np.abs(np.array(x, dtype=np.float64))
    m[..., a] = m[..., b] = np.hypot(x[..., a], x[..., b])
    return m


# ---- 8-bit values ----------------------------------------------------------------------------------
def e4m3_values() -> np.ndarray:
    """The 127 non-negative values of e4m3 (4 exponent bits of bias 7, 3 mantissa bits, no infinities), ascending."""
    v = []
    for code in range(127):
        e, m = code >> 3, code & 7
        v.append(math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10))
    return np.array(v)


def to_e4m3(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value, ties to the even code; |x| <= 448 or not finite (NaN)."""
    table = e4m3_values()
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(table, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = table[hi] - a, a - table[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(table[hi] == a, hi, code)
    return np.where(np.isfinite(x), np.copysign(table[code], x), np.nan)


def scale_for(top: float) -> float:
    """Smallest 2^e, e >= -120, with top <= 448 * 2^e."""
    e = MIN_SCALE_EXPONENT
    while top > math.ldexp(E4M3_MAX, e):
        e += 1
    return math.ldexp(1.0, e)


# ---- the cache -------------------------------------------------------------------------------------
def new_tokens(lengths, cu, capacity):
    """(sequence, row, position) of every new token that has a position inside [0, capacity)."""
    for s, length in enumerate(lengths):
        n = cu[s + 1] - cu[s]
        for i in range(n):
            pos = length - n + i
            if 0 <= pos < capacity:
                yield s, cu[s] + i, pos


def append_bf16(pages: np.ndarray, x: np.ndarray, lengths, cu, table) -> np.ndarray:
    """pages [n_pages, heads, page, d], x [heads, tokens, d]; unrounded new values at their places."""
    pages = pages.copy()
    n_pages, _, page, _ = pages.shape
    for s, row, pos in new_tokens(lengths, cu, table.shape[1] * page):
        p = table[s, pos // page]
        if 0 <= p < n_pages:
            pages[p, :, pos % page] = x[:, row]
    return pages


def append_e4m3(pages: np.ndarray, scales: np.ndarray, x: np.ndarray, lengths, cu, table):
    """pages hold e4m3 values (not times their scale).  Returns (pages with x / scale unrounded at the new places, scales,
    mask of the new places, mask of the places that moved to a larger scale)."""
    pages, scales = pages.copy(), scales.copy()
    n_pages, heads, page, _ = pages.shape
    new, moved = np.zeros(pages.shape[:3], bool), np.zeros(pages.shape[:3], bool)
    rows = np.zeros((n_pages, page), int)
    for s, row, pos in new_tokens(lengths, cu, table.shape[1] * page):
        p = table[s, pos // page]
        if 0 <= p < n_pages:
            new[p, :, pos % page] = True
            rows[p, pos % page] = row
    for p in range(n_pages):
        at = np.flatnonzero(new[p, 0])
        if len(at) == 0:
            continue
        for hd in range(heads):
            vals = x[hd, rows[p, at]]
            need = scale_for(np.max(np.abs(np.where(np.isfinite(vals), vals, 0.0)), initial=0.0))
            s = need if at[0] == 0 else max(need, scales[p, hd])
            if at[0] > 0 and s > scales[p, hd]:
                pages[p, hd, :at[0]] *= scales[p, hd] / s
                moved[p, hd, :at[0]] = True
            scales[p, hd] = s
            pages[p, hd, at] = vals / s
    return pages, scales, new, moved


def visible(pos: int, count: int, window: int, sinks: int) -> np.ndarray:
    j = np.arange(count)
    ok = j <= pos
    if window > 0:
        ok &= (j > pos - window) | (j < sinks)
    return ok


def attention(q: np.ndarray, k_pages: np.ndarray, v_pages: np.ndarray, lengths, cu, table, window: int = 0,
              sinks: int = 0, scale: Optional[float] = None):
    """q [h, tokens, d]; pages [n_pages, h_kv, page, d] as the numbers they stand for.  Returns out, lse, and for error
    bounds: spread = sum of P |v|, and reach = largest scale * sum |q||k| over the visible keys of a row; rows that belong to
    no sequence are NaN."""
    h, tokens, d = q.shape
    n_pages, h_kv, page, _ = k_pages.shape
    scale = 1.0 / math.sqrt(d) if not scale else scale
    out, spread = np.full((h, tokens, d), np.nan), np.full((h, tokens, d), np.nan)
    lse, reach = np.full((h, tokens), np.nan), np.full((h, tokens), np.nan)
    for s, length in enumerate(lengths):
        n = cu[s + 1] - cu[s]
        count = min(max(length, 0), table.shape[1] * page)
        j = np.arange(count)
        ids = table[s, j // page] if count else np.zeros(0, int)
        there = (ids >= 0) & (ids < n_pages)
        ids = np.where(there, ids, 0)
        for hd in range(h):
            kv = hd // (h // h_kv)
            k, v = k_pages[ids, kv, j % page], v_pages[ids, kv, j % page]
            for i in range(n):
                pos = length - n + i
                ok = visible(pos, count, window, sinks) & there
                row = cu[s] + i
                if not ok.any():
                    out[hd, row], lse[hd, row], spread[hd, row], reach[hd, row] = 0.0, -np.inf, 0.0, 0.0
                    continue
                x = scale * (k[ok] @ q[hd, row])
                m = x.max()
                p = np.exp(x - m)
                total = p.sum()
                out[hd, row] = p @ v[ok] / total
                spread[hd, row] = p @ np.abs(v[ok]) / total
                lse[hd, row] = m + math.log(total)
                reach[hd, row] = scale * np.max(np.abs(k[ok]) @ np.abs(q[hd, row]))
    return out, lse, spread, reach
