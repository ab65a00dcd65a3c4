"""64-bit reference of the 8-bit K/V cache: e4m3 rounding, append, attention, page selection.

Works on the cache's own layout (codes as uint8) so that the device's bytes can be compared with it
one by one; shares no code with the library.  Sizes are small: everything loops over rows and heads.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import numpy as np

PAGE = 64
SAT = 65504.0


def _table() -> np.ndarray:
    c = np.arange(128)
    e, m = c // 8, c % 8
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[127] = np.nan
    return np.concatenate([v, -v])


VALUES = _table()  # what each of the 256 codes stands for


def encode(x: np.ndarray) -> np.ndarray:
    """Codes of the e4m3 values nearest to x (|x| <= 448 or NaN), ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    mag = VALUES[:127]
    a = np.abs(np.where(np.isnan(x), 0.0, x))
    hi = np.clip(np.searchsorted(mag, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = mag[hi] - a, a - mag[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = np.where(mag[hi] == a, hi, c)
    return np.where(np.isnan(x), 127, c + 128 * np.signbit(x)).astype(np.uint8)


def scale_exponent(a: float) -> int:
    """The least e >= -32 with a <= 448 * 2^e."""
    e = -32
    while a > 448.0 * 2.0 ** e:
        e += 1
    return e


@dataclass
class Cache:
    """k [P][H][64][D], v [P][H][16][D][4] codes; ke, ve [P][H] exponents; bounds [P][H][2][D]; table [rows][ppr]."""
    k: np.ndarray
    v: np.ndarray
    ke: np.ndarray
    ve: np.ndarray
    bounds: np.ndarray
    table: np.ndarray

    @classmethod
    def of(cls, k, v, k_scale, v_scale, bounds, table):
        ke, ve = (np.log2(np.where(s > 0, s, 1.0)).astype(np.int64) for s in (k_scale, v_scale))
        return cls(k.copy(), v.copy(), ke, ve, bounds.copy().astype(np.int64), table.copy())

    def page(self, row: int, lp: int) -> int:
        p = int(self.table[row, lp])
        return p if 0 <= p < self.k.shape[0] else -1


def append(c: Cache, row: int, p0: int, k: np.ndarray, v: np.ndarray) -> None:
    """Stores keys and values [n][H][D] of positions p0 .. of a row."""
    n, H, D = k.shape
    for lp in range(max(p0, 0) // PAGE, (p0 + n - 1) // PAGE + 1 if n else 0):
        a, b = max(p0, lp * PAGE, 0), min(p0 + n, (lp + 1) * PAGE)
        page = c.page(row, lp)
        if page < 0 or a >= b:
            continue
        s0 = a - lp * PAGE
        for h in range(H):
            x, y = k[a - p0:b - p0, h].astype(np.float64), v[a - p0:b - p0, h].astype(np.float64)
            nan = np.isnan(x).any(1) | np.isnan(y).any(1)
            x = np.where(np.isnan(x), np.nan, np.clip(x, -SAT, SAT))
            y = np.where(np.isnan(y), 0.0, np.clip(y, -SAT, SAT))
            x[nan, 0] = np.nan
            for which, z in (("k", x), ("v", y)):
                codes = c.k[page, h] if which == "k" else c.v[page, h].transpose(0, 2, 1).reshape(PAGE, D).copy()
                es = c.ke if which == "k" else c.ve
                amax = float(np.max(np.abs(np.where(np.isnan(z), 0.0, z)))) if z.size else 0.0
                e = scale_exponent(amax)
                shift = 0
                if s0 > 0:
                    e = max(e, int(es[page, h]))
                    shift = int(es[page, h]) - e
                    if shift < 0:
                        codes[:s0] = encode(VALUES[codes[:s0]] * 2.0 ** shift)
                new = encode(z * 2.0 ** -e)
                codes[s0:s0 + b - a] = new
                es[page, h] = e
                if which == "k":
                    val = VALUES[new]
                    hi = np.where(np.isnan(val).all(0), -128, np.ceil(np.nanmax(np.where(np.isnan(val), -1e9, val), 0) / 4))
                    lo = np.where(np.isnan(val).all(0), 127, np.floor(np.nanmin(np.where(np.isnan(val), 1e9, val), 0) / 4))
                    if s0 > 0:
                        up, down = c.bounds[page, h]
                        some = up != -128  # a channel that held NaN only had no bounds
                        hi = np.where(some, np.maximum(hi, np.ceil(up * 2.0 ** shift)), hi)
                        lo = np.where(some, np.minimum(lo, np.floor(down * 2.0 ** shift)), lo)
                    c.bounds[page, h] = np.stack([hi, lo])
                else:
                    c.v[page, h] = codes.reshape(PAGE // 4, 4, D).transpose(0, 2, 1)


def keys_values(c: Cache, row: int, h: int, pages):
    """Keys and values [len(pages) * 64][D] of a row's pages (NaN-free zeros for pages outside the pool), and which are there."""
    D = c.k.shape[3]
    K, V, ok = [], [], []
    for lp in pages:
        p = c.page(row, lp)
        if p < 0:
            K.append(np.zeros((PAGE, D)))
            V.append(np.zeros((PAGE, D)))
        else:
            K.append(VALUES[c.k[p, h]] * 2.0 ** c.ke[p, h])
            V.append(VALUES[c.v[p, h]].transpose(0, 2, 1).reshape(PAGE, D) * 2.0 ** c.ve[p, h])
        ok.append(np.full(PAGE, p >= 0))
    if not K:
        return np.zeros((0, D)), np.zeros((0, D)), np.zeros(0, dtype=bool)
    return np.concatenate(K), np.concatenate(V), np.concatenate(ok)


def select(c: Cache, row: int, h: int, q: np.ndarray, vis: int, n_select: int):
    """The pages that queries q [G][D] of one token (seeing `vis` positions) choose."""
    n = -(-max(vis, 0) // PAGE)
    there = [p for p in range(n) if c.page(row, p) >= 0]
    if n <= n_select:
        return there
    top = float(np.max(np.abs(q)))
    x = 0 if top == 0 else math.frexp(top)[1]
    w = np.clip(np.rint(q.astype(np.float64) * 2.0 ** (7 - x)), -127, 127)
    score = {}
    for p in there:
        page = c.page(row, p)
        hi, lo = c.bounds[page, h, 0].astype(np.float64), c.bounds[page, h, 1].astype(np.float64)
        s = (np.maximum(w, 0) @ hi + np.minimum(w, 0) @ lo).max() * 2.0 ** c.ke[page, h]
        score[p] = math.inf if p == n - 1 else s
    return sorted(sorted(there, key=lambda p: (-score[p], p))[:n_select])


def attend(c: Cache, row: int, h: int, q: np.ndarray, vis: int, scale: float, pages=None):
    """Attention of queries q [G][D] over the first `vis` positions (of the given pages).  Returns (out [G][D], the same
    with |value| in place of value, a bound of sum |q_d k_d| scale over the positions)."""
    G, D = q.shape
    pages = list(range(-(-max(vis, 0) // PAGE))) if pages is None else list(pages)
    K, V, ok = keys_values(c, row, h, pages)
    pos = np.concatenate([np.arange(p * PAGE, (p + 1) * PAGE) for p in pages]) if pages else np.zeros(0, dtype=int)
    ok = ok & (pos < vis)
    K, V = K[ok], V[ok]
    if not len(K):
        return np.zeros((G, D)), np.zeros((G, D)), 0.0
    q = q.astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale * (q @ K.T)
        p = np.exp(s - np.max(s, axis=1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        size = scale * np.nanmax(np.abs(q) @ np.abs(np.nan_to_num(K)).T)
    return p @ V, p @ np.abs(V), float(size)
