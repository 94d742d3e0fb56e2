"""The 8-bit cache, rotary positions and the commit inside it, written out plainly (test infrastructure).

A cached value is code * scale, the scale one number per block of tokens and head.  The codes are the 8-bit floats e4m3
(1 sign, 4 exponent, 3 fraction bits, bias 7, no infinities, 0x7f is NaN) and e5m2 (5, 2, bias 15, like half without its
lower byte).  Everything here works from those definitions: a table of all 256 values and a search for the nearest.

Rotary positions (the model's side of the verification pass): the draft slots of a tree stand in the text at
prefix_len + depth, so two siblings share a position although their cache rows differ."""
from __future__ import annotations

import numpy as np

MOST = {"e4m3": 448.0, "e5m2": 57344.0}
SMALLEST_SCALE = 2.0 ** -100


def values(kv: str) -> np.ndarray:
    """float64 [256]: what every code stands for."""
    frac, bias = (3, 7) if kv == "e4m3" else (2, 15)
    out = np.empty(256)
    for code in range(256):
        e, m = (code & 0x7F) >> frac, code & ((1 << frac) - 1)
        if kv == "e4m3" and (code & 0x7F) == 0x7F:
            x = np.nan
        elif kv == "e5m2" and e == 31:
            x = np.inf if m == 0 else np.nan
        else:
            x = m * 2.0 ** (1 - bias - frac) if e == 0 else (1 + m / 2.0 ** frac) * 2.0 ** (e - bias)
        out[code] = -x if code & 0x80 else x
    return out


_VALUES = {kv: values(kv) for kv in MOST}


def decode(codes: np.ndarray, kv: str) -> np.ndarray:
    return _VALUES[kv][codes]


def encode(x: np.ndarray, kv: str) -> np.ndarray:
    """Nearest code, ties to the even one, saturating; NaN to 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    last = 0x7E if kv == "e4m3" else 0x7B
    table = _VALUES[kv][: last + 1]
    mag = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), MOST[kv])
    lo = np.clip(np.searchsorted(table, mag, side="right") - 1, 0, last)
    hi = np.minimum(lo + 1, last)
    down, up = mag - table[lo], table[hi] - mag
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    code = code | (np.signbit(x).astype(np.uint8) << 7)
    return np.where(np.isnan(x), np.uint8(0x7F), code).astype(np.uint8)


def scale_for(largest: float, kv: str) -> float:
    """The smallest power of two s with largest <= MOST * s, at least SMALLEST_SCALE; 0 for 0."""
    if largest == 0:
        return 0.0
    e = int(np.floor(np.log2(largest / MOST[kv]))) - 2
    while MOST[kv] * 2.0 ** e < largest:
        e += 1
    return max(2.0 ** e, SMALLEST_SCALE)


def depth_of(parent, j: int) -> int:
    d = 0
    while parent[j] >= 0 and j > 0:
        j = int(parent[j])
        d += 1
    return d


def rotate(x: np.ndarray, position: int, inv_freq: np.ndarray, interleaved: bool, factor: float) -> np.ndarray:
    """x float64 [H, D] at one position."""
    half = len(inv_freq)
    t = float(position) * inv_freq.astype(np.float64)
    c, s = factor * np.cos(t), factor * np.sin(t)
    y = x.copy()
    for i in range(half):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[:, lo] = x[:, lo] * c[i] - x[:, hi] * s[i]
        y[:, hi] = x[:, hi] * c[i] + x[:, lo] * s[i]
    return y


def store_rows(codes: np.ndarray, scale: np.ndarray, kv: str, block: int, page_row, prefix: int, rows: np.ndarray):
    """codes uint8 [pages, H, page, D] and scale float32 [pages, H, page / block] are changed in place; rows float64 [n, H, D]
    go to positions prefix .. prefix + n - 1.  Returns the places written: [(page, head, row, slot)]."""
    page = codes.shape[2]
    n, H = rows.shape[:2]
    written = []
    for start in range(prefix // block * block, prefix + n, block):
        pg, r0 = int(page_row[start // page]), start % page
        for h in range(H):
            new = [j for j in range(n) if start <= prefix + j < start + block]
            old = max(0, min(block, prefix - start))
            had = float(scale[pg, h, r0 // block]) if old else 0.0
            now = max(had, scale_for(float(np.max(np.abs(rows[new, h]))), kv)) or 1.0
            if old and now != had:
                ratio = np.float32(had) / np.float32(now)
                y = decode(codes[pg, h, r0:r0 + old], kv).astype(np.float32) * ratio
                codes[pg, h, r0:r0 + old] = encode(y, kv)
            for j in new:
                codes[pg, h, r0 + prefix + j - start] = encode(rows[j, h].astype(np.float64) / now, kv)
                written.append((pg, h, r0 + prefix + j - start, j))
            scale[pg, h, r0 // block] = now
    return written


def commit_rows(codes: np.ndarray, scale: np.ndarray, kv: str, block: int, page_row, prefix: int, path):
    """The accepted slots' rows behind the root, in place; path: the accepted slots."""
    page = codes.shape[2]
    k = len(path)
    if k == 0:
        return
    before, scale_before = codes.copy(), scale.copy()
    src_of = {prefix + 1 + d: prefix + int(path[d]) for d in range(k)}
    place = lambda x: (int(page_row[x // page]), x % page)
    for start in range((prefix + 1) // block * block, prefix + k + 1, block):
        live = [(x, src_of.get(x, x)) for x in range(start, min(start + block, prefix + k + 1))]
        pg, r0 = place(start)
        for h in range(codes.shape[1]):
            now = max(scale_before[place(y)[0], h, place(y)[1] // block] for _, y in live)
            for x, y in live:
                sp, sr = place(y)
                had = scale_before[sp, h, sr // block]
                row = before[sp, h, sr]
                if had != now:
                    row = encode(decode(row, kv).astype(np.float32) * (np.float32(had) / np.float32(now)), kv)
                codes[pg, h, x % page] = row
            scale[pg, h, r0 // block] = now
