"""Plain definitions of the paged 8-bit KV cache in NumPy (test infrastructure only): page planning on Python lists, the
quantising append row by row, and what a sequence's pages stand for, in float64.  Shares no code with the library."""
from __future__ import annotations

import numpy as np

PAGE = 64
MIN_EXP = -100


def e4m3_table() -> np.ndarray:
    """The value of every code: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7F and 0xFF are NaN."""
    out = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        x = np.nan if (e, f) == (15, 7) else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        out[c] = -x if c >> 7 else x
    return out


VALUES = e4m3_table()
_GRID = VALUES[:127]                                         # the magnitudes, ascending


def encode(x: np.ndarray) -> np.ndarray:
    """Codes of float64 values of at most 448 in magnitude: the nearest, ties to the even code; NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert (a <= 448.0).all()
    hi = np.clip(np.searchsorted(_GRID, a), 1, 126)
    down, up = a - _GRID[hi - 1], _GRID[hi] - a
    code = np.where((down < up) | ((down == up) & ((hi - 1) % 2 == 0)), hi - 1, hi)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isfinite(x), code, 0x7F).astype(np.uint8)


def scale_for(amax: float) -> float:
    e = MIN_EXP
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Pages:
    """Block tables, lengths and the list of free pages."""

    def __init__(self, table, kv_len, free, n_free, n_pages):
        self.table = [list(map(int, r)) for r in table]
        self.kv_len = list(map(int, kv_len))
        self.free, self.n_free, self.n_pages = list(map(int, free)), int(n_free), n_pages

    def plan(self, rows):
        """Slots of `rows[b]` new tokens per sequence, one token after the other."""
        slots, overflow = [], False
        for b, n in enumerate(rows):
            stuck = False
            for _ in range(n):
                i, r = divmod(self.kv_len[b], PAGE)
                if r == 0 and not stuck:
                    if i == len(self.table[b]) or self.n_free == 0:
                        stuck = True
                    else:
                        self.n_free -= 1
                        self.table[b][i] = self.free[self.n_free]
                if stuck:
                    slots.append(-1)
                    overflow = True
                    continue
                slots.append(self.table[b][i] * PAGE + r)
                self.kv_len[b] += 1
        return slots, overflow

    def release(self, keep):
        back = []
        for b, n in enumerate(self.kv_len):
            k = max(0, min(keep[b], n))
            for i in range(-(-k // PAGE), -(-n // PAGE)):
                back.append(self.table[b][i])
                self.table[b][i] = -1
            self.kv_len[b] = k
        for p in reversed(back):
            if 0 <= p < self.n_pages and self.n_free < self.n_pages:
                self.free[self.n_free] = p
                self.n_free += 1


def append(codes: np.ndarray, scale: np.ndarray, new: np.ndarray, slots) -> None:
    """codes uint8 [pages, heads, 64, d], scale [pages, heads], new float64 [t, heads, d]; in place, block by block."""
    t = 0
    while t < len(slots):
        if slots[t] < 0:
            t += 1
            continue
        page, r0 = divmod(int(slots[t]), PAGE)
        n = 1
        while t + n < len(slots) and slots[t + n] == slots[t] + n and r0 + n < PAGE:
            n += 1
        for h in range(new.shape[1]):
            x = new[t:t + n, h]
            fine = np.abs(x[np.isfinite(x)])
            s = scale_for(float(fine.max()) if fine.size else 0.0)
            if r0 > 0:
                old = float(scale[page, h])
                if old < s:
                    codes[page, h, :r0] = encode(VALUES[codes[page, h, :r0]] * (old / s))
                s = max(s, old)
            codes[page, h, r0:r0 + n] = encode(x / s)
            scale[page, h] = s
        t += n


def gather(codes: np.ndarray, scale: np.ndarray, row, n: int) -> np.ndarray:
    """float64 [n, heads, d] of the first n positions of a sequence whose pages are `row`."""
    ids = np.asarray(row[:-(-n // PAGE)], dtype=np.int64)
    x = VALUES[codes[ids]] * scale[ids].astype(np.float64)[:, :, None, None]
    return x.transpose(0, 2, 1, 3).reshape(-1, codes.shape[1], codes.shape[3])[:n]
