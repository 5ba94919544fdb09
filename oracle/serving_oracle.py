"""Plain definitions, in float64 NumPy and on Python lists, of what stands around the caches (test infrastructure only): norms and
rotation of heads, pages that change hands and places, attention to the states of an encoder.  Shares no code with the library."""
from __future__ import annotations

import numpy as np

from oracle.paged_oracle import PAGE


def normed(x: np.ndarray, w, eps: float) -> np.ndarray:
    """Rows x [..., D]: x / sqrt(mean(x^2) + eps) * w; w None: x."""
    if w is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def turned(x: np.ndarray, positions, inv_freq, interleaved: bool) -> np.ndarray:
    """Rows x [t, heads, D]: the pairs of the first 2 * len(inv_freq) dimensions turned by position * inv_freq radians."""
    r = 2 * len(inv_freq)
    y = x.copy()
    for i, f in enumerate(inv_freq):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        t = np.asarray(positions, dtype=np.float64) * float(f)
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        y[:, :, p] = x[:, :, p] * c - x[:, :, q] * s
        y[:, :, q] = x[:, :, q] * c + x[:, :, p] * s
    return y


def heads(x, w, eps, positions, inv_freq, interleaved):
    y = normed(x, w, eps)
    return y if inv_freq is None else turned(y, positions, inv_freq, interleaved)


def pages_of(n: int) -> int:
    return -(-n // PAGE)


def fork(o, shares, parent, keep):
    """o: Pages (see paged_oracle), shares: list; in place.  The copies that have to be made, and whether pages ran out."""
    old = [row[:pages_of(n)] for row, n in zip(o.table, o.kv_len)]
    parent = list(range(len(old))) if parent is None else parent
    size = []
    for b, p in enumerate(parent):
        n = o.kv_len[p] if p >= 0 else 0
        size.append(n if keep is None else max(0, min(keep[b], n)))
    rows = [list(old[p][:pages_of(n)]) if p >= 0 else [] for p, n in zip(parent, size)]
    before, after = {}, {}
    for rs, count in ((old, before), (rows, after)):
        for row in rs:
            for p in row:
                count[p] = count.get(p, 0) + 1
    for p in sorted((p for p in before if p not in after), reverse=True):
        o.free[o.n_free] = p
        o.n_free += 1
    # who may go on writing to a page: nobody if some sequence has all of it, else the first that has it
    writer = {}
    for b, row in enumerate(rows):
        for i, p in enumerate(row):
            if (i + 1) * PAGE <= size[b]:
                writer[p] = None
    for b, row in enumerate(rows):
        if size[b] % PAGE:
            writer.setdefault(row[-1], b)
    copies, short = [], False
    for b, row in enumerate(rows):
        if size[b] % PAGE == 0 or writer[row[-1]] == b:
            continue
        p = row[-1]
        after[p] -= 1
        if o.n_free == 0:
            short = True
            row[-1] = -1
            size[b] -= size[b] % PAGE
            continue
        o.n_free -= 1
        row[-1] = o.free[o.n_free]
        copies.append((p, row[-1], size[b] % PAGE))
        after[row[-1]] = 1
    for b, row in enumerate(rows):
        wide = max(len(row), len(old[b]))
        o.table[b][:wide] = row + [-1] * (wide - len(row))
        o.kv_len[b] = size[b]
    for p in range(len(shares)):
        shares[p] = max(0, after.get(p, 0) - 1)
    return copies, short


def compact(o, shares, most):
    free = sorted(o.free[:o.n_free])
    held = set(range(o.n_pages)) - set(free)
    moves = []
    while free and held and len(moves) < most and free[0] < max(held):
        src, dst = max(held), free.pop(0)
        held.remove(src)
        held.add(dst)
        free.append(src)
        free.sort()
        moves.append((src, dst, PAGE))
    to = {s: d for s, d, _ in moves}
    for row, n in zip(o.table, o.kv_len):
        for i in range(pages_of(n)):
            row[i] = to.get(row[i], row[i])
    for s, d, _ in moves:
        if shares is not None:
            shares[d], shares[s] = shares[s], 0
    o.free[:o.n_free] = sorted(free, reverse=True)
    return moves


def copy_pages(codes, scale, entries):
    """codes [pages, heads, 64, d], scale [pages, heads]; in place."""
    for src, dst, rows in entries:
        codes[dst, :, :rows] = codes[src, :, :rows]
        scale[dst] = scale[src]


def cross(q, k, v, scale):
    """Rows q [n, hq, d] against k, v [m, hkv, d]: the result [n, hq, d], and the same with the magnitudes of v."""
    g = q.shape[1] // k.shape[1]
    out, mag = np.zeros_like(q), np.zeros_like(q)
    if k.shape[0] == 0:
        return out, mag
    for h in range(q.shape[1]):
        s = q[:, h] @ k[:, h // g].T * scale
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        out[:, h], mag[:, h] = p @ v[:, h // g], p @ np.abs(v[:, h // g])
    return out, mag
