"""Plain float64 implementation of the paged cache's operators (test infrastructure only; shares no code with the
GPU path).  Pools are numpy arrays [n_pages, Hkv, page, D]; tables, lengths and counts are lists or int arrays."""
from __future__ import annotations

import math

import numpy as np


def e4m3_values() -> np.ndarray:
    """The value of each E4M3 byte (bias 7, subnormals, 0x7F / 0xFF NaN)."""
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = math.nan if b & 0x7F == 0x7F else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[b] = -v if b >> 7 else v
    return out


def to_e4m3(x: np.ndarray, scale: float) -> np.ndarray:
    """Bytes of the E4M3 values nearest to x / scale (float64, ties to the even mantissa), saturated."""
    pos = e4m3_values()[:127]
    q = np.asarray(x, np.float64) / scale
    a = np.minimum(np.abs(q), 448.0)
    nan = np.isnan(q)
    a = np.where(nan, 0.0, a)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    down, up = a - pos[hi - 1], pos[hi] - a
    i = np.where((down < up) | ((down == up) & (hi % 2 == 1)), hi - 1, hi)
    i = np.where(nan, 0x7F, i)
    return (i | np.where(np.signbit(q), 0x80, 0)).astype(np.uint8)


def visible(pos: int, window, first: int) -> np.ndarray:
    t = np.arange(max(0, pos + 1))
    return t if window is None else t[(t > pos - window) | (t < first)]


def attention(q, K, V, table, lens, page, scale, window=None, first=0, sink=None, gate=None, pairs=None):
    """q [B, C, Hq, D]; K, V [n_pages, Hkv, page, D] float64.  Returns (out, weight): weight the same sum over |v|,
    the size that the errors of the probabilities multiply.  pairs: the (b, g) computed (None: all)."""
    B, C, Hq, D = q.shape
    n_pages, Hkv = K.shape[:2]
    G = Hq // Hkv
    out, weight = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        row = np.asarray(table[b], np.int64)
        for g in range(Hkv):
            if pairs is not None and (b, g) not in pairs:
                continue
            for c in range(C):
                t = visible(int(lens[b]) - C + c, window, first)
                p = row[t // page]
                there = (p >= 0) & (p < n_pages)
                p, s = p[there], t[there] % page
                k, v = K[p, g, s], V[p, g, s]
                for h in range(g * G, (g + 1) * G):
                    x = k @ q[b, c, h] * scale
                    m = max(x.max(initial=-math.inf), -math.inf if sink is None else sink[h])
                    if m == -math.inf:
                        continue
                    e = np.exp(x - m)
                    z = e.sum() + (0.0 if sink is None else math.exp(sink[h] - m))
                    f = 1.0 if gate is None else 1 / (1 + np.exp(-gate[b, c, h]))
                    out[b, c, h] = e @ v / z * f
                    weight[b, c, h] = e @ np.abs(v) / z * f
    return out, weight


def append(K, V, k_new, v_new, n_new, table, lens, page, convert):
    """Writes the rows into K and V (arrays of whatever is stored) in place; convert(row, g, which)."""
    for b in range(len(lens)):
        n = k_new.shape[1] if n_new is None else min(max(int(n_new[b]), 0), k_new.shape[1])
        for i in range(n):
            t = int(lens[b]) - n + i
            if t < 0 or not 0 <= table[b][t // page] < K.shape[0]:
                continue
            for which, (X, new) in enumerate(((K, k_new), (V, v_new))):
                for g in range(X.shape[1]):
                    X[table[b][t // page], g, t % page] = convert(new[b, i, g], g, which)


def extend(table, lens, refs, page):
    """(table, refs, counts) with the pages that len[b] tokens need."""
    table, refs = [list(r) for r in table], list(refs)
    free = [p for p, r in enumerate(refs) if r <= 0]
    given = missing = 0
    for b, row in enumerate(table):
        have = max([j + 1 for j, p in enumerate(row) if 0 <= p < len(refs)], default=0)
        for j in range(have, -(-int(lens[b]) // page)):
            if given < len(free):
                row[j] = free[given]
                refs[free[given]] = 1
                given += 1
            else:
                missing += 1
    return table, refs, [given, missing]


def reorder(parent, table, lens, refs, page):
    """(table, lens, refs, moves, counts) with every row its parent's copy."""
    B, n_pages = len(table), len(refs)
    refs = list(refs)
    free = [p for p, r in enumerate(refs) if r <= 0]
    heir = {}
    for b, p in enumerate(parent):
        if 0 <= p < B and (p not in heir or b == p):
            heir[p] = b
    rows, out_lens, moves, cut = [], [], [], 0
    for b, p in enumerate(parent):
        row, n = [-1] * len(table[b]), 0
        if 0 <= p < B:
            n = int(lens[p])
            full, part = divmod(n, page)
            if heir[p] == b:
                row = list(table[p])
            else:
                row[:full] = table[p][:full]
                for x in row[:full]:
                    if 0 <= x < n_pages:
                        refs[x] += 1
                if part and 0 <= table[p][full] < n_pages:
                    if len(moves) < len(free):
                        row[full] = free[len(moves)]
                        refs[row[full]] = 1
                        moves.append([table[p][full], row[full], part])
                    else:
                        cut += 1
                        n = full * page
        rows.append(row)
        out_lens.append(n)
    for p in range(B):
        if p not in heir:
            for x in table[p]:
                if 0 <= x < n_pages:
                    refs[x] -= 1
    return rows, out_lens, refs, moves, [len(moves), cut]


def compact(table, refs, page):
    """(table, refs, moves, counts) with the used pages at the front."""
    used = [p for p, r in enumerate(refs) if r > 0]
    n = len(used)
    src, dst = [p for p in used if p >= n], [p for p in range(n) if refs[p] <= 0]
    to, refs = dict(zip(src, dst)), list(refs)
    for a, e in to.items():
        refs[e], refs[a] = refs[a], 0
    return [[to.get(p, p) for p in r] for r in table], refs, [[a, e, page] for a, e in to.items()], [len(src), n]
