"""CPU oracle (numpy, fp64) of the K/V caches held in 4 bits and in pages, written from the definitions in include/sa.h: the
number format, the place of every byte, attention over the rows that are there, and the page tables, one entry after the other."""
import math

import numpy as np

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TILE = 32
NO_ROW, ONE = 255, 127


def block_exponent(amax: float) -> int:
    """e of 2^e for a block of 32 whose largest magnitude is amax (finite)"""
    if amax == 0:
        return 0
    e = math.frexp(amax)[1] - 1 - 2   # floor(log2 amax) - 2
    if amax / 2.0 ** e > 7:
        e += 1
    return min(max(e, -125), 125)


def element_code(x: float, e: int) -> int:
    """Nearest magnitude, of two equally near ones the even code; sign in bit 3"""
    v = abs(x) / 2.0 ** e
    best = min(range(8), key=lambda c: (abs(MAGNITUDES[c] - v), c & 1))
    return best | (8 if np.signbit(x) else 0)


def value(code: int, byte: int) -> float:
    return (-1.0 if code & 8 else 1.0) * MAGNITUDES[code & 7] * 2.0 ** (byte - 127)


def blocks_held(x):
    """Many blocks at once, fp64 [n, 32] -> the values that they are held as: of the two magnitudes next to an element the nearer, of two equally
    near ones that of the even code (0, 1, 2, 4)"""
    grid = np.array(MAGNITUDES)
    top = np.abs(x).max(1)
    e = np.frexp(np.where(top > 0, top, 1))[1] - 3
    e = np.where(top > 0, np.clip(e + (top / 2.0 ** e > 7), -125, 125), 0)
    v = np.minimum(np.abs(x) / 2.0 ** e[:, None], 6)
    low = np.clip(np.searchsorted(grid, v, side="right") - 1, 0, 6)
    below, above = v - grid[low], grid[low + 1] - v
    code = np.where(below < above, low, np.where(below > above, low + 1, low + (low & 1)))
    return np.copysign(grid[code] * 2.0 ** e[:, None], x)


def quantise_row(k, v):
    """One row of K and of V of one head -> (codes, bytes) of each"""
    bad = not (np.isfinite(k).all() and np.isfinite(v).all())
    out = []
    for x, mark in ((k, NO_ROW), (v, ONE)):
        d = len(x)
        if bad:
            out.append(([0] * d, [mark] * (d // 32)))
            continue
        blocks = [block_exponent(np.abs(x[32 * c:32 * c + 32]).max()) for c in range(d // 32)]
        out.append(([element_code(x[i], blocks[i // 32]) for i in range(d)], [e + 127 for e in blocks]))
    return out


class Cache:
    """The bytes of one layer's pool; every access goes through put() and get()."""

    def __init__(self, Hkv, d, page_rows, pages, fill=0xFF):
        self.Hkv, self.d, self.page_rows, self.pages = Hkv, d, page_rows, pages
        self.bytes = np.full((pages, Hkv, page_rows // TILE, 34 * d), fill, np.uint8)

    def _places(self, row):
        d, r = self.d, row % TILE
        half, g, i = r // 16, r % 16 // 4, r % 4
        x = np.arange(d // 2)                      # bytes of a row's codes
        k_codes = r * (d // 2) + x
        v_codes = 16 * d + (((g * 16 + x // (d // 32)) * 2 + half) * 4 + i) * (d // 32) + x % (d // 32)
        c = np.arange(d // 32)
        k_scales = 32 * d + (c * 16 + r % 16) * 2 + half
        v_scales = 33 * d + ((c * 4 + g) * 2 + half) * 4 + i
        return k_codes, k_scales, v_codes, v_scales

    def put(self, page, head, row, k, v):
        tile = self.bytes[page, head, row // TILE]
        (kc, ks), (vc, vs) = quantise_row(k, v)
        at = self._places(row)
        for codes, scales, a, s in ((kc, ks, at[0], at[1]), (vc, vs, at[2], at[3])):
            codes = np.asarray(codes)
            tile[a] = codes[0::2] | codes[1::2] << 4
            tile[s] = scales

    def get(self, page, head, row):
        tile = self.bytes[page, head, row // TILE]
        at = self._places(row)
        out = []
        for a, s in ((at[0], at[1]), (at[2], at[3])):
            codes = np.stack([tile[a] & 15, tile[a] >> 4], 1).reshape(-1)
            out.append(np.array([value(int(c), int(b)) for c, b in zip(codes, np.repeat(tile[s], 32))]))
        if (tile[at[1]] == NO_ROW).any():
            return np.full(self.d, np.nan), np.full(self.d, np.nan)
        return out


def _page(table, b, pos, page_rows, pages):
    e = pos // page_rows
    if pos < 0 or e >= table.shape[1]:
        return -1
    p = int(table[b, e])
    return p if 0 <= p < pages else -1


def write(cache, table, K, V, starts, counts):
    B, H, T, _ = K.shape
    for b in range(B):
        for t in range(min(max(int(counts[b]), 0), T)):
            pos = int(starts[b]) + t
            p = _page(table, b, pos, cache.page_rows, cache.pages)
            for h in range(H if p >= 0 else 0):
                cache.put(p, h, pos % cache.page_rows, K[b, h, t], V[b, h, t])


def read(cache, table, K, V, starts, counts):
    """In place, rows t >= counts[b] left as they are"""
    B, H, T, _ = K.shape
    for b in range(B):
        for t in range(min(max(int(counts[b]), 0), T)):
            pos = int(starts[b]) + t
            p = _page(table, b, pos, cache.page_rows, cache.pages)
            for h in range(H):
                K[b, h, t], V[b, h, t] = cache.get(p, h, pos % cache.page_rows) if p >= 0 else (0.0, 0.0)


def attention(cache, table, q, lens, max_len, scale):
    """q [B,Hq,T,d] -> Y, LSE and, for the bounds of a test, the largest sum of |q k| scale of each row"""
    B, Hq, T, d = q.shape
    g = Hq // cache.Hkv
    Y, L, A = np.zeros(q.shape), np.full(q.shape[:3], -np.inf), np.zeros(q.shape[:3])
    for b in range(B):
        n = min(max(int(lens[b]), 0), max_len)
        where = [(_page(table, b, pos, cache.page_rows, cache.pages), pos) for pos in range(n)]
        where = [(p, pos) for p, pos in where if p >= 0]
        for h in range(cache.Hkv):
            rows = [cache.get(p, h, pos % cache.page_rows) for p, pos in where]
            for t in range(T):
                seen = [i for i, (_, pos) in enumerate(where) if pos <= n - T + t]
                if not seen:
                    continue
                K, V = np.array([rows[i][0] for i in seen]), np.array([rows[i][1] for i in seen])
                for hq in range(h * g, h * g + g):
                    s = K @ q[b, hq, t] * scale
                    with np.errstate(invalid="ignore"):
                        m = s.max()
                        w = np.exp(s - m)
                        Y[b, hq, t] = w @ V / w.sum()
                        L[b, hq, t] = m + np.log(w.sum())
                    A[b, hq, t] = (np.abs(K) @ np.abs(q[b, hq, t])).max() * scale
    return Y, L, A


# ---- page tables: table [B, M], refs [pages], entry by entry ------------------------------------------------------------------


def _held(rows, page_rows, M):
    return -(-min(max(int(rows), 0), M * page_rows) // page_rows)


def fork(parents, table, lens, refs, page_rows):
    B, M = table.shape
    P = len(refs)
    new, new_lens, refs = table.copy(), lens.copy(), refs.copy()
    for b in range(B):
        p = int(parents[b])
        if p == b:
            continue
        for x in table[b]:
            if 0 <= x < P:
                refs[x] -= 1
        new[b] = -1
        new_lens[b] = 0
        if 0 <= p < B:
            new_lens[b] = lens[p]
            for e in range(_held(lens[p], page_rows, M)):
                if 0 <= table[p, e] < P:
                    new[b, e] = table[p, e]
                    refs[table[p, e]] += 1
    return new, new_lens, refs


def free(keep, table, refs, page_rows):
    table, refs = table.copy(), refs.copy()
    for b in range(table.shape[0]):
        for e in range(_held(keep[b], page_rows, table.shape[1]), table.shape[1]):
            if 0 <= table[b, e] < len(refs):
                refs[table[b, e]] -= 1
            table[b, e] = -1
    return table, refs


def extend(lens, add, table, refs, page_rows):
    """-> table, refs, info, [(page copied, where to)]"""
    B, M = table.shape
    P = len(refs)
    need = []
    for b in range(B):
        lo = min(max(int(lens[b]), 0), M * page_rows)
        hi = min(lo + max(int(add[b]), 0), M * page_rows)
        for e in range(lo // page_rows, -(-hi // page_rows) if hi > lo else 0):
            x = int(table[b, e])
            there = 0 <= x < P
            if not there or refs[x] > 1:
                need.append((b, e, x if there else -1, there and e == lo // page_rows and lo % page_rows > 0))
    spare = [p for p in range(P) if refs[p] <= 0]
    if len(spare) < len(need):
        return table.copy(), refs.copy(), (0, len(need) - len(spare)), []
    table, refs, copies = table.copy(), refs.copy(), []
    for (b, e, old, begun), p in zip(need, spare):
        table[b, e] = p
        refs[p] = 1
        if old >= 0:
            refs[old] -= 1
        if begun:
            copies.append((old, p))
    return table, refs, (len(need), 0), copies


def compact(max_moves, table, refs):
    """-> table, refs, info, [(from, to)]"""
    P = len(refs)
    used = [p for p in range(P) if refs[p] > 0]
    U = len(used)
    moves = list(zip([p for p in reversed(used) if p >= U], [p for p in range(U) if refs[p] <= 0]))[:max_moves]
    table, refs = table.copy(), refs.copy()
    to = dict(moves)
    for i, x in np.ndenumerate(table):
        table[i] = to.get(int(x), x)
    for a, b in moves:
        refs[b], refs[a] = refs[a], 0
    return table, refs, (U, len(moves)), moves
