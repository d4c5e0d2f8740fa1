"""Float64 CPU oracle of contexts kept in 8 bits: e4m3 codes with a power of two for each block of
rows and head, rows appended to them, attention over them.

TEST INFRASTRUCTURE ONLY, like the rest of this package.  Each function is the definition written
out for one block or one query row after another; nothing is shared with the GPU package.
"""

import numpy as np

TOP, E_MIN, E_MAX, NAN = 448.0, 79, 175, 0x7F

# the finite values of codes 0 .. 126: 4 bits of exponent (bias 7), 3 of fraction
_E, _F = np.divmod(np.arange(127), 8)
GRID = np.where(_E > 0, (8 + _F) * 2.0 ** (_E - 10.0), _F * 2.0 ** -9)


def decode(codes):
    """Values of e4m3 codes (uint8)."""
    codes = np.asarray(codes)
    mag = np.append(GRID, np.nan)[codes & 127]
    return np.where(codes & 128, -mag, mag)


def encode(x):
    """The code of the nearest value, of two equally near ones the even code; |x| <= 448, or NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isnan(x), 0.0, x))
    up = np.searchsorted(GRID, a)                # the first value >= a
    dn = np.maximum(up - 1, 0)
    near = np.where(a - GRID[dn] < GRID[up] - a, dn, up)
    tie = a - GRID[dn] == GRID[up] - a
    near = np.where(tie, np.where(dn % 2 == 0, dn, up), near)
    code = near.astype(np.uint8) | (np.signbit(x).astype(np.uint8) << 7)
    return np.where(np.isnan(x), np.uint8(NAN), code)


def power(x):
    """The byte of the least power of two under which 448 holds every finite entry of x that any
    holds."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    a = a[np.isfinite(a) & (a <= TOP * 2.0 ** (E_MAX - 127))]
    e = E_MIN
    while e < E_MAX and a.size and a.max() > TOP * 2.0 ** (e - 127):
        e += 1
    return e


def clamp_power(e):
    return np.clip(np.asarray(e).astype(int), E_MIN, E_MAX)


def page_of(pages, max_pages, n_pages, b, entry):
    """The page of an entry, None for one that is absent."""
    p = b * max_pages + entry if pages is None else int(pages[b, entry])
    return p if 0 <= p < n_pages else None


def append(keys, values, powers, k, v, max_pages, pages=None, lens=None, n_new=None):
    """The pool after k, v [B, L, heads, d] are appended: keys uint8 [n_pages, heads, page, d],
    values uint8 [n_pages, heads, d, page], powers uint8 [n_pages, heads, 2]; new arrays."""
    keys, values, powers = keys.copy(), values.copy(), powers.copy()
    n_pages, heads, page, d = keys.shape
    B, L = k.shape[:2]
    for b in range(B):
        cap = max_pages * page
        first = min(max(int(lens[b]), 0), cap) if lens is not None else 0
        n = min(max(int(n_new[b]), 0), L) if n_new is not None else L
        end = min(first + n, cap)
        at = first
        while at < end:
            entry, had = divmod(at, page)
            stop = min(end, (entry + 1) * page)
            p = page_of(pages, max_pages, n_pages, b, entry)
            if p is not None:
                for h in range(heads):
                    for part, (x, store) in enumerate(((k, keys[p, h]), (v, values[p, h].T))):
                        new = np.asarray(x[b, at - first:stop - first, h], dtype=np.float64)
                        e = power(new)
                        if had:
                            old = int(clamp_power(powers[p, h, part]))
                            e = max(e, old)
                            if e > old:
                                some = ~np.isnan(decode(store[:had]))
                                again = encode(decode(store[:had]) * 2.0 ** (old - e))
                                store[:had] = np.where(some, again, store[:had])
                        ok = np.abs(new) <= TOP * 2.0 ** (E_MAX - 127)
                        code = encode(np.where(ok, new, 0.0) * 2.0 ** (127 - e))
                        store[had:had + stop - at] = np.where(ok, code, np.uint8(NAN))
                        powers[p, h, part] = e
            at = stop
    return keys, values, powers


def rows_of(keys, values, powers, max_pages, pages, b, length, head):
    """Keys, values [n, d] of one sequence and head, and which of the rows are there."""
    n_pages, page = keys.shape[0], keys.shape[2]
    entry, slot = np.divmod(np.arange(length), page)
    p = b * max_pages + entry if pages is None else np.asarray(pages)[b, entry].astype(np.int64)
    here = (p >= 0) & (p < n_pages)
    p = np.where(here, p, 0)
    two = np.where(here[:, None], 2.0 ** (clamp_power(powers[p, head]) - 127), 0.0)
    K = np.where(here[:, None], decode(keys[p, head, slot]) * two[:, :1], 0.0)
    V = np.where(here[:, None], decode(values[p, head, :, slot]) * two[:, 1:], 0.0)
    return K, V, here


def attend(q, keys, values, powers, max_pages, pages, lens, n_rows, scale, causal, max_len=0):
    """out [B, L, heads, d], lse [B, L, heads] and, for bounds, sum p |V|, the largest sum |q k|
    |scale| and the largest |V| that a row sees; NaN rows of out where n_rows leaves them."""
    B, L, H, d = q.shape
    _, kv, page, _ = keys.shape
    out, lse = np.full((B, L, H, d), np.nan), np.full((B, L, H), np.nan)
    mag, sabs, vmax = np.zeros((B, L, H, d)), np.zeros((B, L, H)), np.zeros((B, L, H))
    for b in range(B):
        n = min(max(int(lens[b]), 0), max_pages * page)
        n = min(n, max_len) if max_len else n
        r = min(max(int(n_rows[b]), 0), L) if n_rows is not None else L
        for g in range(kv):
            K, V, here = rows_of(keys, values, powers, max_pages, pages, b, n, g)
            for h in range(g * (H // kv), (g + 1) * (H // kv)):
                for i in range(r):
                    see = here & (np.arange(n) < (n - r + i + 1 if causal else n))
                    if not see.any():
                        out[b, i, h], lse[b, i, h] = 0.0, -np.inf
                        continue
                    x = scale * (K[see] @ q[b, i, h])
                    m = x.max()
                    p = np.exp(x - m)
                    lse[b, i, h] = m + np.log(p.sum())
                    p = p / p.sum()
                    out[b, i, h] = p @ V[see]
                    mag[b, i, h] = p @ np.abs(V[see])
                    sabs[b, i, h] = abs(scale) * (np.abs(K[see]) @ np.abs(q[b, i, h])).max()
                    vmax[b, i, h] = np.abs(np.nan_to_num(V[see])).max()
    return out, lse, mag, sabs, vmax
