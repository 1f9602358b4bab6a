"""Rotation by positions, bounds of pages, the choice of pages and who sees what, computed plainly with numpy (test infrastructure)."""
import numpy as np

import cache4_ref as ref


def angles(n_pos, pairs, base=10000.0):
    """Cosines and sines [n_pos, pairs, 2], fp32 as a table holds them."""
    at = np.arange(n_pos, dtype=np.float64)[:, None] * base ** (-np.arange(pairs) / pairs)
    return np.stack([np.cos(at), np.sin(at)], -1).astype(np.float32)


def turned(x, at, table, axis, adjacent=False, inverse=False, kind=np.float32):
    """x [N, H, d] at positions at [axes, N], in `kind`: products rounded, then their sums.  Positions outside the table: NaN."""
    pairs = len(axis)
    p = at[np.asarray(axis)].T                                                   # [N, pairs]
    ok = (p >= 0) & (p < len(table))
    cs = np.where(ok[..., None], table[np.clip(p, 0, len(table) - 1), np.arange(pairs)], np.nan).astype(kind)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1] * kind(-1 if inverse else 1)
    y = x.astype(kind).copy()
    a = slice(0, 2 * pairs, 2) if adjacent else slice(0, pairs)
    b = slice(1, 2 * pairs, 2) if adjacent else slice(pairs, 2 * pairs)
    u, v = y[..., a].copy(), y[..., b].copy()
    with np.errstate(over="ignore", invalid="ignore"):
        y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    return y


def keys_of(pool, id, live, H, d, page):
    """K [live, H, d] of a page's first entries, as float64."""
    return np.stack([[ref.get(pool, id * page + t, h, d, page)[0] for h in range(H)] for t in range(live)]).reshape(live, H, d)


def bounds(pool, id, live, H, d, page):
    """int [H, 2, d] and scale bytes [H] of one page."""
    k = keys_of(pool, id, live, H, d, page)
    out, scale = np.zeros((H, 2, d), np.int64), np.zeros(H, np.int64)
    for h in range(H):
        if not np.isfinite(k[:, h]).all():
            scale[h] = 255
            continue
        a = np.abs(k[:, h]).max()
        e = -126 if a == 0 else max(int(np.frexp(a)[1]) - 1 - 6, -126)
        out[h, 0], out[h, 1] = np.ceil(k[:, h].max(0) / 2.0 ** e), np.floor(k[:, h].min(0) / 2.0 ** e)
        scale[h] = e + 127
    return out, scale


def whole(q):
    """Queries [G, d] of a token and K/V head as whole numbers."""
    a = np.abs(q).max()
    if not np.isfinite(a) or a == 0:
        return np.zeros(q.shape, np.int64)
    e = int(np.frexp(a)[1]) - 7
    return np.clip(np.rint(q / 2.0 ** e), -127, 127).astype(np.int64)


def score(q, bound, scale):
    """fp32 score of one page: queries [G, d] as whole numbers, bounds [2, d], scale byte."""
    if scale == 255:
        return np.float32(np.inf)
    total = int(np.maximum(q * bound[0], q * bound[1]).sum())
    return np.float32(np.ldexp(np.float32(total), int(scale) - 127))


def seen(length, nq, i, cap):
    """Entries that row i of nq sees."""
    length = min(max(length, 0), cap)
    return min(max(length - nq + i + 1, 0), length)


def choose(q, bounds_, scales, row, length, nq, i, page, first, last, budget, n_pages):
    """The list [budget] of one token and K/V head: queries [G, d]; bounds [pool, 2, d], scales [pool]; row: of the block table."""
    P = -(-seen(length, nq, i, len(row) * page) // page)
    w = whole(q)
    s = [score(w, bounds_[id], scales[id]) if 0 <= id < n_pages else np.float32(-np.inf) for id in row[:P]]
    always = {e for e in range(P) if e < first or e >= P - last}
    rest = sorted((e for e in range(P) if e not in always), key=lambda e: (-float(s[e]), e))
    if P > budget:
        rest = rest[:budget - len(always)]
    picked = sorted(always | set(rest))
    return picked + [-1] * (budget - len(picked))


def listed(entries, max_pages):
    """The entries of a list that count: in the table, and above all such before them."""
    out, top = [], -1
    for e in entries:
        if 0 <= e < max_pages:
            if e > top:
                out.append(int(e))
            top = max(top, int(e))
    return out
