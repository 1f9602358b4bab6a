"""The cache held in 4 bits, computed plainly in 64 bits with numpy: format, pages, rows and attention (test infrastructure)."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """[.., d] -> indices with sign [.., d] (0..15), scale bytes [.., d/32]."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(invalid="ignore"):
        most = np.abs(g).max(-1)
    finite = np.isfinite(g).all(-1)
    part, power = np.frexp(np.where(finite, most, 1.0))                # most = part * 2^power, part in [1/2, 1)
    e = np.where(most == 0, -100, np.clip(power - 3 + (part >= 0.875), -100, 125))
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.abs(g) / np.exp2(e.astype(np.float64))[..., None]
    a = np.where(np.isfinite(a), a, 0.0)
    # nearest level, of two as near the one of the even index
    dist = np.abs(a[..., None] - LEVELS)
    near = dist == dist.min(-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    index = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = index + 8 * np.signbit(g)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def values(code, scale):
    """indices with sign [.., d], scale bytes [.., d/32] -> float64 [.., d]"""
    x = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    size = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return x * np.repeat(size, 32, axis=-1)


def page_bytes(page, d):
    return page * (d + d // 16)


def put(pool, slot, h, k, v, page):
    """Row (k, v) [d] of head h into slot of the pool [n_pages, H, bytes] (uint8)."""
    d = k.shape[-1]
    at, t = divmod(int(slot), page)
    p = pool[at, h]
    code, scale = quantise(k)
    p[t * d // 2:(t + 1) * d // 2] = code[0::2] | (code[1::2] << 4)
    o = page * d // 2
    p[o + t * d // 32:o + (t + 1) * d // 32] = scale
    o += page * d // 32
    code, scale = quantise(v)
    packed = (code[0::2] | (code[1::2] << 4)).reshape(16, d // 32)
    for part in range(16):
        a = o + ((t // 4) * 16 + part) * (d // 8) + (t % 4) * (d // 32)
        p[a:a + d // 32] = packed[part]
    o += page * d // 2
    for g in range(d // 32):
        p[o + (t // 4) * (d // 8) + g * 4 + t % 4] = scale[g]


def get(pool, slot, h, d, page):
    """k, v [d] (float64) of head h in a slot."""
    at, t = divmod(int(slot), page)
    p = pool[at, h]
    b = p[t * d // 2:(t + 1) * d // 2]
    o = page * d // 2
    k = values(np.stack([b & 15, b >> 4], -1).reshape(d), p[o + t * d // 32:o + (t + 1) * d // 32])
    o += page * d // 32
    b = np.concatenate([p[o + ((t // 4) * 16 + part) * (d // 8) + (t % 4) * (d // 32):][:d // 32] for part in range(16)])
    o += page * d // 2
    scale = np.array([p[o + (t // 4) * (d // 8) + g * 4 + t % 4] for g in range(d // 32)], np.uint8)
    return k, values(np.stack([b & 15, b >> 4], -1).reshape(d), scale)


def undefined_codes(pool, page, d):
    """The pool with the codes of groups that read as NaN set to 0: they may be anything."""
    pool = pool.copy()
    for at, h in np.argwhere(np.ones(pool.shape[:2])):
        p = pool[at, h]
        ks, vc, vs = page * d // 2, page * (d // 2 + d // 32), page * (d + d // 32)
        for t in range(page):
            for g in range(d // 32):
                if p[ks + t * d // 32 + g] == 255:
                    p[t * d // 2 + g * 16:t * d // 2 + g * 16 + 16] = 0
                if p[vs + (t // 4) * (d // 8) + g * 4 + t % 4] == 255:
                    for part in range(g * 512 // d, (g + 1) * 512 // d):
                        a = vc + ((t // 4) * 16 + part) * (d // 8) + (t % 4) * (d // 32)
                        p[a:a + d // 32] = 0
    return pool


def pages(new_len, length, table, free, n_free, page, N):
    """One call of the block-table operator on copies; returns (length, table, free, n_free, slots, missing)."""
    length, table, free = length.copy(), table.copy(), free.copy()
    B, entries = table.shape
    cap = entries * page
    old, new = np.clip(length, 0, cap), np.clip(new_len, 0, cap)
    held, need = -(-old // page), -(-new // page)
    slots = np.full((B, N), -1, np.int32)
    gone = [int(table[b, e]) for b in range(B) for e in range(need[b], held[b])]
    wanted = sum(max(0, int(need[b] - held[b])) for b in range(B))
    if wanted > n_free + len(gone):
        return length, table, free, n_free, slots, wanted - n_free - len(gone)
    stack = [int(x) for x in free[:n_free]] + gone[::-1]
    free[:len(stack)] = stack
    for b in range(B):
        for e in range(held[b], need[b]):
            table[b, e] = stack.pop()
        for i in range(N):
            at = old[b] + i
            if at < new[b]:
                slots[b, i] = table[b, at // page] * page + at % page
    return new.astype(np.int32), table, free, len(stack), slots, 0


def attend(q, K, V, there, length, n_query, scale, keep=None):
    """One sample.  q [N, Hq, d]; K, V [cap, H, d] float64; there [cap] (the entry's page exists).  Returns out, lse and, per row and
    head, what rounding bounds need: sum p |v| [N, Hq, d] and max scale sum |q||k| [N, Hq]."""
    N, Hq, d = q.shape
    G = Hq // K.shape[1]
    out, lse = np.zeros((N, Hq, d)), np.full((N, Hq), -np.inf)
    size, score = np.zeros((N, Hq, d)), np.zeros((N, Hq))
    for i in range(n_query):
        at = length - n_query + i
        seen = there & (np.arange(K.shape[0]) <= at) & (np.arange(K.shape[0]) < length)
        if keep is not None:
            seen = seen & (keep != 0)
        j = np.flatnonzero(seen)
        if j.size == 0:
            continue
        for h in range(Hq):
            k, v = K[j, h // G], V[j, h // G]
            x = scale * (k @ q[i, h])
            m = x.max()
            p = np.exp(x - m)
            total = p.sum()
            lse[i, h] = m + np.log(total)
            p = p / total
            out[i, h] = (p[:, None] * v).sum(0)
            size[i, h] = (p[:, None] * np.abs(v)).sum(0)
            score[i, h] = scale * (np.abs(k) @ np.abs(q[i, h])).max()
    return out, lse, size, score


def attend_heads(q, K, V, there, length, n_query, scale, keep=None):
    """As attend(), all rows of a head at once.  A value that is no number reaches the rows that see it, in its channels."""
    N, Hq, d = q.shape
    G, j = Hq // K.shape[1], np.arange(K.shape[0])
    out, lse = np.zeros((N, Hq, d)), np.full((N, Hq), -np.inf)
    size, score = np.zeros((N, Hq, d)), np.zeros((N, Hq))
    n = min(max(n_query, 0), N)
    seen = there & (j < length) & (j <= length - n_query + np.arange(n)[:, None])
    if keep is not None:
        seen = seen & (keep != 0)
    some = seen.any(1)
    for h in range(Hq if n else 0):
        k, v = K[:, h // G], V[:, h // G]
        x = np.where(seen, scale * (q[:n, h] @ k.T), -np.inf)
        m = np.where(some, x.max(1), 0)[:, None]
        p = np.exp(x - m)
        total = np.where(some, p.sum(1), 1)[:, None]
        p /= total
        none = seen.astype(float) @ np.isnan(v) > 0
        clean = np.nan_to_num(v, nan=0.0)
        out[:n, h] = np.where(none, np.nan, p @ clean)
        size[:n, h] = np.where(none, np.nan, p @ np.abs(clean))
        lse[:n, h] = np.where(some, (m + np.log(total))[:, 0], -np.inf)
        score[:n, h] = scale * np.where(seen, np.abs(q[:n, h]) @ np.abs(k).T, 0).max(1)
    return out, lse, size, score


def attend_bounds(out, lse, size, score, d, length, half_step, part):
    """How far a right kernel may be off.  half_step: of the output's type, relative; part: relative error of a probability as it
    enters the product with V.
      scores: sums of d fp32 products and two multiplications: each off by (d + 4) 2^-24 of sum |q||k|; the probability by that and
      a few units of exp2 (2^-21); sums over the keys: chains of length / 32 + 64 fp32 additions.  A relative error of the
      probabilities counts twice: in the numerator and in the sum."""
    ds = (d + 4) * 2.0 ** -24 * score
    chain = (length / 32 + 64) * 2.0 ** -24
    rel = 2 * (2 * ds + 2.0 ** -21 + chain) + part
    return half_step * np.abs(out) + rel[..., None] * size + 1e-37, 2 * ds + 2.0 ** -21 + chain + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0))
