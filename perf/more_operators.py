"""The operators around positions and pages that are chosen, as they are measured: the rotation of queries and keys by positions with
several axes, rows rotated into the cache held in 4 bits, bounds of a page's keys, the choice of pages by them, and attention
over the chosen pages.

A case is one pass as a serving program makes it.  `own` says who computes it: elementary torch operations (the plain form), or the
library's entry points.

Rotation.  Pair i of a row's channels is (i, i + pairs), or (2i, 2i + 1) where `adjacent`; channels from 2 * pairs on stay.  It has an axis
a(i) of its own, and with (c, s) = table[position on that axis][i] becomes (x c - y s, y c + x s), or with -s the way back: in fp32, the
products rounded before they are added, so that what is then held in 4 bits does not depend on who computes it.

Cache.  A group of 32 consecutive channels of one token and head is 32 numbers of 4 bits (sign, and the index of the magnitude in 0,
0.5, 1, 1.5, 2, 3, 4, 6) and one scale 2^e.  With a the largest magnitude of the group and k = floor(log2 a), e = k - 2, or k - 1 where
a >= 1.75 * 2^k, within -100 and 125; -100 where a = 0.  x becomes the nearest value to x / 2^e, the even index where two are as
near.  The scale is stored as the byte e + 127; 255 is a group that reads as NaN.  A pool is uint8 [pages, H, page * (d + d / 16)]: K codes
[page, d / 2] (channel 2i in the low half of byte i), K scales [page, d / 32], V codes [page / 4, 16, 4, d / 32], V scales [page / 4, d / 32, 4].

Bounds.  Of the keys that a page holds for a head: with a the largest magnitude and e = floor(log2 a) - 6, every channel's largest value
over 2^e, rounded up, and its smallest one, rounded down: int8 [pages, H, 2, d]; and the byte e + 127 [pages, H].  a = 0: e = -126; 255
where a key is no number.

Choice.  The G query heads of a token and K/V head are rounded to whole numbers of 2^e, e = floor(log2 of the largest magnitude) - 6, 127
at most.  A page's score is the sum over heads and channels of the larger of q * largest and q * smallest, a whole number, times the
page's 2^e in fp32.  Of the pages that the token sees, the first and last ones are taken, then those of the highest scores, of equal ones
the first, up to the budget; in ascending order, -1 behind them.
"""
from __future__ import annotations

import math

import torch

own = False

MU2 = 3.0             # heavy entries: logits about three standard deviations above the others, as in the decode workload
HEAVY = 0.05


def _rotate(name, batch, rows, tokens, heads, kv_heads, d, pairs, axes, dtype="bf16", layout="tokens", adjacent=False, inverse=False, ragged=False):
    return {"name": name, "op": "rotate", "batch": batch, "rows": rows, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "d": d,
            "pairs": pairs, "axes": axes, "dtype": dtype, "layout": layout, "adjacent": adjacent, "inverse": inverse, "ragged": ragged}


def _append(name, batch, rows, before, heads, kv_heads, d, pairs, axes, page, dtype="bf16", layout="tokens", adjacent=False, ragged=False):
    return {"name": name, "op": "append", "batch": batch, "rows": rows, "before": before, "heads": heads, "kv_heads": kv_heads, "d": d,
            "pairs": pairs, "axes": axes, "page": page, "dtype": dtype, "layout": layout, "adjacent": adjacent, "ragged": ragged}


def _bounds(name, batch, rows, before, kv_heads, d, page, ragged=False):
    return {"name": name, "op": "bounds", "batch": batch, "rows": rows, "before": before, "kv_heads": kv_heads, "d": d, "page": page, "ragged": ragged}


def _choose(name, batch, rows, length, heads, kv_heads, d, page, budget, dtype="bf16", layout="tokens", ragged=False):
    return {"name": name, "op": "choose", "batch": batch, "rows": rows, "length": length, "heads": heads, "kv_heads": kv_heads, "d": d,
            "page": page, "budget": budget, "dtype": dtype, "layout": layout, "ragged": ragged}


def _attend(name, batch, rows, length, heads, kv_heads, d, page, budget, dtype="bf16", layout="tokens", ragged=False, keep=1.0):
    return {"name": name, "op": "attend", "batch": batch, "rows": rows, "length": length, "heads": heads, "kv_heads": kv_heads, "d": d,
            "page": page, "budget": budget, "dtype": dtype, "layout": layout, "ragged": ragged, "keep": keep}


def listed():
    return [
        # one token of one sequence: where latency counts
        _rotate("rotate_step_b1", 1, 1, 1, 32, 8, 128, 64, 1),
        # the tokens of a video that the merge kept, with their places in time, height and width
        _rotate("rotate_video_b4", 4, 2371, 4672, 32, 32, 128, 64, 3, ragged=True),
        # the rows of a decode step, and what the cache then holds of them
        _append("append_step_b64", 64, 1, 1024, 32, 32, 128, 64, 1, 32),
        # kept rows of prompts of different lengths, fp32, head-major, half of the channels rotated, neighbours as pairs
        _append("append_prompts_b16", 16, 777, 100, 40, 8, 64, 16, 3, 16, dtype="f32", layout="heads", adjacent=True, ragged=True),
        # a decode step: the page that got a row, of every sequence
        _bounds("bounds_step_b64", 64, 1, 4000, 32, 128, 32),
        # prompts behind images in tiles: all of their pages
        _bounds("bounds_prompts_b16", 16, 5888, 0, 8, 128, 64, ragged=True),
        # one sequence: an eighth of its pages
        _choose("choose_step_b1", 1, 1, 4096, 32, 32, 128, 32, 16),
        # the decode workload: 64 sequences of up to 4096 entries, 1024 of them looked at
        _choose("choose_step_b64", 64, 1, 4096, 32, 32, 128, 32, 32, ragged=True),
        # drafts of five tokens behind two long documents, eight K/V heads
        _choose("choose_long_b2", 2, 5, 100003, 32, 8, 128, 64, 64, ragged=True),
        # one sequence's step over the chosen pages
        _attend("attend_chosen_b1", 1, 1, 4096, 32, 32, 128, 32, 16),
        # the decode workload again
        _attend("attend_chosen_b64", 64, 1, 4096, 32, 32, 128, 32, 32, ragged=True),
        # a chunk of a prompt behind images in tiles, entries masked by an eviction that has not moved anything yet
        _attend("attend_chosen_chunk_b4", 4, 161, 5888, 32, 8, 128, 64, 16, ragged=True, keep=0.75),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 5e14


def _fits(case):
    """Whether the keys that lie there, and those that the plain form of an attention gathers, are no more than the largest listed case has."""
    c = case
    if c["op"] not in ("choose", "attend"):
        return True
    return max(c["batch"] * c["length"], c["batch"] * c["rows"] * c["budget"] * c["page"] if c["op"] == "attend" else 0) * c["kv_heads"] * c["d"] <= 1 << 30


def draw(rng):
    """One more case of the ranges above, at most as costly as the largest of its operator."""
    op = rng.choice(("rotate", "append", "bounds", "choose", "choose", "attend", "attend"))
    like = [x for x in listed() if x["op"] == op]
    c = _draw(rng, op)
    while _cost(c) > max(_cost(x) for x in like) or not _fits(c):
        c = _draw(rng, op)
    del c["name"]
    return c


def _draw(rng, op):
    page, d = rng.choice((16, 32, 32, 64, 128)), rng.choice((64, 128, 128, 128))
    dtype, layout, ragged = rng.choice(("bf16", "bf16", "bf16", "f32")), rng.choice(("tokens", "heads")), rng.random() < 0.5
    heads, kv_heads = rng.choice(((32, 32), (40, 40), (16, 16), (32, 8), (40, 8), (28, 4), (64, 8), (8, 1)))
    batch, adjacent, axes = _log(rng, 1, 64), rng.random() < 0.3, rng.choice((1, 1, 2, 3))
    if op == "rotate":
        d = rng.choice((64, 80, 128, 128, 128, 256))
        rows = _log(rng, 1, 4000)
        return _rotate("", batch, rows, rows + rng.choice((0, _log(rng, 1, 4000))), heads, kv_heads, d, rng.choice((d // 2, d // 2, d // 4)), axes,
                       dtype, layout, adjacent, rng.random() < 0.3, ragged)
    if op == "append":
        return _append("", batch, _log(rng, 1, 3000), rng.choice((0, _log(rng, 1, 2000))), heads, kv_heads, d, rng.choice((d // 2, d // 2, d // 4)),
                       axes, page, dtype, layout, adjacent, ragged)
    if op == "bounds":
        return _bounds("", batch, _log(rng, 1, 6000), rng.choice((0, _log(rng, 1, 6000))), kv_heads, d, page, ragged)
    rows = rng.choice((1, 1, rng.randint(2, 12), _log(rng, 16, 400)))
    length = max(_log(rng, 2, 120000), rows)
    budget = rng.choice((8, 16, 32, 64, _log(rng, 2, 200)))
    if op == "choose":                  # (there is something to choose)
        length = max(length, 20 * page)
        budget = max(8, min(budget, length // page // 2))
        return _choose("", batch, rows, length, heads, kv_heads, d, page, budget, dtype, layout, ragged)
    return _attend("", batch, rows, length, heads, kv_heads, d, page, budget, dtype, layout, ragged, rng.choice((1.0, 1.0, rng.uniform(0.4, 0.95))))


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _spread(batch, low, high, ragged):
    """Lengths of a batch: all `high`, or spread over low..high, the first one the longest."""
    share = [1.0 if b == 0 or not ragged else (0.6180339887 * b) % 1.0 for b in range(batch)]
    return [low + int(round(s * (high - low))) for s in share]


def _by_layout(t, layout):
    """A [B, rows, heads, d] tensor, or a view of that shape on head-major memory."""
    return t if layout == "tokens" else t.transpose(1, 2).contiguous().transpose(1, 2)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _normal(g, shape, c, size=1.0):
    return _by_layout((torch.empty(shape, device="cuda").normal_(generator=g) * size).to(_type(c)), c["layout"])


def _zeros(shape, c):
    return _by_layout(torch.zeros(shape, dtype=_type(c), device="cuda"), c["layout"])


def _uneven(g, heads, d):
    """Some channels of K are several times larger than the others, as projections give them."""
    return 1.0 + 4.0 * (torch.rand((heads, d), generator=g, device="cuda") < 0.06)


def _table(g, lengths, page, entries):
    """A block table as a pool in use gives it: the pages of a request lie anywhere.  And the number of pages in the pool."""
    held = torch.tensor([-(-n // page) for n in lengths], device="cuda")
    pool = int(held.sum()) + len(lengths) + 8
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    at = (held.cumsum(0) - held)[:, None] + torch.arange(entries, device="cuda")[None]
    own_entry = torch.arange(entries, device="cuda")[None] < held[:, None]
    return torch.where(own_entry, order[at.clamp(max=pool - 1)], -1).to(torch.int32).contiguous(), pool


def _page_bytes(page, d):
    return page * (d + d // 16)


def _sections(pairs, axes):
    """Pairs of each axis: time gets half of what height and width get."""
    if axes == 1:
        return [pairs]
    if axes == 2:
        return [pairs // 2, pairs - pairs // 2]
    return [pairs - 2 * (2 * pairs // 5), 2 * pairs // 5, 2 * pairs // 5]


def _positions(c, tokens, before):
    """[axes, B, tokens]: frames of 24 x 24 tokens, each axis counted from where the sequence stands; the last tokens are text."""
    j = torch.arange(tokens, device="cuda")
    text = j >= tokens - tokens // 8
    frames = torch.stack([j // 576, j // 24 % 24, j % 24])[3 - c["axes"]:] if c["axes"] > 1 else j[None]
    at = torch.where(text, j, frames)[:, None] + torch.tensor(before, device="cuda")[None, :, None]
    return at.to(torch.int32).contiguous()


def _angles(pairs, count):
    """fp32 [count, pairs, 2]: cosine and sine of position * 10000^(-i / pairs), of angles in 64 bits."""
    rate = torch.exp(torch.arange(pairs, dtype=torch.float64, device="cuda") * (-math.log(10000.0) / pairs))
    at = torch.arange(count, dtype=torch.float64, device="cuda")[:, None] * rate
    return torch.stack([at.cos(), at.sin()], dim=-1).float().contiguous()


def prepare(case, seed):
    made = {"rotate": _prepare_rotate, "append": _prepare_append, "bounds": _prepare_bounds, "choose": _prepare_choose, "attend": _prepare_attend}
    return made[case["op"]](case, _generator(seed))


def _rotation(c, tokens, before):
    return {"positions": _positions(c, tokens, before), "angles": _angles(c["pairs"], max(before) + tokens), "sections": _sections(c["pairs"], c["axes"]),
            "axis": torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_sections(c["pairs"], c["axes"]), device="cuda")),
            "adjacent": c["adjacent"]}


def _prepare_rotate(c, g):
    B, N, d = c["batch"], c["rows"], c["d"]
    before = torch.randint(0, 2000, (B,), generator=g, device="cuda").tolist()
    index = None
    if c["tokens"] > N:                 # the rows that a stage before kept, in order
        index = torch.rand((B, c["tokens"]), generator=g, device="cuda").argsort(1)[:, :N].sort(1).values.to(torch.int32).contiguous()
    return {"op": "rotate", "q": _normal(g, (B, N, c["heads"], d), c), "k": _normal(g, (B, N, c["kv_heads"], d), c, _uneven(g, c["kv_heads"], d)),
            "q_out": _zeros((B, N, c["heads"], d), c), "k_out": _zeros((B, N, c["kv_heads"], d), c), "index": index, "inverse": c["inverse"],
            "count": _ints(_spread(B, max(1, N // 8), N, True)) if c["ragged"] else None, **_rotation(c, c["tokens"], before)}


def _slots(table, page, first, length, rows):
    at = first[:, None] + torch.arange(rows, device="cuda", dtype=torch.int32)[None]
    pages = torch.gather(table, 1, (at // page).clamp(max=table.shape[1] - 1).long())
    return torch.where(at < length[:, None], pages * page + at % page, -1).to(torch.int32)


def _prepare_append(c, g):
    B, N, H, d, page = c["batch"], c["rows"], c["kv_heads"], c["d"], c["page"]
    lengths = [c["before"] + n for n in _spread(B, max(1, N // 8), N, c["ragged"])]
    table, pool = _table(g, lengths, page, -(-(c["before"] + N) // page))
    s = {"op": "append", "page": page, "d": d, "table": table, "length": _ints(lengths), "first": _ints([c["before"]] * B),
         "q": _normal(g, (B, N, c["heads"], d), c), "k_new": _normal(g, (B, N, H, d), c, _uneven(g, H, d)), "v_new": _normal(g, (B, N, H, d), c),
         "q_out": _zeros((B, N, c["heads"], d), c), "k_out": _zeros((B, N, H, d), c), "v_out": _zeros((B, N, H, d), c),
         "cache": torch.zeros((pool, H, _page_bytes(page, d)), dtype=torch.uint8, device="cuda"), **_rotation(c, N, [c["before"]] * B)}
    s["slots"] = _slots(table, page, s["first"], s["length"], N)
    return s


def _filled(g, pool, heads, page, d, values=True):
    """A pool with a few heavy entries among the others, written some at a time."""
    cache = torch.zeros((pool, heads, _page_bytes(page, d)), dtype=torch.uint8, device="cuda")
    places, step, mu, size = pool * page, max(1, (1 << 26) // (heads * d)), math.sqrt(MU2 / math.sqrt(d)), _uneven(g, heads, d) if not values else 1.0
    for at in range(0, places, step):
        n = min(step, places - at)
        k = torch.empty((1, n, heads, d), device="cuda").normal_(generator=g) * size
        k += mu * (torch.rand((1, n, 1, 1), generator=g, device="cuda") < HEAVY)
        v = torch.empty((1, n, heads, d), device="cuda").normal_(generator=g) if values else k
        _plain_write(k, v, torch.arange(at, at + n, dtype=torch.int32, device="cuda")[None], cache, d)
    return cache


def _prepare_bounds(c, g):
    B, N, H, d, page = c["batch"], c["rows"], c["kv_heads"], c["d"], c["page"]
    lengths = [c["before"] + n for n in _spread(B, max(1, N // 8), N, c["ragged"])]
    table, pool = _table(g, lengths, page, -(-(c["before"] + N) // page))
    return {"op": "bounds", "page": page, "d": d, "rows": N, "table": table, "length": _ints(lengths), "first": _ints([c["before"]] * B),
            "cache": _filled(g, pool, H, page, d, values=False), "bounds": torch.zeros((pool, H, 2, d), dtype=torch.int8, device="cuda"),
            "scales": torch.zeros((pool, H), dtype=torch.uint8, device="cuda")}


def _queries(c, g):
    shape = (c["batch"], c["rows"], c["heads"], c["d"])
    q = torch.empty(shape, device="cuda").normal_(generator=g) + math.sqrt(MU2 / math.sqrt(c["d"]))
    lengths = _spread(c["batch"], max(c["rows"], c["length"] // 8), c["length"], c["ragged"])
    q_len = _ints(_spread(c["batch"], max(1, c["rows"] // 2), c["rows"], True)) if c["ragged"] and c["rows"] > 1 else None
    return _by_layout(q.to(_type(c)), c["layout"]), lengths, q_len


def _prepare_choose(c, g):
    B, N, H, d, page = c["batch"], c["rows"], c["kv_heads"], c["d"], c["page"]
    q, lengths, q_len = _queries(c, g)
    table, pool = _table(g, lengths, page, -(-c["length"] // page) + 2)
    bounds, scales = torch.zeros((pool, H, 2, d), dtype=torch.int8, device="cuda"), torch.zeros((pool, H), dtype=torch.uint8, device="cuda")
    size, mu, step = _uneven(g, H, d), math.sqrt(MU2 / math.sqrt(d)), max(1, (1 << 27) // (H * d * page))
    for at in range(0, pool, step):     # bounds of keys that were written and are not needed for this
        n = min(step, pool - at)
        k = torch.empty((n, page, H, d), device="cuda").normal_(generator=g) * size
        k += mu * (torch.rand((n, page, 1, 1), generator=g, device="cuda") < HEAVY)
        k = _values(*_quantise(k))
        bounds[at:at + n], scales[at:at + n] = _outward(k.amax(1), k.amin(1))
    return {"op": "choose", "page": page, "q": q, "bounds": bounds, "scales": scales, "table": table, "length": _ints(lengths), "longest": max(lengths),
            "q_len": q_len, "first_pages": min(1, c["budget"] - 1), "last_pages": 1,
            "chosen": torch.full((B, N, H, c["budget"]), -1, dtype=torch.int32, device="cuda")}


def _visible(s, N, page):
    """[B, N]: entries that a row sees, 0 in rows that are none."""
    rows = torch.full_like(s["length"], N) if s["q_len"] is None else s["q_len"]
    i = torch.arange(N, device="cuda")
    seen = (s["length"] - rows)[:, None] + i[None] + 1
    return torch.where(i[None] < rows[:, None], seen.clamp(min=0), 0), i[None] < rows[:, None]


def _prepare_attend(c, g):
    B, N, H, d, page = c["batch"], c["rows"], c["kv_heads"], c["d"], c["page"]
    q, lengths, q_len = _queries(c, g)
    entries = -(-c["length"] // page) + 2
    table, pool = _table(g, lengths, page, entries)
    length, keep = _ints(lengths), None
    if c["keep"] < 1.0:
        keep = torch.rand((B, entries * page), generator=g, device="cuda") < c["keep"]
        keep |= torch.arange(entries * page, device="cuda")[None] >= (length - N)[:, None]      # the new tokens are there
        keep = keep.to(torch.uint8)
    s = {"op": "attend", "page": page, "d": d, "q": q, "cache": _filled(g, pool, H, page, d), "table": table, "length": length, "q_len": q_len,
         "keep": keep, "scale": 1.0 / math.sqrt(d), "out": _zeros((B, N, c["heads"], d), c),
         "lse": torch.zeros((B, c["heads"], N), dtype=torch.float32, device="cuda")}
    # each row's own page and others anywhere before it
    pages = (_visible(s, N, page)[0] + page - 1) // page
    e = torch.arange(entries, device="cuda")
    chosen = torch.full((B, N, H, c["budget"]), -1, dtype=torch.int32, device="cuda")
    for b in range(B):
        r = torch.rand((N, H, entries), generator=g, device="cuda").masked_fill(e >= pages[b, :, None, None], 2.0).masked_fill(e == pages[b, :, None, None] - 1, -1.0)
        best, at = r.sort(dim=-1)
        m = min(c["budget"], entries)
        at = torch.where(best[..., :m] < 1.5, at[..., :m], 1 << 30).sort(dim=-1).values
        chosen[b, :, :, :m] = torch.where(at < (1 << 30), at, -1).to(torch.int32)
    s["chosen"] = chosen
    return s


# ------------------------------------------------------------------------------------------------ the plain forms

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _regions(cache, d):
    """The four parts of every page and head, as views: K codes, K scales, V codes, V scales."""
    P, H, size = cache.shape
    page = size // (d + d // 16)
    ends = [page * d // 2, page * d // 2 + page * d // 32, page * d + page * d // 32, size]
    return (cache[:, :, :ends[0]].unflatten(2, (page, d // 2)), cache[:, :, ends[0]:ends[1]].unflatten(2, (page, d // 32)),
            cache[:, :, ends[1]:ends[2]].unflatten(2, (page // 4, 16, 4, d // 32)),
            cache[:, :, ends[2]:].unflatten(2, (page // 4, d // 32, 4)))


def _quantise(x):
    """[.., d] -> bytes of codes [.., d / 2], bytes of scales [.., d / 32]"""
    x = x.float().unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    part, power = torch.frexp(most)
    e = torch.where(most == 0, -100, (power - 3 + (part >= 0.875)).clamp(-100, 125))
    y = torch.ldexp(x, -e)
    a = y.abs()
    index = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte()
             + (a > 5.0).byte())
    code = (index + 8 * torch.signbit(y).byte()).flatten(-2)
    scale = torch.where(torch.isfinite(most), e + 127, 255).to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], scale.squeeze(-1)


def _values(codes, scales):
    """bytes of codes [.., d / 2], bytes of scales [.., d / 32] -> fp32 [.., d]"""
    one = torch.tensor(MAGNITUDES, device=codes.device)
    pair = torch.stack([torch.cat([one, -one]).repeat(16), torch.cat([one, -one]).repeat_interleave(16)], dim=-1)
    x = torch.index_select(pair, 0, codes.flatten().int()).view(*codes.shape[:-1], -1, 32)
    size = torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)
    return (x * torch.where(scales == 255, math.nan, size)[..., None]).flatten(-2)


def _plain_write(k, v, slots, cache, d):
    kc, ks, vc, vs = _regions(cache, d)
    page = kc.shape[2]
    b, i = torch.nonzero(slots >= 0, as_tuple=True)
    slot = slots[b, i].long()
    at, t = slot // page, slot % page
    codes, scales = _quantise(k[b, i])
    kc[at, :, t], ks[at, :, t] = codes, scales
    codes, scales = _quantise(v[b, i])
    vc[at, :, t // 4, :, t % 4], vs[at, :, t // 4, :, t % 4] = codes.unflatten(-1, (16, -1)), scales


def _plain_read(cache, table, first, length, d, k_out, v_out):
    kc, ks, vc, vs = _regions(cache, d)
    page = kc.shape[2]
    slots = _slots(table, page, first, length, k_out.shape[1])
    b, i = torch.nonzero(slots >= 0, as_tuple=True)
    slot = slots[b, i].long()
    at, t = slot // page, slot % page
    k_out[b, i] = _values(kc[at, :, t], ks[at, :, t]).to(k_out.dtype)
    v_out[b, i] = _values(vc[at, :, t // 4, :, t % 4].flatten(-2), vs[at, :, t // 4, :, t % 4]).to(v_out.dtype)


def _cosines(s, index=None):
    """[B, N, 1, pairs] each: cosines and sines of the rows' pairs."""
    at = s["positions"] if index is None else torch.gather(s["positions"], 2, index.long()[None].expand(s["positions"].shape[0], -1, -1))
    at = at[s["axis"]].permute(1, 2, 0).long()
    both = s["angles"][at, torch.arange(at.shape[2], device="cuda")][:, :, None]
    return both[..., 0], both[..., 1]


def _rotated(x, c, s, adjacent):
    """fp32 rows [B, N, heads, d]: their pairs turned."""
    m = c.shape[-1]
    x = x.float()
    a, b = (x[..., 0:2 * m:2], x[..., 1:2 * m:2]) if adjacent else (x[..., :m], x[..., m:2 * m])
    a, b = a * c - b * s, b * c + a * s
    pairs = torch.stack([a, b], dim=-1).flatten(-2) if adjacent else torch.cat([a, b], dim=-1)
    return torch.cat([pairs, x[..., 2 * m:]], dim=-1)


def _plain_rotate(s):
    c, sine = _cosines(s, s["index"])
    sine = -sine if s["inverse"] else sine
    live = True if s["count"] is None else (torch.arange(s["q"].shape[1], device="cuda")[None] < s["count"][:, None])[:, :, None, None]
    q, k = (_rotated(s[n], c, sine, s["adjacent"]).to(s[n].dtype) for n in "qk")
    s["q_out"].copy_(q if live is True else torch.where(live, q, s["q_out"]))
    s["k_out"].copy_(k if live is True else torch.where(live, k, s["k_out"]))


def _plain_append(s):
    c, sine = _cosines(s)
    q = _rotated(s["q"], c, sine, s["adjacent"]).to(s["q"].dtype)
    s["q_out"].copy_(torch.where((s["slots"] >= 0)[:, :, None, None], q, s["q_out"]))
    _plain_write(_rotated(s["k_new"], c, sine, s["adjacent"]), s["v_new"], s["slots"], s["cache"], s["d"])


def _outward(most, least):
    """Largest and smallest values [.., H, d] -> int8 [.., H, 2, d], bytes [.., H]"""
    a = torch.maximum(most.abs(), least.abs()).amax(-1)
    e = torch.where(a == 0, -126, torch.frexp(a).exponent - 7)
    whole = torch.stack([torch.ldexp(most, -e[..., None]).ceil(), torch.ldexp(least, -e[..., None]).floor()], dim=-2)
    fine = torch.isfinite(a)
    return torch.where(fine[..., None, None], whole, 0.0).to(torch.int8), torch.where(fine, e + 127, 255).to(torch.uint8)


def _plain_bounds(s):
    kc, ks, _, _ = _regions(s["cache"], s["d"])
    page, entries = s["page"], s["table"].shape[1]
    e = torch.arange(entries, device="cuda")[None]
    last = torch.minimum(s["first"] + s["rows"], s["length"])
    b, at = torch.nonzero((e >= (s["first"] // page)[:, None]) & (e * page < last[:, None]), as_tuple=True)
    id = s["table"][b, at].long()
    k = _values(kc[id], ks[id])                                                             # [pages, H, page, d]
    live = (at[:, None] * page + torch.arange(page, device="cuda")[None] < s["length"][b][:, None])[:, None, :, None]
    most, least = torch.where(live, k, -math.inf).amax(2), torch.where(live, k, math.inf).amin(2)
    s["bounds"][id], s["scales"][id] = _outward(most, least)


def _plain_choose(s):
    B, N, Hq, d = s["q"].shape
    H, page, budget = s["bounds"].shape[1], s["page"], s["chosen"].shape[3]
    q = s["q"].float().view(B, N, H, Hq // H, d)
    a = q.abs().amax((-1, -2), keepdim=True)
    whole = torch.ldexp(q, 7 - torch.frexp(a).exponent).round().clamp(-127, 127)
    whole = torch.where(torch.isfinite(a) & (a > 0), whole, 0.0)
    both = torch.stack([whole.clamp(min=0).sum(3), whole.clamp(max=0).sum(3)], dim=3).flatten(3).transpose(1, 2).contiguous().double()       # [B, H, N, 2d]
    P = -(-s["longest"] // page)
    id = s["table"][:, :P].clamp(min=0).long()
    pages = s["bounds"][id].flatten(3).permute(0, 2, 3, 1).contiguous().double()            # [B, H, 2d, P]
    scale = s["scales"][id].transpose(1, 2)[:, :, None]
    score = torch.matmul(both, pages).float() * torch.ldexp(torch.ones((), device="cuda"), scale.int() - 127)
    score = score.double().masked_fill(scale == 255, 1e300)
    seen, live = _visible(s, N, page)
    seen = ((seen + page - 1) // page)[:, None, :, None]
    e = torch.arange(P, device="cuda")
    score = score.masked_fill((s["table"][:, None, None, :P] < 0), -1e300)
    always = (e < s["first_pages"]) | (e >= seen - s["last_pages"])
    score = torch.where(e < seen, torch.where(always, math.inf, score), -math.inf)
    order = score.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    order = torch.where(order < seen, order, 1 << 30).sort(dim=-1).values
    order = torch.where(order < (1 << 30), order, -1).to(torch.int32).transpose(1, 2)
    full = torch.full_like(s["chosen"], -1)
    full[..., :order.shape[3]] = order
    s["chosen"].copy_(torch.where(live[:, :, None, None], full, s["chosen"]))


def _plain_attend(s):
    B, N, Hq, d = s["q"].shape
    kc, ks, vc, vs = _regions(s["cache"], d)
    page, H, budget = s["page"], s["cache"].shape[1], s["chosen"].shape[3]
    at = s["chosen"].transpose(1, 2)                                                        # [B, H, N, budget]
    b, h = torch.arange(B, device="cuda")[:, None, None, None], torch.arange(H, device="cuda")[None, :, None, None]
    id = s["table"][b, at.clamp(min=0).long()].clamp(min=0).long()
    L = budget * page
    place = (at.long()[..., None] * page + torch.arange(page, device="cuda")).flatten(3)    # [B, H, N, L]
    seen, live = _visible(s, N, page)
    ok = (at >= 0).repeat_interleave(page, dim=3) & (place < seen[:, None, :, None])
    if s["keep"] is not None:
        ok = ok & (s["keep"][b, place.clamp(min=0)] != 0)
    q = s["q"].float().view(B, N, H, Hq // H, d).permute(0, 2, 1, 3, 4).reshape(-1, Hq // H, d)
    k = _values(kc[id, h], ks[id, h]).view(B * H * N, L, d)
    x = torch.matmul(q, k.transpose(1, 2)).mul_(s["scale"]).masked_fill_(~ok.reshape(-1, 1, L), -math.inf)
    del k
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = _values(vc[id, h].transpose(5, 6).flatten(6), vs[id, h].transpose(5, 6)).view(B * H * N, L, d)
    o = (torch.matmul(x, v) / total.clamp(min=1e-38)).view(B, H, N, Hq // H, d).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, d)
    lse = (top + total.log()).view(B, H, N, Hq // H).transpose(2, 3).reshape(B, Hq, N)
    s["out"].copy_(torch.where(live[:, :, None, None], o.to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(live[:, None], lse, s["lse"]))


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    return {"rotate": _run_rotate, "append": _run_append, "bounds": _run_bounds, "choose": _run_choose, "attend": _run_attend}[state["op"]](state)


def _handle(s, md):
    if "rotary" not in s:               # a program keeps it: which pair of channels turns by which axis
        s["rotary"] = md.rotary(s["sections"], adjacent=s["adjacent"])
    return s["rotary"]


def _run_rotate(s):
    if own:
        import paper_2411_10803_amd as md
        md.mustdrop_rotate(s["q"], s["positions"], s["angles"], _handle(s, md), k=s["k"], q_out=s["q_out"], k_out=s["k_out"], index=s["index"],
                           rows=s["count"], inverse=s["inverse"])
    else:
        _plain_rotate(s)
    return {"q": s["q_out"], "k": s["k_out"]}


def _run_append(s):
    """Rows in and out again: what the cache holds is told by the values that it gives back."""
    if own:
        import paper_2411_10803_amd as md
        md.mustdrop_cache4_append(s["q"], s["k_new"], s["v_new"], s["positions"], s["angles"], _handle(s, md), s["slots"], s["cache"], q_out=s["q_out"])
        md.mustdrop_cache4_read(s["cache"], s["table"], s["length"], s["k_out"], s["v_out"], first=s["first"])
    else:
        _plain_append(s)
        _plain_read(s["cache"], s["table"], s["first"], s["length"], s["d"], s["k_out"], s["v_out"])
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _run_bounds(s):
    """The bounds are whole numbers, and their scales the bytes of exponents: they have to be equal."""
    if own:
        import paper_2411_10803_amd as md
        md.mustdrop_cache4_bounds(s["cache"], s["table"], s["length"], s["rows"], s["bounds"], s["scales"], first=s["first"])
    else:
        _plain_bounds(s)
    return {"bounds": s["bounds"], "scales": s["scales"]}


def _run_choose(s):
    if own:
        import paper_2411_10803_amd as md
        if "workspace" not in s:        # a program keeps it from step to step
            s["workspace"] = md.cache4_choose_workspace(s["q"], s["bounds"], s["table"])
        md.mustdrop_cache4_choose(s["q"], s["bounds"], s["scales"], s["table"], s["length"], s["page"], s["chosen"], q_len=s["q_len"],
                                  first_pages=s["first_pages"], last_pages=s["last_pages"], workspace=s["workspace"])
    else:
        _plain_choose(s)
    return {"chosen": s["chosen"]}


def _run_attend(s):
    if own:
        import paper_2411_10803_amd as md
        if "workspace" not in s:
            s["workspace"] = md.cache4_attend_chosen_workspace(s["q"], s["cache"], s["chosen"])
        md.mustdrop_cache4_attend_chosen(s["q"], s["cache"], s["table"], s["length"], s["chosen"], s["scale"], out=s["out"], lse=s["lse"],
                                         q_len=s["q_len"], keep=s["keep"], workspace=s["workspace"])
    else:
        _plain_attend(s)
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------ accounting

def work(case):
    """Bytes and operations of one pass: every input that it needs once, every output once."""
    c = case
    B, d, Hk = c["batch"], c["d"], c["kv_heads"]
    size = 4 if c.get("dtype") == "f32" else 2
    if c["op"] == "rotate":
        rows = sum(_spread(B, max(1, c["rows"] // 8), c["rows"], True)) if c["ragged"] else B * c["rows"]
        heads = c["heads"] + Hk
        return {"bytes": rows * (2.0 * heads * d * size + 8 * c["pairs"] + 4 * c["axes"]), "flops": 6.0 * rows * heads * c["pairs"]}
    if c["op"] == "append":             # in, and out again
        rows = sum(_spread(B, max(1, c["rows"] // 8), c["rows"], c["ragged"]))
        return {"bytes": rows * (2.0 * c["heads"] * d * size + 2.0 * Hk * d * (2 * size + 17.0 / 32) + 8 * c["pairs"] + 4 * c["axes"]),
                "flops": rows * (6.0 * (c["heads"] + Hk) * c["pairs"] + 6.0 * Hk * d)}
    if c["op"] == "bounds":
        lengths = [c["before"] + n for n in _spread(B, max(1, c["rows"] // 8), c["rows"], c["ragged"])]
        begin = c["before"] // c["page"]
        entries, pages = sum(n - begin * c["page"] for n in lengths), sum(-(-n // c["page"]) - begin for n in lengths)
        return {"bytes": Hk * (entries * d * 17.0 / 32 + pages * (2 * d + 1)), "flops": 2.0 * entries * Hk * d}
    N, H = c["rows"], c["heads"]
    lengths = _spread(B, max(N, c["length"] // 8), c["length"], c["ragged"])
    rows = _spread(B, max(1, N // 2), N, True) if c["ragged"] and N > 1 else [N] * B
    pages = [-(-n // c["page"]) for n in lengths]
    if c["op"] == "choose":
        flops = sum(4.0 * m * p for m, p in zip(rows, pages)) * H * d
        return {"bytes": sum(pages) * (Hk * (2.0 * d + 1) + 4) + sum(rows) * (H * d * size + Hk * c["budget"] * 4.0), "flops": flops}
    taken = [min(n, c["budget"] * c["page"]) * c["keep"] for n in lengths]
    live = sum(min(t * m, n * c["keep"]) for t, m, n in zip(taken, rows, lengths))
    return {"bytes": live * Hk * d * 17.0 / 16 + sum(rows) * (H * (2.0 * d * size + 4) + Hk * c["budget"] * 4.0),
            "flops": 4.0 * sum(t * m for t, m in zip(taken, rows)) * H * d}


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits

def exact(case, seed):
    """What `run` gives for these inputs, in 64 bits, request by request."""
    if case["batch"] * case["rows"] > 3000 and case["op"] in ("choose", "attend"):
        return None
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "bounds": _exact_bounds, "choose": _exact_choose, "attend": _exact_attend}[case["op"]](s)


def _turned(x, s, b, at):
    """Rows [n, heads, d] of request b at positions `at` [axes, n], in 64 bits: each pair as a complex number times another."""
    m = s["axis"].shape[0]
    both = s["angles"].double()[at.long()[s["axis"]], torch.arange(m, device="cuda")[:, None]]               # [pairs, n, 2]
    by = torch.view_as_complex(both.contiguous()).transpose(0, 1)[:, None]
    by = by.conj() if s.get("inverse") else by
    y = x.double().clone()
    first, second = (slice(0, 2 * m, 2), slice(1, 2 * m, 2)) if s["adjacent"] else (slice(0, m), slice(m, 2 * m))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * by
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_rotate(s):
    out = {n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in "qk"}
    for b in range(s["q"].shape[0]):
        n = s["q"].shape[1] if s["count"] is None else int(s["count"][b])
        at = s["positions"][:, b] if s["index"] is None else s["positions"][:, b][:, s["index"][b].long()]
        for x in "qk":
            out[x][b, :n] = _turned(s[x][b, :n], s, b, at[:, :n])
    return out


def _held_as(x):
    """The values that the cache holds for [.., 32 n] numbers: of the fifteen values times the scale the nearest."""
    x = x.double().unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)
    k = torch.floor(torch.log2(most.clamp(min=2.0 ** -200)))
    k = k + (torch.exp2(k + 1) <= most).double() - (torch.exp2(k) > most).double()        # log2 may round up to a whole number
    e = torch.where(most == 0, -100.0, (k - 2 + (most >= 1.75 * torch.exp2(k))).clamp(-100, 125))
    levels = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    a = x.abs() / torch.exp2(e)
    below = (torch.searchsorted(levels, a, right=True) - 1).clamp(0, 7)
    above = (below + 1).clamp(max=7)
    down, up = a - levels[below], levels[above] - a
    index = torch.where((down > up) | ((down == up) & (below % 2 == 1)), above, below)
    return (torch.copysign(levels[index], x) * torch.exp2(e)).flatten(-2)


def _exact_append(s):
    out = {n: torch.zeros(s[n + "_out"].shape, dtype=torch.float64, device="cuda") for n in "qkv"}
    for b, n in enumerate((s["length"] - s["first"]).tolist()):
        at = s["positions"][:, b, :n]
        out["q"][b, :n] = _turned(s["q"][b, :n], s, b, at)
        out["k"][b, :n], out["v"][b, :n] = _held_as(_turned(s["k_new"][b, :n], s, b, at)), _held_as(s["v_new"][b, :n])
    return out


def _signed(code):
    return torch.tensor(MAGNITUDES, dtype=torch.float64, device=code.device)[(code & 7).long()] * (1 - 2 * (code >> 3).double())


def _numbers(code_bytes, scale_bytes):
    """[.., d / 2] and [.., d / 32] bytes -> [.., d] in 64 bits"""
    x = torch.stack([_signed(code_bytes & 15), _signed(code_bytes >> 4)], dim=-1).flatten(-2)
    return x * torch.exp2(scale_bytes.double() - 127.0).repeat_interleave(32, dim=-1)


def _keys_values(raw, page, d):
    """Bytes of pages [.., page * (d + d / 16)] -> K and V [.., page, d], in 64 bits"""
    c = page * d // 2
    lead = raw.shape[:-1]
    k = _numbers(raw[..., :c].reshape(*lead, page, d // 2), raw[..., c:c + page * d // 32].reshape(*lead, page, d // 32))
    vc = raw[..., c + page * d // 32:2 * c + page * d // 32].reshape(*lead, page // 4, 16, 4, d // 32).transpose(-3, -2).reshape(*lead, page, d // 2)
    vs = raw[..., 2 * c + page * d // 32:].reshape(*lead, page // 4, d // 32, 4).transpose(-2, -1).reshape(*lead, page, d // 32)
    return k, _numbers(vc, vs)


def _exact_bounds(s):
    page, d, bounds, scales = s["page"], s["d"], s["bounds"].clone(), s["scales"].clone()
    for b, n in enumerate(s["length"].tolist()):
        e0 = int(s["first"][b]) // page
        id = s["table"][b, e0:-(-n // page)].long()
        k, _ = _keys_values(s["cache"][id], page, d)                                        # [pages, H, page, d]
        dead = torch.arange(e0 * page, e0 * page + id.numel() * page, device="cuda").view(-1, 1, page, 1) >= n
        most, least = k.masked_fill(dead, -math.inf).amax(2), k.masked_fill(dead, math.inf).amin(2)
        a = torch.maximum(most, -least).amax(-1)
        e = torch.where(a > 0, torch.floor(torch.log2(a.clamp(min=1e-60)) + 1e-9) - 6, -126.0)
        bounds[id] = torch.stack([(most / torch.exp2(e)[..., None]).ceil(), (least / torch.exp2(e)[..., None]).floor()], dim=2).to(torch.int8)
        scales[id] = (e + 127).to(torch.uint8)
    return {"bounds": bounds, "scales": scales}


def _exact_choose(s):
    B, N, Hq, d = s["q"].shape
    H, page, chosen = s["bounds"].shape[1], s["page"], s["chosen"].clone()
    budget, G = chosen.shape[3], Hq // H
    for b, n in enumerate(s["length"].tolist()):
        rows = N if s["q_len"] is None else int(s["q_len"][b])
        id = s["table"][b, :-(-n // page)].long()
        hi, lo = s["bounds"][id, :, 0].double(), s["bounds"][id, :, 1].double()             # [pages, H, d]
        size = torch.exp2(s["scales"][id].double() - 127).T
        for i in range(rows):
            q = s["q"][b, i].double().view(H, G, d)
            step = torch.exp2(torch.floor(torch.log2(q.abs().amax((1, 2), keepdim=True))) - 6)
            q = (q / step).round().clamp(-127, 127)
            score = sum(torch.maximum(q[None, :, g] * hi, q[None, :, g] * lo).sum(-1) for g in range(G)).T * size
            pages = (n - rows + i) // page + 1
            score = score[:, :pages].clone()
            score[:, :s["first_pages"]], score[:, max(0, pages - s["last_pages"]):] = math.inf, math.inf
            best = score.sort(dim=-1, descending=True, stable=True).indices[:, :budget].sort(-1).values
            chosen[b, i], chosen[b, i, :, :best.shape[1]] = -1, best.int()
    return {"chosen": chosen}


def _exact_attend(s):
    B, N, Hq, d = s["q"].shape
    page, H = s["page"], s["cache"].shape[1]
    G = Hq // H
    out, lse = torch.zeros((B, N, Hq, d), dtype=torch.float64, device="cuda"), torch.zeros((B, Hq, N), dtype=torch.float64, device="cuda")
    head = torch.arange(H, device="cuda")[:, None]
    for b, n in enumerate(s["length"].tolist()):
        rows = N if s["q_len"] is None else int(s["q_len"][b])
        for i in range(rows):
            at = s["chosen"][b, i].long()                                                   # [H, budget]
            id = s["table"][b, at.clamp(min=0)].long().clamp(min=0)
            k, v = (x.flatten(1, 2) for x in _keys_values(s["cache"][id, head], page, d))
            place = (at[..., None] * page + torch.arange(page, device="cuda")).flatten(1)
            seen = (at >= 0).repeat_interleave(page, 1) & (place <= n - rows + i)
            if s["keep"] is not None:
                seen &= s["keep"][b, place.clamp(min=0)] != 0
            x = (s["q"][b, i].double().view(H, G, d) @ k.transpose(1, 2) * s["scale"]).masked_fill(~seen[:, None], -math.inf)
            lse[b, :, i] = torch.logsumexp(x, dim=-1).flatten()
            out[b, i] = (torch.softmax(x, dim=-1) @ v).flatten(0, 1)
    return {"out": out, "lse": lse}
