"""The operators behind the cache held in 4 bits, as they are measured: block tables and slot maps from request lengths, rows
into the cache, rows out of it, and the attention that reads it.

A case is one pass as a serving program makes it.  `own` says who computes it: elementary torch operations (the plain form),
or the library's entry points.

The cache.  A group of 32 consecutive channels of one token and head is held as 32 numbers of 4 bits (sign, and the index of
the magnitude in 0, 0.5, 1, 1.5, 2, 3, 4, 6) and one scale 2^e.  With a the largest magnitude of the group and k = floor(log2 a),
e = k - 2, or k - 1 where a >= 1.75 * 2^k (so that a is rounded to 6 at most, not cut down to it), within -100 and 125; -100
where a = 0.  x becomes the nearest value to x / 2^e, the even index where two are as near.  The scale is stored as the byte
e + 127; a group with an infinity or a NaN has 255 there and reads as NaN.

A pool is uint8 [pages, H, page * (d + d / 16)]: per page and head, one after the other,
  K codes   [page, d / 2]                 channel 2i in the low half of byte i
  K scales  [page, d / 32]
  V codes   [page / 4, 16, 4, d / 32]     the d / 16 channels of a sixteenth of the row, of four tokens side by side
  V scales  [page / 4, d / 32, 4]
A request's row in the block table names its pages; a slot is page number * page + place in the page.
"""
from __future__ import annotations

import math

import torch

own = False

MU2 = 3.0             # heavy entries: logits about three standard deviations above the others, as in the decode workload
HEAVY = 0.05


def _pages(name, batch, rows, before, page, capacity):
    return {"name": name, "op": "pages", "batch": batch, "rows": rows, "before": before, "page": page, "capacity": capacity}


def _rows(name, op, batch, rows, before, heads, d, page, dtype="bf16", layout="tokens", ragged=False):
    return {"name": name, "op": op, "batch": batch, "rows": rows, "before": before, "heads": heads, "d": d, "page": page,
            "dtype": dtype, "layout": layout, "ragged": ragged}


def _attend(name, batch, rows, length, heads, kv_heads, d, page, capacity, dtype="bf16", layout="tokens", ragged=False, keep=1.0):
    return {"name": name, "op": "attend", "batch": batch, "rows": rows, "length": length, "heads": heads, "kv_heads": kv_heads,
            "d": d, "page": page, "capacity": capacity, "dtype": dtype, "layout": layout, "ragged": ragged, "keep": keep}


def listed():
    return [
        # a decode step of many sequences: one token more each, and back (a draft that is not taken)
        _pages("pages_step_b64", 64, 1, 1024, 32, 4352),
        # requests with high-resolution images come and go: five tiles and a prompt
        _pages("pages_prompts_b256", 256, 3008, 0, 64, 4096),
        # the rows of a decode step, and what the cache then holds of them
        _rows("store_step_b64", "store", 64, 1, 1024, 32, 128, 32),
        # the rows that the prefill stage kept, for a batch of requests with prompts of different lengths
        _rows("store_prompts_b16", "store", 16, 640, 0, 32, 128, 32, ragged=True),
        # fp32 rows of a head-major tensor
        _rows("store_f32_heads40_b4", "store", 4, 777, 100, 40, 64, 16, dtype="f32", layout="heads"),
        # a turn is over: the cache comes back as dense rows for the eviction
        _rows("load_turn_b64", "load", 64, 1025, 0, 32, 128, 32),
        # the last rows of a few sequences, head-major
        _rows("load_heads40_b4", "load", 4, 160, 617, 40, 128, 64, layout="heads", ragged=True),
        # one sequence with an image and a short question: the shortest call, where latency counts
        _attend("attend_step_b1", 1, 1, 640, 32, 32, 128, 32, 1024),
        # the decode workload: 64 sequences of up to 4096 entries
        _attend("attend_step_b64", 64, 1, 4096, 32, 32, 128, 32, 4352, ragged=True),
        # two long documents, eight K/V heads
        _attend("attend_step_long_b2", 2, 1, 100003, 32, 8, 128, 64, 131072, ragged=True),
        # drafts of five tokens, entries masked by an eviction that has not moved anything yet
        _attend("attend_draft_b16", 16, 5, 2009, 40, 40, 128, 16, 4096, ragged=True, keep=0.75),
        # a chunk of a prompt behind images in tiles
        _attend("attend_prompt_b4", 4, 512, 5888, 32, 8, 128, 64, 8192, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 5e14


def draw(rng):
    """One more case of the ranges above, at most as costly as the largest of its operator."""
    c = _draw(rng)
    while _cost(c) > max(_cost(x) for x in listed() if x["op"] == c["op"]):
        c = _draw(rng)
    del c["name"]
    return c


def _draw(rng):
    op = rng.choice(("pages", "store", "load", "attend", "attend", "attend"))
    page = rng.choice((16, 32, 32, 64, 128))
    if op == "pages":
        rows, before = _log(rng, 1, 3008), rng.choice((0, _log(rng, 1, 5000)))
        return _pages("", _log(rng, 1, 1000), rows, before, page, before + rows + _log(rng, 1, 2000))
    d, dtype, layout, ragged = rng.choice((64, 128, 128, 128)), rng.choice(("bf16", "bf16", "bf16", "f32")), rng.choice(("tokens", "heads")), rng.random() < 0.5
    if op != "attend":
        return _rows("", op, _log(rng, 1, 64), _log(rng, 1, 4000), rng.choice((0, _log(rng, 1, 2000))), rng.choice((4, 8, 16, 32, 40)), d, page,
                     dtype, layout, ragged)
    heads, kv_heads = rng.choice(((32, 32), (40, 40), (16, 16), (32, 8), (40, 8), (28, 4), (64, 8), (8, 1)))
    rows = rng.choice((1, 1, rng.randint(2, 12), _log(rng, 16, 700)))
    length = max(_log(rng, 2, 120000), rows)
    return _attend("", _log(rng, 1, 64), rows, length, heads, kv_heads, d, page, length + _log(rng, 1, 4000), dtype, layout, ragged,
                   rng.choice((1.0, 1.0, rng.uniform(0.4, 0.95))))


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


def _table(g, lengths, page, entries, pool=None):
    """A block table as a pool in use gives it: the pages of a request lie anywhere.  And the number of pages in the pool."""
    held = torch.tensor([-(-n // page) for n in lengths], device="cuda")
    pool = pool or int(held.sum()) + len(lengths) + 8
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    at = (held.cumsum(0) - held)[:, None] + torch.arange(entries, device="cuda")[None]
    own_entry = torch.arange(entries, device="cuda")[None] < held[:, None]
    return torch.where(own_entry, order[at.clamp(max=pool - 1)], -1).to(torch.int32).contiguous(), pool


def _page_bytes(page, d):
    return page * (d + d // 16)


def prepare(case, seed):
    made = {"pages": _prepare_pages, "store": _prepare_store, "load": _prepare_load, "attend": _prepare_attend}
    return made[case["op"]](case, _generator(seed))


def _prepare_pages(c, g):
    B, page, entries = c["batch"], c["page"], -(-c["capacity"] // c["page"])
    # requests at lengths of their own, from half of `before` on; each gets up to `rows` tokens more, two thirds of them at least
    span = lambda n, low: torch.randint(low, n + 1, (B,), generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    length = span(c["before"], c["before"] // 2)
    longer = length + span(c["rows"], (2 * c["rows"] + 2) // 3)
    table, pool = _table(g, length.tolist(), page, entries, B * -(-(c["before"] + c["rows"]) // page) + 8)
    taken = torch.zeros(pool, dtype=torch.bool, device="cuda")
    taken[table[table >= 0].long()] = True
    rank = torch.rand(pool, generator=g, device="cuda").masked_fill(taken, 2.0).argsort()
    free = torch.where(torch.arange(pool, device="cuda") < (~taken).sum(), rank, -1).to(torch.int32)
    s = {"op": "pages", "page": page, "length": length, "shorter": length.clone(), "longer": longer, "table": table, "free": free,
         "n_free": _ints([int((~taken).sum())]), "missing": _ints([0]),
         "slots": torch.zeros((B, c["rows"]), dtype=torch.int32, device="cuda")}
    s["result"] = {k: s[k] for k in ("slots", "table", "length", "free", "n_free", "missing")}
    return s


def _slots(table, page, first, length, rows):
    at = first[:, None] + torch.arange(rows, device="cuda", dtype=torch.int32)[None]
    pages = torch.gather(table, 1, (at // page).clamp(max=table.shape[1] - 1).long())
    return torch.where(at < length[:, None], pages * page + at % page, -1).to(torch.int32)


def _row_state(c, g):
    B, page = c["batch"], c["page"]
    count = _spread(B, max(1, c["rows"] // 8), c["rows"], c["ragged"])
    lengths = [c["before"] + n for n in count]
    table, pool = _table(g, lengths, page, -(-(c["before"] + c["rows"]) // page))
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    rows = lambda: _by_layout(torch.zeros((B, c["rows"], c["heads"], c["d"]), dtype=dtype, device="cuda"), c["layout"])  # noqa: E731
    s = {"op": c["op"], "page": page, "d": c["d"], "table": table, "length": _ints(lengths), "first": _ints([c["before"]] * B),
         "cache": torch.zeros((pool, c["heads"], _page_bytes(page, c["d"])), dtype=torch.uint8, device="cuda"),
         "k_out": rows(), "v_out": rows()}
    s["slots"] = _slots(table, page, s["first"], s["length"], c["rows"])
    return s, dtype


def _made_rows(c, g, dtype):
    """Rows as projections give them: some channels of K are several times larger than the others."""
    shape = (c["batch"], c["rows"], c["heads"], c["d"])
    size = 1.0 + 4.0 * (torch.rand((c["heads"], c["d"]), generator=g, device="cuda") < 0.06)
    k = torch.empty(shape, device="cuda").normal_(generator=g) * size
    return _by_layout(k.to(dtype), c["layout"]), _by_layout(torch.empty(shape, device="cuda").normal_(generator=g).to(dtype), c["layout"])


def _prepare_store(c, g):
    s, dtype = _row_state(c, g)
    s["k_new"], s["v_new"] = _made_rows(c, g, dtype)
    return s


def _prepare_load(c, g):
    s, dtype = _row_state(c, g)
    k, v = _made_rows(c, g, dtype)
    _plain_write(k, v, s["slots"], s["cache"], c["d"])
    return s


def _prepare_attend(c, g):
    B, N, page, d, Hk = c["batch"], c["rows"], c["page"], c["d"], c["kv_heads"]
    lengths = _spread(B, max(N, c["length"] // 8), c["length"], c["ragged"])
    entries = -(-c["capacity"] // page)
    table, pool = _table(g, lengths, page, entries)
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    mu = math.sqrt(MU2 / math.sqrt(d))
    cache = torch.zeros((pool, Hk, _page_bytes(page, d)), dtype=torch.uint8, device="cuda")
    places, length, step = pool * page, _ints(lengths), max(1, (1 << 26) // (Hk * d))
    for at in range(0, places, step):       # the contents of the pool, some at a time: a few heavy entries among the others
        n = min(step, places - at)
        k = torch.empty((1, n, Hk, d), device="cuda").normal_(generator=g)
        k += mu * (torch.rand((1, n, 1, 1), generator=g, device="cuda") < HEAVY)
        v = torch.empty((1, n, Hk, d), device="cuda").normal_(generator=g)
        _plain_write(k, v, torch.arange(at, at + n, dtype=torch.int32, device="cuda")[None], cache, d)
    q = torch.empty((B, N, c["heads"], d), device="cuda").normal_(generator=g) + mu
    q_len = _ints(_spread(B, max(1, N // 2), N, True)) if c["ragged"] and N > 1 else None
    keep = None
    if c["keep"] < 1.0:
        keep = torch.rand((B, entries * page), generator=g, device="cuda") < c["keep"]
        keep |= torch.arange(entries * page, device="cuda")[None] >= (length - N)[:, None]      # the new tokens are there
        keep = keep.to(torch.uint8)
    s = {"op": "attend", "page": page, "d": d, "q": _by_layout(q.to(dtype), c["layout"]), "cache": cache, "table": table, "length": length,
         "longest": max(lengths), "q_len": q_len, "keep": keep, "scale": 1.0 / math.sqrt(d),
         "out": _by_layout(torch.zeros((B, N, c["heads"], d), dtype=dtype, device="cuda"), c["layout"]),
         "lse": torch.zeros((B, c["heads"], N), dtype=torch.float32, device="cuda")}
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


def _plain_pages(new_len, length, table, free, n_free, page, slots, missing):
    entries, pool = table.shape[1], free.shape[0]
    held, need = (length + page - 1) // page, (new_len + page - 1) // page
    index = torch.arange(entries, device="cuda")[None]
    leave, come = (index >= need[:, None]) & (index < held[:, None]), (index >= held[:, None]) & (index < need[:, None])
    R, T = leave.sum(), come.sum()
    short = (T - n_free - R).clamp(min=0)
    fits = short == 0
    rank = leave.flatten().cumsum(0) - 1
    to = torch.where(leave.flatten() & fits, n_free + R - 1 - rank, pool)
    stack = torch.cat([free, free[:1]])
    stack[to] = table.flatten()
    rank = (come.flatten().cumsum(0) - 1).view_as(come)
    table.copy_(torch.where(come & fits, stack[(n_free + R - 1 - rank).clamp(0, pool - 1)], table))
    free.copy_(stack[:pool])
    if slots is not None:
        slots.copy_(torch.where(fits, _slots(table, page, length, new_len, slots.shape[1]), -1))
    length.copy_(torch.where(fits, new_len, length))
    n_free.copy_(torch.where(fits, n_free + R - T, n_free))
    missing.copy_(short)


def _plain_attend(s):
    B, N, H, d = s["q"].shape
    kc, ks, vc, vs = _regions(s["cache"], d)
    page, Hk = s["page"], s["cache"].shape[1]
    pages = s["table"][:, :-(-s["longest"] // page)].clamp(min=0).long()
    L = pages.shape[1] * page
    by_head = lambda t: t.transpose(1, 2)  # noqa: E731  [B, pages, Hk, ..] -> [B, Hk, pages, ..]
    k = _values(by_head(kc[pages]), by_head(ks[pages])).view(B, Hk, L, d)
    q = s["q"].float().view(B, N, Hk, H // Hk, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, H // Hk * N, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(B, Hk, H // Hk, N, L)
    del k
    j, i = torch.arange(L, device="cuda"), torch.arange(N, device="cuda")
    rows = torch.full_like(s["length"], N) if s["q_len"] is None else s["q_len"]
    seen = j[None, None] <= (s["length"] - rows)[:, None, None] + i[None, :, None]
    seen = seen & (j < s["length"][:, None])[:, None]
    if s["keep"] is not None:
        seen = seen & (s["keep"][:, None, :L] != 0)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = _values(by_head(vc[pages].transpose(4, 5).flatten(5)), by_head(vs[pages].transpose(4, 5)))
    o = torch.matmul(x.view(B, Hk, H // Hk * N, L), v.view(B, Hk, L, d)).view(B, Hk, H // Hk, N, d) / total.clamp(min=1e-38)
    lse = (top + total.log()).squeeze(-1).reshape(B, H, N)
    live = i[None] < rows[:, None]
    s["out"].copy_(torch.where(live[:, :, None, None], o.permute(0, 3, 1, 2, 4).reshape(B, N, H, d).to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(live[:, None], lse, s["lse"]))


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    s = state
    if s["op"] == "pages":
        return _run_pages(s)
    if s["op"] == "attend":
        return _run_attend(s)
    return _run_rows(s)


def _run_pages(s):
    """The tokens come and go again: the pool is then what it was."""
    if own:
        import paper_2411_10803_amd as md
        if "workspace" not in s:        # a program keeps it from step to step
            s["workspace"] = md.cache4_pages_workspace(s["length"].shape[0])
        md.mustdrop_cache4_pages(s["longer"], s["length"], s["table"], s["free"], s["n_free"], s["missing"], s["page"], slots=s["slots"],
                                 workspace=s["workspace"])
        md.mustdrop_cache4_pages(s["shorter"], s["length"], s["table"], s["free"], s["n_free"], s["missing"], s["page"],
                                 workspace=s["workspace"])
    else:
        _plain_pages(s["longer"], s["length"], s["table"], s["free"], s["n_free"], s["page"], s["slots"], s["missing"])
        _plain_pages(s["shorter"], s["length"], s["table"], s["free"], s["n_free"], s["page"], None, s["missing"])
    return s["result"]


def _run_rows(s):
    """Rows in and out again, or only out: what the cache holds is told by the values that it gives back."""
    if own:
        import paper_2411_10803_amd as md
        if s["op"] == "store":
            md.mustdrop_cache4_write(s["k_new"], s["v_new"], s["slots"], s["cache"])
        md.mustdrop_cache4_read(s["cache"], s["table"], s["length"], s["k_out"], s["v_out"], first=s["first"])
    else:
        if s["op"] == "store":
            _plain_write(s["k_new"], s["v_new"], s["slots"], s["cache"], s["d"])
        _plain_read(s["cache"], s["table"], s["first"], s["length"], s["d"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _run_attend(s):
    if own:
        import paper_2411_10803_amd as md
        if "workspace" not in s:
            s["workspace"] = md.cache4_workspace(s["q"], s["cache"], s["table"])
        md.mustdrop_cache4_attend(s["q"], s["cache"], s["table"], s["length"], s["scale"], out=s["out"], lse=s["lse"], q_len=s["q_len"],
                                  keep=s["keep"], workspace=s["workspace"])
    else:
        _plain_attend(s)
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------ accounting

def work(case):
    """Bytes and operations of one pass: every input that it needs once, every output once."""
    c = case
    if c["op"] == "pages":
        more = c["rows"] * 5.0 / 6
        each = 12.0 + 8.0 * more / c["page"] + 4.0 * c["rows"]
        return {"bytes": c["batch"] * each, "flops": c["batch"] * (2.0 * c["rows"] + 8.0)}
    if c["op"] in ("store", "load"):
        rows = sum(_spread(c["batch"], max(1, c["rows"] // 8), c["rows"], c["ragged"]))
        n = 2.0 * rows * c["heads"] * c["d"]
        size = 4 if c["dtype"] == "f32" else 2
        return {"bytes": n * (17.0 / 32 + size * (2 if c["op"] == "store" else 1)), "flops": n * (3.0 if c["op"] == "store" else 1.0)}
    N, H, d = c["rows"], c["heads"], c["d"]
    lengths = _spread(c["batch"], max(N, c["length"] // 8), c["length"], c["ragged"])
    rows = _spread(c["batch"], max(1, N // 2), N, True) if c["ragged"] and N > 1 else [N] * c["batch"]
    live = sum(lengths) * c["keep"]
    pairs = sum(m * (n - (m - 1) / 2.0) for n, m in zip(lengths, rows)) * c["keep"]
    size = 4 if c["dtype"] == "f32" else 2
    return {"bytes": live * c["kv_heads"] * d * 17.0 / 16 + sum(rows) * H * (2.0 * d * size + 4), "flops": 4.0 * pairs * H * d}


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits

def exact(case, seed):
    """What `run` gives for these inputs, in 64 bits, request by request."""
    s = prepare(case, seed)
    return {"pages": _exact_pages, "store": _exact_store, "load": _exact_load, "attend": _exact_attend}[case["op"]](s)


def _exact_pages(s):
    page, table, free = s["page"], s["table"].tolist(), s["free"].tolist()
    top, length, longer = int(s["n_free"]), s["length"].tolist(), s["longer"].tolist()
    slots = [[-1] * s["slots"].shape[1] for _ in length]
    grown, left = [], top
    for b, (old, new) in enumerate(zip(length, longer)):
        for e in range((old + page - 1) // page, (new + page - 1) // page):
            left -= 1
            table[b][e] = free[left]
            grown.append(left)
        for p in range(old, new):
            slots[b][p - old] = table[b][p // page] * page + p % page
    # the way back puts the pages where they were: the stack is as before, the table keeps its entries
    assert grown == sorted(grown, reverse=True)
    return {"slots": _ints(slots), "table": _ints(table), "length": s["length"], "free": s["free"], "n_free": s["n_free"], "missing": _ints([0])}


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


def _exact_store(s):
    k, v = torch.zeros_like(s["k_out"], dtype=torch.float64), torch.zeros_like(s["v_out"], dtype=torch.float64)
    for b, n in enumerate((s["length"] - s["first"]).tolist()):
        k[b, :n], v[b, :n] = _held_as(s["k_new"][b, :n]), _held_as(s["v_new"][b, :n])
    return {"k": k, "v": v}


def _signed(code):
    return torch.tensor(MAGNITUDES, dtype=torch.float64, device=code.device)[(code & 7).long()] * (1 - 2 * (code >> 3).double())


def _numbers(code_bytes, scale_bytes):
    """[.., d / 2] and [.., d / 32] bytes -> [.., d] in 64 bits"""
    x = torch.stack([_signed(code_bytes & 15), _signed(code_bytes >> 4)], dim=-1).flatten(-2)
    return x * torch.exp2(scale_bytes.double() - 127.0).repeat_interleave(32, dim=-1)


def _request(s, b, n):
    """K and V of a request's first n entries, [n, H, d] each, read out of its pages' bytes."""
    page, d, H = s["page"], s["d"], s["cache"].shape[1]
    raw = s["cache"][s["table"][b, :-(-n // page)].long()]                  # [pages, H, bytes]
    m, c = raw.shape[0], page * d // 2
    part = lambda at, size: raw[:, :, at:at + size]  # noqa: E731
    tokens = lambda t: t.reshape(m, H, page, -1).transpose(1, 2).reshape(m * page, H, -1)[:n]  # noqa: E731
    k = _numbers(tokens(part(0, c)), tokens(part(c, page * d // 32)))
    vc = part(c + page * d // 32, c).reshape(m, H, page // 4, 16, 4, d // 32).permute(0, 1, 2, 4, 3, 5)
    vs = part(2 * c + page * d // 32, page * d // 32).reshape(m, H, page // 4, d // 32, 4).permute(0, 1, 2, 4, 3)
    return k, _numbers(tokens(vc), tokens(vs))


def _exact_load(s):
    out = {n: torch.zeros_like(s[n + "_out"], dtype=torch.float64) for n in "kv"}
    for b, (lo, hi) in enumerate(zip(s["first"].tolist(), s["length"].tolist())):
        k, v = _request(s, b, hi)
        out["k"][b, :hi - lo], out["v"][b, :hi - lo] = k[lo:], v[lo:]
    return out


def _exact_attend(s):
    B, N, H, d = s["q"].shape
    out, lse = torch.zeros((B, N, H, d), dtype=torch.float64, device="cuda"), torch.zeros((B, H, N), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["length"].tolist()):
        rows = N if s["q_len"] is None else int(s["q_len"][b])
        k, v = _request(s, b, n)
        seen = torch.ones((rows, n), dtype=torch.bool, device="cuda").tril(n - rows)
        if s["keep"] is not None:
            seen &= s["keep"][b, :n] != 0
        group = H // k.shape[1]
        for h in range(H):
            x = (s["q"][b, :rows, h].double() @ k[:, h // group].T * s["scale"]).masked_fill(~seen, -math.inf)
            lse[b, h, :rows] = torch.logsumexp(x, dim=-1)
            out[b, :rows, h] = torch.softmax(x, dim=-1) @ v[:, h // group]
    return {"out": out, "lse": lse}
