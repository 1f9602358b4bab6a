"""Rotation, rows rotated into the cache held in 4 bits, bounds, the choice of pages and attention over them, on the GPU against the plain
references (chosen_ref.py, cache4_ref.py): rows, bytes, bounds and choices exactly, attention within bounds that follow from its arithmetic."""
import numpy as np
import pytest

import cache4_ref as ref
import chosen_ref as cr
from test_gpu_cache4 import BF16, F32, dev, host, make_rows, rows_on_gpu, scattered

pytestmark = pytest.mark.gpu


def rounded(x, dtype):
    """float32 as the rows' type holds it, as float64."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32))
    return (t.bfloat16() if dtype == BF16 else t).double().numpy()


def same(got, want):
    return np.array_equal(got, want, equal_nan=True)


# ------------------------------------------------------------------------------------------------ rotation

ROTATIONS = [
    # B, N, Hq, H, d, sections, dtype, layout, adjacent, inverse, what else
    (1, 1, 1, 1, 64, [32], BF16, "tokens", False, False, ""),
    (3, 5, 4, 2, 128, [64], BF16, "tokens", False, False, "rows"),
    (2, 7, 5, 3, 128, [16, 24, 24], F32, "heads", False, True, "index rows"),
    (2, 33, 3, 1, 128, [16, 16], BF16, "heads", True, False, "index"),
    (1, 9, 2, 2, 80, [20, 20], BF16, "tokens", False, False, ""),               # pairs in eights, but rows of five
    (1, 9, 2, 2, 72, [12, 12, 12], F32, "tokens", False, False, ""),             # pairs in fours
    (2, 3, 7, 0, 72, [4, 8], BF16, "heads", True, True, "rows"),                 # no k; channels that stay
    (1, 4, 2, 1, 8, [4], BF16, "tokens", True, False, ""),
    (1, 3, 2, 1, 256, [32, 32, 32, 32], BF16, "tokens", False, False, "index"),
    (1, 3, 2, 1, 256, [64, 0, 12], F32, "heads", True, True, ""),
    (2, 1500, 13, 9, 128, [64], BF16, "heads", False, False, "rows"),            # many rows: four heads to a thread, twenty-two of them
    (1, 5003, 11, 3, 64, [16, 8], F32, "tokens", True, False, "index"),
    (1, 9001, 7, 5, 72, [36], BF16, "tokens", False, True, ""),
    (3, 40, 3, 2, 128, [40, 8], BF16, "tokens", True, False, "rows"),            # neighbours as pairs, that end in a row's second half
    (1, 5003, 11, 3, 128, [24, 16], BF16, "tokens", True, True, "rows index"),
    (1, 4001, 11, 3, 128, [8, 12], F32, "heads", False, False, ""),
    (1, 9001, 7, 5, 96, [24], BF16, "tokens", False, False, "rows"),
]


@pytest.mark.parametrize("place", ["out", "in place"])
@pytest.mark.parametrize("i", range(len(ROTATIONS)))
def test_rotate(i, place):
    import torch
    import paper_2411_10803_amd as md
    B, N, Hq, H, d, sections, dtype, layout, adjacent, inverse, more = ROTATIONS[i]
    rng = np.random.default_rng(100 + i)
    pairs, axes, n_pos = sum(sections), len(sections), 4000
    axis = np.repeat(np.arange(axes), sections)
    rng.shuffle(axis)
    L = 2 * N + 3 if "index" in more else N
    pos = rng.integers(0, n_pos, (axes, B, L)).astype(np.int32)
    index = np.stack([rng.permutation(L)[:N] for _ in range(B)]).astype(np.int32) if "index" in more else None
    rows = rng.integers(0, N + 1, B).astype(np.int32) if "rows" in more else None
    if rows is not None:
        rows[0] = N
    table = cr.angles(n_pos, pairs)
    turn = md.rotary(sections, adjacent=adjacent, axis=axis)
    given = [rows_on_gpu(rng.standard_normal((B, N, h, d)), dtype, layout, pad=2) for h in (Hq, H) if h]
    before = [g[0]._base.clone() if g[0]._base is not None else g[0].clone() for g in given]
    outs = [None, None] if place == "in place" else [rows_on_gpu(np.full(g[1].shape, 7.0), dtype, "tokens" if layout == "heads" else "heads", pad=1)[0] for g in given]
    opt = lambda a: None if a is None else dev(a)  # noqa: E731
    got = md.mustdrop_rotate(given[0][0], dev(pos), dev(table), turn, k=given[1][0] if H else None, q_out=outs[0], k_out=outs[1] if H else None,
                             index=opt(index), rows=opt(rows), inverse=inverse)
    torch.cuda.synchronize()
    for (t, x), y in zip(given, got):
        if place == "in place":
            assert y is t
        for b in range(B):
            n = N if rows is None else rows[b]
            at = pos[:, b] if index is None else pos[:, b][:, index[b]]
            want = rounded(cr.turned(x[b].astype(np.float32), at[:, :N], table, axis, adjacent, inverse), dtype)
            assert same(host(y)[b, :n], want[:n]), (i, b)
            # near the 64-bit value: three roundings of fp32, one of the type
            exact = cr.turned(x[b], at[:, :N], table, axis, adjacent, inverse, np.float64)
            size = np.abs(cr.turned(np.abs(x[b]), at[:, :N], np.abs(table), axis, adjacent, False, np.float64)) + np.abs(x[b]).max()
            assert (np.abs(want - exact) <= 2.0 ** -22 * size + (2.0 ** -8 if dtype == BF16 else 0) * np.abs(exact)).all()
            left = x[b, n:] if place == "in place" else np.full_like(x[b, n:], 7.0)
            assert np.array_equal(host(y)[b, n:], left), "rows behind the last were written"
    if place == "in place":                              # nothing between the rows was written, either
        for (t, x), was in zip(given, before):
            whole = t._base if t._base is not None else t
            assert np.array_equal(np.isnan(host(whole)), np.isnan(host(was)))
    else:
        for (t, _), was in zip(given, before):
            assert same(host(t._base if t._base is not None else t), host(was))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_positions_out_of_the_table_are_nan_there(dtype):
    import paper_2411_10803_amd as md
    rng = np.random.default_rng(3)
    table, axis = cr.angles(10, 16), np.repeat([0, 1], 8)
    pos = np.array([[[0, 3, -1, 9]], [[10, 9, 5, 2 ** 31 - 1]]], np.int32)
    index = np.array([[0, 1, 2, 3, 4, -1, 1]], np.int32)
    x, xh = rows_on_gpu(rng.standard_normal((1, 7, 2, 64)), dtype)
    y, _ = md.mustdrop_rotate(x, dev(pos), dev(table), md.rotary([8, 8]), q_out=rows_on_gpu(xh, dtype)[0], index=dev(index))
    at = np.where((index >= 0) & (index < 4), pos[:, 0][:, np.clip(index[0], 0, 3)], -1)
    want = rounded(cr.turned(xh[0].astype(np.float32), at, table, axis), dtype)
    assert same(host(y)[0], want)
    assert np.isnan(want).any(-1).any(-1).tolist() == [True, False, True, True, True, True, False] and not np.isnan(want[..., 32:]).any()


def test_inverse_is_the_gradient():
    """<g, turned x> = <inverse g, x>, and differences of <g, turned x> over single channels."""
    import torch
    import paper_2411_10803_amd as md
    torch.manual_seed(5)
    x, g = (torch.randn((2, 6, 3, 64), device="cuda") for _ in range(2))
    table = md.rotary_table(500, 24) * 1.25                                       # (a table may carry a factor)
    pos = torch.randint(0, 500, (3, 2, 6), dtype=torch.int32, device="cuda")
    turn = md.rotary([8, 8, 8])
    run = lambda t, inverse=False: md.mustdrop_rotate(t, pos, table, turn, q_out=torch.empty_like(t), inverse=inverse)[0].double()  # noqa: E731
    back = run(g, True)
    size = float(g.double().norm() * x.double().norm()) * 1.25
    assert abs(float((g.double() * run(x)).sum() - (back * x.double()).sum())) <= 2.0 ** -22 * size
    for at in ((0, 0, 0, 0), (1, 5, 2, 30), (0, 3, 1, 47), (1, 2, 0, 60)):
        h = 0.5
        up, down = x.clone(), x.clone()
        up[at] += h
        down[at] -= h
        moved = float(((run(up) - run(down)) * g.double()).sum()) / float(up[at].double() - down[at].double())
        # the two sides differ in the channel's pair alone: a few roundings of numbers of up to 4
        assert abs(moved - float(back[at])) <= 2.0 ** -20 * 16, at


# ------------------------------------------------------------------------------------------------ rows into the cache

@pytest.mark.parametrize("B, N, Hq, H, d, page, sections, dtype, layout, adjacent, index", [
    (1, 1, 1, 1, 128, 16, [64], BF16, "tokens", False, False), (3, 5, 4, 2, 64, 32, [16, 8, 8], F32, "tokens", False, True),
    (2, 17, 3, 3, 128, 64, [16], BF16, "heads", False, False), (2, 9, 5, 1, 64, 16, [8, 0, 8], BF16, "heads", False, True),
    (2, 18, 2, 2, 128, 16, [32, 32], F32, "heads", True, False), (1, 70, 2, 1, 64, 128, [16], BF16, "tokens", True, True),
    (2, 7, 0, 2, 128, 32, [64], BF16, "tokens", False, False), (1, 40, 3, 2, 128, 256, [48], F32, "tokens", False, True)])
@pytest.mark.parametrize("place", ["out", "in place"])
def test_append(B, N, Hq, H, d, page, sections, dtype, layout, adjacent, index, place):
    import torch
    import paper_2411_10803_amd as md
    rng = np.random.default_rng(d + N)
    pairs, axes, n_pos = sum(sections), len(sections), 900
    axis = np.repeat(np.arange(axes), sections)
    rng.shuffle(axis)
    L = N + 4 if index else N
    pos = rng.integers(0, n_pos, (axes, B, L)).astype(np.int32)
    idx = np.stack([np.sort(rng.permutation(L)[:N]) for _ in range(B)]).astype(np.int32) if index else None
    table = cr.angles(n_pos, pairs)
    n_pages = -(-B * N // page) + 3
    slots = rng.permutation(n_pages * page)[:B * N].reshape(B, N).astype(np.int32)
    if N > 4:
        slots[0, 1], slots[0, 3], slots[B - 1, N - 1] = -1, n_pages * page, -(2 ** 31)
    kx, vx = make_rows(rng, B, N, H, d), make_rows(rng, B, N, H, d)
    k, kh = rows_on_gpu(kx, dtype, layout, pad=1)
    v, vh = rows_on_gpu(vx, dtype, layout, pad=1)
    q, qh = rows_on_gpu(rng.standard_normal((B, N, Hq, d)), dtype, layout) if Hq else (None, None)
    out = None if place == "in place" or not Hq else rows_on_gpu(np.full((B, N, Hq, d), 7.0), dtype, "tokens", pad=1)[0]
    pool = np.full((n_pages, H, ref.page_bytes(page, d)), 0x55, np.uint8)
    cache = dev(pool)
    got = md.mustdrop_cache4_append(q, k, v, dev(pos), dev(table), md.rotary(sections, adjacent, axis), dev(slots), cache, q_out=out,
                                    index=None if idx is None else dev(idx))
    torch.cuda.synchronize()
    for b in range(B):
        at = pos[:, b] if idx is None else pos[:, b][:, idx[b]]
        tk = cr.turned(kh[b].astype(np.float32), at[:, :N], table, axis, adjacent)
        on = (slots[b] >= 0) & (slots[b] < n_pages * page)
        for i in np.flatnonzero(on):
            for h in range(H):
                ref.put(pool, slots[b, i], h, tk[i, h], vh[b, i, h], page)
        if Hq:
            tq = rounded(cr.turned(qh[b].astype(np.float32), at[:, :N], table, axis, adjacent), dtype)
            assert same(host(got)[b][on], tq[on])
            assert np.array_equal(host(got)[b][~on], qh[b][~on] if place == "in place" else np.full_like(qh[b][~on], 7.0))
    assert np.array_equal(ref.undefined_codes(host(cache), page, d), ref.undefined_codes(pool, page, d))


@pytest.mark.parametrize("d, dtype, sections, adjacent", [(128, BF16, [64], False), (64, F32, [8, 8], False), (128, F32, [16, 16], True),
                                                        (128, F32, [64], False), (128, F32, [8, 16], False), (128, F32, [40, 8], True)])
def test_many_appended_rows_are_what_few_are(d, dtype, sections, adjacent):
    """Enough rows for two heads to a wave, against the same rows in calls of a few."""
    import torch
    import paper_2411_10803_amd as md
    torch.manual_seed(7)
    B, N, Hq, H, page = 1, 9001, 5, 3, 32
    kind = torch.bfloat16 if dtype == BF16 else torch.float32
    q, k, v = (torch.randn((B, N, h, d), device="cuda").to(kind) for h in (Hq, H, H))
    n_pages = -(-N // page)
    slots = torch.randperm(n_pages * page, device="cuda")[:N].to(torch.int32)[None].contiguous()
    pos = torch.randint(0, 700, (len(sections), B, N), dtype=torch.int32, device="cuda")
    table, turn = md.rotary_table(700, sum(sections)), md.rotary(sections, adjacent)
    caches = [md.cache4_buffer(n_pages, page, H, d) for _ in range(2)]
    whole = md.mustdrop_cache4_append(q, k, v, pos, table, turn, slots, caches[0], q_out=torch.zeros_like(q))
    parts = torch.zeros_like(q)
    for at in range(0, N, 1000):
        s = slice(at, min(at + 1000, N))
        md.mustdrop_cache4_append(q[:, s], k[:, s], v[:, s], pos[:, :, s].contiguous(), table, turn, slots[:, s].contiguous(), caches[1], q_out=parts[:, s])
    torch.cuda.synchronize()
    assert torch.equal(whole, parts) and torch.equal(*caches)


# ------------------------------------------------------------------------------------------------ bounds

def filled_pool(rng, n_pages, H, d, page, spread=0):
    """A pool whose entries are all written: [n_pages, H, bytes], and K, V [n_pages * page, H, d] as float64."""
    pool = np.zeros((n_pages, H, ref.page_bytes(page, d)), np.uint8)
    k, v = rng.standard_normal((2, n_pages * page, H, d))
    if spread:
        k *= np.exp2(rng.integers(-spread, spread + 1, (n_pages * page, H, d // 32, 1)).astype(float)).repeat(32, -1).reshape(k.shape)
    for t in range(n_pages * page):
        for h in range(H):
            ref.put(pool, t, h, k[t, h], v[t, h], page)
    return pool, ref.values(*ref.quantise(k)), ref.values(*ref.quantise(v))


@pytest.mark.parametrize("d, page, H, spread", [(128, 16, 2, 0), (64, 16, 3, 6), (128, 32, 1, 9), (64, 64, 2, 0), (128, 128, 2, 3), (64, 256, 1, 2)])
def test_bounds(d, page, H, spread):
    import torch
    import paper_2411_10803_amd as md
    rng = np.random.default_rng(d + page)
    n_pages, entries = 9, 4
    pool, _, _ = filled_pool(rng, n_pages, H, d, page, spread)
    zero = np.zeros(d)
    for t in range(page):
        for h in range(H):
            ref.put(pool, 8 * page + t, h, zero, zero, page)                     # a page of zeros
    nan = np.ones(d)
    nan[d - 3] = np.nan
    ref.put(pool, 7 * page + page - 1, H - 1, nan, zero, page)                   # a key that is no number, in the last place of page 7
    table = np.array([[3, 0, 8, 7], [5, 2, -1, 1], [4, n_pages, 6, 6], [7, 7, 7, 7]], np.int32)
    cap = entries * page
    for first, length, n in (([0, 0, 0, 0], [cap, 2 * page + 1, page, page - 1], cap), ([page - 1, -5, 2 * page, 0], [page + 1, cap + 7, cap, 1], 2),
                             ([0, 5, cap, 0], [0, -3, cap, page], 1), (None, [1, page + 1, 3 * page - 1, 0], page + 1)):
        b, s = md.cache4_bounds_buffer(n_pages, H, d)
        b.fill_(99)
        s.fill_(77)
        md.mustdrop_cache4_bounds(dev(pool), dev(table), dev(np.array(length, np.int32)), n, b, s, first=None if first is None else dev(np.array(first, np.int32)))
        torch.cuda.synchronize()
        wb, ws = np.full((n_pages, H, 2, d), 99), np.full((n_pages, H), 77)
        live = {}                                        # (a page that two entries name as differently full holds parts of both)
        for x in range(4):
            lo, to = max(0 if first is None else first[x], 0), min(max(length[x], 0), cap)
            for e in range(entries):
                if e * page < min(lo + n, to) and (e + 1) * page > lo and 0 <= table[x, e] < n_pages:
                    wb[table[x, e]], ws[table[x, e]] = cr.bounds(pool, table[x, e], min(page, to - e * page), H, d, page)
                    live.setdefault(int(table[x, e]), set()).add(min(page, to - e * page))
        one = [p for p in range(n_pages) if len(live.get(p, [])) < 2]
        assert len(one) >= 7 and np.array_equal(host(b)[one], wb[one]) and np.array_equal(host(s)[one], ws[one]), (first, length, n)


def test_bounds_of_pages_with_keys_that_are_no_numbers():
    """One such key in any group and head marks that head's page, and only while it is below the length."""
    import torch
    import paper_2411_10803_amd as md
    rng = np.random.default_rng(12)
    d, page, H = 128, 32, 2
    pool, _, _ = filled_pool(rng, 4, H, d, page)
    for id, t, h, c in ((0, 0, 1, 0), (1, 31, 0, 127), (2, 17, 1, 40), (3, 5, 0, 95)):
        bad = np.ones(d)
        bad[c] = np.inf
        ref.put(pool, id * page + t, h, bad, bad, page)
    b, s = md.cache4_bounds_buffer(4, H, d)
    md.mustdrop_cache4_bounds(dev(pool), dev(np.arange(4, dtype=np.int32)[:, None]), dev(np.array([1, 31, 32, 6], np.int32)), 32, b, s)
    torch.cuda.synchronize()
    for id, live in enumerate((1, 31, 32, 6)):
        wb, ws = cr.bounds(pool, id, live, H, d, page)
        assert np.array_equal(host(b)[id], wb) and host(s)[id].tolist() == ws.tolist()
    assert (host(s) == 255).tolist() == [[False, True], [False, False], [False, True], [True, False]]


# ------------------------------------------------------------------------------------------------ the choice

def made_bounds(rng, n_pages, H, d, few=False):
    """Bounds as pages have them; few: of few values, so that many scores are equal."""
    lo = rng.integers(-96, 97, (n_pages, H, d)) if not few else rng.integers(-1, 2, (n_pages, H, d)) * (rng.random((n_pages, H, d)) < 0.02)
    hi = np.maximum(lo, rng.integers(-96, 97, lo.shape)) if not few else np.maximum(lo, 0)
    return np.stack([hi, lo], 2).astype(np.int8), (rng.integers(120, 123, (n_pages, H)) if not few else np.full((n_pages, H), 127)).astype(np.uint8)


CHOICES = [
    # lengths, N, Hq, H, d, page, first, last, budget, dtype, what else
    ([0, 1, 16, 17, 160, 161], 1, 2, 2, 128, 16, 0, 1, 4, BF16, ""),
    ([100, 900, 640], 1, 8, 2, 64, 32, 1, 2, 7, F32, "heads"),
    ([5000, 4000], 1, 3, 3, 128, 16, 0, 0, 64, BF16, "few"),                     # equal scores by the dozen
    ([3000, 2999], 3, 5, 1, 64, 16, 2, 1, 50, BF16, "few heads"),
    ([70, 300, 2], 5, 28, 4, 128, 16, 1, 1, 3, F32, "q_len"),                    # heads that share: 7
    ([1000], 2, 40, 1, 128, 64, 0, 1, 5, BF16, ""),                              # 40 to one: three tiles of them
    ([700, 650], 37, 3, 1, 64, 16, 1, 1, 9, BF16, "q_len heads"),
    ([400], 19, 2, 2, 128, 32, 0, 3, 3, F32, ""),                                # nothing left for scores
    ([9, 0, 4], 7, 2, 1, 64, 16, 1, 1, 4, BF16, ""),                             # rows before the first entry
    ([40000, 39000, 100], 1, 4, 2, 64, 16, 1, 1, 1200, BF16, "few"),             # 2500 pages
    ([33000], 2, 2, 1, 128, 16, 0, 1, 3, F32, "few"),
    ([1 << 30, -5], 1, 1, 1, 64, 16, 0, 1, 2, BF16, ""),                         # lengths out of range
    ([140000, 131], 1, 2, 1, 64, 16, 0, 1, 37, BF16, "few"),                     # 8750 pages
    ([112000, 40000], 2, 2, 1, 64, 16, 1, 1, 300, F32, "few"),                   # 7000
    ([900, 901], 1, 1024, 1, 128, 64, 0, 1, 4, BF16, ""),                        # 1024 heads to one
    # scores and choice in one launch: many tiles of query rows, up to 256, 768 and 2048 pages
    ([300 * (b % 14) + b for b in range(17)], 1, 16, 16, 128, 16, 1, 1, 20, BF16, "few"),
    ([600 * (b % 10) + 17 * b for b in range(18)], 1, 30, 15, 64, 16, 0, 1, 40, F32, ""),
    ([1500 * (b % 12) for b in range(26)], 1, 30, 10, 128, 16, 1, 0, 130, BF16, "few heads"),
    ([3000 + 90 * b for b in range(11)], 23, 12, 2, 64, 64, 1, 1, 8, BF16, "q_len"),
    ([1500 * (b % 12) for b in range(53)], 1, 20, 10, 128, 16, 1, 2, 77, F32, "few"),
]


@pytest.mark.parametrize("i", range(len(CHOICES)))
def test_choose(i):
    import torch
    import paper_2411_10803_amd as md
    lengths, N, Hq, H, d, page, first, last, budget, dtype, more = CHOICES[i]
    rng = np.random.default_rng(200 + i)
    B, G = len(lengths), Hq // H
    entries = max(1, -(-max(n for n in lengths if n < 1 << 29) // page)) if max(lengths) < 1 << 29 else 6
    n_pages = 50
    table = rng.integers(0, n_pages, (B, entries)).astype(np.int32)              # (pages may be named twice)
    table[rng.random(table.shape) < 0.02] = n_pages
    bounds, scales = made_bounds(rng, n_pages, H, d, "few" in more)
    scales[rng.random(scales.shape) < 0.03] = 255
    x = rng.standard_normal((B, N, Hq, d)) * np.exp2(rng.integers(-3, 4, (B, N, Hq, 1)).astype(float))
    q, qh = rows_on_gpu(x, dtype, "heads" if "heads" in more else "tokens", pad=1)
    q_len = rng.integers(-1, N + 2, B).astype(np.int32) if "q_len" in more else None
    if q_len is not None:
        q_len[0] = N
    chosen = torch.full((B, N, H, budget), 99, dtype=torch.int32, device="cuda")
    md.mustdrop_cache4_choose(q, dev(bounds), dev(scales), dev(table), dev(np.array(lengths, np.int32)), page, chosen,
                              q_len=None if q_len is None else dev(q_len), first_pages=first, last_pages=last)
    torch.cuda.synchronize()
    got = host(chosen)
    for b in range(B):
        nq = N if q_len is None else min(max(q_len[b], 0), N)
        assert (got[b, nq:] == 99).all()
        for r in range(nq):
            for h in range(H):
                want = cr.choose(qh[b, r, h * G:(h + 1) * G], bounds[:, h].astype(np.int64), scales[:, h], table[b], lengths[b], nq, r, page, first, last, budget, n_pages)
                assert got[b, r, h].tolist() == want, (b, r, h)


def test_choice_by_queries_that_are_no_numbers_or_nothing():
    """Such queries count as 0: the first pages, by index; one query's does not reach the other heads and tokens."""
    import torch
    import paper_2411_10803_amd as md
    rng = np.random.default_rng(9)
    bounds, scales = made_bounds(rng, 30, 2, 64)
    q = torch.randn((1, 4, 4, 64), device="cuda")
    plain = q.clone()
    q[0, 0, 1, 5], q[0, 1, 0, 63], q[0, 2, 2:] = float("nan"), float("-inf"), 0.0
    q[0, 3, :2] *= 1e-42                                                         # numbers below the normal ones keep their order
    plain[0, 3, :2] = (q[0, 3, :2].double() * 2.0 ** 100).float()
    assert bool(torch.isfinite(plain).all()) and bool((plain[0, 3, 0] != 0).any())
    table, length = dev(np.arange(30, dtype=np.int32)[None]), dev(np.array([480], np.int32))
    a, b = (torch.zeros((1, 4, 2, 5), dtype=torch.int32, device="cuda") for _ in range(2))
    for x, c in ((q, a), (plain, b)):
        md.mustdrop_cache4_choose(x, dev(bounds), dev(scales), table, length, 16, c, last_pages=1)
    torch.cuda.synchronize()
    a, b = host(a)[0], host(b)[0]
    zero = [0, 1, 2, 3, 29]
    assert a[0, 0].tolist() == zero and a[1, 0].tolist() == zero and a[2, 1].tolist() == zero
    assert np.array_equal(a[0, 1], b[0, 1]) and np.array_equal(a[1, 1], b[1, 1]) and np.array_equal(a[2, 0], b[2, 0]) and np.array_equal(a[3], b[3])


@pytest.mark.parametrize("sign", (1.0, -1.0))
def test_the_largest_sums_fit(sign):
    """1024 heads of 128 channels with the largest whole numbers and bounds of all ones or their ends: sums of nearly 2^31."""
    import torch
    import paper_2411_10803_amd as md
    G, d, pages = 1024, 128, 6
    bounds = np.zeros((pages, 1, 2, d), np.int8)
    bounds[:, 0, 0], bounds[:, 0, 1] = 127, -128
    for p in range(pages):                               # one after the other a little less
        bounds[p, 0, 0, :8 * p], bounds[p, 0, 1, :8 * p] = 120, -120
    order = np.array([3, 0, 5, 1, 4, 2])
    scales = np.full((pages, 1), 127, np.uint8)
    q = torch.full((1, 1, G, d), sign * 1.99, device="cuda")
    chosen = torch.zeros((1, 1, 1, 3), dtype=torch.int32, device="cuda")
    md.mustdrop_cache4_choose(q, dev(bounds), dev(scales), dev(order[None].astype(np.int32)), dev(np.array([16 * pages], np.int32)), 16, chosen, last_pages=0)
    torch.cuda.synchronize()
    w = cr.whole(host(q)[0, 0].astype(np.float64))
    assert abs(int(w[0, 0])) == 127 and cr.score(w, bounds[0, 0].astype(np.int64), 127) > 2.0 ** 30.9
    want = cr.choose(host(q)[0, 0].astype(np.float64), bounds[:, 0].astype(np.int64), scales[:, 0], order, 16 * pages, 1, 0, 16, 0, 0, 3, pages)
    assert host(chosen)[0, 0, 0].tolist() == want == [1, 3, 5]


# ------------------------------------------------------------------------------------------------ attention

class Chosen:
    """Inputs of one call over chosen pages, on both sides."""

    def __init__(self, seed, lengths, N, Hq, H, d, page, budget, dtype, q_len=None, keep=None, layout="tokens", size=1.0, kind="sorted", spare=1):
        rng = np.random.default_rng(seed)
        B = len(lengths)
        self.B, self.N, self.Hq, self.H, self.d, self.page, self.budget, self.dtype, self.layout, self.lengths = B, N, Hq, H, d, page, budget, dtype, layout, lengths
        self.entries = max(1, -(-max(lengths) // page)) + spare
        self.table, n_pages = scattered(rng, [max(n, 0) for n in lengths], page, self.entries, fill=2 ** 31 - 1)
        self.pool, k, v = filled_pool(rng, n_pages, H, d, page)
        if size != 1.0:
            for t in range(n_pages * page):
                for h in range(H):
                    ref.put(self.pool, t, h, k[t, h] * size, v[t, h], page)
                    k[t, h] = ref.values(*ref.quantise(k[t, h] * size))
        self.k, self.v = k, v
        self.q, self.qh = rows_on_gpu(rng.standard_normal((B, N, Hq, d)) + 0.3, dtype, layout, pad=1)
        self.q_len = None if q_len is None else np.asarray(q_len, np.int32)
        cap = self.entries * page
        self.keep = None if keep is None else (rng.random((B, cap)) < keep).astype(np.uint8) * rng.integers(1, 256, (B, cap)).astype(np.uint8)
        self.scale = 1.0 / np.sqrt(d)
        lists = np.full((B, N, H, budget), -1, np.int32)
        for b, i, h in np.ndindex(B, N, H):
            if kind == "sorted":
                pick = np.sort(rng.permutation(self.entries)[:budget])
            elif kind == "any":                          # twice, out of order, out of range
                pick = rng.integers(-2, self.entries + 2, budget)
                pick[rng.random(budget) < 0.3] = 2 ** 31 - 1
                pick[rng.random(budget) < 0.1] = -(2 ** 31)
            else:
                pick = np.arange(self.entries)[:budget]
            lists[b, i, h, :len(pick)] = pick
        self.lists = lists

    def args(self):
        return [self.q, dev(self.pool), dev(self.table), dev(np.asarray(self.lengths, np.int32)), dev(self.lists), self.scale]

    def call(self, md, args=None, **kw):
        import torch
        out, _ = rows_on_gpu(np.full((self.B, self.N, self.Hq, self.d), 7.0), self.dtype, self.layout, pad=1)
        lse = torch.full((self.B, self.Hq, self.N), 7.0, device="cuda")
        opt = lambda a: None if a is None else dev(a)  # noqa: E731
        md.mustdrop_cache4_attend_chosen(*(args or self.args()), out=out, lse=lse, q_len=opt(self.q_len), keep=opt(self.keep), **kw)
        torch.cuda.synchronize()
        return host(out).astype(np.float64), host(lse).astype(np.float64)

    def check(self, out, lse):
        # a probability enters the product with V in two bf16 parts, 16 bits, or in three, 24 bits; the output is off by half a step
        step, part = (2.0 ** -8, 2.0 ** -16) if self.dtype == BF16 else (2.0 ** -24, 2.0 ** -23)
        G, cap, page = self.Hq // self.H, self.entries * self.page, self.page
        for b in range(self.B):
            nq = self.N if self.q_len is None else int(np.clip(self.q_len[b], 0, self.N))
            assert (out[b, nq:] == 7).all() and (lse[b, :, nq:] == 7).all(), f"sample {b}: rows behind the last were written"
            ids = self.table[b]
            slot = np.where((ids >= 0) & (ids < len(self.pool)), ids, 0)[:, None] * page + np.arange(page)
            K, V = self.k[slot.reshape(-1)], self.v[slot.reshape(-1)]
            there = np.repeat((ids >= 0) & (ids < len(self.pool)), page)
            for i in range(nq):
                n = cr.seen(self.lengths[b], nq, i, cap)
                for h in range(self.H):
                    on = np.zeros(self.entries, bool)
                    on[cr.listed(self.lists[b, i, h], self.entries)] = True
                    see = there & np.repeat(on, page) & (np.arange(cap) < n)
                    if self.keep is not None:
                        see &= self.keep[b] != 0
                    g = slice(h * G, (h + 1) * G)
                    want, wlse, size, score = ref.attend_heads(self.qh[b, i:i + 1, g], K[:, h:h + 1], V[:, h:h + 1], see, cap, 1, self.scale)
                    bound, lb = ref.attend_bounds(want, wlse, size, score, self.d, see.sum(), step, part)
                    got, gl = out[b, i, g], lse[b, g, i]
                    assert np.array_equal(np.isnan(got), np.isnan(want[0])), (b, i, h, "NaN")
                    off = np.where(np.isnan(got), 0, np.abs(got - want[0]) - bound[0])
                    assert (off <= 0).all(), (b, i, h, off.max())
                    empty = np.isneginf(wlse[0])
                    assert np.array_equal(np.isneginf(gl), empty) and (got[empty] == 0).all(), (b, i, h, "empty rows")
                    assert np.where(empty | np.isnan(wlse[0]), True, np.abs(gl - np.where(empty, 0, wlse[0])) <= lb[0]).all(), (b, i, h, "lse")


ATTENDS = [
    dict(lengths=[0, 1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 100], N=1, Hq=2, H=2, d=128, page=16, budget=3, dtype=BF16),
    dict(lengths=[0, 1, 31, 32, 33, 63, 64, 65, 100, 129], N=1, Hq=2, H=2, d=64, page=32, budget=2, dtype=F32),
    dict(lengths=[130, 77], N=1, Hq=6, H=2, d=128, page=32, budget=1, dtype=BF16),
    dict(lengths=[300, 5], N=1, Hq=20, H=4, d=64, page=64, budget=4, dtype=BF16),
    dict(lengths=[200, 129], N=2, Hq=7, H=1, d=128, page=16, budget=9, dtype=F32),
    dict(lengths=[500], N=1, Hq=40, H=1, d=64, page=256, budget=2, dtype=BF16),                  # three tiles of query heads
    dict(lengths=[90], N=3, Hq=18, H=1, d=128, page=16, budget=5, dtype=F32),
    # drafts and pieces of a prompt; rows that stand before the first entry; samples with fewer rows, none, or out of range
    dict(lengths=[5, 4, 40, 0, 3], N=5, Hq=4, H=2, d=128, page=16, budget=3, dtype=BF16),
    dict(lengths=[90, 60, 17, 31], N=17, Hq=2, H=2, d=64, page=32, budget=2, dtype=BF16, q_len=[17, 3, -4, 99]),
    dict(lengths=[70, 200], N=33, Hq=4, H=2, d=128, page=64, budget=2, dtype=F32, q_len=[33, 20]),
    # masks
    dict(lengths=[100, 50, 333], N=1, Hq=4, H=4, d=128, page=32, budget=5, dtype=BF16, keep=0.5),
    dict(lengths=[100, 50, 333], N=6, Hq=4, H=2, d=64, page=16, budget=7, dtype=F32, keep=0.05),
    dict(lengths=[100, 50], N=4, Hq=4, H=2, d=128, page=16, budget=4, dtype=BF16, keep=0.0),
    # lists out of order, with repeats and entries that are none
    dict(lengths=[300, 150, 20], N=3, Hq=4, H=2, d=128, page=16, budget=12, dtype=BF16, kind="any"),
    dict(lengths=[300, 150, 20], N=1, Hq=2, H=2, d=64, page=32, budget=70, dtype=F32, kind="any", keep=0.6),
    # head-major and padded views; large scores
    dict(lengths=[97, 160], N=9, Hq=8, H=4, d=128, page=32, budget=3, dtype=BF16, layout="heads"),
    dict(lengths=[97, 160], N=2, Hq=4, H=4, d=64, page=32, budget=3, dtype=F32, layout="heads", keep=0.7),
    dict(lengths=[260, 31], N=2, Hq=4, H=2, d=128, page=32, budget=4, dtype=BF16, size=30.0),
    dict(lengths=[260, 31], N=1, Hq=4, H=2, d=128, page=32, budget=4, dtype=F32, size=2000.0),
    # long lists: parts that are joined, few and many of them
    dict(lengths=[3000, 700], N=1, Hq=4, H=2, d=128, page=16, budget=150, dtype=BF16),
    dict(lengths=[3000, 700], N=2, Hq=2, H=1, d=64, page=16, budget=190, dtype=F32, keep=0.8, q_len=[2, 1]),
    dict(lengths=[700], N=1, Hq=18, H=1, d=128, page=16, budget=1500, dtype=F32, kind="any"),
    dict(lengths=[600, 90], N=1, Hq=2, H=2, d=64, page=16, budget=2100, dtype=BF16, kind="all"),
    dict(lengths=[9000, 40], N=1, Hq=20, H=1, d=64, page=16, budget=560, dtype=BF16, keep=0.7),
    dict(lengths=[4500], N=2, Hq=3, H=1, d=128, page=32, budget=140, dtype=F32),
    # several tokens together (1536 tokens and K/V heads and more, eight heads to one at most): 2, 2, 4, 16, 3, 5 and 8 tokens
    dict(lengths=[390, 300], N=391, Hq=16, H=2, d=64, page=16, budget=6, dtype=BF16, keep=0.8),
    dict(lengths=[400, 250], N=400, Hq=14, H=2, d=128, page=32, budget=3, dtype=F32, q_len=[399, 250]),
    dict(lengths=[230, 150], N=200, Hq=16, H=4, d=128, page=16, budget=4, dtype=BF16, q_len=[200, 133]),
    dict(lengths=[120, 70], N=65, Hq=13, H=13, d=64, page=32, budget=2, dtype=BF16, keep=0.5),
    dict(lengths=[300, 200], N=261, Hq=15, H=3, d=64, page=64, budget=3, dtype=F32, kind="any", layout="heads"),
    dict(lengths=[100, 391], N=390, Hq=6, H=2, d=128, page=16, budget=9, dtype=F32, keep=0.7, q_len=[-1, 390]),
    dict(lengths=[66, 5, 33, 0], N=100, Hq=8, H=4, d=64, page=16, budget=2, dtype=BF16, kind="any", layout="heads"),     # rows before the first entry
    dict(lengths=[3, 2], N=800, Hq=1, H=1, d=128, page=256, budget=1, dtype=F32),
    dict(lengths=[97], N=97, Hq=16, H=16, d=128, page=16, budget=7, dtype=BF16, kind="all"),
]


@pytest.mark.parametrize("i", range(len(ATTENDS)))
def test_attend_chosen(i):
    import paper_2411_10803_amd as md
    c = Chosen(300 + i, **ATTENDS[i])
    c.check(*c.call(md))


def test_attend_chosen_over_lengths_out_of_range_and_bad_pages():
    import paper_2411_10803_amd as md
    c = Chosen(41, [100, 90, 80], 2, 4, 2, 128, 16, 5, BF16)
    c.table[1, 2], c.table[2, :] = -7, 2 ** 31 - 1
    c.lengths = [10 ** 9, 90, 80]
    c.check(*c.call(md))
    c.lengths = [-1, 90, 80]
    c.check(*c.call(md))


@pytest.mark.parametrize("dtype, d", ((BF16, 128), (F32, 64)))
def test_attend_chosen_nan_reaches_only_the_rows_that_see_it(dtype, d):
    import paper_2411_10803_amd as md
    c = Chosen(43, [75, 75, 75], 6, 4, 2, d, 16, 4, dtype, keep=1.0)
    bad = np.full(d, 1.0)
    bad[33] = np.nan
    one = np.full(d, 1.0)
    for b, t, h, k, v in ((0, 72, 0, one, bad), (1, 20, 1, bad, one), (2, 10, 0, bad, bad), (2, 40, 1, one, bad)):
        slot = c.table[b, t // 16] * 16 + t % 16
        ref.put(c.pool, slot, h, k, v, 16)
        c.k[slot, h], c.v[slot, h] = ref.values(*ref.quantise(k)), ref.values(*ref.quantise(v))
    c.keep[2, 10] = 0                                    # masked: may hold anything
    out, lse = c.call(md)
    assert np.isnan(out).any() and not np.isnan(out).all()
    c.check(out, lse)


@pytest.mark.parametrize("masked", (True, False))
@pytest.mark.parametrize("dtype, d", ((BF16, 64), (F32, 128)))
def test_nan_reaches_only_the_tokens_that_have_chosen_its_page(dtype, d, masked):
    """Tokens that go together: a V or K that is no number counts for the tokens whose lists name its page and which see it."""
    import paper_2411_10803_amd as md
    c = Chosen(45, [400, 400], 97, 8, 8, d, 16, 6, dtype, keep=0.9 if masked else None)      # sixteen tokens together
    bad = np.full(d, 1.0)
    bad[40] = np.nan
    one = np.full(d, 1.0)
    for b, t, h, k, v in ((0, 350, 0, one, bad), (0, 12, 1, bad, one), (1, 100, 2, bad, bad), (1, 399, 3, one, bad), (1, 64, 4, one, bad)):
        slot = c.table[b, t // 16] * 16 + t % 16
        ref.put(c.pool, slot, h, k, v, 16)
        c.k[slot, h], c.v[slot, h] = ref.values(*ref.quantise(k)), ref.values(*ref.quantise(v))
        if masked:
            c.keep[b, t] = 1
    if masked:
        c.keep[1, 64] = 0
    out, lse = c.call(md)
    assert np.isnan(out).any() and not np.isnan(out).all()
    c.check(out, lse)


@pytest.mark.parametrize("N, H, dtype, d", ((1, 3, BF16, 128), (1, 3, F32, 64), (110, 8, BF16, 128), (110, 8, F32, 64)))
def test_places_that_nobody_sees_may_hold_anything(N, H, dtype, d):
    """Entries that are masked and those behind the length hold any bytes, scales beyond every finite number among them; so do pages that are
    not chosen."""
    import paper_2411_10803_amd as md
    page, lengths = 16, [150, 131]
    c = Chosen(49, lengths, N, 2 * H, H, d, page, 5, dtype, keep=0.6)
    rng = np.random.default_rng(50)
    for b, n in enumerate(lengths):
        used = np.zeros(c.entries, bool)
        for i, h in np.ndindex(N, H):
            used[cr.listed(c.lists[b, i, h], c.entries)] = True
        for t in range(-(-n // page) * page):
            if t < n and c.keep[b, t] and used[t // page]:
                continue
            at, p = c.table[b, t // page], t % page
            for h in range(H):
                x = c.pool[at, h]
                any_bytes = lambda m: rng.choice(np.array([0, 1, 127, 128, 252, 253, 254, 255], np.uint8), m)  # noqa: E731
                x[p * d // 2:(p + 1) * d // 2] = rng.integers(0, 256, d // 2)
                o = page * d // 2
                x[o + p * d // 32:o + (p + 1) * d // 32] = any_bytes(d // 32)
                o += page * d // 32
                for part in range(16):
                    a = o + ((p // 4) * 16 + part) * (d // 8) + (p % 4) * (d // 32)
                    x[a:a + d // 32] = rng.integers(0, 256, d // 32)
                o += page * d // 2
                for g in range(d // 32):
                    x[o + (p // 4) * (d // 8) + g * 4 + p % 4] = any_bytes(1)[0]
    out, lse = c.call(md)
    assert not np.isnan(out).any()
    c.check(out, lse)


def test_tokens_together_are_tokens_apart():
    """A call whose tokens go together against calls of one token each."""
    import torch
    import paper_2411_10803_amd as md
    c = Chosen(46, [500, 333], 100, 16, 8, 128, 32, 5, BF16, keep=0.8)
    a = c.args()
    keep = dev(c.keep)
    out, lse = torch.zeros((2, 100, 16, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 16, 100), device="cuda")
    md.mustdrop_cache4_attend_chosen(*a, out=out, lse=lse, keep=keep)
    for i in range(0, 100, 9):
        o, l = torch.zeros((2, 1, 16, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 16, 1), device="cuda")
        md.mustdrop_cache4_attend_chosen(a[0][:, i:i + 1], a[1], a[2], a[3] - (99 - i), a[4][:, i:i + 1].contiguous(), a[5], out=o, lse=l, keep=keep)
        torch.cuda.synchronize()
        x, y = host(out[:, i:i + 1]), host(o)
        assert (np.abs(x - y) <= 2.0 ** -7 * np.abs(y) + 2.0 ** -14).all() and np.allclose(host(lse[:, :, i:i + 1]), host(l), atol=1e-5)


def test_attend_chosen_in_a_pool_beyond_four_gigabytes():
    """Pages, bounds and the choice behind 2^32 bytes."""
    import torch
    import paper_2411_10803_amd as md
    c = Chosen(47, [70, 40], 2, 8, 8, 128, 32, 2, BF16)
    n_pages, H = 131072, 8
    far = n_pages - len(c.pool)
    cache = torch.empty((n_pages, H, ref.page_bytes(32, 128)), dtype=torch.uint8, device="cuda")
    cache[far:] = dev(c.pool)
    valid = (c.table >= 0) & (c.table < len(c.pool))
    table = np.where(valid, c.table + far, c.table).astype(np.int32)
    args = [c.q, cache, dev(table), dev(np.array([70, 40], np.int32)), dev(c.lists), c.scale]
    c.check(*c.call(md, args))
    bounds, scales = torch.zeros((n_pages, H, 2, 128), dtype=torch.int8, device="cuda"), torch.zeros((n_pages, H), dtype=torch.uint8, device="cuda")
    md.mustdrop_cache4_bounds(cache, args[2], args[3], 100, bounds, scales)
    small = md.cache4_bounds_buffer(len(c.pool), H, 128)
    md.mustdrop_cache4_bounds(dev(c.pool), dev(c.table), args[3], 100, *small)
    assert torch.equal(bounds[far:], small[0]) and torch.equal(scales[far:], small[1])
    picks = [torch.zeros((2, 2, 8, 2), dtype=torch.int32, device="cuda") for _ in range(2)]
    md.mustdrop_cache4_choose(c.q, bounds, scales, args[2], args[3], 32, picks[0])
    md.mustdrop_cache4_choose(c.q, *small, dev(c.table), args[3], 32, picks[1])
    torch.cuda.synchronize()
    assert torch.equal(*picks)
    # rows into the last pages
    k, q = (torch.randn((1, 3, h, 128), device="cuda").bfloat16() for h in (H, 2))
    at, table, turn = torch.tensor([[[5, 600, 31]]], dtype=torch.int32, device="cuda"), md.rotary_table(700, 64), md.rotary([64])
    slots = torch.arange(n_pages * 32 - 3, n_pages * 32, dtype=torch.int32, device="cuda")[None].contiguous()
    qo = md.mustdrop_cache4_append(q, k, k, at, table, turn, slots, cache, q_out=torch.zeros_like(q))
    want, kt = md.mustdrop_rotate(q, at, table, turn, k=k.clone(), q_out=torch.zeros_like(q))
    ko, vo = torch.zeros_like(k), torch.zeros_like(k)
    md.mustdrop_cache4_read(cache, dev(np.array([[n_pages - 1]], np.int32)), dev(np.array([32], np.int32)), ko, vo, first=dev(np.array([29], np.int32)))
    torch.cuda.synchronize()
    tk = cr.turned(host(k)[0].astype(np.float32), host(at)[:, 0], host(table), np.zeros(64, np.int64))
    assert torch.equal(qo, want) and same(host(kt)[0], rounded(tk, BF16))
    assert same(host(ko)[0], ref.values(*ref.quantise(tk))) and same(host(vo)[0], ref.values(*ref.quantise(host(k)[0])))


def test_all_pages_chosen_is_the_attention_over_all():
    import torch
    import paper_2411_10803_amd as md
    c = Chosen(53, [333, 64, 200], 3, 8, 2, 128, 32, 12, BF16, kind="all", keep=0.7)
    out, lse = c.call(md)
    dense = torch.zeros((3, 8, 3), device="cuda")
    want = md.mustdrop_cache4_attend(*c.args()[:4], c.scale, lse=dense, keep=dev(c.keep))
    torch.cuda.synchronize()
    # both within half a step of bf16 of one value, and a few units of fp32
    assert (np.abs(out - host(want)) <= 2.0 ** -7 * np.abs(out) + 2.0 ** -14 * np.abs(host(want)).max()).all()
    assert (np.abs(lse - host(dense)) <= 1e-5).all()


# ------------------------------------------------------------------------------------------------ used together

def decode_program(md, torch, B, H, Hq, d, page, entries, N, budget):
    """What a serving loop keeps, and its step: pages, rows turned into the cache, their pages' bounds, the choice and the attention."""
    s = {"cache": md.cache4_buffer(B * entries, page, H, d), "table": torch.full((B, entries), -1, dtype=torch.int32, device="cuda"),
         "length": torch.zeros(B, dtype=torch.int32, device="cuda"), "new_len": torch.zeros(B, dtype=torch.int32, device="cuda"),
         "before": torch.zeros(B, dtype=torch.int32, device="cuda"), "free": torch.arange(B * entries, dtype=torch.int32, device="cuda"),
         "n_free": dev(np.array([B * entries], np.int32)), "missing": torch.zeros(1, dtype=torch.int32, device="cuda"),
         "slots": torch.zeros((B, N), dtype=torch.int32, device="cuda"), "chosen": torch.zeros((B, N, H, budget), dtype=torch.int32, device="cuda"),
         "q": torch.zeros((B, N, Hq, d), dtype=torch.bfloat16, device="cuda"), "out": torch.zeros((B, N, Hq, d), dtype=torch.bfloat16, device="cuda"),
         "lse": torch.zeros((B, Hq, N), device="cuda"), "pos": torch.zeros((1, B, N), dtype=torch.int32, device="cuda")}
    s["bounds"], s["scales"] = md.cache4_bounds_buffer(B * entries, H, d)
    keep = {"turn": md.rotary([d // 2]), "angles": md.rotary_table(entries * page, d // 2), "pages": md.cache4_pages_workspace(B),
            "choose": md.cache4_choose_workspace(s["q"], s["bounds"], s["table"]), "attend": md.cache4_attend_chosen_workspace(s["q"], s["cache"], s["chosen"]),
            "rows": torch.arange(N, dtype=torch.int32, device="cuda")}

    def step(k, v, q, grow, stream=None):
        s["before"].copy_(s["length"])
        torch.add(s["length"], grow, out=s["new_len"])
        torch.add(s["length"][None, :, None], keep["rows"], out=s["pos"])
        md.mustdrop_cache4_pages(s["new_len"], s["length"], s["table"], s["free"], s["n_free"], s["missing"], page, slots=s["slots"],
                                 workspace=keep["pages"], stream=stream)
        md.mustdrop_cache4_append(q, k, v, s["pos"], keep["angles"], keep["turn"], s["slots"], s["cache"], q_out=s["q"], stream=stream)
        md.mustdrop_cache4_bounds(s["cache"], s["table"], s["length"], N, s["bounds"], s["scales"], first=s["before"], stream=stream)
        md.mustdrop_cache4_choose(s["q"], s["bounds"], s["scales"], s["table"], s["length"], page, s["chosen"], first_pages=1, last_pages=1,
                                  workspace=keep["choose"], stream=stream)
        md.mustdrop_cache4_attend_chosen(s["q"], s["cache"], s["table"], s["length"], s["chosen"], 1.0 / np.sqrt(d), out=s["out"], lse=s["lse"],
                                         workspace=keep["attend"], stream=stream)
    return s, step


def test_steps_against_the_plain_computation():
    """A prompt, then single tokens, through all five operators: each step's choice and attention as the references give them."""
    import torch
    import paper_2411_10803_amd as md
    B, H, Hq, d, page, entries, budget = 2, 2, 4, 64, 16, 12, 4
    torch.manual_seed(11)
    keys, vals = [[] for _ in range(B)], [[] for _ in range(B)]
    table = cr.angles(entries * page, d // 2)
    axis = np.zeros(d // 2, np.int64)
    kept = None
    for n in [90, 1, 1, 3, 1]:
        s, step = decode_program(md, torch, B, H, Hq, d, page, entries, n, budget)
        if kept is not None:                             # another number of rows: the same cache
            for name in ("cache", "table", "length", "free", "n_free", "bounds", "scales"):
                s[name].copy_(kept[name])
        q, k, v = (torch.randn((B, n, h, d), device="cuda").bfloat16() for h in (Hq, H, H))
        step(k, v, q, n)
        torch.cuda.synchronize()
        kept = s
        for b in range(B):
            at = np.arange(len(keys[b]), len(keys[b]) + n)[None]
            tk = cr.turned(host(k)[b], at, table, axis)
            tq = rounded(cr.turned(host(q)[b], at, table, axis), BF16)
            assert np.array_equal(host(s["q"])[b], tq)
            keys[b] += list(ref.values(*ref.quantise(tk)))
            vals[b] += list(ref.values(*ref.quantise(host(v)[b])))
            K, V, total = np.stack(keys[b]), np.stack(vals[b]), len(keys[b])
            pages = -(-total // page)
            row, pool = host(s["table"])[b], host(s["cache"])
            wb, ws = zip(*[cr.bounds(pool, row[e], min(page, total - e * page), H, d, page) for e in range(pages)])
            wb, ws = np.stack(wb), np.stack(ws)
            for i in range(n):
                for h in range(H):
                    g = slice(2 * h, 2 * h + 2)
                    want = cr.choose(tq[i, g], wb[:, h], ws[:, h], np.arange(entries), total, n, i, page, 1, 1, budget, pages)
                    assert host(s["chosen"])[b, i, h].tolist() == want, (n, b, i, h)
                    see = np.isin(np.arange(total) // page, want) & (np.arange(total) <= total - n + i)
                    o, l, size, score = ref.attend_heads(tq[i:i + 1, g], K[:, h:h + 1], V[:, h:h + 1], see, total, 1, 1 / np.sqrt(d))
                    bound, lb = ref.attend_bounds(o, l, size, score, d, total, 2.0 ** -8, 2.0 ** -16)
                    assert (np.abs(host(s["out"])[b, i, g] - o[0]) <= bound[0]).all()
                    assert (np.abs(host(s["lse"])[b, g, i] - l[0]) <= lb[0]).all()


NAMES = ("cache", "table", "length", "free", "n_free", "slots", "bounds", "scales", "chosen", "q", "out", "lse")


@pytest.mark.parametrize("entries, budget", [(8, 3), (150, 100)])
def test_steps_in_a_graph(entries, budget):
    """All calls of a step in one graph, replayed with eager steps of a second program between; both agree bit for bit."""
    import torch
    import paper_2411_10803_amd as md
    B, H, Hq, d, page = 5, 2, 8, 128, 16
    made = [decode_program(md, torch, B, H, Hq, d, page, entries, 1, budget) for _ in range(2)]
    k, v = (torch.zeros((B, 1, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((B, 1, Hq, d), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)

    def fresh():
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    for s, step in made:
        g.manual_seed(3)
        fresh()
        step(k, v, q, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made[0][1](k, v, q, 1)
    for n in range(100):
        fresh()
        torch.cuda.synchronize()
        graph.replay()
        made[1][1](k, v, q, 1)
        torch.cuda.synchronize()
        for name in NAMES:
            assert torch.equal(made[0][0][name], made[1][0][name]), (n, name)
    assert host(made[0][0]["length"]).tolist() == [101] * B


def test_two_graphs_with_one_workspace():
    """What a call leaves in its workspace is nobody's: two graphs that take turns on one give what eager calls give, replay after replay."""
    import torch
    import paper_2411_10803_amd as md
    cases = [Chosen(61, [2000, 900], 1, 4, 2, 128, 16, 120, BF16), Chosen(62, [70, 1500], 2, 4, 2, 128, 16, 90, BF16)]
    args = [c.args() for c in cases]
    lists = []
    for c, a in zip(cases, args):
        b, s = md.cache4_bounds_buffer(len(c.pool), c.H, c.d)
        md.mustdrop_cache4_bounds(a[1], a[2], a[3], 4000, b, s)
        lists.append((a[0], b, s, a[2], a[3], c.page, torch.zeros_like(a[4])))
    sizes = [md.cache4_attend_chosen_workspace(a[0], a[1], a[4]).numel() for a in args] + [md.cache4_choose_workspace(x[0], x[1], x[3]).numel() for x in lists]
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    want = []
    for a, x in zip(args, lists):
        picked = md.mustdrop_cache4_choose(*x).clone()
        want.append((picked, md.mustdrop_cache4_attend_chosen(*a[:4], picked, a[5])))
    out = [torch.zeros_like(w[1]) for w in want]

    def both(i):
        md.mustdrop_cache4_choose(*lists[i], workspace=ws)
        md.mustdrop_cache4_attend_chosen(*args[i][:4], lists[i][6], args[i][5], out=out[i], workspace=ws)
    graphs = []
    for i in range(2):
        both(i)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            both(i)
    for n in range(5):
        for i in range(2):
            out[i].fill_(9)
            lists[i][6].fill_(9)
        ws.fill_(255)
        graphs[n % 2].replay()
        graphs[1 - n % 2].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(lists[i][6], want[i][0]) and torch.equal(out[i], want[i][1]), n


def test_two_programs_on_two_streams():
    """Two batches in flight at once, each with its own state and workspaces, give what each gives alone; one by a given stream."""
    import torch
    import paper_2411_10803_amd as md
    B, H, Hq, d, page, entries, n = 3, 4, 4, 64, 32, 30, 150
    streams = [torch.cuda.Stream() for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(5)
    inputs = [[tuple(torch.randn((B, n, h, d), generator=g, device="cuda").bfloat16() for h in (H, H, Hq)) for _ in range(3)] for _ in range(2)]
    results = []
    for together in (False, True):
        made = [decode_program(md, torch, B, H, Hq, d, page, entries, n, 4) for _ in range(2)]
        torch.cuda.synchronize()
        for i in range(3):
            for p in range(2):
                k, v, q = inputs[p][i]
                with torch.cuda.stream(streams[p]):
                    made[p][1](k, v, q, n, stream=streams[p] if p else None)
                if not together:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        results.append([{x: s[x].clone() for x in NAMES} for s, _ in made])
    for a, b in zip(*results):
        for x in NAMES:
            assert torch.equal(a[x], b[x]), x


def test_what_a_call_makes_belongs_to_its_stream():
    """Workspaces and `out` that calls on a given stream make: the current stream may not get that memory while they run."""
    import torch
    import paper_2411_10803_amd as md
    c = Chosen(71, [3000, 1700], 1, 4, 2, 128, 16, 180, BF16, kind="sorted")
    a = c.args()
    want = md.mustdrop_cache4_attend_chosen(*a)
    b, s = md.cache4_bounds_buffer(len(c.pool), c.H, c.d)
    md.mustdrop_cache4_bounds(a[1], a[2], a[3], 4000, b, s)
    pick = [torch.zeros((2, 1, 2, 9), dtype=torch.int32, device="cuda") for _ in range(2)]
    md.mustdrop_cache4_choose(a[0], b, s, a[2], a[3], 16, pick[0])
    size = max(md.cache4_attend_chosen_workspace(a[0], a[1], a[4]).numel(), md.cache4_choose_workspace(a[0], b, a[2]).numel())
    stream = torch.cuda.Stream()
    busy = torch.ones(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(8):
            busy @ busy
    out = md.mustdrop_cache4_attend_chosen(*a, stream=stream)
    md.mustdrop_cache4_choose(a[0], b, s, a[2], a[3], 16, pick[1], stream=stream)
    over = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)] + [torch.full_like(want, 9) for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(*pick) and len(over) == 8


def test_the_kept_rows_of_a_prompt_at_their_own_positions():
    """The prefill stage's kept index says where its rows stood: rotation by it is what rotation before the filter gives."""
    import torch
    import paper_2411_10803_amd as md
    import workloads as wl
    from paper_2411_10803_amd import harness
    cfg = wl.tiny(wl.CONFIGS[2], B=3, H=4)
    t = wl.prefill_inputs(cfg)
    R, Mv, N, H, d, B = 40, cfg.M, cfg.N, cfg.H, cfg.d, 3
    pre = md.mustdrop_prefill_filter(harness.to_dev(t["q_txt"], True), harness.to_dev(t["k"], True), harness.to_dev(t["v"], True),
                                     harness.to_dev(t["hidden"], True), None, None, None, Mv, 1 / np.sqrt(d), md.FILTER_BUDGET, R, 1.0 / Mv, 2.0 / (Mv + N), Rcap=R)
    torch.cuda.synchronize()
    ids, length = host(pre["out_ids"]), host(pre["out_len"])
    L = int(ids.max()) + 1
    j = np.arange(L)
    pos = np.stack([np.broadcast_to(j // 16, (B, L)), np.broadcast_to(j % 16, (B, L))]).astype(np.int32)
    table, turn = cr.angles(L, 32), md.rotary([16, 16])
    k = pre["k_out"]
    y, _ = md.mustdrop_rotate(k, dev(pos), dev(table), turn, q_out=torch.zeros_like(k), index=dev(ids[:, :k.shape[1]]), rows=dev(length))
    torch.cuda.synchronize()
    for b in range(B):
        n = int(length[b])
        want = rounded(cr.turned(host(k)[b, :n], pos[:, b][:, ids[b, :n]], table, np.repeat([0, 1], 16)), BF16)
        assert np.array_equal(host(y)[b, :n], want) and (host(y)[b, n:] == 0).all()


def test_nothing_is_written_beside_outputs_and_workspaces():
    """Every output, the cache and workspaces of the size that is asked for, between bands of memory that stay as they were."""
    import torch
    import paper_2411_10803_amd as md
    bands = []

    def between(shape, dtype):
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        whole = torch.full((n + 16384,), 0xA5, dtype=torch.uint8, device="cuda")
        bands.append((whole, n))
        return whole[8192:8192 + n].view(dtype).view(shape)

    def untouched():
        torch.cuda.synchronize()
        return all(bool((w[:8192] == 0xA5).all()) and bool((w[8192 + n:] == 0xA5).all()) for w, n in bands)
    torch.manual_seed(21)
    rng = np.random.default_rng(22)
    for B, N, Hq, H, d, page, entries, budget in ((3, 5, 6, 2, 64, 16, 21, 4), (2, 1, 8, 8, 128, 32, 9, 9), (1, 1, 18, 1, 128, 16, 3000, 1500),
                                                  (2, 130, 8, 8, 64, 16, 40, 3), (1, 2, 4, 4, 128, 16, 330, 200), (1, 7, 40, 1, 64, 16, 700, 5)):
        n_pages = entries + 2
        length = dev(np.array([entries * page - 3 * b for b in range(B)], np.int32))
        table = dev(np.stack([rng.permutation(n_pages)[:entries] for _ in range(B)]).astype(np.int32))
        cache = between((n_pages, H, ref.page_bytes(page, d)), torch.uint8)
        cache.zero_()
        q, k = (torch.randn((B, N, h, d), device="cuda").bfloat16() for h in (Hq, H))
        at = torch.randint(0, 99, (1, B, N), dtype=torch.int32, device="cuda")
        angles, turn = md.rotary_table(99, d // 2), md.rotary([d // 2])
        slots = dev(np.concatenate([rng.permutation(n_pages * page)[:B * N - 1], [n_pages * page - 1]]).reshape(B, N).astype(np.int32))
        qo, ko = between(q.shape, torch.bfloat16), between(k.shape, torch.bfloat16)
        md.mustdrop_rotate(q, at, angles, turn, k=k, q_out=qo, k_out=ko)
        md.mustdrop_cache4_append(q, k, k, at, angles, turn, slots, cache, q_out=qo)
        bounds, scales = between((n_pages, H, 2, d), torch.int8), between((n_pages, H), torch.uint8)
        md.mustdrop_cache4_bounds(cache, table, length, entries * page, bounds, scales)
        chosen = between((B, N, H, budget), torch.int32)
        lib = md.library()
        ws = between((lib.mustdrop_cache4_choose_workspace_bytes(B, N, Hq, H, d, entries, page),), torch.uint8)
        md.mustdrop_cache4_choose(qo, bounds, scales, table, length, page, chosen, workspace=ws)
        ws = between((lib.mustdrop_cache4_attend_chosen_workspace_bytes(B, N, Hq, H, d, budget, page),), torch.uint8)
        out, lse = between(q.shape, torch.bfloat16), between((B, Hq, N), torch.float32)
        md.mustdrop_cache4_attend_chosen(qo, cache, table, length, chosen, 0.1, out=out, lse=lse, workspace=ws)
        assert untouched(), (B, N, Hq, H, d)
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
        bands.clear()
