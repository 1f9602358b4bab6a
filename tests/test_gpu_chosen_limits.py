"""Calls at the ends of what the rotation, the bounds, the choice and the attention over chosen pages take: views of one projection, samples
without new entries, millions of lists and of pages, lists and tables as long as a block holds."""
import numpy as np
import pytest

import cache4_ref as ref
import chosen_ref as cr
from test_gpu_cache4 import BF16, F32, dev, host
from test_gpu_chosen import Chosen

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ views of one projection

def projection(torch, B, N, heads, d, dtype, layout):
    """What one product gives, and its views [B, N, h, d] for each of `heads`; two heads between the last one and the next row."""
    kind = torch.bfloat16 if dtype == BF16 else torch.float32
    total = sum(heads) + 2
    shape = {"tokens": (B, N, total, d), "heads": (B, total, N, d), "samples last": (N, B, total, d)}[layout]
    whole = torch.randn(shape, device="cuda").to(kind)
    view = {"tokens": lambda t: t, "heads": lambda t: t.transpose(1, 2), "samples last": lambda t: t.transpose(0, 1)}[layout](whole)
    return whole, list(view.split([*heads, 2], dim=2))[:-1]


FUSED = [
    # B, N, Hq, H, d, sections, dtype, layout, adjacent
    (2, 3, 8, 4, 128, [64], BF16, "tokens", False),
    (3, 7, 4, 4, 64, [16, 8], F32, "tokens", True),
    (2, 5, 6, 2, 128, [32, 16], BF16, "heads", False),
    (2, 9, 3, 1, 64, [32], F32, "heads", False),
    (3, 4, 5, 1, 128, [24, 24], BF16, "samples last", True),
    (1, 40, 4, 2, 128, [64], F32, "tokens", False),
    (40, 1, 4, 2, 64, [16], BF16, "tokens", False),
    (2, 2600, 13, 3, 128, [64], BF16, "tokens", False),      # several heads to a thread
    (2, 1300, 12, 4, 128, [40], F32, "tokens", False),
]


@pytest.mark.parametrize("i", range(len(FUSED)))
def test_rotation_in_place_of_views_of_one_projection(i):
    import torch
    import paper_2411_10803_amd as md
    torch.manual_seed(i)
    B, N, Hq, H, d, sections, dtype, layout, adjacent = FUSED[i]
    whole, (q, k, v) = projection(torch, B, N, (Hq, H, H), d, dtype, layout)
    table, turn = md.rotary_table(500, sum(sections)), md.rotary(sections, adjacent)
    pos = torch.randint(0, 500, (len(sections), B, N), dtype=torch.int32, device="cuda")
    before, copies = whole.clone(), [t.contiguous().clone() for t in (q, k)]
    want = md.mustdrop_rotate(copies[0], pos, table, turn, k=copies[1], q_out=torch.zeros_like(copies[0]), k_out=torch.zeros_like(copies[1]))
    got = md.mustdrop_rotate(q, pos, table, turn, k=k)
    torch.cuda.synchronize()
    assert got[0] is q and got[1] is k and torch.equal(q, want[0]) and torch.equal(k, want[1])
    q.copy_(copies[0])
    k.copy_(copies[1])
    assert torch.equal(whole, before), "something beside the queries and keys was written"
    # out into another view of the same memory that shares no byte with any
    if Hq == H and not layout == "samples last":
        md.mustdrop_rotate(q, pos, table, turn, q_out=v)
        torch.cuda.synchronize()
        assert torch.equal(v, want[0]) and torch.equal(q, copies[0]) and torch.equal(k, copies[1])


@pytest.mark.parametrize("i", range(len(FUSED)))
def test_append_of_views_of_one_projection(i):
    import torch
    import paper_2411_10803_amd as md
    torch.manual_seed(50 + i)
    B, N, Hq, H, d, sections, dtype, layout, adjacent = FUSED[i]
    page = 16
    whole, (q, k, v) = projection(torch, B, N, (Hq, H, H), d, dtype, layout)
    table, turn = md.rotary_table(500, sum(sections)), md.rotary(sections, adjacent)
    pos = torch.randint(0, 500, (len(sections), B, N), dtype=torch.int32, device="cuda")
    n_pages = -(-B * N // page) + 1
    slots = torch.randperm(n_pages * page, device="cuda")[:B * N].to(torch.int32).reshape(B, N).contiguous()
    caches = [md.cache4_buffer(n_pages, page, H, d) for _ in range(2)]
    before, copies = whole.clone(), [t.contiguous().clone() for t in (q, k, v)]
    want = md.mustdrop_cache4_append(*copies, pos, table, turn, slots, caches[0], q_out=torch.zeros_like(copies[0]))
    got = md.mustdrop_cache4_append(q, k, v, pos, table, turn, slots, caches[1])
    torch.cuda.synchronize()
    assert got is q and torch.equal(q, want) and torch.equal(*caches)
    q.copy_(copies[0])
    assert torch.equal(whole, before), "something beside the queries was written"


def test_views_that_share_bytes_are_refused():
    import torch
    import paper_2411_10803_amd as md
    whole = torch.randn((2, 6, 10, 64), device="cuda").bfloat16()
    table, turn = md.rotary_table(9, 32), md.rotary([32])
    pos = torch.zeros((1, 2, 6), dtype=torch.int32, device="cuda")
    before = whole.clone()
    q = whole[:, :, :4]
    for other in (dict(q_out=whole[:, :, 1:5]), dict(q_out=whole[:, :, 3:7]), dict(k=whole[:, :, 2:5]), dict(k=whole[:, :, 3:4]),
                  dict(q_out=whole[:, :, 4:8], k=whole[:, :, 7:9]), dict(k=whole[:, :, 4:6], k_out=whole[:, :, 5:7]),
                  dict(q_out=torch.zeros_like(q), k=whole[:, :, 4:6], k_out=whole[:, :, 2:4])):
        with pytest.raises(md.MustDropError, match="overlap"):
            md.mustdrop_rotate(q, pos, table, turn, **other)
    cache = md.cache4_buffer(2, 16, 3, 64)
    slots = torch.arange(12, dtype=torch.int32, device="cuda").reshape(2, 6).contiguous()
    for k in (whole[:, :, 2:5], whole[:, :, 3:6]):
        with pytest.raises(md.MustDropError, match="overlap"):
            md.mustdrop_cache4_append(q, k, whole[:, :, 7:], pos, table, turn, slots, cache)
        with pytest.raises(md.MustDropError, match="overlap"):
            md.mustdrop_cache4_append(q, whole[:, :, 7:], k, pos, table, turn, slots, cache)
    torch.cuda.synchronize()
    assert torch.equal(whole, before) and not bool(cache.any())


# ------------------------------------------------------------------------------------------------ bounds

@pytest.mark.parametrize("d, page", [(128, 32), (64, 16), (64, 256)])
def test_bounds_of_samples_without_new_entries(d, page):
    """Only pages that hold an entry first .. min(first + n, length) - 1 are written: none where first is the length or behind it."""
    import torch
    import paper_2411_10803_amd as md
    from test_gpu_chosen import filled_pool
    rng = np.random.default_rng(d)
    H, entries, n = 2, 3, 7
    cap = entries * page
    #         first, length: at the length, behind it, at the pool's end, one entry in the same page, none at all, negative
    samples = [(page + 1, page + 1), (page + 3, page + 1), (cap, cap), (page + 1, page + 2), (0, 0), (-4, 0), (5, 1), (-3, 1), (2 ** 31 - 1, cap), (page - 1, page + 1)]
    B = len(samples)
    pool, _, _ = filled_pool(rng, 4, H, d, page)
    pool = np.concatenate([pool] * 8)
    table = rng.permutation(len(pool))[:B * entries].reshape(B, entries).astype(np.int32)
    b, s = md.cache4_bounds_buffer(len(pool), H, d)
    b.fill_(99)
    s.fill_(77)
    first, length = (dev(np.array(x, np.int32)) for x in zip(*samples))
    md.mustdrop_cache4_bounds(dev(pool), dev(table), length, n, b, s, first=first)
    torch.cuda.synchronize()
    wb, ws, written = np.full((len(pool), H, 2, d), 99), np.full((len(pool), H), 77), 0
    for x, (lo, to) in enumerate(samples):
        for e in sorted({t // page for t in range(max(lo, 0), min(max(lo, 0) + n, to))}):
            wb[table[x, e]], ws[table[x, e]] = cr.bounds(pool, table[x, e], min(page, to - e * page), H, d, page)
            written += 1
    assert written == 4 and np.array_equal(host(b), wb) and np.array_equal(host(s), ws)


# ------------------------------------------------------------------------------------------------ the attention's workspace

def test_tokens_together_with_long_lists_have_no_use_for_a_workspace():
    """Lists padded to 1100 entries in a table of 26: a workspace of 256 bytes, between bands that stay as they were."""
    import torch
    import paper_2411_10803_amd as md
    c = Chosen(81, [390], 391, 8, 4, 64, 16, 1100, BF16, kind="any")
    whole = torch.full((256 + 16384,), 0xA5, dtype=torch.uint8, device="cuda")
    out, lse = c.call(md, workspace=whole[8192:8448])
    assert bool((whole[:8192] == 0xA5).all()) and bool((whole[8448:] == 0xA5).all())
    c.check(out, lse)


@pytest.mark.parametrize("Hq, H, dtype", [(3, 3, BF16), (10, 2, F32), (20, 1, BF16), (33, 1, F32)])
def test_parts_leave_their_sums_in_the_workspace_that_is_asked_for(Hq, H, dtype):
    """Lists in parts, with 1, 5, 20 and 33 query heads to one: exactly the workspace's size, between bands."""
    import torch
    import paper_2411_10803_amd as md
    c = Chosen(82, [1500, 900], 2, Hq, H, 64, 16, 1300, dtype, kind="any", keep=0.8)
    n = md.library().mustdrop_cache4_attend_chosen_workspace_bytes(2, 2, Hq, H, 64, 1300, 16)
    whole = torch.full((n + 16384,), 0xA5, dtype=torch.uint8, device="cuda")
    out, lse = c.call(md, workspace=whole[8192:8192 + n])
    assert bool((whole[:8192] == 0xA5).all()) and bool((whole[8192 + n:] == 0xA5).all())
    c.check(out, lse)


# ------------------------------------------------------------------------------------------------ the choice

def test_choice_for_millions_of_lists():
    """4.2 million lists in tables of more than 2048 pages: more threads than one row of blocks has."""
    import torch
    import paper_2411_10803_amd as md
    B, N, d, page, entries, budget, n_pages = 5, 840000, 64, 16, 2049, 4, 40
    free, _ = torch.cuda.mem_get_info()
    need = md.library().mustdrop_cache4_choose_workspace_bytes(B, N, 1, 1, d, entries, page)
    if free < need + (8 << 30):
        pytest.skip(f"{need >> 30} GiB of workspace")
    rng = np.random.default_rng(91)
    lo = rng.integers(-96, 97, (n_pages, 1, d))
    bounds = np.stack([np.maximum(lo, rng.integers(-96, 97, lo.shape)), lo], 2).astype(np.int8)
    scales = np.full((n_pages, 1), 127, np.uint8)
    table = rng.integers(0, n_pages, (B, entries)).astype(np.int32)
    lengths = [entries * page - 37, 300, 0, entries * page, 5000]
    torch.manual_seed(92)
    q = torch.randn((B, N, 1, d), device="cuda").bfloat16()
    chosen = torch.full((B, N, 1, budget), 99, dtype=torch.int32, device="cuda")
    ws = torch.empty((need,), dtype=torch.uint8, device="cuda")
    md.mustdrop_cache4_choose(q, dev(bounds), dev(scales), dev(table), dev(np.array(lengths, np.int32)), page, chosen, first_pages=1, last_pages=1, workspace=ws)
    torch.cuda.synchronize()
    for b, n in enumerate(lengths):
        assert bool((chosen[b, :N - n] == -1).all()), b
        for i in sorted({N - n, N - n + 65, N - n + 70, N - 1, N - 2, *(N - 1 - rng.integers(0, max(n, 1), 20))} if n else ()):
            want = cr.choose(host(q[b, i]).astype(np.float64), bounds[:, 0].astype(np.int64), scales[:, 0], table[b], n, N, i, page, 1, 1, budget, n_pages)
            assert chosen[b, i, 0].tolist() == want, (b, i)
    del ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", ["equal", "few", "nothing"])
def test_choice_of_millions_of_pages(kind):
    """More than 2^22 pages to take of five million: equal scores, a few values, and queries that are nothing."""
    import torch
    import paper_2411_10803_amd as md
    d, page, entries, budget, n_pages = 64, 16, 5000000, 4600000, 12
    rng = np.random.default_rng(93)
    bounds, scales = np.zeros((n_pages, 1, 2, d), np.int8), np.full((n_pages, 1), 127, np.uint8)
    if kind != "equal":
        bounds[:, 0, 0, 0] = np.arange(n_pages)
    q = torch.zeros((1, 1, 1, d), device="cuda")
    if kind != "nothing":
        q[..., 0] = 1.0
    table = rng.integers(0, n_pages, (1, entries)).astype(np.int32)
    if kind == "few":                                    # nine of ten pages are the same
        table[rng.random(table.shape) < 0.9] = 2
    table[0, rng.integers(0, entries, 50)] = -1          # (their scores are below all others)
    length, last = entries * page - 5, 3
    chosen = torch.full((1, 1, 1, budget), 99, dtype=torch.int32, device="cuda")
    md.mustdrop_cache4_choose(q, dev(bounds), dev(scales), dev(table), dev(np.array([length], np.int32)), page, chosen, first_pages=2, last_pages=last)
    torch.cuda.synchronize()
    w = cr.whole(host(q)[0, 0].astype(np.float64))
    by_page = np.array([cr.score(w, bounds[p, 0].astype(np.int64), 127) for p in range(n_pages)] + [-np.inf])
    score = by_page[table[0]].astype(np.float64)
    score[:2], score[entries - last:] = np.inf, np.inf
    want = np.sort(np.argsort(-score, kind="stable")[:budget])
    assert np.array_equal(host(chosen)[0, 0, 0], want)
