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


@pytest.mark.parametrize("axis", ["batch", "tokens", "heads"])
def test_in_place_whatever_the_stride_of_an_axis_with_one_place(axis):
    """The same rows by two layouts of the C ABI that differ in nothing but such a stride."""
    import ctypes as C
    import torch
    from paper_2411_10803_amd import binding
    import paper_2411_10803_amd as md
    torch.manual_seed(5)
    at = ("batch", "tokens", "heads").index(axis)
    shape = [3, 4, 5, 64]
    whole = torch.randn(shape, device="cuda").bfloat16()
    q = whole.narrow(at, 0, 1)
    strides = list(q.stride()[:3])
    lay = C.byref(md.KvLayout(*strides))
    strides[at] = 4096
    other = C.byref(md.KvLayout(*strides))
    B, N, H, d = q.shape
    table, turn = md.rotary_table(50, 32), md.rotary([32])
    pos = torch.randint(0, 50, (1, B, N), dtype=torch.int32, device="cuda")
    before = whole.clone()
    want = md.mustdrop_rotate(q.contiguous(), pos, table, turn, q_out=torch.zeros(q.shape, dtype=q.dtype, device="cuda"))[0]
    angles, by, stream = (pos.data_ptr(), None, table.data_ptr()), C.byref(turn), torch.cuda.current_stream().cuda_stream
    binding._call("mustdrop_rotate", q.data_ptr(), None, 1, *angles, None, B, N, N, H, 0, d, 50, by, 0, q.data_ptr(), None, lay, None, other, None, stream)
    torch.cuda.synchronize()
    assert torch.equal(q, want)
    q.copy_(before.narrow(at, 0, 1))
    cache, k = md.cache4_buffer(2, 16, 2, 64), torch.randn((B, N, 2, d), device="cuda").bfloat16()
    slots = torch.arange(B * N, dtype=torch.int32, device="cuda").reshape(B, N).contiguous()
    binding._call("mustdrop_cache4_append", q.data_ptr(), k.data_ptr(), k.data_ptr(), 1, *angles, slots.data_ptr(), cache.data_ptr(), B, N, N, H, 2, d, 50, 2, 16, by,
                  q.data_ptr(), lay, None, other, stream)
    torch.cuda.synchronize()
    assert torch.equal(q, want)
    q.copy_(before.narrow(at, 0, 1))
    assert torch.equal(whole, before)


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


# ------------------------------------------------------------------------------------------------ lists and tables as long as a block holds

def decoded(pool, d, page):
    """K and V [pages * page, H, d] of all slots, as float64."""
    n, H = pool.shape[:2]
    at = np.cumsum([0, page * d // 2, page * d // 32, page * d // 2, page * d // 32])
    kc, ks, vc, vs = (pool[:, :, a:b] for a, b in zip(at, at[1:]))
    nibbles = lambda x: np.stack([x & 15, x >> 4], -1)  # noqa: E731
    k = ref.values(nibbles(kc.reshape(n, H, page, d // 2)).reshape(n, H, page, d), ks.reshape(n, H, page, d // 32))
    vc = vc.reshape(n, H, page // 4, 16, 4, d // 32).transpose(0, 1, 2, 4, 3, 5).reshape(n, H, page, d // 2)      # tokens, then their sixteenths
    vs = vs.reshape(n, H, page // 4, d // 32, 4).transpose(0, 1, 2, 4, 3).reshape(n, H, page, d // 32)
    v = ref.values(nibbles(vc).reshape(n, H, page, d), vs)
    return [x.transpose(0, 2, 1, 3).reshape(n * page, H, d) for x in (k, v)]


class Wide(Chosen):
    """Tables of many entries over a pool of any bytes (entries may name a page again), lists of many entries; some rows are checked."""

    def __init__(self, seed, lengths, N, Hq, H, d, page, budget, dtype, entries, n_pages=40, q_len=None, keep=None, kind="sorted"):
        import torch
        rng = np.random.default_rng(seed)
        B = len(lengths)
        self.B, self.N, self.Hq, self.H, self.d, self.page, self.budget, self.dtype, self.layout, self.lengths = B, N, Hq, H, d, page, budget, dtype, "tokens", lengths
        self.entries, self.scale = entries, 1 / np.sqrt(d)
        self.pool = rng.integers(0, 256, (n_pages, H, ref.page_bytes(page, d))).astype(np.uint8)
        codes = page * d // 2
        for o in (codes, 2 * codes + page * d // 32):
            self.pool[:, :, o:o + page * d // 32] = rng.integers(124, 128, (n_pages, H, page * d // 32))
        self.k, self.v = decoded(self.pool, d, page)
        self.table = rng.integers(0, n_pages, (B, entries)).astype(np.int32)
        self.table[rng.random(self.table.shape) < 0.02] = n_pages
        q = torch.from_numpy(rng.standard_normal((B, N, Hq, d)) * 0.3).to(torch.bfloat16 if dtype == BF16 else torch.float32)
        self.q, self.qh = q.cuda(), q.double().numpy()
        self.q_len = None if q_len is None else np.asarray(q_len, np.int32)
        self.keep = None if keep is None else (rng.random((B, entries * page)) < keep).astype(np.uint8)
        self.lists = np.full((B, N, H, budget), -1, np.int32)
        for b, i, h in np.ndindex(B, N, H):
            if kind == "any":
                pick = rng.integers(-2, entries + 2, budget)
                if i % 3 == 0:                           # long runs that ascend, and some that do not
                    pick[:budget * 3 // 4] = np.sort(pick[:budget * 3 // 4])
            else:
                pick = np.sort(rng.choice(entries, min(budget, entries), replace=False))
            self.lists[b, i, h, :len(pick)] = pick

    def check_some(self, out, lse, seed=0, n=60):
        rng = np.random.default_rng(seed)
        step, part = (2.0 ** -8, 2.0 ** -16) if self.dtype == BF16 else (2.0 ** -24, 2.0 ** -23)
        G, cap, page = self.Hq // self.H, self.entries * self.page, self.page
        rows = [self.N if self.q_len is None else int(np.clip(self.q_len[b], 0, self.N)) for b in range(self.B)]
        for b, nq in enumerate(rows):
            assert (out[b, nq:] == 7).all() and (lse[b, :, nq:] == 7).all(), f"sample {b}: rows behind the last were written"
        picks = [(b, i, h) for b, nq in enumerate(rows) for i in {0, 1, nq - 1, nq - 2} if 0 <= i < nq for h in (0, self.H - 1)]
        picks = [picks[x] for x in rng.permutation(len(picks))[:n // 2]]
        while len(picks) < n:
            b = int(rng.integers(self.B))
            if rows[b]:
                picks.append((b, int(rng.integers(rows[b])), int(rng.integers(self.H))))
        for b, i, h in picks:
            seen = cr.seen(self.lengths[b], rows[b], i, cap)
            pages = np.array([e for e in cr.listed(self.lists[b, i, h], self.entries) if 0 <= self.table[b, e] < len(self.pool)], np.int64)
            at = (pages[:, None] * page + np.arange(page)).reshape(-1)
            on = at < seen
            if self.keep is not None:
                on &= self.keep[b, at] != 0
            slot = (self.table[b, at // page].astype(np.int64) * page + at % page)[on]
            g = slice(h * G, (h + 1) * G)
            there = np.ones(len(slot), bool)
            want, wlse, size, score = ref.attend_heads(self.qh[b, i:i + 1, g], self.k[slot, h:h + 1], self.v[slot, h:h + 1], there, len(slot), 1, self.scale) \
                if len(slot) else (np.zeros((1, G, self.d)), np.full((1, G), -np.inf), np.zeros((1, G, self.d)), np.zeros((1, G)))
            bound, lb = ref.attend_bounds(want, wlse, size, score, self.d, len(slot), step, part)
            off = np.abs(out[b, i, g] - want[0]) - bound[0]
            assert (off <= 0).all(), (b, i, h, len(slot), off.max())
            empty = np.isneginf(wlse[0])
            assert np.array_equal(np.isneginf(lse[b, g, i]), empty), (b, i, h, "empty rows")
            assert np.where(empty, True, np.abs(lse[b, g, i] - np.where(empty, 0, wlse[0])) <= lb[0]).all(), (b, i, h, "lse")


WIDE = [
    # several tokens together: sixteen over a table of 601 entries, blocks of eight waves
    dict(lengths=[9000], N=768, Hq=2, H=2, d=64, page=16, budget=64, dtype=BF16, entries=601),
    # four over a table of 4096, joint lists of up to 1024: the most LDS, eight waves
    dict(lengths=[65500], N=192, Hq=32, H=8, d=128, page=16, budget=256, dtype=BF16, entries=4096),
    # two over a table of 4096, joint lists of 1024, more than 512 blocks of four waves
    dict(lengths=[65536, 40000], N=130, Hq=64, H=8, d=64, page=16, budget=512, dtype=BF16, entries=4096, q_len=[130, 77]),
    # fp32: eight over 1100 entries, a mask, a last group of fewer tokens, a sample of none
    dict(lengths=[17000, 9000, 400], N=131, Hq=16, H=8, d=128, page=16, budget=100, dtype=F32, entries=1100, keep=0.6, q_len=[131, 90, 0]),
    # lists in any order of more than 64 entries, rows before the first entry
    dict(lengths=[40, 30000], N=300, Hq=4, H=4, d=64, page=32, budget=130, dtype=F32, entries=950, kind="any"),
    dict(lengths=[20000, 100], N=400, Hq=6, H=2, d=128, page=16, budget=200, dtype=BF16, entries=1030, kind="any", keep=0.5),
    # joint lists as long as the table, in pages of 64: 990 entries of 1000 tokens' sixteenths
    dict(lengths=[63300], N=400, Hq=4, H=4, d=64, page=64, budget=500, dtype=BF16, entries=990),
    # one token: lists of 1024 entries in one part, eight waves
    dict(lengths=[17600 - 11 * b for b in range(38)], N=1, Hq=16, H=8, d=128, page=16, budget=1024, dtype=BF16, entries=1100),
    dict(lengths=[17600 - 11 * b for b in range(70)], N=1, Hq=20, H=5, d=64, page=16, budget=1024, dtype=F32, entries=1100, keep=0.7, kind="any"),
    # and of 1025: two parts
    dict(lengths=[17600 - 11 * b for b in range(38)], N=1, Hq=16, H=8, d=128, page=16, budget=1025, dtype=BF16, entries=1100, keep=0.7),
]


@pytest.mark.parametrize("i", range(len(WIDE)))
def test_attention_over_many_chosen_pages(i):
    import paper_2411_10803_amd as md
    c = Wide(400 + i, **WIDE[i])
    c.check_some(*c.call(md), seed=i)
