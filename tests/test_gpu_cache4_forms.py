"""The attention over the cache held in 4 bits, in every form that a call may take (csrc/cache4_plan.hpp, c4_attend): blocks and runs, 16 and 32
rows together, plain and streaming loads; and its entries on streams of their own.  tests/test_cache4_forms.py says on the CPU which form each case
takes."""
import numpy as np
import pytest

import cache4_forms as forms
import cache4_ref as ref
import test_gpu_cache4 as base
from test_gpu_cache4 import BF16, F32, Case, dev, host

pytestmark = pytest.mark.gpu


def check(c, out, lse):
    """Every row within the bounds of the formula; a probability as it enters the product with V is off by a part in 2^16 of itself for bf16
    rows (two bf16 parts, of 8 bits each), in 2^23 for fp32 ones (three parts), whatever form the call takes."""
    step, part = (2.0 ** -8, 2.0 ** -16) if c.dtype == BF16 else (2.0 ** -24, 2.0 ** -23)
    for b in range(c.B):
        nq = c.N if c.q_len is None else int(np.clip(c.q_len[b], 0, c.N))
        n = int(np.clip(c.lengths[b], 0, c.table.shape[1] * c.page))
        want, wlse, size, score = ref.attend_heads(c.qh[b], c.K[b], c.V[b], c.there[b], n, nq, c.scale, None if c.keep is None else c.keep[b, :c.K.shape[1]])
        bound, lbound = ref.attend_bounds(want, wlse, size, score, c.d, n, step, part)
        assert (out[b, nq:] == 7).all() and (lse[b, :, nq:] == 7).all(), f"sample {b}: rows behind the last were written"
        got, gl, wl = out[b, :nq], lse[b, :, :nq].T, wlse[:nq]
        assert np.array_equal(np.isnan(got), np.isnan(want[:nq])), f"sample {b}: NaN"
        off = np.where(np.isnan(got), 0, np.abs(got - want[:nq]) - bound[:nq])
        assert (off <= 0).all(), f"sample {b}: {(off > 0).sum()} values, {np.argwhere(off > 0)[:3]}, off by up to {off.max()} more than the bound"
        empty = np.isneginf(wl)
        assert np.array_equal(np.isneginf(gl), empty) and (got[empty] == 0).all(), f"sample {b}: empty rows"
        ok = np.where(empty | np.isnan(wl), True, np.abs(gl - np.where(empty, 0, wl)) <= lbound[:nq])
        assert ok.all(), f"sample {b}: lse"


@pytest.mark.parametrize("i", range(len(forms.MANY_ROWS)))
def test_probabilities_keep_16_bits_where_rows_go_together(i):
    """The same accuracy for a request whatever else is in the batch: where 32 rows of a K/V head are taken together too.  Small scores: their own
    rounding is then far below what one bf16 part of a probability would be off."""
    import paper_2411_10803_amd as md
    c = Case(400 + i, **forms.MANY_ROWS[i], size=0.25, heavy=False)
    check(c, *c.call(md))


@pytest.mark.parametrize("kind, d, runs", forms.FORMS)
def test_entries_of_a_table_behind_the_length_change_nothing(kind, d, runs):
    """They may name no page, other samples' pages, or pages whose rows are no numbers."""
    import paper_2411_10803_amd as md
    c = Case(500, **forms.form(kind, d, runs))
    live = np.arange(c.table.shape[1]) < -(-np.asarray(c.lengths)[:, None] // c.page)
    used = c.table[live]
    spare = [p for p in range(len(c.pool)) if p not in set(used.tolist())]     # never written: all scales 255
    assert spare and (c.pool[spare] == 255).all()
    rng = np.random.default_rng(1)
    shape, own = c.table.shape, c.table
    results = []
    for behind in (np.full(shape, -1), rng.choice(used, shape), rng.choice(spare, shape), rng.integers(-2 ** 31, 2 ** 31, shape)):
        c.table = np.where(live, own, behind).astype(np.int32)
        results.append(c.call(md))
    check(c, *results[0])
    for out, lse in results[1:]:
        assert np.array_equal(out, results[0][0]) and np.array_equal(lse, results[0][1])


@pytest.mark.parametrize("page, masks", ((16, False), (64, True), (256, False), (256, True)))
@pytest.mark.parametrize("kind, d, runs", forms.FORMS)
def test_no_number_reaches_the_rows_that_see_it(kind, d, runs, page, masks):
    """Groups that are no numbers in K and V, at entries that all rows of a sample see, that the last of them see, and that `keep` leaves out; in
    any place of a page, and in parts of a unit that a join adds up."""
    import paper_2411_10803_amd as md
    c = Case(800 + page, **dict(forms.form(kind, d, runs, page=page, keep=0.9 if masks else None), lengths=forms.nan_lengths(kind)))
    rng = np.random.default_rng(page + d)
    poisoned = partly = 0
    for b, n in enumerate(c.lengths):
        first = max(0, n - c.N + 1)                  # from here on not all rows see an entry
        late = [*rng.integers(first, n, 2), n - 1] if b % 3 else []
        early = rng.integers(0, max(first, 1), 3) if b % 2 else []
        for x, t in enumerate([*late, *early]):
            h, g, in_k = rng.integers(0, c.H), rng.integers(0, d // 32), x == 0 and b % 4 == 1
            kk, vv = c.K[b, t, h].copy(), c.V[b, t, h].copy()
            kk[np.isnan(kk)], vv[np.isnan(vv)] = 1.0, 1.0
            (kk if in_k else vv)[g * 32 + 7] = np.nan
            ref.put(c.pool, c.table[b, t // page] * page + t % page, h, kk, vv, page)
            c.K[b, t, h], c.V[b, t, h] = ref.values(*ref.quantise(kk)), ref.values(*ref.quantise(vv))
            if masks:
                c.keep[b, t] = x < 3 or x == 4       # two of the early ones are left out
            poisoned += 1
    out, lse = c.call(md)
    for b in range(c.B):
        bad = np.isnan(out[b]).any((1, 2))
        partly += bad.any() and not bad.all()
    assert poisoned > c.B and partly >= 2            # some rows, not all of them
    check(c, out, lse)


@pytest.mark.parametrize("kind, d, runs", forms.FORMS)
def test_a_query_that_is_no_number_reaches_its_own_rows(kind, d, runs):
    import torch
    import paper_2411_10803_amd as md
    c = Case(900, **dict(forms.form(kind, d, runs), lengths=forms.nan_lengths(kind)))
    rng = np.random.default_rng(d)
    bad = np.zeros((c.B, c.N, c.Hq), bool)
    for b in range(1, c.B):
        i, h = rng.integers(0, c.N), rng.integers(0, c.Hq)
        if c.lengths[b] - c.N + i < 30:              # (many keys: an infinite query then has scores of both signs)
            i = c.N - 1
        c.q[b, i, h, rng.integers(0, d)] = float("nan") if b % 2 else float("inf")
        bad[b, i, h] = True
    with np.errstate(invalid="ignore"):
        out, lse = c.call(md)
        c.qh = np.where(bad[..., None], np.nan, c.qh)
        check(c, out, lse)
    assert np.array_equal(np.isnan(out).all(3), bad) and np.array_equal(np.isnan(lse.transpose(0, 2, 1)), bad)


@pytest.mark.parametrize("entries", (8, 1100))       # of a table with pages of 16: blocks, runs
@pytest.mark.parametrize("dtype", (BF16, F32))
def test_scores_at_the_ends_of_the_range(dtype, entries):
    """Rows that see one key whose only channel is 1: their score is the query's.  Beyond 2.3e38 it is infinite to base 2 and the row NaN, below
    -2e38 the row is as one that sees nothing; in between lse is the score, but for five roundings of 2^-24 each (log2(e), its product with the score,
    the sum with log2 of a sum near 1, ln 2, its product) and a unit each of exp2 and log2 near 1, 2^-22 together."""
    import paper_2411_10803_amd as md
    d, scores = 64, np.array([2.2e38, 3e38, -1.9e38, -2.2e38, -3e38, 1.0, 0.0, 1e30])
    c = Case(950, [1] * 4, 1, len(scores), 1, d, 16, dtype, entries=entries)
    k = np.zeros(d)
    k[5] = 1.0
    for b in range(4):
        ref.put(c.pool, int(c.table[b, 0]) * 16, 0, k, c.V[b, 0, 0], 16)
    q = np.zeros(c.qh.shape)
    q[..., 5] = scores
    c.q, c.qh = base.rows_on_gpu(q, dtype)
    c.scale = 1.0
    out, lse = c.call(md)
    want = np.where(scores > 2.3e38, np.nan, np.where(scores < -2e38, -np.inf, c.qh[0, 0, :, 5]))
    for b in range(4):
        assert np.array_equal(np.isnan(lse[b, :, 0]), np.isnan(want)) and np.array_equal(np.isneginf(lse[b, :, 0]), np.isneginf(want))
        ok = np.isfinite(want)
        assert (np.abs(lse[b, ok, 0] - want[ok]) <= 5 * 2.0 ** -24 * np.abs(want[ok]) + 2.0 ** -22).all()
        assert np.isnan(out[b, 0, np.isnan(want)]).all() and (out[b, 0, np.isneginf(want)] == 0).all()
        assert (out[b, 0, ok] == c.V[b, 0, 0]).all()             # (one probability of 1: V itself, exact in bf16)


@pytest.mark.parametrize("masks", (False, True))
@pytest.mark.parametrize("kind, d, runs", forms.FORMS)
def test_scores_of_every_size(kind, d, runs, masks):
    """Queries of one channel, from 1 to 2^120: a score is one exact product, so keys of one value tie at any size, and where scores are large only those
    of the largest count.  Off by: the factor to base 2, 2^-23 of a difference of scores of which no more than 150 count, 2^-21 for exp2, the
    sums over the keys, 2^-16 or 2^-23 for the parts of a probability (twice each, in the product and in the sum), and the output's rounding."""
    import paper_2411_10803_amd as md
    c = Case(970, **dict(forms.form(kind, d, runs, keep=0.9 if masks else None), lengths=forms.nan_lengths(kind)))
    rng = np.random.default_rng(d + runs)
    for b, n in enumerate(c.lengths):
        for t in range(n):
            for h in range(c.H):
                k = np.zeros(d)
                k[3] = rng.choice([6, 4, 3, 2, 1.5, 1, 0.5, 0, -1, -6])
                ref.put(c.pool, c.table[b, t // c.page] * c.page + t % c.page, h, k, c.V[b, t, h], c.page)
                c.K[b, t, h] = k
    q = np.zeros(c.qh.shape)
    q[..., 3] = np.exp2(rng.integers(0, 121, q.shape[:3]).astype(float)) * rng.choice([1, -1, 1.5, 1.25], q.shape[:3])
    c.q, c.qh = base.rows_on_gpu(q, c.dtype)
    assert np.array_equal(c.qh, q)
    c.scale = float(np.float32(c.scale))
    out, lse = c.call(md)
    step, part = (2.0 ** -8, 2.0 ** -16) if c.dtype == BF16 else (2.0 ** -24, 2.0 ** -23)
    for b, n in enumerate(c.lengths):
        want, wlse, size, _ = ref.attend_heads(c.qh[b], c.K[b], c.V[b], c.there[b], n, c.N, c.scale, None if c.keep is None else c.keep[b, :c.K.shape[1]])
        bound = step * np.abs(want) + 2 * (150 * 2.0 ** -23 + 2.0 ** -21 + (n / 32 + 64) * 2.0 ** -24 + part) * size + 1e-37
        assert (np.abs(out[b] - want) <= bound).all(), b
        gl, empty = lse[b].T, np.isneginf(wlse)
        assert np.array_equal(np.isneginf(gl), empty)
        gl, wlse = gl[~empty], wlse[~empty]
        assert (np.abs(gl - wlse) <= 6 * 2.0 ** -24 * np.abs(wlse) + 150 * 2.0 ** -23 + 2.0 ** -21 + (n / 32 + 64) * 2.0 ** -24).all(), b


@pytest.mark.parametrize("entries", (8, 1100))
@pytest.mark.parametrize("d", (64, 128))
def test_fp32_queries_at_the_ends_of_their_range(d, entries):
    """One key of 2^k in one channel, queries of 24 bits: a score is one exact product.  Off by five roundings of 2^-24, a unit each of exp2 and log2
    near 1, and by what a query has below 2^-134 (half the smallest bf16 number)."""
    import paper_2411_10803_amd as md
    for k, queries in ((125, np.exp2([-110.0, -109, -100, -112, -120, -126, -133]) * (2 - 2.0 ** -23)), (-90, np.array([3.389e38, -3.389e38, 1e38, 3.4e38]))):
        c = Case(990, [1] * 2, 1, len(queries), 1, d, 16, F32, entries=entries)
        key = np.zeros(d)
        key[9] = 2.0 ** k
        for b in range(2):
            ref.put(c.pool, int(c.table[b, 0]) * 16, 0, key, c.V[b, 0, 0], 16)
        q = np.zeros(c.qh.shape)
        q[..., 9] = queries.astype(np.float32)
        c.q, c.qh = base.rows_on_gpu(q, F32)
        c.scale = 1.0
        out, lse = c.call(md)
        want = c.qh[0, 0, :, 9] * 2.0 ** k
        over = np.abs(queries) > 3.3895e38
        assert np.array_equal(np.isnan(lse[0, :, 0]), over) and np.isnan(out[:, 0, over]).all()
        bound = 5 * 2.0 ** -24 * np.abs(want) + 2.0 ** -22 + 2.0 ** (k - 134)
        assert (np.abs(lse[:, :, 0] - want) <= bound)[:, ~over].all() and np.isfinite(out[:, 0, ~over]).all()


@pytest.mark.parametrize("scale", (1e-44, 1e-20, 1e20))
@pytest.mark.parametrize("kind, d, runs", [f for f in forms.FORMS if f[1] == 64])
def test_scales_of_every_size(kind, d, runs, scale):
    """Tiny ones (a factor that fp32 holds with few bits): all keys count alike.  A large one, with queries that make up for it."""
    import paper_2411_10803_amd as md
    c = Case(980, **forms.form(kind, d, runs))
    if scale > 1:
        c.q, c.qh = base.rows_on_gpu(c.qh * 2.0 ** -67, c.dtype)
    c.scale = float(np.float32(scale))
    check(c, *c.call(md))


def test_a_sample_of_seventy_million_entries():
    """4.8 GB of one sample's pages; its keys are 0, so that a row's output is the mean of the values.  The sums of a part are exact (multiples of 1/2
    below 2^22), the join of at most 1024 parts and four waves adds them up: 2^-24 of all of it each."""
    import torch
    import paper_2411_10803_amd as md
    n, d, page = 70_000_001, 64, 256
    n_pages = -(-n // page)
    cache = md.cache4_buffer(n_pages, page, 1, d)
    g = torch.Generator(device="cuda").manual_seed(1)
    at = page * (d // 2 + d // 32)                   # codes of V: [page / 4, 16, 4, d / 32], magnitudes without a sign
    cache[:, 0, page * d // 2:at] = 127
    cache[:, 0, at + page * d // 2:] = 127
    codes = cache[:, 0, at:at + page * d // 2].view(n_pages, page // 4, 16, 4, d // 32)
    levels = torch.tensor(ref.LEVELS, dtype=torch.float64, device="cuda")
    total = torch.zeros((16, d // 32, 2), dtype=torch.float64, device="cuda")
    for i in range(0, n_pages, 8192):
        part = torch.randint(0, 256, codes[i:i + 8192].shape, generator=g, dtype=torch.uint8, device="cuda") & 0x77
        codes[i:i + 8192] = part
        live = (torch.arange(i * page, i * page + part.shape[0] * page, device="cuda") < n).view(part.shape[0], page // 4, 1, 4, 1)
        for half in range(2):
            total[..., half] += (levels[((part >> (4 * half)) & 7).int()] * live).sum((0, 1, 3))
    mean = (total / n).reshape(d).cpu().numpy()
    ends = cache[0].clone()
    cache[0], cache[-1] = cache[-1].clone(), ends
    order = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    order[0], order[-1] = n_pages - 1, 0             # entry 0 in the last page of the pool, the last entry in its first
    table = order[None].contiguous()
    length = torch.full((1,), n, dtype=torch.int32, device="cuda")
    q = torch.randn((1, 1, 3, d), generator=g, device="cuda")
    lse = torch.zeros((1, 3, 1), device="cuda")
    out = md.mustdrop_cache4_attend(q, cache, table, length, 0.125, lse=lse)
    torch.cuda.synchronize()
    assert (np.abs(host(out)[0, 0] - mean) <= 1100 * 2.0 ** -24 * mean).all()
    assert (np.abs(host(lse) - np.log(n)) <= 1100 * 2.0 ** -24 + 2.0 ** -22 * np.log(n)).all()
    # rows out of its end, and one more in
    rows = [torch.zeros((1, 4, 1, d), device="cuda") for _ in range(2)]
    md.mustdrop_cache4_read(cache, table, length, *rows, first=length - 2)
    slot = torch.tensor([[int(order[n // page]) * page + n % page]], dtype=torch.int32, device="cuda")
    new = torch.full((1, 1, 1, d), 6.0, device="cuda")
    md.mustdrop_cache4_write(new, new, slot, cache)
    after = [torch.zeros((1, 1, 1, d), device="cuda") for _ in range(2)]
    md.mustdrop_cache4_read(cache, table, length + 1, *after, first=length)
    torch.cuda.synchronize()
    assert (rows[0] == 0).all() and rows[1][0, :2].any() and not rows[1][0, 2:].any() and all(torch.equal(x, new) for x in after)


@pytest.mark.parametrize("dtype, d", ((BF16, 128), (F32, 64)))
def test_rows_from_one_buffer_of_queries_keys_and_values(dtype, d):
    """[B, N, (Hq + 2 H) d], as one projection gives it: rows in and queries as views of it."""
    import torch
    import paper_2411_10803_amd as md
    B, N, Hq, H, page = 3, 9, 6, 2, 16
    g = torch.Generator(device="cuda").manual_seed(d)
    one = torch.randn((B, N, Hq + 2 * H, d), generator=g, device="cuda").to(torch.bfloat16 if dtype == BF16 else torch.float32)
    q, k, v = one[:, :, :Hq], one[:, :, Hq:Hq + H], one[:, :, Hq + H:]
    slots = torch.arange(B * page, dtype=torch.int32, device="cuda").view(B, page)[:, :N].contiguous()
    table, length = torch.arange(B, dtype=torch.int32, device="cuda")[:, None].contiguous(), torch.full((B,), N, dtype=torch.int32, device="cuda")
    got = []
    for x in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
        cache = md.cache4_buffer(B, page, H, d)
        md.mustdrop_cache4_write(x[1], x[2], slots, cache)
        got.append((cache, md.mustdrop_cache4_attend(x[0], cache, table, length, 0.1)))
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and bool(got[0][1].any())


# ------------------------------------------------------------------------------------------------ streams

def busy_for_a_while(torch, stream, work):
    """About 50 ms of products on the stream: what is put behind them there has not begun when the host has made its next calls."""
    with torch.cuda.stream(stream):
        for _ in range(40):
            torch.mm(work, work, out=work)


@pytest.mark.parametrize("name", ("pages", "write", "read", "attend", "attend runs"))
def test_a_call_follows_what_its_stream_does_before(name):
    """The inputs are made on the call's stream, behind 50 ms of other work, and nothing else is waited for: a call on any other stream, the current
    one among them, would take the zeros that stand there until then."""
    import torch
    import paper_2411_10803_amd as md
    c = Case(23, **forms.form("few", 128, int(name.endswith("runs"))))
    H, d, page, B = c.H, c.d, c.page, c.B
    table, length = dev(c.table), dev(np.asarray(c.lengths, np.int32))
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = [torch.randn((B, 7, H, d), generator=g, device="cuda").bfloat16() for _ in range(2)]
    slots = torch.arange(B * 7, dtype=torch.int32, device="cuda").view(B, 7)
    entries, n_pages = 4, 4 * B

    def pages(x, stream=None):
        zero = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
        s = [zero(B), zero(B, entries) - 1, torch.arange(n_pages, dtype=torch.int32, device="cuda"), zero(1) + n_pages, zero(1) + 9, zero(B, 64)]
        torch.cuda.current_stream().synchronize()
        return s, lambda: md.mustdrop_cache4_pages(x, *s[:5], page, slots=s[5], stream=stream)

    def write(x, stream=None):
        cache = torch.zeros((n_pages, H, ref.page_bytes(page, d)), dtype=torch.uint8, device="cuda")
        torch.cuda.current_stream().synchronize()
        return [cache], lambda: md.mustdrop_cache4_write(x, rows[1], slots, cache, stream=stream)

    def read(x, stream=None):
        out = [torch.zeros((B, 80, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        torch.cuda.current_stream().synchronize()
        return out, lambda: md.mustdrop_cache4_read(x, table, length, *out, stream=stream)

    def attend(x, stream=None):
        out, lse = torch.zeros_like(c.q, memory_format=torch.contiguous_format), torch.zeros((B, c.Hq, c.N), device="cuda")
        torch.cuda.current_stream().synchronize()
        return [out, lse], lambda: md.mustdrop_cache4_attend(c.q, x, table, length, c.scale, out=out, lse=lse, stream=stream)
    make, true = {"pages": (pages, torch.tensor([(11 * b) % 64 for b in range(B)], dtype=torch.int32, device="cuda")), "write": (write, rows[0]),
                  "read": (read, dev(c.pool)), "attend": (attend, dev(c.pool))}[name.split()[0]]
    want, call = make(true)
    call()
    stale, call = make(torch.zeros_like(true))
    call()
    work = torch.eye(4096, device="cuda")
    torch.mm(work, work, out=torch.empty_like(work))
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    x = torch.zeros_like(true)
    torch.cuda.synchronize()
    assert not all(torch.equal(a.nan_to_num(1e9) if a.is_floating_point() else a, b.nan_to_num(1e9) if b.is_floating_point() else b)
                   for a, b in zip(want, stale))
    with torch.cuda.stream(other):                   # (what the call itself makes, it makes on its own stream: not on this one)
        got, call = make(x, stream=s)
        busy_for_a_while(torch, s, work)
        with torch.cuda.stream(s):
            x.copy_(true)
        call()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b) or np.array_equal(host(a), host(b), equal_nan=True)


def test_nobody_gets_the_memory_of_a_call_on_its_own_stream():
    """What a call makes for itself on a given stream goes back to that stream: tensors made on the current one while the call has not begun
    yet keep what is written into them."""
    import torch
    import paper_2411_10803_amd as md
    c = Case(22, [3000, 1700], 1, 4, 2, 128, 32, BF16, entries=600)              # in runs: with sums in the workspace
    args = [c.q, dev(c.pool), dev(c.table), dev(np.asarray(c.lengths, np.int32)), c.scale]
    want = md.mustdrop_cache4_attend(*args)
    size, pages_size = md.cache4_workspace(args[0], args[1], args[2]).numel(), md.cache4_pages_workspace(2).numel()
    work = torch.eye(4096, device="cuda")
    torch.mm(work, work, out=torch.empty_like(work))
    i32 = dict(dtype=torch.int32, device="cuda")
    # (many samples: two launches, the first of which leaves the plan in its workspace)
    B, entries = 2000, 2
    state = [torch.full((B,), 20, **i32), torch.zeros(B, **i32), torch.full((B, entries), -1, **i32), torch.arange(B * entries, **i32),
             torch.full((1,), B * entries, **i32), torch.zeros(1, **i32)]
    slots = torch.zeros((B, 20), **i32)
    pages_size = md.cache4_pages_workspace(B).numel()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()                         # (what was given back before is gone: new tensors do not take it)
    busy_for_a_while(torch, s, work)
    out = md.mustdrop_cache4_attend(*args, stream=s)
    md.mustdrop_cache4_pages(*state, 16, slots=slots, stream=s)
    sizes = [size, pages_size, out.numel() * out.element_size()] * 6
    over = [torch.full((n,), 170, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda.synchronize()
    for n, t in zip(sizes, over):
        assert (t == 170).all(), n
    assert torch.equal(out, want)
    assert state[1].tolist() == [20] * B and int(state[4]) == 0 and int(state[5]) == 0
    assert sorted(slots[:, ::16].flatten().tolist()) == list(range(0, 16 * B * entries, 16))


# ------------------------------------------------------------------------------------------------ joins, and pools that are streamed

@pytest.mark.parametrize("i", range(len(forms.JOINS)))
def test_joins(i):
    import paper_2411_10803_amd as md
    c = Case(600 + i, **forms.JOINS[i])
    out, lse = c.call(md)
    check(c, out, lse)
    again, lse2 = c.call(md)
    assert np.array_equal(out, again) and np.array_equal(lse, lse2)             # the same bits


@pytest.mark.parametrize("dtype, d", ((BF16, 128), (F32, 64), (BF16, 64), (F32, 128)))
def test_a_long_sample_among_short_ones(dtype, d):
    """A row in more than 256 parts that four waves add up, each of them more than 64."""
    import torch
    import paper_2411_10803_amd as md
    lengths, page, entries = forms.LONG["lengths"], forms.LONG["page"], forms.LONG["entries"]
    rng = np.random.default_rng(d)
    table, n_pages = base.scattered(rng, lengths, page, entries)
    B, most = len(lengths), max(lengths)
    cache = torch.full_like(md.cache4_buffer(n_pages, page, 1, d), 255)
    K, V = np.zeros((B, most, 1, d)), np.zeros((B, most, 1, d))
    for b, n in enumerate(lengths):                  # (rows in are tested byte by byte elsewhere)
        k, v = rng.standard_normal((n, 1, d)) + 1.2 * (rng.random((n, 1, 1)) < 0.02), rng.standard_normal((n, 1, d))
        at = np.arange(n)
        rows = [torch.from_numpy(x[None]).float().cuda() for x in (k, v)]
        md.mustdrop_cache4_write(*rows, dev((table[b, at // page] * page + at % page)[None].astype(np.int32)), cache)
        K[b, :n], V[b, :n] = (ref.values(*ref.quantise(host(x)[0])) for x in rows)
    q, qh = base.rows_on_gpu(rng.standard_normal((B, 1, 1, d)) + 0.3, dtype)
    out, lse = md.mustdrop_cache4_attend(q, cache, dev(table), dev(np.asarray(lengths, np.int32)), 1 / np.sqrt(d),
                                         lse=(l := torch.zeros((B, 1, 1), device="cuda"))), l
    torch.cuda.synchronize()
    out, lse = host(out).astype(np.float64), host(lse).astype(np.float64)
    step, part = (2.0 ** -8, 2.0 ** -16) if dtype == BF16 else (2.0 ** -24, 2.0 ** -23)
    for b, n in enumerate(lengths):
        want, wlse, size, score = ref.attend(qh[b], K[b, :n], V[b, :n], np.ones(n, bool), n, 1, 1 / np.sqrt(d))
        bound, lbound = ref.attend_bounds(want, wlse, size, score, d, n, step, part)
        assert (np.abs(out[b] - want) <= bound).all() and (np.abs(lse[b].T - wlse) <= lbound).all(), b


@pytest.mark.parametrize("kind, d, runs", forms.FORMS)
def test_a_pool_that_is_streamed_gives_the_same_bits(kind, d, runs):
    """Pools of more than 128 MiB are read by streaming loads: the same pages behind others, in one of 140."""
    import torch
    import paper_2411_10803_amd as md
    c = Case(700, **forms.form(kind, d, runs, page=32, keep=0.8))
    out, lse = c.call(md)
    check(c, out, lse)
    n_pages = (140 << 20) // (c.pool.shape[1] * c.pool.shape[2])
    far = n_pages - len(c.pool)
    cache = torch.full((n_pages,) + c.pool.shape[1:], 255, dtype=torch.uint8, device="cuda")
    cache[far:] = dev(c.pool)
    table = np.where((c.table >= 0) & (c.table < len(c.pool)), c.table + far, c.table).astype(np.int32)
    big, lse2 = base.rows_on_gpu(np.full(out.shape, 7.0), c.dtype, c.layout, pad=1)[0], torch.full(lse.shape, 7.0, device="cuda")
    md.mustdrop_cache4_attend(c.q, cache, dev(table), dev(np.asarray(c.lengths, np.int32)), c.scale, out=big, lse=lse2, keep=dev(c.keep))
    torch.cuda.synchronize()
    assert cache.numel() > 128 << 20 and np.array_equal(host(big), out) and np.array_equal(host(lse2), lse)


def test_a_step_in_a_graph_with_eight_waves():
    """As in a graph of short and of very long tables: tables of 512 entries, whose blocks have eight waves."""
    base.test_decode_step_in_a_graph(32)
