"""The cache held in 4 bits on the GPU against the plain 64-bit reference (cache4_ref.py): pages and slots and the bytes of the cache
exactly, attention within bounds that follow from its arithmetic."""
import numpy as np
import pytest

import cache4_ref as ref
import workloads as wl

pytestmark = pytest.mark.gpu

BF16, F32 = "bf16", "f32"


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def rows_on_gpu(x, dtype, layout="tokens", pad=0):
    """float64 [B, N, H, d] -> (a view on the GPU in that layout, what it holds as float64).  pad: rows of memory with NaN between."""
    import torch
    t = torch.from_numpy(x).to(torch.bfloat16 if dtype == BF16 else torch.float32).cuda()
    B, N, H, d = t.shape
    if layout == "heads":
        m = torch.full((B, H, N + pad, d), float("nan"), dtype=t.dtype, device="cuda")
        v = m.transpose(1, 2)[:, :N]
    else:
        m = torch.full((B, N, H * d + 8 * pad), float("nan"), dtype=t.dtype, device="cuda")
        v = m[:, :, :H * d].unflatten(2, (H, d))
    v.copy_(t)
    return v, t.double().cpu().numpy()


def scattered(rng, lengths, page, entries, spare=3, fill=-1):
    """A block table whose pages lie anywhere in the pool, entries behind the length `fill`; and the pool's pages."""
    held = [-(-n // page) for n in lengths]
    n_pages = sum(held) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(lengths), entries), fill, np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


# ------------------------------------------------------------------------------------------------ pages and slots

def run_pages(new_len, length, table, free, n_free, page, N, ws=None):
    import torch
    import paper_2411_10803_amd as md
    t = [dev(np.asarray(a, np.int32)) for a in (new_len, length, table, free, [n_free])]
    missing = dev(np.array([77], np.int32))
    slots = torch.full((len(length), N), 99, dtype=torch.int32, device="cuda") if N else None
    md.mustdrop_cache4_pages(t[0], t[1], t[2], t[3], t[4], missing, page, slots=slots, workspace=ws)
    torch.cuda.synchronize()
    return host(t[1]), host(t[2]), host(t[3]), int(host(t[4])[0]), host(slots) if N else np.zeros((len(length), 0), np.int32), int(host(missing)[0])


def same_pages(got, want):
    for name, g, w in zip(("length", "table", "free", "n_free", "slots", "missing"), got, want):
        assert np.array_equal(g, w), name


@pytest.mark.parametrize("B, entries, page, N, spare, seed", [
    (1, 1, 16, 1, 0, 0), (1, 7, 16, 200, 2, 1), (3, 5, 32, 0, 1, 2), (64, 40, 32, 1, 9, 3), (65, 9, 64, 33, 0, 4), (7, 300, 16, 5000, 50, 5),
    (1023, 3, 16, 2, 5, 6), (1024, 3, 16, 40, 0, 7), (1025, 3, 128, 1, 4, 8), (3000, 2, 256, 3, 10, 9)])
def test_pages_and_slots(B, entries, page, N, spare, seed):
    rng = np.random.default_rng(seed)
    cap = entries * page
    length = rng.integers(0, cap + 1, B).astype(np.int32)
    new_len = rng.integers(0, cap + 1, B).astype(np.int32)
    new_len[rng.random(B) < 0.2] = 0
    table, n_pages = scattered(rng, length, page, entries, spare=0)
    need = int(sum(-(-n // page) for n in new_len))
    n_pages = max(n_pages, need) + spare
    held = set(table[table >= 0].tolist())
    free = rng.permutation([p for p in range(n_pages) if p not in held]).astype(np.int32)
    n_free = len(free)
    free = np.concatenate([free, np.full(n_pages - n_free, -5, np.int32)])
    want = ref.pages(new_len, length, table, free, n_free, page, N)
    assert want[5] == 0
    same_pages(run_pages(new_len, length, table, free, n_free, page, N), want)
    back = ref.pages(length, want[0], want[1], want[2], want[3], page, N)
    same_pages(run_pages(length, want[0], want[1], want[2], want[3], page, N), back)


def test_pages_that_the_pool_is_short_of():
    page, entries = 16, 10
    length, new_len = np.array([0, 33, 16], np.int32), np.array([100, 0, 160], np.int32)      # 7 + 9 pages wanted, 3 come back
    table = np.full((3, entries), -1, np.int32)
    table[1, :3], table[2, 0] = (4, 0, 7), 2
    free = np.array([9, 1, 3, 5, 6, 8, 10, 11, 12, 13, 14, 15, -1, -1, -1, -1], np.int32)
    for n_free, missing in ((12, 1), (5, 8), (0, 13)):
        want = ref.pages(new_len, length, table, free, n_free, page, 4)
        assert want[5] == missing
        same_pages(run_pages(new_len, length, table, free, n_free, page, 4), want)
    free[12] = 0
    want = ref.pages(new_len, length, table, free[:16], 13, page, 4)
    assert want[5] == 0
    same_pages(run_pages(new_len, length, table, free, 13, page, 4), want)


def test_pages_of_lengths_out_of_range():
    """Lengths below 0 or beyond the table's capacity are taken as its ends; pages that name nothing give no slot."""
    page, entries = 32, 4
    length, new_len = np.array([-7, 40, 0, 5], np.int32), np.array([1 << 30, -1, 33, 2 ** 31 - 1], np.int32)
    table = np.full((4, entries), -1, np.int32)
    table[1, :2], table[3, 0] = (3, 5), 1
    free = np.array([0, 2, 4, 6, 7, 8, 9, 10, 11, 12, 13, 14], np.int32)
    free = np.concatenate([free, np.full(4, -1, np.int32)])
    want = ref.pages(new_len, length, table, free, 12, page, 130)
    assert want[0].tolist() == [128, 0, 33, 128]
    same_pages(run_pages(new_len, length, table, free, 12, page, 130), want)
    table[3, 0] = 400                                                                       # no page of the pool
    got = run_pages([20], [5], table[3:], free, 12, page, 20)
    assert got[4].tolist() == [[-1] * 20] and got[5] == 0


# ------------------------------------------------------------------------------------------------ rows in and out

SPECIAL = np.array([0.0, -0.0, 1e-45, 1e-38, 2.0 ** -126, 2.0 ** -103, 2.0 ** -99, 3.3e38, -3.38e38, 6.5e4, 1.75, 1.7499, 3.5, 7.0, 6.99, 0.25, 2.5])


def make_rows(rng, B, N, H, d):
    """Rows of all sizes: groups of one magnitude, groups with borders between two levels, zeros, the ends of the range."""
    x = rng.standard_normal((B, N, H, d)) * np.exp2(rng.integers(-40, 40, (B, N, H, 1)).astype(float))
    ties = rng.random((B, N, H, 1)) < 0.2
    x = np.where(ties, rng.choice([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0, 4.0, 0.5], x.shape), x)
    special = rng.random((B, N, H, 1)) < 0.1
    x = np.where(special, rng.choice(SPECIAL, x.shape), x)
    return np.where(rng.random((B, N, H, 1)) < 0.05, 0.0, x)


@pytest.mark.parametrize("B, N, H, d, page, dtype, layout", [
    (1, 1, 1, 128, 16, BF16, "tokens"), (1, 1, 1, 64, 16, F32, "heads"), (3, 5, 4, 128, 32, BF16, "heads"), (2, 33, 3, 64, 32, BF16, "tokens"),
    (4, 1, 5, 128, 64, F32, "tokens"), (2, 18, 2, 64, 128, F32, "tokens"), (5, 7, 1, 128, 256, BF16, "tokens"), (1, 70, 2, 128, 16, F32, "heads")])
def test_rows_in_and_out(B, N, H, d, page, dtype, layout):
    import torch
    import paper_2411_10803_amd as md
    rng = np.random.default_rng(B * 1000 + N)
    k, kh = rows_on_gpu(make_rows(rng, B, N, H, d), dtype, layout, pad=2)
    v, vh = rows_on_gpu(make_rows(rng, B, N, H, d), dtype, layout, pad=2)
    if N > 4:                                          # a group with an infinity, one with a NaN
        k[0, 1, 0, 3], v[0, 2, H - 1, d - 1] = float("inf"), float("nan")
        kh[0, 1, 0, 3], vh[0, 2, H - 1, d - 1] = np.inf, np.nan
    first = rng.integers(0, 2 * page, B).astype(np.int32)
    length = first + rng.integers(1, N + 1, B).astype(np.int32)
    length[0] = first[0] + N
    entries = int(-(-length.max() // page)) + 1
    table, n_pages = scattered(rng, length, page, entries)
    slots = np.full((B, N), -1, np.int32)
    pool = rng.integers(0, 256, (n_pages, H, ref.page_bytes(page, d)), dtype=np.uint8)
    want = pool.copy()
    for b in range(B):
        for i in range(length[b] - first[b]):
            at = first[b] + i
            slots[b, i] = table[b, at // page] * page + at % page
            for h in range(H):
                ref.put(want, slots[b, i], h, kh[b, i, h], vh[b, i, h], page)
    slots[slots < 0] = rng.choice([-1, -2 ** 31, n_pages * page, 2 ** 31 - 1], int((slots < 0).sum()))      # none of these is a slot
    cache = dev(pool)
    assert tuple(md.cache4_buffer(n_pages, page, H, d).shape) == tuple(cache.shape)
    md.mustdrop_cache4_write(k, v, dev(slots), cache)
    torch.cuda.synchronize()
    assert np.array_equal(ref.undefined_codes(host(cache), page, d), ref.undefined_codes(want, page, d))
    for out_type, out_layout in ((dtype, layout), (F32 if dtype == BF16 else BF16, "tokens")):
        ko, _ = rows_on_gpu(np.full((B, N, H, d), 7.0), out_type, out_layout, pad=1)
        vo, _ = rows_on_gpu(np.full((B, N, H, d), 7.0), out_type, out_layout, pad=1)
        md.mustdrop_cache4_read(cache, dev(table), dev(length), ko, vo, first=dev(first))
        torch.cuda.synchronize()
        ko, vo = host(ko), host(vo)
        for b in range(B):
            n = length[b] - first[b]
            assert (ko[b, n:] == 7).all() and (vo[b, n:] == 7).all()
            for i in range(n):
                for h in range(H):
                    gk, gv = ref.get(want, slots[b, i], h, d, page)
                    assert np.array_equal(ko[b, i, h], gk.astype(np.float32), equal_nan=True), (b, i, h)
                    assert np.array_equal(vo[b, i, h], gv.astype(np.float32), equal_nan=True), (b, i, h)


@pytest.mark.parametrize("B, N, H, d, dtype, layout", [(3, 3001, 9, 128, BF16, "heads"), (2, 5003, 7, 64, F32, "tokens"), (1, 16400, 5, 128, F32, "heads"),
                                                       (5, 1300, 13, 64, BF16, "tokens")])
def test_many_rows_are_what_few_rows_are(B, N, H, d, dtype, layout):
    """A call of many rows takes several heads per wave: the same bytes as its pieces of few rows, which the test above checks."""
    import torch
    import paper_2411_10803_amd as md
    page = 64
    rng = np.random.default_rng(N)
    length = np.full(B, N, np.int32)
    length[-1] -= 77
    table, n_pages = scattered(rng, length, page, -(-N // page))
    at = np.arange(N)
    slots = dev(np.where(at < length[:, None], table[:, at // page] * page + at % page, -1).astype(np.int32))
    k, _ = rows_on_gpu(rng.standard_normal((B, N, H, d)), dtype, layout, pad=1)
    v, _ = rows_on_gpu(rng.standard_normal((B, N, H, d)), dtype, layout, pad=1)
    whole, parts = (torch.full_like(md.cache4_buffer(n_pages, page, H, d), 0x5A) for _ in range(2))
    md.mustdrop_cache4_write(k, v, slots, whole)
    for i in range(0, N, 999):
        md.mustdrop_cache4_write(k[:, i:i + 999], v[:, i:i + 999], slots[:, i:i + 999].contiguous(), parts)
    torch.cuda.synchronize()
    assert torch.equal(whole, parts)
    table, length = dev(table), dev(length)
    out = [rows_on_gpu(np.full((B, N, H, d), 7.0), dtype, layout, pad=1)[0] for _ in range(4)]
    md.mustdrop_cache4_read(whole, table, length, out[0], out[1])
    for i in range(0, N, 999):
        first = torch.full((B,), i, dtype=torch.int32, device="cuda")
        md.mustdrop_cache4_read(whole, table, length, out[2][:, i:i + 999], out[3][:, i:i + 999], first=first)
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    assert (out[0][-1, -77:] == 7).all() and not (out[0][-1, :-77] == 7).all()


def test_rows_out_of_bad_pages_and_places_are_left_alone():
    import torch
    import paper_2411_10803_amd as md
    d, H, page = 64, 2, 16
    cache = dev(np.random.default_rng(0).integers(0, 200, (4, H, ref.page_bytes(page, d)), dtype=np.uint8))
    table = dev(np.array([[0, 4, -1, 2 ** 31 - 1], [-2 ** 31, 1, 2, 3]], np.int32))
    length, first = dev(np.array([64, 1000], np.int32)), dev(np.array([-3, 60], np.int32))
    ko, vo = (torch.full((2, 70, H, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    md.mustdrop_cache4_read(cache, table, length, ko, vo, first=first)
    torch.cuda.synchronize()
    there = np.zeros((2, 70), bool)
    there[0, 3:19] = True                              # entries 0..15 of the one page that exists
    there[1, :4] = True                                # entries 60..63: the table ends there
    for t in (ko, vo):
        left = (host(t) == 7).all((2, 3))
        assert np.array_equal(~left, there)


# ------------------------------------------------------------------------------------------------ attention

class Case:
    """Inputs of one attention call, on both sides."""

    def __init__(self, seed, lengths, N, Hq, H, d, page, dtype, q_len=None, keep=None, layout="tokens", entries=None, size=1.0, heavy=True, spread=0):
        import torch
        rng = np.random.default_rng(seed)
        B = len(lengths)
        self.B, self.N, self.Hq, self.H, self.d, self.page, self.dtype, self.lengths = B, N, Hq, H, d, page, dtype, list(lengths)
        entries = entries or max(1, -(-max(lengths) // page) + 1)
        self.table, n_pages = scattered(rng, lengths, page, entries, fill=2 ** 31 - 1)
        # what nobody wrote reads as NaN
        self.pool = np.full((n_pages, H, ref.page_bytes(page, d)), 255, np.uint8)
        reach = min(entries, -(-max(max(lengths), 1) // page)) * page
        self.K, self.V = np.zeros((B, reach, H, d)), np.zeros((B, reach, H, d))
        for b, n in enumerate(lengths):
            k, v = rng.standard_normal((n, H, d)) * size, rng.standard_normal((n, H, d))
            if heavy and n:
                k += 1.2 * (rng.random((n, 1, 1)) < 0.05)
            for t in range(n):
                for h in range(H):
                    ref.put(self.pool, self.table[b, t // page] * page + t % page, h, k[t, h], v[t, h], page)
                    self.K[b, t, h], self.V[b, t, h] = ref.values(*ref.quantise(k[t, h])), ref.values(*ref.quantise(v[t, h]))
        q = rng.standard_normal((B, N, Hq, d)) + 0.3
        if spread:                                     # channels of all sizes
            q *= np.exp2(rng.integers(-spread, 1, q.shape).astype(float))
        self.q, self.qh = rows_on_gpu(q, dtype, layout, pad=1)
        self.there = np.ones((B, reach), bool)
        self.q_len = None if q_len is None else np.asarray(q_len, np.int32)
        self.keep = keep
        if keep is not None and not isinstance(keep, np.ndarray):
            self.keep = (rng.random((B, entries * page)) < keep).astype(np.uint8) * rng.integers(1, 256, (B, entries * page)).astype(np.uint8)
        self.scale = 1.0 / np.sqrt(d)
        self.layout = layout

    def call(self, md, **kw):
        import torch
        out, _ = rows_on_gpu(np.full((self.B, self.N, self.Hq, self.d), 7.0), self.dtype, self.layout, pad=1)
        lse = torch.full((self.B, self.Hq, self.N), 7.0, device="cuda")
        opt = lambda a: None if a is None else dev(a)  # noqa: E731
        md.mustdrop_cache4_attend(self.q, dev(self.pool), dev(self.table), dev(np.asarray(self.lengths, np.int32)), self.scale, out=out, lse=lse,
                                  q_len=opt(self.q_len), keep=opt(self.keep), **kw)
        torch.cuda.synchronize()
        return host(out).astype(np.float64), host(lse).astype(np.float64)

    def check(self, out, lse, nan_rows=()):
        # bf16 rows: probabilities in two bf16 parts, 16 bits; where 32 rows go together, in one, whose rounding is off by half a
        # step, 2^-8, at most; fp32 rows: in three bf16 parts, 24 bits
        rows = self.N * self.Hq // self.H
        many = self.dtype == BF16 and rows > 16 and self.B * self.H * -(-rows // 16) > 512
        step, part = (2.0 ** -8, 2.0 ** -8 if many else 2.0 ** -16) if self.dtype == BF16 else (2.0 ** -24, 2.0 ** -23)
        for b in range(self.B):
            nq = self.N if self.q_len is None else int(np.clip(self.q_len[b], 0, self.N))
            n = int(np.clip(self.lengths[b], 0, self.table.shape[1] * self.page))
            want, wl_, size, score = ref.attend(self.qh[b], self.K[b], self.V[b], self.there[b], n, nq, self.scale,
                                                None if self.keep is None else self.keep[b, :self.K.shape[1]])
            assert (out[b, nq:] == 7).all() and (lse[b, :, nq:] == 7).all(), f"sample {b}: rows behind the last were written"
            bound, lbound = ref.attend_bounds(want, wl_, size, score, self.d, n, step, part)
            got = out[b, :nq]
            assert np.array_equal(np.isnan(got), np.isnan(want[:nq])), f"sample {b}: NaN"
            off = np.where(np.isnan(got), 0, np.abs(got - want[:nq]) - bound[:nq])
            assert (off <= 0).all(), f"sample {b}: {np.argwhere(off > 0)[:3]} off by {off.max()} more than the bound"
            gl, wlse = lse[b, :, :nq].T, wl_[:nq]
            empty = np.isneginf(wlse)
            assert np.array_equal(np.isneginf(gl), empty) and (got[empty] == 0).all(), f"sample {b}: empty rows"
            ok = np.where(empty | np.isnan(wlse), True, np.abs(gl - np.where(empty, 0, wlse)) <= lbound[:nq])
            assert ok.all(), f"sample {b}: lse"


CASES = [
    # lengths of nothing, one, and around the 16- and 32-key steps
    dict(lengths=[0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 100], N=1, Hq=2, H=2, d=128, page=16, dtype=BF16),
    dict(lengths=[0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 100], N=1, Hq=2, H=2, d=64, page=32, dtype=F32),
    # heads that share: 3, 4, 5, 7 and 8 to one; more than one tile of query rows
    dict(lengths=[130, 77], N=1, Hq=6, H=2, d=128, page=32, dtype=BF16),
    dict(lengths=[300, 5], N=1, Hq=20, H=4, d=64, page=64, dtype=BF16),
    dict(lengths=[200, 129], N=2, Hq=7, H=1, d=128, page=16, dtype=F32),
    dict(lengths=[64, 33], N=3, Hq=8, H=1, d=128, page=128, dtype=BF16),
    dict(lengths=[500], N=1, Hq=40, H=1, d=64, page=256, dtype=BF16),
    # drafts and pieces of a prompt; rows that stand before the first entry; samples with fewer rows, none, or out of range
    dict(lengths=[5, 4, 40, 0, 3], N=5, Hq=4, H=2, d=128, page=16, dtype=BF16),
    dict(lengths=[90, 60, 17, 31], N=17, Hq=2, H=2, d=64, page=32, dtype=BF16, q_len=[17, 3, -4, 99]),
    dict(lengths=[70, 70, 200], N=70, Hq=4, H=2, d=128, page=64, dtype=F32, q_len=[70, 33, 0]),
    dict(lengths=[150, 400], N=130, Hq=3, H=1, d=128, page=32, dtype=BF16, q_len=[130, 129]),
    # masks
    dict(lengths=[100, 50, 333], N=1, Hq=4, H=4, d=128, page=32, dtype=BF16, keep=0.5),
    dict(lengths=[100, 50, 333], N=6, Hq=4, H=2, d=64, page=16, dtype=F32, keep=0.05),
    dict(lengths=[100, 50], N=4, Hq=4, H=2, d=128, page=16, dtype=BF16, keep=0.0),
    # head-major and padded views; large scores
    dict(lengths=[97, 160], N=9, Hq=8, H=4, d=128, page=32, dtype=BF16, layout="heads"),
    dict(lengths=[97, 160], N=2, Hq=4, H=4, d=64, page=32, dtype=F32, layout="heads", keep=0.7),
    dict(lengths=[260, 31], N=2, Hq=4, H=2, d=128, page=32, dtype=BF16, size=30.0),
    dict(lengths=[260, 31], N=1, Hq=4, H=2, d=128, page=32, dtype=F32, size=2000.0),
    # longer: every wave has many steps
    dict(lengths=[3001, 1500, 1], N=1, Hq=2, H=1, d=128, page=32, dtype=BF16),
    dict(lengths=[2500, 700], N=20, Hq=4, H=2, d=64, page=64, dtype=BF16),
    dict(lengths=[2000], N=40, Hq=4, H=1, d=128, page=16, dtype=F32),
    # runs of equal work over the borders of samples, some of them empty; more than 64 samples; many rows
    dict(lengths=[0, 700, 1, 33, 0, 1234, 64], N=3, Hq=4, H=2, d=128, page=16, dtype=BF16, entries=200, q_len=[3, 3, 1, 0, 2, 3, 3]),
    dict(lengths=[0, 700, 1, 33, 0, 1234, 64], N=3, Hq=4, H=2, d=64, page=16, dtype=F32, entries=200, keep=0.6),
    dict(lengths=[(37 * b) % 90 for b in range(150)], N=1, Hq=1, H=1, d=64, page=256, dtype=BF16, entries=65),
    dict(lengths=[300, 40, 90], N=90, Hq=12, H=2, d=64, page=256, dtype=BF16, entries=65, q_len=[90, 41, 90]),
    dict(lengths=[1], N=1, Hq=3, H=3, d=128, page=32, dtype=BF16, entries=400),
    # eight waves to a block: short sequences in tables of 512 entries
    dict(lengths=[500, 3, 130, 0], N=1, Hq=5, H=5, d=128, page=64, dtype=BF16, entries=8),
    dict(lengths=[500, 3, 130, 0], N=2, Hq=6, H=3, d=64, page=64, dtype=F32, entries=8, keep=0.5),
    # 32 rows together, in blocks per unit and in runs
    dict(lengths=[(29 * b) % 80 for b in range(22)], N=20, Hq=13, H=13, d=64, page=32, dtype=BF16, entries=16, q_len=[(7 * b) % 24 for b in range(22)]),
    dict(lengths=[(29 * b) % 80 for b in range(22)], N=20, Hq=13, H=13, d=128, page=256, dtype=BF16, entries=65),
    dict(lengths=[50] * 40, N=9, Hq=28, H=7, d=128, page=16, dtype=BF16, entries=16, keep=0.7, layout="heads"),
    # queries whose channels are far apart
    dict(lengths=[260, 31], N=2, Hq=4, H=2, d=128, page=32, dtype=BF16, spread=30, size=8.0),
    dict(lengths=[260, 31], N=2, Hq=4, H=2, d=128, page=32, dtype=BF16, spread=13, size=8.0),
    dict(lengths=[260, 31], N=2, Hq=4, H=2, d=64, page=32, dtype=BF16, spread=30, size=8.0),
    # 32 rows together in more than 64 samples, which are taken by their length; many are as long as others, some have no rows
    dict(lengths=[(23 * b) % 61 for b in range(70)], N=40, Hq=4, H=2, d=64, page=16, dtype=BF16, entries=8, q_len=[(7 * b) % 44 - 2 for b in range(70)]),
    dict(lengths=[40 - b % 3 for b in range(66)], N=33, Hq=4, H=2, d=128, page=32, dtype=BF16, entries=2),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_attend(i):
    import paper_2411_10803_amd as md
    c = Case(100 + i, **CASES[i])
    out, lse = c.call(md)
    c.check(out, lse)
    again, lse2 = c.call(md)
    assert np.array_equal(out, again) and np.array_equal(lse, lse2)             # the same bits


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_are_exact_where_fp32_sums_are(d, dtype):
    """Integers whose products and partial sums stay below 2^24 have the same sum in fp32 in any order: a row that sees one key has its score
    as lse but for six roundings of 2^-24 each (log2(e), its product with the scale, that with the score, the sum with log2 of a sum near 1, ln 2, its
    product) and a unit each of exp2 and log2 near 1, 2^-22 together."""
    rng = np.random.default_rng(d)
    c = Case(5, [1] * 40, 1, 8, 4, d, 16, dtype)
    q = rng.integers(-127, 128, c.qh.shape) * np.exp2(rng.integers(0, 3, c.qh.shape))
    q[..., rng.integers(0, d)] = 2.0 ** 14                       # a product of 12 * 2^14 beside sums of many small ones
    c.q, c.qh = rows_on_gpu(q, dtype)
    assert np.array_equal(c.qh, q)
    for b in range(40):
        for h in range(4):
            k = rng.integers(-12, 13, d).astype(float)
            ref.put(c.pool, int(c.table[b, 0]) * 16, h, k, k, 16)
            c.K[b, 0, h] = ref.values(*ref.quantise(k))
    assert np.array_equal(c.K[:, 0], np.round(c.K[:, 0] * 4) / 4) and (np.abs(c.K[:, 0]).max() * np.abs(q)).sum(-1).max() * 4 < 2 ** 24
    _, lse = c.call(__import__("paper_2411_10803_amd"))
    want = np.einsum("bhd,bhd->bh", c.qh[:, 0], np.repeat(c.K[:, 0], 2, axis=1)) * np.float64(np.float32(c.scale))
    assert (np.abs(lse[:, :, 0] - want) <= 6 * 2.0 ** -24 * np.abs(want) + 2.0 ** -22).all()


def test_attend_over_lengths_out_of_range_and_bad_pages():
    import paper_2411_10803_amd as md
    c = Case(7, [96, 96, 96, 80], 3, 4, 2, 128, 16, BF16, entries=6)
    c.lengths = [10 ** 6, -3, 96, 80]                                            # taken as 96 (six pages of 16) and 0
    for b, e, bad in ((0, 1, -1), (0, 5, 10 ** 9), (2, 0, -2 ** 31), (2, 3, len(c.pool)), (3, 4, 2 ** 31 - 1)):
        c.table[b, e] = bad
        c.there[b, e * 16:e * 16 + 16] = False
    c.check(*c.call(md))
    c.table[:] = -1
    c.there[:] = False
    c.check(*c.call(md))


@pytest.mark.parametrize("dtype, d", ((BF16, 128), (F32, 64)))
def test_attend_nan_reaches_only_the_rows_that_see_it(dtype, d):
    import paper_2411_10803_amd as md
    c = Case(9, [75, 75, 75, 40], 6, 4, 2, d, 16, dtype, keep=1.0)
    page = c.page

    def poison(b, t, h, k=False, v=False):
        nan = np.full(d, 1.0)
        nan[33] = np.nan                                                         # the second group only
        kk, vv = c.K[b, t, h].copy(), c.V[b, t, h].copy()
        if k:
            kk[33] = np.nan
        if v:
            vv[33] = np.nan
        ref.put(c.pool, c.table[b, t // page] * page + t % page, h, kk, vv, page)
        if k:
            c.K[b, t, h, 32:64] = np.nan
        if v:
            c.V[b, t, h, 32:64] = np.nan
    poison(0, 72, 0, v=True)                                                     # rows 0..2 of six stand before entry 72
    poison(1, 73, 1, k=True)
    poison(2, 10, 0, k=True, v=True)
    c.keep[2, 10] = 0                                                            # masked: may hold anything
    poison(3, 5, 1, v=True)                                                      # all rows see it
    want = ref.attend(c.qh[3], c.K[3], c.V[3], c.there[3], 40, 6, c.scale)[0]
    assert np.isnan(want[:, 2:, 32:64]).all() and not np.isnan(want[:, 2:, :32]).any()
    # entries that a row does not see take no part: the reference sums over the seen ones only
    c.check(*c.call(md))


def test_attend_in_a_pool_beyond_four_gigabytes():
    import torch
    import paper_2411_10803_amd as md
    c = Case(11, [70, 40], 2, 8, 8, 128, 32, BF16)
    n_pages, H = 131072, 8                                                       # 4.56 GB of pages; the last ones are used
    far = n_pages - len(c.pool)
    assert (n_pages - 1) * H * ref.page_bytes(32, 128) > 1 << 32
    cache = torch.empty((n_pages, H, ref.page_bytes(32, 128)), dtype=torch.uint8, device="cuda")
    cache[far:] = dev(c.pool)
    table = np.where((c.table >= 0) & (c.table < len(c.pool)), c.table + far, c.table).astype(np.int32)
    out = torch.full((2, 2, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((2, 8, 2), 7.0, device="cuda")
    md.mustdrop_cache4_attend(c.q, cache, dev(table), dev(np.array([70, 40], np.int32)), c.scale, out=out, lse=lse)
    torch.cuda.synchronize()
    c.check(host(out).astype(np.float64), host(lse).astype(np.float64))
    # rows in and out there
    k = torch.randn((1, 3, 8, 128), device="cuda").bfloat16()
    slots = torch.arange(n_pages * 32 - 3, n_pages * 32, dtype=torch.int32, device="cuda")[None].contiguous()
    md.mustdrop_cache4_write(k, k, slots, cache)
    ko, vo = torch.zeros_like(k), torch.zeros_like(k)
    md.mustdrop_cache4_read(cache, dev(np.array([[n_pages - 1]], np.int32)), dev(np.array([32], np.int32)), ko, vo, first=dev(np.array([29], np.int32)))
    torch.cuda.synchronize()
    want = ref.values(*ref.quantise(host(k)))
    assert np.array_equal(host(ko), want) and np.array_equal(host(vo), want)


# ------------------------------------------------------------------------------------------------ used together

def decode_program(md, torch, B, H, Hq, d, page, prompt, steps, entries, N):
    """What a serving loop keeps: pool, tables, lengths; and its step."""
    s = {"cache": md.cache4_buffer(B * entries, page, H, d), "table": torch.full((B, entries), -1, dtype=torch.int32, device="cuda"),
         "length": torch.zeros(B, dtype=torch.int32, device="cuda"), "new_len": torch.zeros(B, dtype=torch.int32, device="cuda"),
         "free": torch.arange(B * entries, dtype=torch.int32, device="cuda"), "n_free": dev(np.array([B * entries], np.int32)),
         "missing": torch.zeros(1, dtype=torch.int32, device="cuda"), "slots": torch.zeros((B, N), dtype=torch.int32, device="cuda"),
         "out": torch.zeros((B, N, Hq, d), dtype=torch.bfloat16, device="cuda"), "lse": torch.zeros((B, Hq, N), device="cuda"),
         "pages_ws": md.cache4_pages_workspace(B)}

    def step(k, v, q, grow, q_len=None, stream=None):
        torch.add(s["length"], grow, out=s["new_len"])
        md.mustdrop_cache4_pages(s["new_len"], s["length"], s["table"], s["free"], s["n_free"], s["missing"], page, slots=s["slots"],
                                 workspace=s["pages_ws"], stream=stream)
        md.mustdrop_cache4_write(k, v, s["slots"], s["cache"], stream=stream)
        if "ws" not in s:
            s["ws"] = md.cache4_workspace(q, s["cache"], s["table"])
        md.mustdrop_cache4_attend(q, s["cache"], s["table"], s["length"], 1.0 / np.sqrt(d), out=s["out"], lse=s["lse"], q_len=q_len,
                                  workspace=s["ws"], stream=stream)
    return s, step


def test_prefill_to_cache_to_decode_to_eviction():
    """The rows that the prefill stage keeps go into the cache; decode steps append and attend; the cache comes back as dense rows
    and the eviction stage runs on them."""
    import torch
    import paper_2411_10803_amd as md
    from paper_2411_10803_amd import harness
    cfg = wl.tiny(wl.CONFIGS[2], B=3, H=4)
    t = wl.prefill_inputs(cfg)
    R, Mv, N, H, d, B, page = 40, cfg.M, cfg.N, cfg.H, cfg.d, 3, 16
    txt_len = np.array([N, 1, N // 2], np.int32)
    pre = md.mustdrop_prefill_filter(harness.to_dev(t["q_txt"], True), harness.to_dev(t["k"], True), harness.to_dev(t["v"], True),
                                     harness.to_dev(t["hidden"], True), None, harness.to_dev(txt_len), None, Mv, 1 / np.sqrt(d), md.FILTER_BUDGET,
                                     R, 1.0 / Mv, 2.0 / (Mv + N), Rcap=R)
    entries = -(-(R + N + 5) // page)
    s, step = decode_program(md, torch, B, H, H, d, page, R + N, 4, entries, R + N)
    # the whole kept prompt as one piece: every sample has its own number of rows
    q = torch.randn((B, R + N, H, d), device="cuda").bfloat16()
    step(pre["k_out"], pre["v_out"], q, pre["out_len"], q_len=pre["out_len"])
    rng = np.random.default_rng(1)
    keys = [[host(pre["k_out"])[b, i] for i in range(int(pre["out_len"][b]))] for b in range(B)]
    vals = [[host(pre["v_out"])[b, i] for i in range(int(pre["out_len"][b]))] for b in range(B)]
    K = lambda b: ref.values(*ref.quantise(np.stack(keys[b])))  # noqa: E731
    V = lambda b: ref.values(*ref.quantise(np.stack(vals[b])))  # noqa: E731

    def check(q, out, lse, rows):
        for b in range(B):
            n = len(keys[b])
            want, wlse, size, score = ref.attend(host(q)[b].astype(np.float64), K(b), V(b), np.ones(n, bool), n, rows[b], 1 / np.sqrt(d))
            bound, lb = ref.attend_bounds(want, wlse, size, score, d, n, 2.0 ** -8, 2.0 ** -16)
            assert (np.abs(host(out)[b, :rows[b]] - want[:rows[b]]) <= bound[:rows[b]]).all()
            assert (np.abs(host(lse)[b, :, :rows[b]].T - wlse[:rows[b]]) <= lb[:rows[b]]).all()
    torch.cuda.synchronize()
    check(q, s["out"], s["lse"], [len(k) for k in keys])
    one = {"slots": torch.zeros((B, 1), dtype=torch.int32, device="cuda"), "out": torch.zeros((B, 1, H, d), dtype=torch.bfloat16, device="cuda"),
           "lse": torch.zeros((B, H, 1), device="cuda")}
    s.update(one)
    del s["ws"]
    for _ in range(4):
        k, v, q = (torch.from_numpy(rng.standard_normal((B, 1, H, d))).cuda().bfloat16() for _ in range(3))
        step(k, v, q, 1)
        torch.cuda.synchronize()
        for b in range(B):
            keys[b].append(host(k)[b, 0])
            vals[b].append(host(v)[b, 0])
        check(q, s["out"], s["lse"], [1] * B)
    assert int(s["missing"][0]) == 0
    # back to dense rows, and the eviction on them
    cap = entries * page
    dense = {n: torch.zeros((B, cap, H, d), dtype=torch.bfloat16, device="cuda") for n in "kv"}
    md.mustdrop_cache4_read(s["cache"], s["table"], s["length"], dense["k"], dense["v"])
    torch.cuda.synchronize()
    for b in range(B):
        n = len(keys[b])
        assert np.array_equal(host(dense["k"])[b, :n], K(b)) and np.array_equal(host(dense["v"])[b, :n], V(b))
    acc = torch.zeros((B, cap), device="cuda")
    ids = torch.arange(cap, dtype=torch.int32, device="cuda").repeat(B, 1).contiguous()
    protect = torch.zeros((B, cap), dtype=torch.uint8, device="cuda")
    length = s["length"].clone()
    md.mustdrop_decode_evict(q[:, 0].contiguous(), dense["k"], dense["v"], acc, ids, protect, length, 1 / np.sqrt(d), 1.0, 24)
    torch.cuda.synchronize()
    assert host(length).tolist() == [min(24, len(k)) for k in keys]
    for b in range(B):
        n = int(length[b])
        left = host(ids)[b, :n]
        assert np.array_equal(host(dense["k"])[b, :n], K(b)[left]) and np.array_equal(host(dense["v"])[b, :n], V(b)[left])


@pytest.mark.parametrize("entries", [8, 800])                                    # of a block table; 800: attention in runs
def test_decode_step_in_a_graph(entries):
    """Pages, rows and attention of a step in one graph, replayed with eager steps of a second program between; both agree bit for bit."""
    import torch
    import paper_2411_10803_amd as md
    B, H, Hq, d, page = 5, 2, 8, 128, 16
    made = [decode_program(md, torch, B, H, Hq, d, page, 0, 0, entries, 1) for _ in range(2)]
    k, v = (torch.zeros((B, 1, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((B, 1, Hq, d), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)

    def fresh():
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    for s, step in made:                                # warm up, one eager step each
        g.manual_seed(3)
        fresh()
        step(k, v, q, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made[0][1](k, v, q, 1)
    for n in range(40):                                 # over several pages
        fresh()
        torch.cuda.synchronize()
        graph.replay()
        made[1][1](k, v, q, 1)
        torch.cuda.synchronize()
        for name in ("cache", "table", "length", "free", "n_free", "missing", "slots", "out", "lse"):
            assert torch.equal(made[0][0][name], made[1][0][name]), (n, name)
    assert host(made[0][0]["length"]).tolist() == [41] * B


def test_two_graphs_with_one_workspace():
    """What a call leaves in its workspace is nobody's: two graphs that take turns on one give what eager calls give, replay after replay."""
    import torch
    import paper_2411_10803_amd as md
    cases = [Case(31, [2000, 900], 1, 4, 2, 128, 32, BF16, entries=600), Case(32, [70, 4000], 2, 4, 2, 128, 32, BF16, entries=600)]
    args = [[c.q, dev(c.pool), dev(c.table), dev(np.asarray(c.lengths, np.int32)), c.scale] for c in cases]
    ws = max((md.cache4_workspace(a[0], a[1], a[2]) for a in args), key=lambda w: w.numel())
    want = [md.mustdrop_cache4_attend(*a) for a in args]
    out = [torch.zeros_like(w) for w in want]
    graphs = []
    for a, o in zip(args, out):
        md.mustdrop_cache4_attend(*a, out=o, workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            md.mustdrop_cache4_attend(*a, out=o, workspace=ws)
    for n in range(5):
        for o in out:
            o.fill_(9)
        ws.fill_(255)
        graphs[n % 2].replay()
        graphs[1 - n % 2].replay()
        md.mustdrop_cache4_attend(*args[0], workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), n


def test_two_programs_on_two_streams():
    """Two batches in flight at once, each with its own state and workspaces, give what each gives alone."""
    import torch
    import paper_2411_10803_amd as md
    B, H, Hq, d, page, entries = 7, 4, 4, 64, 32, 30
    streams = [torch.cuda.Stream() for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(5)
    inputs = [[tuple(torch.randn((B, n, h, d), generator=g, device="cuda").bfloat16() for h in (H, H, Hq)) for n in [300] * 3] for _ in range(2)]
    results = []
    for together in (False, True):
        got = []
        made = [decode_program(md, torch, B, H, Hq, d, page, 0, 0, entries, 300) for _ in range(2)]
        torch.cuda.synchronize()
        for i in range(3):
            for p in range(2):
                with torch.cuda.stream(streams[p]):
                    made[p][1](*inputs[p][i], 300)
                if not together:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        results.append([{n: s[n].clone() for n in ("cache", "table", "length", "out", "lse")} for s, _ in made])
    for a, b in zip(*results):
        for n in a:
            assert torch.equal(a[n], b[n]), n


def test_a_given_stream_is_used():
    import torch
    import paper_2411_10803_amd as md
    c = Case(21, [200, 90], 1, 4, 2, 128, 32, BF16)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, lse = c.call(md, stream=s)
    c.check(out, lse)


def test_what_a_call_makes_belongs_to_its_stream():
    """The workspace and `out` of a call on a given stream, which the call makes: the current stream may not get that memory while the call runs."""
    import torch
    import paper_2411_10803_amd as md
    c = Case(22, [3000, 1700], 1, 4, 2, 128, 32, BF16, entries=600)              # in runs: with sums in the workspace
    args = [c.q, dev(c.pool), dev(c.table), dev(np.asarray(c.lengths, np.int32)), c.scale]
    want = md.mustdrop_cache4_attend(*args)
    size = md.cache4_workspace(args[0], args[1], args[2]).numel()
    s = torch.cuda.Stream()
    busy = torch.ones(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(8):
            busy @ busy
    out = md.mustdrop_cache4_attend(*args, stream=s)
    over = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)] + [torch.full_like(want, 9) for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and len(over) == 8
