"""The cache held in 4 bits without a GPU: its page arithmetic, the 64-bit reference that the GPU tests use, and every refusal."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

import cache4_ref as ref
import paper_2411_10803_amd as md

HERE = os.path.dirname(os.path.abspath(__file__))
OK, EINVAL, ESHAPE, EALIGN, EALIAS, EWORKSPACE, EDTYPE = range(7)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
def test_page_arithmetic(tmp_path):
    exe = str(tmp_path / "cache4_plan")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           os.path.join(HERE, "plan", "cache4_plan_main.cpp"), "-o", exe])
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]


# ---- the reference itself
def test_reference_rounds_to_the_nearest_and_ties_to_even():
    x = np.zeros(32)
    x[:12] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.26, -0.74, 6.9, -1.0]
    code, scale = ref.quantise(x)
    assert scale.tolist() == [127]                             # 6.9 rounds to 6: the scale stays 1
    got = ref.values(code, scale)[:12]
    assert got.tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.5, -0.5, 6.0, -1.0]
    x[10] = 7.0                                                # would be cut down: the next scale
    assert ref.quantise(x)[1].tolist() == [128]


def test_reference_errors_stay_within_what_the_header_says():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4000, 32)) * np.exp2(rng.integers(-30, 30, (4000, 1)).astype(float))
    y = ref.values(*ref.quantise(x))
    most = np.abs(x).max(-1, keepdims=True)
    assert np.all(np.abs(y - x) <= most / 5)
    large = np.abs(x) >= most / 4
    assert np.all(np.abs(y - x)[large] <= np.abs(x)[large] / 5)


def test_reference_edges():
    assert ref.quantise(np.zeros(32))[1].tolist() == [27]
    assert ref.quantise(np.full(32, 2.0 ** -140))[1].tolist() == [27]
    top = np.full(32, 3.38e38)
    code, scale = ref.quantise(top)
    assert scale.tolist() == [252] and ref.values(code, scale)[0] == 6 * 2.0 ** 125
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(64)
        x[40] = bad
        code, scale = ref.quantise(x)
        y = ref.values(code, scale)
        assert scale.tolist()[1] == 255 and np.isnan(y[32:]).all() and (y[:32] == 1).all()


def test_reference_pages_round_trip():
    rng = np.random.default_rng(1)
    for d, page in ((64, 16), (128, 32)):
        pool = rng.integers(0, 256, (3, 2, ref.page_bytes(page, d)), dtype=np.uint8)
        rows = {}
        for slot in rng.permutation(3 * page)[:40]:
            for h in range(2):
                k, v = rng.standard_normal(d), rng.standard_normal(d)
                ref.put(pool, slot, h, k, v, page)
                rows[slot, h] = k, v
        for (slot, h), (k, v) in rows.items():
            gk, gv = ref.get(pool, slot, h, d, page)
            assert np.array_equal(gk, ref.values(*ref.quantise(k))) and np.array_equal(gv, ref.values(*ref.quantise(v)))


# ---- refusals of the C entries, before any launch: the pointers are never followed
def P(i):
    return C.c_void_p(0x100000000 + i * 0x40000000)


BIG = C.c_size_t(1 << 40)


@pytest.fixture(scope="module")
def lib():
    return md.library()


def pages(lib, **kw):
    a = dict(new_len=P(1), len=P(2), table=P(3), free=P(4), n_free=P(5), slots=P(6), missing=P(7), B=3, max_pages=8, n_pages=30, page=32, N=2,
             ws=P(8), wsb=BIG)
    a.update(kw)
    return lib.mustdrop_cache4_pages(*[a[n] for n in ("new_len", "len", "table", "free", "n_free", "slots", "missing", "B", "max_pages", "n_pages",
                                                      "page", "N", "ws", "wsb")], None)


def test_pages_refusals(lib):
    for n in ("new_len", "len", "table", "free", "n_free", "slots", "missing"):
        assert pages(lib, **{n: None}) == EINVAL and b"cache4_pages" in lib.mustdrop_last_error()
    for n in ("B", "max_pages", "n_pages", "page"):
        assert pages(lib, **{n: 0}) == EINVAL and pages(lib, **{n: -3}) == EINVAL
    assert pages(lib, N=-1) == EINVAL
    for page in (8, 24, 33, 512):
        assert pages(lib, page=page) == ESHAPE
    assert pages(lib, B=65536) == ESHAPE and pages(lib, B=1, N=(1 << 30) + 1) == ESHAPE
    assert pages(lib, n_pages=1 << 27, page=16) == ESHAPE                        # 2^31 slots
    assert pages(lib, max_pages=(1 << 30) // 32) == ESHAPE                       # 2^30 entries per request
    assert pages(lib, B=65535, max_pages=40000) == ESHAPE                        # a table of more than 2^31 entries
    assert pages(lib, B=1024, max_pages=(1 << 21) - 9, n_pages=1 << 24) == ESHAPE     # places of the stack beyond 31 bits
    assert pages(lib, len=P(1)) == EALIAS and pages(lib, free=P(3)) == EALIAS and pages(lib, ws=P(3)) == EALIAS
    assert pages(lib, slots=P(7)) == EALIAS
    assert pages(lib, ws=None) == EWORKSPACE and pages(lib, wsb=C.c_size_t(8)) == EWORKSPACE
    assert pages(lib, ws=C.c_void_p(P(8).value + 64)) == EALIGN
    need = lib.mustdrop_cache4_pages_workspace_bytes(3)
    assert need % 256 == 0 and need > 0 and lib.mustdrop_cache4_pages_workspace_bytes(0) == 0
    assert pages(lib, wsb=C.c_size_t(need - 1)) == EWORKSPACE


def layout(b, t, h):
    return C.byref(md.KvLayout(b, t, h))


def write(lib, **kw):
    a = dict(k=P(1), v=P(2), dtype=1, slots=P(3), cache=P(4), B=2, N=3, H=4, d=128, n_pages=10, page=32, lay=None)
    a.update(kw)
    return lib.mustdrop_cache4_write(*[a[n] for n in ("k", "v", "dtype", "slots", "cache", "B", "N", "H", "d", "n_pages", "page", "lay")], None)


def read(lib, **kw):
    a = dict(cache=P(4), table=P(5), len=P(6), first=P(7), k=P(1), v=P(2), dtype=1, B=2, N=3, H=4, d=128, n_pages=10, page=32, max_pages=6, lay=None)
    a.update(kw)
    return lib.mustdrop_cache4_read(*[a[n] for n in ("cache", "table", "len", "first", "k", "v", "dtype", "B", "N", "H", "d", "n_pages", "page",
                                                     "max_pages", "lay")], None)


@pytest.mark.parametrize("call", (write, read))
def test_rows_refusals(lib, call):
    for n in ("k", "v", "cache") + (("slots",) if call is write else ("table", "len")):
        assert call(lib, **{n: None}) == EINVAL and lib.mustdrop_last_error() != b""
    for n in ("B", "N", "H", "d", "n_pages", "page"):
        assert call(lib, **{n: 0}) == EINVAL and call(lib, **{n: -1}) == EINVAL
    for d in (16, 32, 96, 256):
        assert call(lib, d=d) == ESHAPE
    assert call(lib, page=48) == ESHAPE and call(lib, H=65536) == ESHAPE
    for t in (-1, 2, 7):
        assert call(lib, dtype=t) == EDTYPE
    for n in ("k", "v", "cache"):
        assert call(lib, **{n: C.c_void_p(P(9).value + 8)}) == EALIGN
    assert call(lib, k=P(4)) == EALIAS                                           # the rows lie over the pool
    assert call(lib, lay=layout(3 * 512, 512, 100)) == EINVAL                    # a stride that is no multiple of 8
    assert call(lib, lay=layout(3 * 512, 512, 0)) == EINVAL
    assert call(lib, lay=layout(3 * 512, 512, 64)) == ESHAPE                     # heads overlap
    assert call(lib, B=1 << 20, N=1 << 20, H=1) == ESHAPE
    assert call(lib, B=1 << 8, N=1 << 20, H=1) == ESHAPE and b"rows" in lib.mustdrop_last_error()   # 2^28
    if call is read:
        assert call(lib, v=P(1)) == EALIAS and call(lib, k=P(5)) == EALIAS and call(lib, max_pages=0) == EINVAL


def attend(lib, **kw):
    a = dict(q=P(1), dtype=1, cache=P(2), table=P(3), len=P(4), q_len=P(5), keep=P(6), B=2, N=3, Hq=8, H=4, d=128, n_pages=10, page=32, max_pages=6,
             scale=C.c_float(0.09), out=P(7), lse=P(8), ql=None, ol=None, ws=P(9), wsb=BIG)
    a.update(kw)
    return lib.mustdrop_cache4_attend(*[a[n] for n in ("q", "dtype", "cache", "table", "len", "q_len", "keep", "B", "N", "Hq", "H", "d", "n_pages", "page",
                                                       "max_pages", "scale", "out", "lse", "ql", "ol", "ws", "wsb")], None)


def test_attend_refusals(lib):
    for n in ("q", "cache", "table", "len", "out"):
        assert attend(lib, **{n: None}) == EINVAL and b"cache4_attend" in lib.mustdrop_last_error()
    for n in ("B", "N", "Hq", "H", "d", "n_pages", "page", "max_pages"):
        assert attend(lib, **{n: 0}) == EINVAL and attend(lib, **{n: -2}) == EINVAL
    assert attend(lib, Hq=9) == ESHAPE and attend(lib, Hq=3) == ESHAPE           # heads that do not share evenly
    assert attend(lib, d=96) == ESHAPE and attend(lib, page=100) == ESHAPE
    assert attend(lib, dtype=2) == EDTYPE
    for s in (0.0, -1.0, float("nan"), float("inf")):
        assert attend(lib, scale=C.c_float(s)) == EINVAL
    for n in ("q", "cache", "out"):
        assert attend(lib, **{n: C.c_void_p(P(10).value + 4)}) == EALIGN
    assert attend(lib, keep=C.c_void_p(P(6).value + 2)) == EALIGN
    assert attend(lib, out=P(1)) == EALIAS and attend(lib, out=P(2)) == EALIAS and attend(lib, lse=P(7)) == EALIAS and attend(lib, lse=P(4)) == EALIAS
    assert attend(lib, ws=P(7)) == EALIAS and attend(lib, ws=P(2)) == EALIAS
    assert attend(lib, ws=None) == EWORKSPACE and attend(lib, wsb=C.c_size_t(1)) == EWORKSPACE
    assert attend(lib, ws=C.c_void_p(P(9).value + 16)) == EALIGN
    assert attend(lib, ql=layout(3 * 1024, 1024, 4)) == EINVAL and attend(lib, ol=layout(512, 1024, 128)) == ESHAPE
    assert attend(lib, N=1 << 30, Hq=8, H=1) == ESHAPE
    assert attend(lib, B=1 << 21, N=1, Hq=4, H=4, ql=layout(512, 512, 128), ol=layout(512, 512, 128)) == ESHAPE   # 2^23 tiles: 2^32 threads
    assert b"tiles" in lib.mustdrop_last_error()
    size = lib.mustdrop_cache4_attend_workspace_bytes
    need = size(2, 3, 8, 4, 128, 6, 32)
    assert need > 0 and need % 256 == 0 and attend(lib, wsb=C.c_size_t(need - 1)) == EWORKSPACE
    assert size(0, 3, 8, 4, 128, 6, 32) == 0 and size(2, 3, 9, 4, 128, 6, 32) == 0 and size(2, 3, 8, 4, 96, 6, 32) == 0


def test_pool_bytes(lib):
    assert lib.mustdrop_cache4_bytes(10, 32, 4, 128) == 10 * 4 * 32 * 136 == 10 * 4 * ref.page_bytes(32, 128)
    assert lib.mustdrop_cache4_bytes(100000, 128, 64, 128) == 100000 * 64 * 128 * 136          # beyond 2^32
    for bad in ((0, 32, 4, 128), (10, 20, 4, 128), (10, 32, 4, 80), (1 << 27, 16, 1, 64), (1 << 24, 32, 8, 128)):
        assert lib.mustdrop_cache4_bytes(*bad) == 0


# ---- refusals of the Python entries
def test_binding_refusals():
    import torch
    i32 = dict(dtype=torch.int32)
    table, length, one = torch.zeros((2, 6), **i32), torch.zeros(2, **i32), torch.zeros(1, **i32)
    cache = torch.zeros((10, 4, 32 * 136), dtype=torch.uint8)
    rows = torch.zeros((2, 3, 4, 128), dtype=torch.bfloat16)
    slots = torch.zeros((2, 3), **i32)
    with pytest.raises(ValueError, match="GPU"):                                 # no CPU fallback
        md.mustdrop_cache4_write(rows, rows, slots, cache)
    with pytest.raises(ValueError, match="GPU"):
        md.mustdrop_cache4_read(cache, table, length, rows, rows)
    with pytest.raises(ValueError, match="GPU"):
        md.mustdrop_cache4_attend(rows, cache, table, length, 0.1)
    with pytest.raises(ValueError, match="GPU"):
        md.mustdrop_cache4_pages(length, length.clone(), table, one, one, one, 32)
    with pytest.raises(TypeError, match="slots"):
        md.mustdrop_cache4_write(rows, rows, slots.long(), cache)
    with pytest.raises(ValueError, match="slots"):
        md.mustdrop_cache4_write(rows, rows, slots[:1], cache)
    with pytest.raises(TypeError, match="v_new"):
        md.mustdrop_cache4_write(rows, rows.float(), slots, cache)
    with pytest.raises(ValueError, match="heads"):
        md.mustdrop_cache4_write(rows[:, :, :2], rows[:, :, :2], slots, cache)
    with pytest.raises(ValueError, match="layout"):
        md.mustdrop_cache4_write(rows, rows.transpose(1, 2).contiguous().transpose(1, 2), slots, cache)
    with pytest.raises(ValueError, match="contiguous d"):
        md.mustdrop_cache4_write(rows.transpose(2, 3).contiguous().transpose(2, 3), rows, slots, cache)
    with pytest.raises(ValueError, match="cache"):
        md.mustdrop_cache4_write(rows, rows, slots, cache[:, :, :1000])
    with pytest.raises(TypeError, match="cache"):
        md.mustdrop_cache4_attend(rows, cache.to(torch.int8), table, length, 0.1)
    with pytest.raises(ValueError, match="keep"):
        md.mustdrop_cache4_attend(rows, cache, table, length, 0.1, keep=torch.zeros((2, 100), dtype=torch.uint8))
    with pytest.raises(TypeError, match="lse"):
        md.mustdrop_cache4_attend(rows, cache, table, length, 0.1, lse=torch.zeros((2, 4, 3), dtype=torch.float64))
    with pytest.raises(ValueError, match="lse"):
        md.mustdrop_cache4_attend(rows, cache, table, length, 0.1, lse=torch.zeros((2, 3, 4)))
    with pytest.raises(ValueError, match="length"):
        md.mustdrop_cache4_attend(rows, cache, table, torch.zeros(3, **i32), 0.1)
    with pytest.raises(TypeError, match="table"):
        md.mustdrop_cache4_read(cache, table.long(), length, rows, rows)
    with pytest.raises(ValueError, match="page"):
        md.cache4_buffer(10, 24, 4, 128, device="cpu")
    assert tuple(md.cache4_buffer(10, 32, 4, 128, device="cpu").shape) == (10, 4, 32 * 136)
