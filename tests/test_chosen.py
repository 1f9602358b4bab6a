"""Rotation, rows rotated into the cache and pages that are chosen, without a GPU: the plain references, and every refusal."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

import cache4_ref as ref
import chosen_ref as cr
import paper_2411_10803_amd as md

OK, EINVAL, ESHAPE, EALIGN, EALIAS, EWORKSPACE, EDTYPE = range(7)
BIG = C.c_size_t(1 << 40)


def P(n):
    """Fake device pointers far apart: never dereferenced on the host."""
    return C.c_void_p((n + 1) << 36)


def moved(p, by):
    return C.c_void_p(p.value + by)


def layout(*strides):
    return C.byref(md.KvLayout(*strides))


@pytest.fixture(scope="module")
def lib():
    return md.library()


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
def test_how_calls_are_cut(tmp_path):
    exe = str(tmp_path / "cache4_chosen")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           os.path.join(os.path.dirname(os.path.abspath(__file__)), "plan", "cache4_chosen_main.cpp"), "-o", exe])
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]


# ---- the references
def test_turning_keeps_lengths_and_differences_of_positions():
    """Scores of turned rows depend on the difference of their positions alone, and the way back gives the rows again."""
    rng = np.random.default_rng(0)
    for adjacent in (False, True):
        table, axis = cr.angles(200, 16).astype(np.float64), [0] * 5 + [1] * 11
        q, k = rng.standard_normal((2, 1, 1, 40))
        at = lambda t, w: np.array([[t], [w]])  # noqa: E731
        dots = [(cr.turned(q, at(t + 3, w + 50), table, axis, adjacent, kind=np.float64) * cr.turned(k, at(t, w), table, axis, adjacent, kind=np.float64)).sum()
                for t, w in ((0, 0), (10, 7), (100, 149))]
        assert np.allclose(dots, dots[0], atol=1e-5)                             # (the table is fp32)
        y = cr.turned(q, at(17, 180), table, axis, adjacent, kind=np.float64)
        assert np.allclose(cr.turned(y, at(17, 180), table, axis, adjacent, True, kind=np.float64), q, atol=1e-6)
        assert np.array_equal(y[..., 32:], q[..., 32:])


def test_a_pages_score_is_no_less_than_its_keys():
    rng = np.random.default_rng(1)
    page, d, H, G = 16, 64, 2, 3
    pool = np.zeros((1, H, ref.page_bytes(page, d)), np.uint8)
    for t in range(page):
        for h in range(H):
            k = rng.standard_normal(d) * np.exp2(rng.integers(-6, 2, d))
            ref.put(pool, t, h, k, k, page)
    b, s = cr.bounds(pool, 0, page, H, d, page)
    assert np.abs(b).max() <= 96 and (b[:, 0] >= b[:, 1]).all()
    k = cr.keys_of(pool, 0, page, H, d, page)
    for h in range(H):
        w = cr.whole(rng.standard_normal((G, d)) * 3)
        assert cr.score(w, b[h], s[h]) >= (k[:, h] @ w.T).sum(1).max()
        assert (b[h, 0] * 2.0 ** (s[h] - 127) >= k[:, h].max(0)).all() and (b[h, 1] * 2.0 ** (s[h] - 127) <= k[:, h].min(0)).all()


def test_reference_choice():
    bounds, scales = np.zeros((6, 2, 64), np.int64), np.full(6, 127)
    bounds[:, 0, 0] = [5, 9, 9, 1, 9, 0]
    q = np.zeros((1, 64))
    q[0, 0] = 64
    row = np.arange(6)
    pick = lambda first, last, budget, length=96: cr.choose(q, bounds, scales, row, length, 1, 0, 16, first, last, budget, 6)  # noqa: E731
    assert pick(0, 0, 2) == [1, 2] and pick(0, 1, 3) == [1, 2, 5] and pick(1, 1, 3) == [0, 1, 5] and pick(0, 0, 4) == [0, 1, 2, 4]
    assert pick(0, 1, 4, 33) == [0, 1, 2, -1] and pick(2, 1, 3, 33) == [0, 1, 2] and pick(0, 1, 2, 0) == [-1, -1]
    assert cr.listed([3, 3, 1, 5, 9, 4, 6], 8) == [3, 5, 6]


# ---- refusals of the C ABI
def turn(pairs=64, axes=2, adjacent=0, axis=None):
    r = md.Rotary(pairs, axes, adjacent)
    for i in range(min(pairs, 128)):
        r.axis[i] = i % max(axes, 1) if axis is None else axis
    return C.byref(r)


def rotate(lib, **kw):
    a = dict(q=P(1), k=P(2), dtype=1, pos=P(3), index=P(4), table=P(5), rows=P(6), B=2, N=3, L=7, Hq=8, H=4, d=128, n_pos=100, turn=turn(), inverse=0,
             qo=P(7), ko=P(8), ql=None, kl=None, qol=None, kol=None)
    a.update(kw)
    return lib.mustdrop_rotate(*[a[n] for n in ("q", "k", "dtype", "pos", "index", "table", "rows", "B", "N", "L", "Hq", "H", "d", "n_pos", "turn", "inverse",
                                                "qo", "ko", "ql", "kl", "qol", "kol")], None)


def append(lib, **kw):
    a = dict(q=P(1), k=P(2), v=P(9), dtype=1, pos=P(3), index=P(4), table=P(5), slots=P(6), cache=P(8), B=2, N=3, L=7, Hq=8, H=4, d=128, n_pos=100, n_pages=10,
             page=32, turn=turn(), qo=P(7), ql=None, lay=None, qol=None)
    a.update(kw)
    return lib.mustdrop_cache4_append(*[a[n] for n in ("q", "k", "v", "dtype", "pos", "index", "table", "slots", "cache", "B", "N", "L", "Hq", "H", "d", "n_pos",
                                                       "n_pages", "page", "turn", "qo", "ql", "lay", "qol")], None)


@pytest.mark.parametrize("call, name", [(rotate, b"rotate"), (append, b"cache4_append")])
def test_rotation_refusals(lib, call, name):
    for n in ("pos", "table", "turn", "q", "qo"):
        assert call(lib, **{n: None}) == EINVAL and name in lib.mustdrop_last_error()
    for n in ("B", "N", "L", "Hq", "H", "d", "n_pos"):
        assert call(lib, **{n: 0}) == EINVAL and call(lib, **{n: -2}) == EINVAL
    assert call(lib, dtype=2) == EDTYPE
    for t in (turn(pairs=66), turn(pairs=72), turn(pairs=6), turn(axes=5), turn(axes=0)):
        assert call(lib, turn=t) == ESHAPE
    assert call(lib, turn=turn(pairs=0)) == ESHAPE and call(lib, turn=turn(pairs=-4)) == ESHAPE and call(lib, turn=turn(pairs=132)) == ESHAPE
    assert call(lib, turn=turn(axis=2)) == EINVAL and b"axis" in lib.mustdrop_last_error()
    assert call(lib, index=None, L=2) == ESHAPE                                  # fewer positions than rows
    for n in ("q", "k", "qo"):
        assert call(lib, **{n: moved(P(10), 4)}) == EALIGN
    assert call(lib, table=moved(P(10), 8)) == EALIGN
    for n in ("k", "pos", "index", "table"):
        assert call(lib, **{n: P(7)}) == EALIAS                                  # an input over an output
    assert call(lib, qo=moved(P(1), 16)) == EALIAS                               # shifted over its own input
    assert call(lib, qo=P(1), qol=layout(3 * 2048, 2048, 256)) == EALIAS         # in place in another layout
    assert call(lib, ql=layout(4 * 1024, 1024, 4)) == EINVAL and call(lib, qol=layout(4 * 1024, 512, 128)) == ESHAPE
    assert call(lib, B=1 << 14, N=1 << 15, L=1 << 15) == ESHAPE


def test_rotate_refusals(lib):
    assert rotate(lib, k=None) == EINVAL and rotate(lib, ko=None) == EINVAL
    assert rotate(lib, d=132) == ESHAPE and rotate(lib, d=264) == ESHAPE
    assert rotate(lib, ko=P(7)) == EALIAS and rotate(lib, rows=P(8)) == EALIAS and rotate(lib, ko=P(1)) == EALIAS
    assert rotate(lib, ko=moved(P(10), 8)) == EALIGN
    assert rotate(lib, B=1 << 12, N=1 << 12, L=1 << 12, Hq=1 << 10) == ESHAPE    # 2^34 rows and heads
    few = dict(k=None, ko=None, B=1 << 8, N=(1 << 20) - 1, L=1 << 20, Hq=8, d=8, turn=turn(pairs=4))      # 2^31 - 2^11 pieces of 8 channels
    assert rotate(lib, **dict(few, N=1 << 20)) == ESHAPE and b"too many" in lib.mustdrop_last_error()
    assert rotate(lib, **dict(few, dtype=2)) == EDTYPE and rotate(lib, **dict(few, q=moved(P(1), 8))) == EALIGN


def test_append_refusals(lib):
    for n in ("k", "v", "slots", "cache"):
        assert append(lib, **{n: None}) == EINVAL
    assert append(lib, d=96) == ESHAPE and append(lib, page=24) == ESHAPE and append(lib, n_pages=0) == EINVAL
    assert append(lib, turn=turn(pairs=60)) == ESHAPE                            # pairs in eights
    assert append(lib, Hq=65535) == ESHAPE
    assert append(lib, q=P(8)) == EALIAS and append(lib, q=P(8), qo=P(8)) == EALIAS and append(lib, slots=P(8)) == EALIAS and append(lib, k=P(8)) == EALIAS
    assert append(lib, lay=layout(3 * 512, 512, 100)) == EINVAL


def bounds(lib, **kw):
    a = dict(cache=P(1), table=P(2), len=P(3), first=P(4), bounds=P(5), scales=P(6), B=2, N=3, H=4, d=128, n_pages=10, page=32, max_pages=6)
    a.update(kw)
    return lib.mustdrop_cache4_bounds(*[a[n] for n in ("cache", "table", "len", "first", "bounds", "scales", "B", "N", "H", "d", "n_pages", "page", "max_pages")], None)


def test_bounds_refusals(lib):
    for n in ("cache", "table", "len", "bounds", "scales"):
        assert bounds(lib, **{n: None}) == EINVAL and b"cache4_bounds" in lib.mustdrop_last_error()
    for n in ("B", "N", "H", "d", "n_pages", "page", "max_pages"):
        assert bounds(lib, **{n: 0}) == EINVAL and bounds(lib, **{n: -2}) == EINVAL
    assert bounds(lib, d=96) == ESHAPE and bounds(lib, page=8) == ESHAPE
    assert bounds(lib, cache=moved(P(1), 8)) == EALIGN and bounds(lib, bounds=moved(P(5), 4)) == EALIGN
    for n in ("cache", "table", "len", "first", "scales"):
        assert bounds(lib, **{n: P(5)}) == EALIAS
    assert bounds(lib, len=P(6)) == EALIAS
    assert bounds(lib, B=65536, N=1 << 20, max_pages=1 << 20) == ESHAPE


def choose(lib, **kw):
    a = dict(q=P(1), dtype=1, bounds=P(2), scales=P(3), table=P(4), len=P(5), q_len=P(6), B=2, N=3, Hq=8, H=4, d=128, n_pages=10, page=32, max_pages=6,
             first=1, last=1, budget=4, chosen=P(7), ql=None, ws=P(8), wsb=BIG)
    a.update(kw)
    return lib.mustdrop_cache4_choose(*[a[n] for n in ("q", "dtype", "bounds", "scales", "table", "len", "q_len", "B", "N", "Hq", "H", "d", "n_pages", "page",
                                                       "max_pages", "first", "last", "budget", "chosen", "ql", "ws", "wsb")], None)


def test_choose_refusals(lib):
    for n in ("q", "bounds", "scales", "table", "len", "chosen"):
        assert choose(lib, **{n: None}) == EINVAL and b"cache4_choose" in lib.mustdrop_last_error()
    for n in ("B", "N", "Hq", "H", "d", "n_pages", "page", "max_pages", "budget"):
        assert choose(lib, **{n: 0}) == EINVAL and choose(lib, **{n: -2}) == EINVAL
    assert choose(lib, first=-1) == EINVAL and choose(lib, last=-1) == EINVAL and choose(lib, first=3, last=2) == EINVAL
    assert choose(lib, first=2 ** 31 - 1, last=2 ** 31 - 1) == EINVAL
    assert choose(lib, Hq=9) == ESHAPE and choose(lib, d=96) == ESHAPE and choose(lib, page=100) == ESHAPE and choose(lib, dtype=3) == EDTYPE
    assert choose(lib, q=moved(P(1), 4)) == EALIGN and choose(lib, bounds=moved(P(2), 8)) == EALIGN
    for n in ("q", "bounds", "scales", "table", "len", "q_len", "ws"):
        assert choose(lib, **{n: P(7)}) == EALIAS
    assert choose(lib, ws=P(2)) == EALIAS and choose(lib, ws=None) == EWORKSPACE and choose(lib, ws=moved(P(8), 16)) == EALIGN
    assert choose(lib, ql=layout(4 * 1024, 1024, 4)) == EINVAL
    assert choose(lib, Hq=1025, H=1, N=1) == ESHAPE and b"query heads" in lib.mustdrop_last_error()
    assert choose(lib, N=1 << 20) == ESHAPE and choose(lib, B=1 << 22, N=1, H=2, Hq=2) == ESHAPE
    size = lib.mustdrop_cache4_choose_workspace_bytes
    need = size(2, 3, 8, 4, 128, 6, 32)
    assert need > 0 and need % 256 == 0 and choose(lib, wsb=C.c_size_t(need - 1)) == EWORKSPACE
    assert size(0, 3, 8, 4, 128, 6, 32) == 0 and size(2, 3, 9, 4, 128, 6, 32) == 0 and size(2, 3, 8, 4, 96, 6, 32) == 0


def attend(lib, **kw):
    a = dict(q=P(1), dtype=1, cache=P(2), table=P(3), len=P(4), q_len=P(5), keep=P(6), chosen=P(10), B=2, N=3, Hq=8, H=4, d=128, n_pages=10, page=32, max_pages=6,
             budget=4, scale=C.c_float(0.09), out=P(7), lse=P(8), ql=None, ol=None, ws=P(9), wsb=BIG)
    a.update(kw)
    return lib.mustdrop_cache4_attend_chosen(*[a[n] for n in ("q", "dtype", "cache", "table", "len", "q_len", "keep", "chosen", "B", "N", "Hq", "H", "d", "n_pages",
                                                              "page", "max_pages", "budget", "scale", "out", "lse", "ql", "ol", "ws", "wsb")], None)


def test_attend_chosen_refusals(lib):
    for n in ("q", "cache", "table", "len", "out", "chosen"):
        assert attend(lib, **{n: None}) == EINVAL and b"cache4_attend_chosen" in lib.mustdrop_last_error()
    for n in ("B", "N", "Hq", "H", "d", "n_pages", "page", "max_pages", "budget"):
        assert attend(lib, **{n: 0}) == EINVAL and attend(lib, **{n: -2}) == EINVAL
    assert attend(lib, Hq=9) == ESHAPE and attend(lib, d=96) == ESHAPE and attend(lib, page=100) == ESHAPE and attend(lib, dtype=2) == EDTYPE
    for s in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        assert attend(lib, scale=C.c_float(s)) == EINVAL
    for n in ("q", "cache", "out"):
        assert attend(lib, **{n: moved(P(11), 4)}) == EALIGN
    assert attend(lib, keep=moved(P(6), 2)) == EALIGN and attend(lib, ws=moved(P(9), 16)) == EALIGN
    for n in ("q", "cache", "table", "len", "q_len", "keep", "chosen", "lse", "ws"):
        assert attend(lib, **{n: P(7)}) == EALIAS
    assert attend(lib, lse=P(10)) == EALIAS and attend(lib, ws=P(10)) == EALIAS
    assert attend(lib, ws=None) == EWORKSPACE and attend(lib, wsb=C.c_size_t(1)) == EWORKSPACE
    assert attend(lib, ql=layout(4 * 1024, 1024, 4)) == EINVAL and attend(lib, ol=layout(512, 1024, 128)) == ESHAPE
    assert attend(lib, B=1 << 21, N=1, Hq=4, H=4, ql=layout(512, 512, 128), ol=layout(512, 512, 128)) == ESHAPE
    assert attend(lib, budget=1 << 30) == ESHAPE
    size = lib.mustdrop_cache4_attend_chosen_workspace_bytes
    assert size(2, 3, 8, 4, 128, 5000, 32) % 256 == 0 and size(2, 3, 8, 4, 128, 5000, 32) > 0
    assert size(0, 3, 8, 4, 128, 6, 32) == 0 and size(2, 3, 9, 4, 128, 6, 32) == 0 and size(2, 3, 8, 4, 96, 6, 32) == 0


# ---- refusals of the Python entries
def test_binding_refusals():
    import torch
    i32 = dict(dtype=torch.int32)
    q, k = torch.zeros((2, 3, 8, 128), dtype=torch.bfloat16), torch.zeros((2, 3, 4, 128), dtype=torch.bfloat16)
    pos, table, t = torch.zeros((2, 2, 5), **i32), torch.zeros((50, 64, 2)), md.rotary([24, 40])
    slots, cache = torch.zeros((2, 3), **i32), torch.zeros((10, 4, 32 * 136), dtype=torch.uint8)
    length, rows = torch.zeros(2, **i32), torch.zeros((2, 6), **i32)
    bounds, scales = md.cache4_bounds_buffer(10, 4, 128, device="cpu")
    chosen = torch.zeros((2, 3, 4, 5), **i32)
    for call in (lambda: md.mustdrop_rotate(q, pos, table, t, k=k), lambda: md.mustdrop_cache4_append(q, k, k, pos, table, t, slots, cache),
                 lambda: md.mustdrop_cache4_bounds(cache, rows, length, 3, bounds, scales),
                 lambda: md.mustdrop_cache4_choose(q, bounds, scales, rows, length, 32, chosen),
                 lambda: md.mustdrop_cache4_attend_chosen(q, cache, rows, length, chosen, 0.1)):
        with pytest.raises(ValueError, match="GPU"):                             # no CPU fallback
            call()
    for bad in (dict(sections=[64, 65]), dict(sections=[0]), dict(sections=[4, 4], axis=[0] * 7), dict(sections=[4, 4], axis=[2] * 8), dict(sections=[-1, 5])):
        with pytest.raises(ValueError, match="pairs"):
            md.rotary(**bad)
    t2 = md.rotary([2, 2], adjacent=True, axis=[0, 1, 0, 1])
    assert (t2.pairs, t2.axes, t2.adjacent, list(t2.axis[:4])) == (4, 2, 1, [0, 1, 0, 1])
    for error, match, call in (
            (ValueError, "positions", lambda: md.mustdrop_rotate(q, pos[:1], table, t)),
            (TypeError, "positions", lambda: md.mustdrop_rotate(q, pos.long(), table, t)),
            (ValueError, "table", lambda: md.mustdrop_rotate(q, pos, table[:, :32], t)),
            (TypeError, "table", lambda: md.mustdrop_rotate(q, pos, table.double(), t)),
            (ValueError, "index", lambda: md.mustdrop_rotate(q, pos, table, t, index=torch.zeros((2, 4), **i32))),
            (ValueError, "rows", lambda: md.mustdrop_rotate(q, pos, table, t, rows=torch.zeros(3, **i32))),
            (TypeError, "q_out", lambda: md.mustdrop_rotate(q, pos, table, t, q_out=q.float())),
            (TypeError, "k", lambda: md.mustdrop_rotate(q, pos, table, t, k=k.float())),
            (ValueError, "k_out", lambda: md.mustdrop_rotate(q, pos, table, t, k_out=k)),
            (ValueError, "k must", lambda: md.mustdrop_rotate(q, pos, table, t, k=k[:, :2])),
            (ValueError, "q_out", lambda: md.mustdrop_cache4_append(None, k, k, pos, table, t, slots, cache, q_out=q)),
            (TypeError, "q must", lambda: md.mustdrop_cache4_append(q.float(), k, k, pos, table, t, slots, cache)),
            (ValueError, "heads", lambda: md.mustdrop_cache4_append(q, q, q, pos, table, t, slots, cache)),
            (TypeError, "slots", lambda: md.mustdrop_cache4_append(q, k, k, pos, table, t, slots.long(), cache)),
            (ValueError, "bounds", lambda: md.mustdrop_cache4_bounds(cache, rows, length, 3, bounds[:9], scales[:9])),
            (ValueError, "scales", lambda: md.mustdrop_cache4_bounds(cache, rows, length, 3, bounds, scales[:9])),
            (TypeError, "bounds", lambda: md.mustdrop_cache4_bounds(cache, rows, length, 3, bounds.to(torch.uint8), scales)),
            (ValueError, "first", lambda: md.mustdrop_cache4_bounds(cache, rows, length, 3, bounds, scales, first=torch.zeros(3, **i32))),
            (ValueError, "channels", lambda: md.mustdrop_cache4_choose(q[..., :64], bounds, scales, rows, length, 32, chosen)),
            (ValueError, "chosen", lambda: md.mustdrop_cache4_choose(q, bounds, scales, rows, length, 32, chosen[:, :2])),
            (TypeError, "chosen", lambda: md.mustdrop_cache4_attend_chosen(q, cache, rows, length, chosen.long(), 0.1)),
            (ValueError, "chosen", lambda: md.mustdrop_cache4_attend_chosen(q, cache, rows, length, chosen[:, :, :2], 0.1)),
            (ValueError, "keep", lambda: md.mustdrop_cache4_attend_chosen(q, cache, rows, length, chosen, 0.1, keep=torch.zeros((2, 9), dtype=torch.uint8)))):
        with pytest.raises(error, match=match):
            call()


def test_table_of_angles():
    t = md.rotary_table(300, 32, base=500.0, device="cpu").numpy()
    assert t.shape == (300, 32, 2) and np.array_equal(t, cr.angles(300, 32, 500.0))
    far = md.rotary_table(1 << 17, 4, device="cpu").numpy()
    x = (np.arange(1 << 17, dtype=np.longdouble) * np.longdouble(10000) ** (-np.longdouble(1) / 4))      # as far out as this, still to half a step
    assert np.abs(far[:, 1, 0] - np.cos(x)).max() <= 2.0 ** -25 + 1e-11
