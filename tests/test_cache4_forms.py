"""The cache held in 4 bits without a GPU: which form of the attention the cases of cache4_forms.py take, from csrc/cache4_plan.hpp compiled for
the CPU; and what include/mustdrop.h says of its numbers, on the 64-bit reference."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import cache4_forms as forms
import cache4_ref as ref
import test_cache4 as refusals

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """cases -> a dict(rows, tiles, waves, runs) of each"""
    if shutil.which("g++") is None:
        pytest.skip("g++ not found")
    exe = str(tmp_path_factory.mktemp("plan") / "cache4_forms")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", os.path.join(HERE, "plan", "cache4_forms_main.cpp"), "-o", exe])

    def run(cases):
        lines = [f"{int(c['dtype'] == forms.F32)} {len(c['lengths'])} {c['N']} {c['Hq'] // c['H']} {c['H']} {c['d']} {c['entries'] * c['page']}" for c in cases]
        out = subprocess.run([exe], input="\n".join(lines), stdout=subprocess.PIPE, text=True, timeout=60, check=True).stdout
        return [dict(zip(("rows", "tiles", "waves", "runs"), map(int, x.split()))) for x in out.splitlines()]
    return run


def test_many_rows_go_together(plan):
    got = plan(forms.MANY_ROWS)
    assert [p["rows"] for p in got] == [32] * len(forms.MANY_ROWS)
    assert [p["runs"] for p in got] == [0, 0, 1, 1, 0]
    fewer = dict(forms.MANY_ROWS[4], lengths=forms.MANY_ROWS[4]["lengths"][:32])
    assert plan([fewer])[0]["rows"] == 16                     # one sample less: sixteen rows at a time


@pytest.mark.parametrize("page", (16, 64, 256))
def test_every_form_is_there(plan, page):
    for (kind, d, runs), p in zip(forms.FORMS, plan([forms.form(*f, page=page) for f in forms.FORMS])):
        assert (p["rows"], p["runs"]) == (32 if kind == "many" else 16, runs), (kind, d, runs)


def test_joins_are_reached(plan):
    for c, (rows, many) in zip(forms.JOINS, ((16, False), (16, True), (16, True), (32, True))):
        p = plan([c])[0]
        assert p["runs"] == 1 and p["rows"] == rows and (len(c["lengths"]) * c["Hq"] * c["N"] > 2048) == many, c
    for dtype in (forms.BF16, forms.F32):
        for d in (64, 128):
            p = plan([dict(forms.LONG, dtype=dtype, d=d)])[0]
            units, parts = len(forms.LONG["lengths"]), forms.parts_of(forms.LONG["lengths"], 1, 1, 1, 16)
            assert p["runs"] == 1 and units > 1024 / 8 / 5           # four waves to a row: 1024 / units / 8, four at least
            assert parts > 4 * 64, parts


# ---- what the header says of a value's error, over all scales
def groups(rng, n, low, high):
    """[n, 32] with the largest magnitude between 2^low and 2^high, and what they are held as."""
    x = rng.standard_normal((n, 32)) * np.exp2(rng.uniform(-6, 0, (n, 32)))
    x *= np.exp2(rng.uniform(low, high, (n, 1))) / np.abs(x).max(-1, keepdims=True)
    return x, ref.values(*ref.quantise(x)), np.abs(x).max(-1, keepdims=True)


def test_errors_where_the_scale_follows_the_largest_magnitude():
    low, high = np.log2(3.5) - 100, np.log2(7.0) + 125
    rng = np.random.default_rng(0)
    for a, b in ((low, high), (low, low + 3), (high - 3, high)):
        x, y, most = groups(rng, 20000, a, b - 1e-9)
        off = np.abs(y - x)
        assert (off <= most / 5).all() and (off <= np.abs(x) / 5)[np.abs(x) >= most / 4].all()


def test_errors_where_the_scale_ends():
    rng = np.random.default_rng(1)
    x, y, _ = groups(rng, 20000, -150, np.log2(3.5) - 100 - 1e-9)
    assert (np.abs(y - x) <= 2.0 ** -101).all() and (y[np.abs(x) <= 2.0 ** -102] == 0).all()
    assert (np.abs(y - x) > np.abs(x) / 5)[np.abs(x) >= np.abs(x).max(-1, keepdims=True) / 4].any()      # (no fifth here)
    x, y, most = groups(rng, 20000, np.log2(7.0) + 125, 128 - 1e-9)
    cut = np.abs(x) > 6 * 2.0 ** 125
    assert (np.abs(y)[cut] == 6 * 2.0 ** 125).all() and (np.abs(y - x)[cut] <= np.abs(x)[cut] / 4).all()
    assert (np.abs(y - x) <= most / 5)[~cut].all() and (np.abs(y - x) > most / 5).any()
    # both ends: what the bound without a range would have promised
    for top, off in ((3.38e38, 0.24), (6e-31, 0.3), (2.0 ** -103, 0.99)):
        v = np.full(32, top)
        assert np.abs(ref.values(*ref.quantise(v)) - v).max() > off * top


# ---- the reference of all rows at once against that of a row at a time
@pytest.mark.parametrize("n_query, length, nan", ((7, 30, False), (5, 33, True), (9, 4, True), (3, 0, False), (0, 20, False)))
def test_reference_of_all_rows_at_once(n_query, length, nan):
    rng = np.random.default_rng(length)
    q, K, V = rng.standard_normal((9, 6, 64)), rng.standard_normal((36, 2, 64)), rng.standard_normal((36, 2, 64))
    there, keep = np.arange(36) // 16 != 1, rng.integers(0, 3, 36)
    if nan:
        K[1, 0, 3], V[2, 1, 5], V[35, 0, 7] = np.nan, np.nan, np.nan
        keep[1:3] = 1
        V[max(0, length - 1), 1, 60] = np.nan
    for mask in (None, keep):
        for a, b in zip(ref.attend(q, K, V, there, length, n_query, 0.3, mask), ref.attend_heads(q, K, V, there, length, n_query, 0.3, mask)):
            np.testing.assert_allclose(a, b, rtol=1e-12, atol=1e-14)


# ---- refusals
def test_a_scale_that_is_infinite_to_base_2_is_refused():
    import ctypes as C
    import paper_2411_10803_amd as md
    lib = md.library()
    for scale in (2.4e38, 3.4e38):
        assert refusals.attend(lib, scale=C.c_float(scale)) == refusals.EINVAL and b"softmax_scale" in lib.mustdrop_last_error()
    # the largest one that is taken, as far as the next check: no workspace
    assert refusals.attend(lib, scale=C.c_float(2.3e38), ws=None) == refusals.EWORKSPACE


def test_outputs_between_other_rows_are_refused_and_inputs_are_not():
    """K and V side by side in one buffer [B, N, 2, H, d]: as inputs (far enough for the next check to be reached), not as outputs."""
    import ctypes as C
    import paper_2411_10803_amd as md
    lib = md.library()
    k, H, d, N = refusals.P(1), 4, 128, 3
    v, lay = C.c_void_p(k.value + H * d * 2), refusals.layout(N * 2 * H * d, 2 * H * d, d)
    assert refusals.read(lib, k=k, v=v, lay=lay) == refusals.EALIAS
    assert refusals.write(lib, k=k, v=v, lay=lay, slots=refusals.P(4)) == refusals.EALIAS and b"overlap" in lib.mustdrop_last_error()   # (slots over the pool)
    assert refusals.attend(lib, q=k, out=v, Hq=H, ql=lay, ol=lay) == refusals.EALIAS
    assert refusals.attend(lib, q=k, Hq=H, ql=lay, ws=None) == refusals.EWORKSPACE
