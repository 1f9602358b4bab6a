"""The ends of what the rotation and the calls on chosen pages take, without a GPU: what shares a byte, refusals."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from test_chosen import EALIAS, ESHAPE, EWORKSPACE, append, attend, choose, layout, lib, moved, P, rotate  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
@pytest.mark.parametrize("name", ["row_overlap", "cache4_lists"])
def test_plain_arithmetic(tmp_path, name):
    """Rows that share a byte, against every byte of small grids; blocks of a launch for any number of lists."""
    exe = str(tmp_path / name)
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           os.path.join(HERE, "plan", name + "_main.cpp"), "-o", exe])
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]


def test_views_of_one_projection_that_share_bytes_are_refused(lib):  # noqa: F811
    """Rows of 16 heads of 128, of which 8 are queries and four each keys and values, in bf16."""
    lay, head = layout(3 * 2048, 2048, 128), 256
    q, k, v = P(1), moved(P(1), 8 * head), moved(P(1), 12 * head)
    one = dict(ql=lay, qol=lay)
    turned = dict(q=q, qo=q, kl=lay, kol=lay, **one)
    assert rotate(lib, **dict(turned, k=moved(q, 7 * head), ko=P(8))) == EALIAS            # the last query head and the first key head
    assert rotate(lib, **dict(turned, k=k, ko=moved(k, head))) == EALIAS                   # in place, but for a head
    assert rotate(lib, **dict(turned, k=k, ko=moved(k, 12 * head))) == EALIAS              # the last heads are the next row's first queries
    assert rotate(lib, **dict(turned, k=k, ko=k, pos=v)) == EALIAS                         # anything else goes by first and last byte
    assert rotate(lib, **dict(turned, k=v, ko=v, kl=layout(3 * 2048, 2048, 256), kol=layout(3 * 2048, 2048, 256))) == EALIAS        # every other head
    assert rotate(lib, **dict(turned, k=k, ko=k, qol=layout(3 * 4096, 4096, 128))) == EALIAS
    rows = dict(q=q, qo=q, lay=lay, **one)
    assert append(lib, **dict(rows, k=moved(q, 7 * head), v=v)) == EALIAS and append(lib, **dict(rows, k=k, v=moved(q, 16 * head))) == EALIAS
    assert append(lib, **dict(rows, k=k, v=v, qo=moved(q, 2 * head))) == EALIAS and append(lib, **dict(rows, k=k, v=v, slots=v)) == EALIAS
    assert append(lib, **dict(rows, k=k, v=v, cache=v)) == EALIAS and append(lib, **dict(rows, k=k, v=v, cache=q)) == EALIAS


# ---- the workspace of the attention over chosen pages
@pytest.mark.parametrize("B, N, Hq, H, d", [(4, 512, 32, 32, 128), (1, 4000, 32, 32, 128), (4, 512, 64, 8, 64), (2, 900, 16, 1, 128), (2, 900, 40, 1, 64)])
def test_workspace_of_lists_of_more_than_a_part(lib, B, N, Hq, H, d):  # noqa: F811
    """A sum of d channels and two numbers for each query head and part of 1024 entries; nothing where there is one part."""
    size = lib.mustdrop_cache4_attend_chosen_workspace_bytes
    G = Hq // H
    tile = min(G, 16) * -(-G // 16)                          # (the last sixteen heads of more take whole places)
    for budget, parts in ((1024, 1), (1025, 2), (2048, 2), (2049, 3), (9000, 9)):
        want = B * N * H * tile * parts * (d + 2) * 4 if parts > 1 else 0
        assert max(want, 256) <= size(B, N, Hq, H, d, budget, 16) <= want + 512, budget


def test_workspace_of_tokens_that_go_together(lib):  # noqa: F811
    """Lists that are padded beyond 1024 entries, in a table of fewer: no parts, and none asked for."""
    for dtype in (0, 1):
        few = dict(B=4, N=512, Hq=32, H=32, budget=1025, page=16, max_pages=100, dtype=dtype)
        assert attend(lib, **few, wsb=C.c_size_t(255)) == EWORKSPACE and b"256 bytes needed" in lib.mustdrop_last_error()
        assert attend(lib, **dict(few, max_pages=5000), wsb=C.c_size_t(256)) == EWORKSPACE       # (such tables are not shared in)


# ---- the choice
def test_lists_that_are_too_long_are_refused(lib):  # noqa: F811
    """A list's places are counted in 31 bits, in steps of up to 1024: a budget near 2^31 would not end."""
    for max_pages in (6, 900, 3000, 9000):
        for budget in (2 ** 26 + 1, 2 ** 31 - 1024, 2 ** 31 - 1):
            few = dict(B=1, N=1, H=1, Hq=1, max_pages=max_pages, page=16, budget=budget)
            assert choose(lib, **few, ws=None) == ESHAPE and b"too long" in lib.mustdrop_last_error()
    assert choose(lib, B=1, N=1, H=1, Hq=1, budget=2 ** 26, ws=None) == EWORKSPACE


def test_choice_in_tables_that_are_too_wide(lib):  # noqa: F811
    """What no call takes has no workspace, either."""
    size = lib.mustdrop_cache4_choose_workspace_bytes
    most = 2 ** 23 - 128
    assert size(1, 1, 1, 1, 64, most, 16) == most * 4 and size(1, 1, 1, 1, 64, most + 1, 16) == 0
    few = dict(B=1, N=1, H=1, Hq=1, d=64, page=16, ws=None)
    assert choose(lib, max_pages=most, **few) == EWORKSPACE and choose(lib, max_pages=most + 1, **few) == ESHAPE
