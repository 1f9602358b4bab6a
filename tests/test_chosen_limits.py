"""The ends of what the rotation and the calls on chosen pages take, without a GPU: what shares a byte, refusals."""
import os
import shutil
import subprocess

import pytest

from test_chosen import EALIAS, append, layout, lib, moved, P, rotate  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
def test_rows_that_share_a_byte(tmp_path):
    exe = str(tmp_path / "row_overlap")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           os.path.join(HERE, "plan", "row_overlap_main.cpp"), "-o", exe])
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
