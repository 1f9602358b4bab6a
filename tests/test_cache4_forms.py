"""Which form of the attention over the cache held in 4 bits the cases of cache4_forms.py take, from csrc/cache4_plan.hpp compiled for the CPU."""
import os
import shutil
import subprocess

import pytest

import cache4_forms as forms

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
