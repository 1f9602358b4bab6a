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
        want, wlse, size, score = ref.attend(c.qh[b], c.K[b], c.V[b], c.there[b], n, nq, c.scale, None if c.keep is None else c.keep[b, :c.K.shape[1]])
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
