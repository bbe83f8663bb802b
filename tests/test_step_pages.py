"""The pages of a step whose rows are not all kept: the definition (plain integers) keeps every page, and the call's refusals. No GPU needed."""
import numpy as np
import pytest

from paper_2512_23966_amd import binding as B
from tests import step_reference as R
from tests.step_pages import Pool, step_tables_held

ERR_NULL, ERR_SHAPE, ERR_ALIGN = -1, -2, -6
A = 4096


def _held(**k):
    a = dict(cache=A, new=2 * A, parents=3 * A, free=4 * A, count=5 * A, held=13 * A, table=6 * A, B=2, n=8, num_free=10, num_pages=100, page=64, most=16,
             granted=7 * A, seqlens=8 * A, pos=9 * A, slots=10 * A, masks=11 * A, left=12 * A, after=14 * A)
    a.update(k)
    return B.lib().loza_ssa_step_tables_held(*a.values(), None)


def test_refusals():
    for name in ("cache", "new", "count", "table", "granted", "seqlens", "pos", "slots", "left", "free", "parents", "masks", "held", "after"):
        assert _held(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(B=65537), dict(n=0), dict(n=65), dict(page=48), dict(granted=2 * A), dict(seqlens=A), dict(left=5 * A), dict(after=13 * A)):
        assert _held(**bad) == ERR_SHAPE, bad
    assert _held(held=A * 20 + 2) == ERR_ALIGN and _held(after=A * 20 + 2) == ERR_ALIGN


def test_nothing_held_is_what_the_caches_need():
    rng = np.random.default_rng(1)
    cache, new = rng.integers(0, 300, size=9).astype(np.int32), rng.integers(0, 6, size=9).astype(np.int32)
    table, free = rng.permutation(90).astype(np.int32).reshape(9, 10), rng.permutation(90).astype(np.int32)
    parents = np.stack([R.random_parents(rng, 5) for _ in range(9)])
    a = step_tables_held(cache, new, parents, free, 3, np.zeros(9, np.int32), table, 5, 90, 32)
    for x, y in zip(a, R.step_tables(cache, new, parents, free, 3, table, 5, 90, 32)):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("B_,n,page,most,pages,tree", [(3, 9, 32, 12, 36, True), (16, 64, 32, 20, 200, True), (5, 8, 64, 6, 22, True), (4, 40, 32, 9, 30, False)])
def test_the_definition_loses_no_page(B_, n, page, most, pages, tree):
    pool = Pool(np.random.default_rng(n), B_, most, page, pages, step_tables_held)
    for _ in range(300):
        pool.step(n, tree)
    assert pool.ended > 3                              # (far beyond what the pool holds once)
