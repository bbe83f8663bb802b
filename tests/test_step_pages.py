"""The pages of a step whose rows are not all kept: the definition (plain integers) keeps every page, and the call's refusals. No GPU needed."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
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


@pytest.mark.parametrize("held", [True, False])
def test_no_result_may_lie_on_another_array(held):
    """Workgroups read what others write: requests would get the same page. (Refused before anything is launched.)"""
    B_, n, most = 2, 8, 16
    sizes = dict(granted=4 * B_, seqlens=4 * B_, pos=4 * B_ * n, slots=4 * B_ * n, masks=8 * B_ * n, left=4, after=4 * B_, table=4 * B_ * most,
                 cache=4 * B_, new=4 * B_, parents=4 * B_ * n, free=40, count=4, held=4 * B_)
    results = ["granted", "seqlens", "pos", "slots", "masks", "left", "table"] + (["after"] if held else [])
    at = dict(cache=1, new=2, parents=3, free=4, count=5, held=13, table=6, granted=7, seqlens=8, pos=9, slots=10, masks=11, left=12, after=14)

    def call(**k):
        if held:
            return _held(**k)
        a = dict(cache=A, new=2 * A, parents=3 * A, free=4 * A, count=5 * A, table=6 * A, B=2, n=8, num_free=10, num_pages=100, page=64, most=16,
                 granted=7 * A, seqlens=8 * A, pos=9 * A, slots=10 * A, masks=11 * A, left=12 * A)
        a.update(k)
        return B.lib().loza_ssa_step_tables(*a.values(), None)
    for r in results:
        for other in sizes:
            if other == r or (not held and other in ("held", "after")):
                continue
            step = 8 if r == "masks" else 4
            assert call(**{r: at[other] * A}) == ERR_SHAPE, (r, other)
            assert call(**{r: at[other] * A + (sizes[other] - 4) // step * step}) == ERR_SHAPE, (r, other)        # its last word
            assert call(**{r: at[other] * A - (sizes[r] - 1) // step * step}) == ERR_SHAPE, (r, other)            # this one's last word


def test_binding_takes_both_counts_or_none():
    z = torch.zeros(2, 4, dtype=torch.int32)
    args = (z[:, 0], z[:, 0], None, z[0], z[0, :1], z, 4, 64, z[:, 0], z[:, 0], z, z, None, z[0, :1])
    for one in (dict(held=z[:, 0]), dict(held_after=z[:, 0])):
        with pytest.raises(ValueError):
            loza.loza_ssa_step_tables(*args, **one)
    with pytest.raises(TypeError):
        loza.loza_ssa_step_tables(*args, held=z[:, 0], held_after=z[:, 0])
