"""Forks of requests whose own numbers are out of range: left out, as every call on pages does with such requests."""
import numpy as np
import pytest

from tests import beside_reference as N
from tests.test_gpu_pages import Pool, _fork

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [10, 200])                     # one workgroup for all of them, and one each
def test_a_source_that_holds_an_impossible_number_of_pages_is_not_forked(gpu_device, B):
    page, most = 32, 6
    p = Pool(np.random.default_rng(B), B, page, most)
    p.lens[:5], p.held[:5] = [70, 70, 64, 70, 70], [-1, most + 1, -2 ** 31, most, 2 ** 31 - 1]
    p.table[:5, :3] = np.arange(15).reshape(5, 3)
    p.lens[5:], p.held[5:] = 0, 0
    source = np.full(B, -1, np.int32)
    source[5:10] = [0, 1, 2, 3, 4]
    got = _fork(gpu_device, p, source, 0, 1)
    taken = source.copy()
    for b in np.nonzero(source >= 0)[0]:
        if not 0 <= p.held[source[b]] <= most:
            taken[b] = -1
    ref = N.pages_fork(taken, p.lens, p.held, p.trimmed, p.free, p.count, p.shared, p.table, page, 0)
    for k in ref:
        assert np.array_equal(got[k], ref[k]), k
    assert got["forked"].sum() == 1 and got["forked"][8] == 1 and got["lens"][8] == 70
