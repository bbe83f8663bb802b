"""Verification where single probabilities are no probabilities: a token weighs 0 whose target probability is negative or a NaN, or whose draft
probability is a NaN, with draft probabilities and without."""
import numpy as np
import pytest

from tests import step_reference as R
from tests.test_gpu_step_ops import _probs, _verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B,n,V,kind", [(4, 6, 7, "star"), (6, 40, 500, "tree"), (3, 9, 32003, "tree"), (2, 30, 66000, "star")])
def test_tokens_without_a_probability_weigh_nothing(gpu_device, B, n, V, kind, draft):
    rng = np.random.default_rng(V)
    target, dr = _probs(rng, B, n, V, 1.0)
    parents = np.stack([R.random_parents(rng, n, kind) for _ in range(B)])
    tokens = np.array([[rng.choice(V, p=dr[b, max(0, parents[b, r])].astype(np.float64) / dr[b, max(0, parents[b, r])].astype(np.float64).sum())
                        for r in range(n)] for b in range(B)], np.int32)
    bad = rng.random((B, n, V)) < min(0.3, 20 / V)
    for b in range(B):                                  # some of them at drafted tokens
        for r in range(1, n):
            if rng.random() < 0.3:
                bad[b, parents[b, r], tokens[b, r]] = True
    kind_of = rng.integers(0, 3 if draft else 2, size=bad.shape)
    clean_t, clean_d = np.where(bad, np.float32(0), target), np.where(bad, np.float32(0), dr)
    target, dr = target.copy(), dr.copy()
    target[bad & (kind_of == 0)] = np.nan
    target[bad & (kind_of == 1)] *= -1
    dr[bad & (kind_of == 2)] = np.nan
    # where the target alone is at fault the draft's probability still counts
    clean_d = np.where(bad & (kind_of != 2), dr, clean_d)
    lens = np.full(B, n, np.int32)
    ua, un = rng.random((B, n), dtype=np.float32), rng.random(B, dtype=np.float32)
    got = _verify(gpu_device, target, dr if draft else None, tokens, parents, lens, ua, un)
    for name, g, r in zip(("path", "path_lens", "next_token"), got, R.verify_tree(clean_t, clean_d if draft else None, tokens, parents, lens, ua, un)):
        assert np.array_equal(g, r), name
