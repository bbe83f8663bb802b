"""Greedy rows of very small logits: each operation rounded by itself, there too."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import beside_reference as N
from tests.test_gpu_token_probs import _bits

pytestmark = pytest.mark.gpu
F = np.float32


@pytest.mark.parametrize("V", [1000, 30_000])               # a workgroup a row, and slices
@pytest.mark.parametrize("repetition", [1.2, 1.3, 0.7, 3.0, 1.3 * 2.0 ** 19, 1.3 * 2.0 ** 30, 1.3 * 2.0 ** 90, 1.3 * 2.0 ** -30])
def test_quotients_of_tiny_logits(gpu_device, V, repetition):
    """A token that was said, of the logit l, and one that was not, of the logit l / repetition rounded once: the two are equal, and the first of them wins, whichever it is.
    From the smallest number there is to beyond 2^-70, and where the quotient is small."""
    rng = np.random.default_rng(int(V + 10 * repetition))
    exponents = np.concatenate([rng.integers(-149, -70, size=30), np.clip(rng.integers(-149, -120, size=10) + int(np.log2(repetition)), -149, 0)])
    l = np.ldexp(1 + rng.random(40), exponents).astype(F)
    quotient = l / F(repetition)
    keep = quotient > 0
    l, quotient = l[keep], quotient[keep]
    B = 2 * len(l)
    logits = np.full((B, 1, V), -1.0, F)
    seen = np.zeros((B, (V + 7) // 8 * 8), np.int16)
    for i in range(len(l)):
        logits[2 * i, 0, [5, 9]] = quotient[i], l[i]
        seen[2 * i, 9] = 1
        logits[2 * i + 1, 0, [5, 9]] = l[i], quotient[i]
        seen[2 * i + 1, 5] = 1
    full = lambda x: torch.full((B,), x, dtype=torch.float32, device=gpu_device)
    probs = torch.empty(B, 1, V, device=gpu_device)
    for rows in (slice(0, B), slice(0, 2)):
        sub = torch.from_numpy(logits[rows]).to(gpu_device)
        loza.loza_ssa_token_probs_f32(sub, probs[rows], seen=torch.from_numpy(seen[rows]).to(gpu_device), repetition=full(repetition)[rows], temperature=full(0.0)[rows])
        got = probs[rows, 0].cpu().numpy()
        assert (got.argmax(-1) == 5).all() and (got.sum(-1) == 1.0).all(), np.nonzero(got.argmax(-1) != 5)[0] // 2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("frequency,presence", [(0.0, 0.0), (2.0 ** -60, 0.0), (-(2.0 ** -60), 2.0 ** -49), (2.0 ** -45, -(2.0 ** -45)), (0.0, 2.0 ** -70), (0.0, -(2.0 ** -70)), (0.0, -(2.0 ** -51)), (-(2.0 ** -49), 2.0 ** -49)])
def test_tiny_logits_under_penalties(gpu_device, frequency, presence, dtype):
    """Every token that was said has another, not said, with exactly what the penalties leave of it, before it or behind it: the largest are always two, and the first has to win. Tokens
    of ordinary size are there as well and not allowed."""
    rng = np.random.default_rng(5)
    B, V = 24, 2000
    rep = np.resize(np.array([1.3, 0.7, 1.2, 1.0], F), B)
    to = lambda a: torch.from_numpy(a).to(dtype).float().numpy()
    logits, seen = np.full((B, 1, V), 3.0, F), np.zeros((B, V), np.int16)
    ok, want = np.zeros((B, 1, V), bool), []
    for b in range(B):
        at = rng.permutation(V)[:400]
        said, copies = at[:200], at[200:]
        lo = int(rng.integers(-149, -100))
        l = to(np.ldexp(1 + rng.random(200), rng.integers(lo, lo + 30, size=200)).astype(F) * rng.choice(np.array([1, -1], F), size=200))
        counts = rng.integers(1, 4, size=200)
        changed = N.changed_logits(l, counts, np.ones(200, bool), rep[b], frequency, presence, [], None)
        logits[b, 0, said], logits[b, 0, copies], seen[b, said] = l, changed, counts
        logits[b, 0] = to(logits[b, 0])
        ok[b, 0, at] = True
        c, o = np.zeros(V, np.int64), np.zeros(V, bool)
        c[said], o[said] = counts, True
        want.append(int(np.argmax(N.changed_logits(logits[b, 0], c, o, rep[b], frequency, presence, [], ok[b, 0]))))
    full = lambda x: torch.full((B,), x, dtype=torch.float32, device=gpu_device)
    probs = torch.empty(B, 1, V, device=gpu_device)
    fn = loza.loza_ssa_token_probs_f32 if dtype == torch.float32 else loza.loza_ssa_token_probs
    fn(torch.from_numpy(logits).to(gpu_device).to(dtype), probs, seen=torch.from_numpy(seen).to(gpu_device), repetition=torch.from_numpy(rep).to(gpu_device), frequency=full(frequency),
       presence=full(presence), temperature=full(0.0), allowed=torch.from_numpy(_bits(ok)).to(gpu_device))
    got = probs[:, 0].cpu().numpy()
    assert got.argmax(-1).tolist() == want and (got.sum(-1) == 1.0).all()
