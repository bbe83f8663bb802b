"""Probabilities from logits and the record of tokens on the GPU against their definition."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import beside_reference as N
from tests import step_reference as R

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
FN = {BF: loza.loza_ssa_token_probs, F32: loza.loza_ssa_token_probs_f32}


def _dev(x, dev):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(dev)


def _bits(ok):
    """[B, n, V] truth values as words of 32."""
    B, n, V = ok.shape
    padded = np.zeros((B, n, (V + 31) // 32 * 32), dtype=bool)
    padded[..., :V] = ok
    return np.packbits(padded, axis=-1, bitorder="little").view(np.int32)


class Call:
    """Inputs of a call with everything in it; parts can be left out."""

    def __init__(self, B, n, V, dtype, seed, bias=7, dev="cuda"):
        rng = np.random.default_rng(seed)
        self.B, self.n, self.V, self.dtype, self.dev, self.rng = B, n, V, dtype, dev, rng
        g = torch.Generator(device=dev).manual_seed(seed)
        self.logits = (torch.randn(B, n, V, generator=g, device=dev) * 3).to(dtype)
        self.parents = np.stack([R.random_parents(rng, n) for _ in range(B)])
        self.lens = rng.integers(1, n + 1, size=B).astype(np.int32)
        self.masks = np.stack([R.masks_of(self.parents[b], int(self.lens[b])) for b in range(B)]).view(np.int64)
        few = max(1, min(V, 30))
        self.tokens = rng.integers(0, few, size=(B, n)).astype(np.int32)
        row = (V + 7) // 8 * 8
        self.seen = np.zeros((B, row), dtype=np.uint16)
        hit = rng.random((B, row)) < 0.2
        self.seen[hit] = rng.choice([1, 2, 5, 0x8000, 0x8003, 0xffff], size=int(hit.sum()))
        self.rep, self.fre, self.pre = (rng.choice(x, size=B).astype(np.float32) for x in ([1.0, 1.2, 0.8], [0.0, 0.1, -0.3], [0.0, 0.7, -0.2]))
        self.temp = rng.choice([1.0, 0.7, 0.0, 2.5], size=B).astype(np.float32)
        self.bt = rng.integers(0, V, size=(B, bias)).astype(np.int32) if bias else None
        self.bv = rng.normal(0, 3, size=(B, bias)).astype(np.float32) if bias else None
        if bias > 3:
            self.bt[:, 1], self.bt[:, 2], self.bt[0, 3] = self.bt[:, 0], self.tokens[:, 0], -1     # twice the same, one of the tree's own, none
            if B > 1:
                self.bt[1, 3] = V
        self.ok = rng.random((B, n, V)) < 0.6
        self.ok[0, 0] = False                               # a grammar that leaves nothing
        if V > 40:
            self.ok[-1, -1, 40:] = False

    def run(self, probs=None, logits=None, stream=None, ws=None):
        d = self.dev
        probs = torch.full((self.B, self.n, self.V), 9.0, device=d) if probs is None else probs
        FN[self.dtype](self.logits if logits is None else logits, probs, ws, tree_lens=_dev(self.lens, d), tokens=_dev(self.tokens, d), masks=_dev(self.masks, d),
                       seen=None if self.seen is None else _dev(self.seen.view(np.int16), d), repetition=_dev(self.rep, d), frequency=_dev(self.fre, d),
                       presence=_dev(self.pre, d), temperature=_dev(self.temp, d), bias_tokens=_dev(self.bt, d), bias_values=_dev(self.bv, d),
                       allowed=None if self.ok is None else _dev(_bits(self.ok), d), stream=stream)
        return probs

    def check(self, probs, rows=None):
        got, l = probs.double().cpu().numpy(), self.logits.float().cpu().numpy()
        pick = lambda a, b, other: other if a is None else a[b]
        worst = 0.0
        for b in range(self.B):
            count = self.n if self.lens is None else max(0, int(self.lens[b]))
            for r in range(self.n) if rows is None else rows:
                if r >= count:
                    assert (got[b, r] == 9.0).all()
                    continue
                z = np.zeros(self.V, np.int64) if self.seen is None else self.seen[b, :self.V].astype(np.int64)
                said, occurs = z & 0x7fff, z != 0
                if self.masks is not None:
                    for a in range(min(self.n, count)):
                        if int(np.uint64(self.masks[b, r])) >> a & 1 and 0 <= self.tokens[b, a] < self.V:
                            said[self.tokens[b, a]] += 1
                            occurs[self.tokens[b, a]] = True
                bias = [] if self.bt is None else list(zip(self.bt[b].tolist(), self.bv[b]))
                c = N.changed_logits(l[b, r], said, occurs, pick(self.rep, b, 1.0), pick(self.fre, b, 0.0), pick(self.pre, b, 0.0), bias,
                                     None if self.ok is None else self.ok[b, r])
                with np.errstate(all="ignore"):
                    rep, row = float(pick(self.rep, b, 1.0)), np.abs(l[b, r].astype(np.float64))
                    size = 4 * occurs * (row * max(rep, 1 / rep) + abs(float(pick(self.fre, b, 0.0))) * said + abs(float(pick(self.pre, b, 0.0))))
                ref, bound = N.probabilities(c, float(pick(self.temp, b, 1.0)), np.where(np.isfinite(size), size, 0.0))
                err = np.abs(got[b, r] - ref)
                assert (err <= bound).all(), (b, r, float(err.max()), int(err.argmax()))
                worst = max(worst, float((err / np.maximum(bound, 1e-37)).max()))
        return worst


SIZES = [(1, 1, 1), (1, 1, 7), (2, 3, 8), (3, 5, 33), (1, 1, 2047), (2, 64, 2049), (5, 2, 4096), (1, 1, 32003), (70, 1, 5001), (4, 9, 20011), (2100, 1, 700), (40, 60, 333)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,n,V", SIZES)
def test_everything(gpu_device, B, n, V, dtype):
    c = Call(B, n, V, dtype, B + n + V)
    c.check(c.run())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("without", ["masks", "seen", "rep", "fre", "pre", "temp", "bt", "ok", "lens", "all"])
def test_without(gpu_device, without, dtype):
    c = Call(3, 6, 6001, dtype, 5)
    parts = ["masks", "seen", "rep", "fre", "pre", "temp", "bt", "ok", "lens"] if without == "all" else [without]
    for part in parts:
        setattr(c, part, None)
        if part == "masks":
            c.tokens = None
        if part == "bt":
            c.bv = None
    c.check(c.run())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_rows(gpu_device, dtype):
    """Rows of several slices, of one, and longer than a slice can be."""
    for B, n, V, rows in ((1, 1, 300_001, None), (16, 64, 40_007, (0, 31)), (1, 2, 2_000_003, None)):
        c = Call(B, n, V, dtype, 11)
        c.check(c.run(), rows)


def test_many_biases(gpu_device):
    c = Call(2, 3, 3001, F32, 3, bias=1024)
    c.check(c.run())


def test_rows_that_lie_apart_and_in_place(gpu_device):
    """Logits of a padded vocabulary, at any alignment of its elements; probabilities in the place of the logits."""
    for dtype in (BF, F32):
        for row, begin in ((5056, 0), (5001, 0), (5011, 3)):
            c = Call(3, 4, 5001, dtype, 8)
            ref = c.run()
            c.check(ref)
            wide = torch.full((3, 4, row + begin), float("nan"), dtype=dtype, device=gpu_device)
            part = wide[..., begin:begin + 5001]
            part.copy_(c.logits)
            assert torch.equal(c.run(logits=part), ref)
    for V in (5001, 70_003):
        c = Call(3, 4, V, F32, 8)
        c.lens[:] = 4
        c.masks = np.stack([R.masks_of(c.parents[b], 4) for b in range(3)]).view(np.int64)
        ref, x = c.run(), c.logits.clone()
        assert torch.equal(c.run(probs=x, logits=x), ref)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_that_are_not_finite(gpu_device, dtype):
    """NaN and infinities where nothing is allowed do not matter; where it is, a NaN weighs nothing, -inf nothing, and +inf shares the row."""
    c = Call(4, 2, 3001, dtype, 4)
    c.temp[:] = [1.0, 0.0, 0.5, 1.0]
    c.lens[:] = 2
    c.masks = np.stack([R.masks_of(c.parents[b], 2) for b in range(4)]).view(np.int64)
    ref = c.run()
    bad = torch.from_numpy(~c.ok).to(gpu_device)
    for value in (float("nan"), float("inf"), -float("inf")):
        l = torch.where(bad, torch.full_like(c.logits, value), c.logits)
        assert torch.equal(c.run(logits=l), ref)
    c.seen[:, 100:200] = 0
    c.bt[(c.bt >= 100) & (c.bt < 200)] = 5
    c.ok[:, :, 100:200] = True
    c.logits[:, 0, 100:150] = float("nan")
    c.logits[:, 1, 120], c.logits[:, 1, 170], c.logits[:, 1, 130:160] = float("inf"), float("inf"), -float("inf")
    got = c.run()
    c.check(got)
    assert bool((got[[0, 2, 3], 1, 120] == 0.5).all()) and bool((got[[0, 2, 3], 1, 170] == 0.5).all()) and bool((got[1, 1, 120] == 1.0).all())
    c.logits[:] = -float("inf")
    assert not bool(c.run().any())
    c.logits[:] = float("nan")
    assert not bool(c.run().any())


def test_ties_and_temperatures(gpu_device):
    """Greedy rows take the first of equals, also one of the tokens that are done apart; temperatures that divide by nothing are greedy, too."""
    V, B = 9000, 6
    c = Call(B, 1, V, BF, 6, bias=0)
    c.ok = c.seen = c.masks = c.tokens = None
    c.logits.zero_()
    c.temp = np.array([0.0, -1.0, np.nan, np.inf, 1e-40, 1.0], dtype=np.float32)
    got = c.run()
    assert bool((got[:5, 0, 0] == 1.0).all()) and not bool(got[:5, 0, 1:].any()) and float((got[5] - 1.0 / V).abs().max()) <= 1e-9
    c.bt, c.bv = np.tile(np.array([[4000, 5000, 4000]], np.int32), (B, 1)), np.tile(np.array([[0.25, 0.5, 0.25]], np.float32), (B, 1))
    got = c.run()
    assert bool((got[:5, 0, 4000] == 1.0).all()) and bool((got[:5].sum(-1) == 1.0).all())
    c.check(got)
    c.temp = np.array([2.0 ** -100, 2.0 ** 100, 2.0 ** -20, 100.0, 2.0 ** -101, 1e-10], dtype=np.float32)
    c.logits = torch.randn(B, 1, V, device=gpu_device).mul(30).to(BF)
    c.check(c.run())


def test_a_mask_of_nothing_and_nodes_beyond_the_tree(gpu_device):
    """A row whose mask is 0 has no path; bits of nodes at or beyond tree_lens and tokens that are none do not count; lens of 0 leave all rows."""
    c = Call(4, 8, 2500, F32, 2)
    c.masks[:] = -1
    c.masks[:, 2] = 0
    c.tokens[0, 1], c.tokens[1, 0] = -5, 2500
    c.lens[:] = [8, 5, 0, -3]
    c.check(c.run())


def test_probabilities_beyond_2_31(gpu_device):
    B, n, V = 260, 64, 131072                               # 2.2 billion
    c = Call(1, 1, V, BF, 1)
    c.temp[:], c.ok, c.bt, c.bv, c.masks, c.tokens, c.seen, c.lens, c.rep, c.fre, c.pre = 0.7, None, None, None, None, None, None, None, None, None, None
    ref = c.run()
    c.check(ref)
    logits = torch.zeros(B, n, V, dtype=BF, device=gpu_device)
    logits[-1, -1] = c.logits[0, 0]
    probs = torch.empty(B, n, V, device=gpu_device)
    loza.loza_ssa_token_probs(logits, probs, temperature=torch.full((B,), 0.7, device=gpu_device))
    # (one slice a row here, several there: another order of the sums, by the bound of both)
    _, bound = N.probabilities(N.changed_logits(c.logits[0, 0].float().cpu().numpy(), np.zeros(V), np.zeros(V, bool), 1, 0, 0, [], None), float(np.float32(0.7)))
    assert ((probs[-1, -1] - ref[0, 0]).double().abs().cpu().numpy() <= 2 * bound).all()
    assert float((probs[-1, -2] - 1.0 / V).abs().max()) <= 1e-9 and float((probs[0, 0] - 1.0 / V).abs().max()) <= 1e-9
    del logits, probs
    torch.cuda.empty_cache()


def test_same_bits_again_on_another_stream_and_in_a_graph(gpu_device):
    c = Call(4, 7, 30_011, BF, 7)
    ref = c.run()
    s, ws = torch.cuda.Stream(), torch.empty(loza.loza_ssa_token_probs_workspace_bytes(4, 7, 30_011), dtype=torch.uint8, device=gpu_device)
    s.wait_stream(torch.cuda.current_stream())
    other = torch.full_like(ref, 9.0)
    d = gpu_device
    parts = dict(tree_lens=_dev(c.lens, d), tokens=_dev(c.tokens, d), masks=_dev(c.masks, d), seen=_dev(c.seen.view(np.int16), d), repetition=_dev(c.rep, d),
                 frequency=_dev(c.fre, d), presence=_dev(c.pre, d), temperature=_dev(c.temp, d), bias_tokens=_dev(c.bt, d), bias_values=_dev(c.bv, d),
                 allowed=_dev(_bits(c.ok), d))
    torch.cuda.synchronize()
    loza.loza_ssa_token_probs(c.logits, other, ws, stream=s, **parts)
    s.synchronize()
    assert torch.equal(other, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loza.loza_ssa_token_probs(c.logits, other, ws, **parts)
    for k in range(3):
        c.logits.copy_(c.logits.flip(-1))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(other, c.run()), k
    with pytest.raises(loza.LozaError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            loza.loza_ssa_token_probs(c.logits, other)


# ---- the record -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("B,n,V", [(1, 1, 1), (3, 9, 97), (2, 3000, 50), (5, 700, 32003), (300, 5, 1000), (2, 70_000, 20_001), (3, 5000, 200_000)])
@pytest.mark.parametrize("path", [False, True])
def test_count(gpu_device, B, n, V, path):
    rng = np.random.default_rng(B + n + V)
    row = (V + 7) // 8 * 8 + 8 * (V % 3)
    seen = rng.choice(np.array([0, 0, 0, 1, 0x8000, 0x7ffe, 0x7fff, 0xfffe, 0xffff], np.uint16), size=(B, row))
    tokens = rng.integers(-2, V + 2, size=(B, n)).astype(np.int32)
    tokens[:, : n // 3] = rng.integers(0, min(V, 5), size=(B, n // 3))           # the same again and again
    lens = rng.integers(-1, n + 3, size=B).astype(np.int32)
    lens[0] = n
    prompt = rng.integers(-1, n + 1, size=B).astype(np.int32)
    fresh = (rng.random(B) < 0.5).astype(np.int32) * 7
    at = rng.integers(-1, n + 1, size=(B, n)).astype(np.int32) if path else None
    for p, f in ((None, None), (prompt, None), (None, fresh), (prompt, fresh)):
        t = _dev(seen.view(np.int16), gpu_device)
        loza.loza_ssa_count_tokens(_dev(tokens, gpu_device), _dev(lens, gpu_device), t, V, path=_dev(at, gpu_device), prompt_lens=_dev(p, gpu_device), fresh=_dev(f, gpu_device))
        assert np.array_equal(t.cpu().numpy().view(np.uint16), N.count(seen, tokens, lens, V, at, p, f))


def test_count_stops_at_its_largest(gpu_device):
    n = 40_000
    tokens = torch.full((1, n), 3, dtype=I32, device=gpu_device)
    seen = torch.zeros(1, 8, dtype=torch.int16, device=gpu_device)
    loza.loza_ssa_count_tokens(tokens, torch.tensor([n], dtype=I32, device=gpu_device), seen, 5)
    assert seen[0].tolist() == [0, 0, 0, 32767, 0, 0, 0, 0]
    loza.loza_ssa_count_tokens(tokens, torch.tensor([n], dtype=I32, device=gpu_device), seen, 5, prompt_lens=torch.tensor([1], dtype=I32, device=gpu_device))
    assert seen[0].tolist() == [0, 0, 0, -1, 0, 0, 0, 0]


@pytest.mark.parametrize("B,V", [(1, 8191), (3, 8193), (2, 16_384), (2, 1_048_576), (1, 1_048_577)])
@pytest.mark.parametrize("n", [255, 256, 4095, 4096, 16_385, 32_771])
def test_count_around_its_steps(gpu_device, B, V, n):
    """One entry a thread or slices of the vocabulary; loads of four, alone or four under way; requests of no entries, fresh or not."""
    rng = np.random.default_rng(n + V)
    row = (V + 7) // 8 * 8 + 16
    seen = rng.choice(np.array([0, 0, 1, 0x8000, 0x7fff], np.uint16), size=(B, row))
    tokens = rng.integers(-1, V + 1, size=(B, n)).astype(np.int32)
    tokens[:, 0], tokens[:, -1], tokens[:, n // 2] = V - 1, -2 ** 31, 2 ** 31 - 1
    lens = np.array([n, 0, n - 1][:B], np.int32)
    prompt = np.array([n // 2, 5, n][:B], np.int32)
    for fresh in (None, np.array([0, 1, 0][:B], np.int32), np.array([1, 0, 1][:B], np.int32)):
        t = _dev(seen.view(np.int16), gpu_device)
        loza.loza_ssa_count_tokens(_dev(tokens, gpu_device), _dev(lens, gpu_device), t, V, prompt_lens=_dev(prompt, gpu_device), fresh=_dev(fresh, gpu_device))
        assert np.array_equal(t.cpu().numpy().view(np.uint16), N.count(seen, tokens, lens, V, None, prompt, fresh))


# ---- penalties that change nothing, grammars that leave little, tokens done apart -----------------------------------------

@pytest.mark.parametrize("temp", [0.0, 0.9])
@pytest.mark.parametrize("rep", [1.0, 1.3, 0.7])
@pytest.mark.parametrize("fre", [0.0, -0.0, 0.2, float("inf"), float("-inf")])
@pytest.mark.parametrize("pre", [0.0, 0.4, float("inf")])
def test_each_penalty_alone_and_together(gpu_device, pre, fre, rep, temp):
    for dtype in (BF, F32):
        c = Call(2, 3, 2600, dtype, 21)
        for name, x in (("rep", rep), ("fre", fre), ("pre", pre), ("temp", temp)):
            getattr(c, name)[:] = x
        if np.isinf(fre) or np.isinf(pre):                  # (tokens that were said are sure or barred then: some have to be left)
            c.seen[:, 1::2] = 0
        c.check(c.run())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,n,V", [(1, 2, 40_000), (4, 64, 5003), (2, 3, 9001)])
def test_grammars_that_leave_little(gpu_device, B, n, V, dtype):
    """Whole blocks of 512 tokens are barred, NaNs and infinities in them; what is left: one token, one of a tree's own, a biased one, the last ones."""
    c = Call(B, n, V, dtype, 31)
    c.ok[:] = False
    c.ok[0, 0, 3] = True
    c.ok[0, 1, int(c.tokens[0, 0])] = True
    c.ok[-1, 0, int(c.bt[-1, 0])] = True
    c.ok[-1, -1, V - 2:] = True
    c.ok[-1, 1, 512:1024] = True
    c.ok[-1, 1, 2048:2050] = True
    c.temp[:] = [(0.0, 1.3)[b % 2] for b in range(B)]
    barred = torch.from_numpy(~c.ok).to(gpu_device)
    c.logits[barred] = torch.tensor([float("nan"), float("inf"), -1.0], device=gpu_device).to(dtype)[torch.arange(int(barred.sum()), device=gpu_device) % 3]
    got = c.run()
    finite = c.logits.clone()
    finite[barred] = -1.0
    c.logits = finite
    assert torch.equal(c.run(), got)
    c.check(got)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,n,V", [(1, 2, 1500), (1, 2, 20_000), (70, 4, 5003)])
def test_tokens_done_apart_side_by_side(gpu_device, B, n, V, dtype):
    """Many biased tokens of one block, in its two halves, at its edges, at the end of a vocabulary, some of them barred, said, on a path."""
    c = Call(B, n, V, dtype, 41, bias=300)
    c.bt[:, :280] = c.rng.permuted(np.tile(np.arange(500, 780), (B, 1)), axis=1)
    c.bt[:, 280:290] = np.arange(V - 10, V)
    c.bt[:, 290:] = c.bt[:, :10]
    c.tokens[:, 0], c.tokens[:, 1] = 511, V - 1
    c.temp[:] = [(1.3, 0.0, 0.8)[b % 3] for b in range(B)]
    c.check(c.run())


@pytest.mark.parametrize("parts", ["all of it", "no record", "nothing"])
@pytest.mark.parametrize("B,n,V", [(256, 1, 66_001), (4, 64, 131_072), (4, 64, 65_536), (800, 1, 16_384), (12, 64, 16_385), (800, 1, 8192), (768, 1, 8193), (800, 1, 1025), (400, 2, 513), (800, 1, 511)])
def test_rows_of_each_number_of_threads(gpu_device, B, n, V, parts):
    for dtype in (BF, F32):
        c = Call(B, n, V, dtype, V, bias=9)
        if parts != "all of it":
            c.seen = None
        if parts == "nothing":
            c.masks = c.tokens = c.bt = c.bv = c.ok = None
        c.check(c.run(), (0, n // 2, n - 1) if B < 100 else None)


@pytest.mark.parametrize("B,V", [(256, 131_073), (256, 200_003), (260, 262_144), (256, 262_145)])
def test_many_rows_of_large_vocabularies(gpu_device, B, V):
    c = Call(B, 1, V, BF, V)
    c.ok = None                                            # (a truth value for each token is all of the test's time)
    got = c.run()
    keep = [0, B // 2, B - 1]
    for name in ("seen", "rep", "fre", "pre", "temp", "bt", "bv", "lens", "masks", "tokens"):
        setattr(c, name, getattr(c, name)[keep])
    c.B, c.logits = 3, c.logits[keep]
    c.check(got[keep])


@pytest.mark.parametrize("B,n,V", [(256, 1, 66_001), (800, 1, 4001), (300, 1, 20_001)])
def test_rows_in_place(gpu_device, B, n, V):
    c = Call(B, n, V, F32, 77)
    c.lens[:] = n
    ref, x = c.run(), c.logits.clone()
    assert torch.equal(c.run(probs=x, logits=x), ref)
