"""Steps of a speculative decode in which requests draft nothing, a part or all of a tree, are refused for lack of pages, and end: the calls together as in
test_gpu_step_together.py, over many page borders, on a pool that could not hold the pages of rows that were not kept; eager, and as one captured graph."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import step_reference as R
from tests.test_gpu_step_together import B, HQ, LAYERS, LOCAL, MOST, N, PAGE, SCALE, SINK, V, Engine

pytestmark = pytest.mark.gpu
I32 = torch.int32
POOL = 9                                               # pages; three requests of up to 12


class Running(Engine):
    def __init__(self, dev, seed):
        super().__init__(dev, seed)
        self.free[:POOL].copy_(torch.randperm(POOL, generator=torch.Generator().manual_seed(seed)).to(I32))
        self.count.fill_(POOL)
        self.held, self.after = torch.zeros(B, dtype=I32, device=dev), torch.zeros(B, dtype=I32, device=dev)

    def step(self):
        loza.loza_ssa_step_tables(self.cache_lens, self.new_lens, self.parents, self.free, self.count, self.table, B * MOST, PAGE, self.granted, self.seqlens,
                                  self.positions, self.slots, self.masks, self.left, held=self.held, held_after=self.after)
        self.count.copy_(self.left)
        self.held.copy_(self.after)
        tok = self.tokens.long()
        self.q.fill_(float("nan"))                     # what rope_append does not write is nobody's
        for layer in range(LAYERS):
            x, k, cache = self.wq[layer][tok], self.wk[layer][tok], self.cache[layer]
            there = (self.positions >= 0)[..., None, None]
            self.q[..., :512].copy_(torch.where(there, x[..., :512], self.q[..., :512]))
            loza.loza_ssa_rope_append(x.view(B * N, HQ, 576)[..., 512:], k.view(B * N, 1, 576), None, self.positions.view(-1), self.slots.view(-1), self.freq,
                                      self.q.view(B * N, HQ, 576)[..., 512:], cache, None, 0, 512, True, self.m)
            loza.loza_ssa_extend_tree(self.q, cache, cache, self.seqlens, self.granted, self.masks, self.out[layer], self.lse,
                                      SINK, LOCAL, 1, SCALE, block_table=self.table, workspace=self.ws)
        logits = sum(self.out[layer].float().view(B * N, HQ * 512) for layer in range(LAYERS)) @ self.head
        self.target.copy_(torch.softmax(logits, -1).view(B, N, V))
        loza.loza_ssa_verify_tree(self.target, self.draft, self.tokens, self.parents, self.granted, self.ua, self.un, self.path, self.path_lens, self.next, self.vws)
        loza.loza_ssa_keep_accepted(self.cache, None, self.slots, self.path, self.path_lens)
        self.cache_lens.add_(self.path_lens)

    def end(self, b):
        """The request gives its pages back."""
        h, c = int(self.held[b]), int(self.count)
        self.free[c:c + h] = self.table[b, :h]
        self.count.add_(h)
        self.held[b] = 0
        self.cache_lens[b] = 0

    def check_pages(self):
        owned = torch.cat([*(self.table[b, :int(self.held[b])] for b in range(B)), self.free[:int(self.count)]])
        assert torch.equal(owned.sort().values.cpu(), torch.arange(POOL, dtype=I32))

    def check_step(self, history, par, tok, new, deep):
        granted, path, lens, nxt = (x.cpu().numpy() for x in (self.granted, self.path, self.path_lens, self.next))
        ref = R.verify_tree(self.target.cpu().numpy(), self.draft.cpu().numpy(), tok, par, granted, self.ua.cpu().numpy(), self.un.cpu().numpy())
        assert all(np.array_equal(a, b) for a, b in zip((path, lens, nxt), ref))
        for b in range(B):
            count = int(granted[b])
            assert count in (0, int(new[b]))
            assert bool((self.out[:, b, count:] == 0).all()) and bool((self.lse[b, :, count:] == -float("inf")).all())
            assert bool(torch.isfinite(self.out[:, b, :count].float()).all()) and bool(torch.isfinite(self.lse[b, :, :count]).all())
            for r in {0, count - 1} if deep and count else ():
                line = [a for a in range(N) if int(R.masks_of(par[b], N)[r]) >> a & 1]
                want = self.decode(history[b] + [int(tok[b, a]) for a in line])
                for layer in range(LAYERS):            # both are within a half ulp and 1e-2 of the exact value
                    assert torch.allclose(self.out[layer, b, r].float(), want[layer].float(), atol=2e-2, rtol=2 ** -7), (b, r, layer)
            history[b] += [int(tok[b, a]) for a in path[b, :lens[b]]]
            assert int(self.cache_lens[b]) == len(history[b])
            if deep and history[b]:
                at = torch.arange(len(history[b]), device=self.dev)
                for layer in range(LAYERS):
                    rows = self.cache[layer][self.table[b].long()[at // PAGE], at % PAGE, 0]
                    assert torch.equal(rows, self.rows(layer, history[b])[:, 0]), (b, layer)


def _steps(rng, engines, run, steps, check):
    """`steps` steps of all engines alike; returns how often a request was refused, ended and ran without a draft."""
    history, first, seen = [[] for _ in range(B)], np.array([1, 2, 3]), [0, 0, 0]
    for step in range(steps):
        new = rng.integers(0, N + 1, size=B).astype(np.int32)
        seed = int(rng.integers(1 << 30))
        for e in engines:
            e.new_lens.copy_(torch.from_numpy(new))
            par, tok = e.set_inputs(np.random.default_rng(seed), first)
        run()
        torch.cuda.synchronize()
        e = engines[0]
        e.check_pages()
        check(step)
        e.check_step(history, par, tok, new, step % 8 == 0)
        nxt, refused = e.next.cpu().numpy(), (e.granted.cpu().numpy() < new)
        first = np.where(nxt >= 0, nxt, first)
        seen[0], seen[2] = seen[0] + int(refused.sum()), seen[2] + int((new == 0).sum())
        over = {int(np.argmax([len(h) for h in history]))} if refused.any() else set()
        over |= {b for b in range(B) if len(history[b]) + N > MOST * PAGE}
        for b in over:
            history[b] = []
            seen[1] += 1
            for e in engines:
                e.end(b)
    return seen


def test_steps_with_partial_work(gpu_device):
    e = Running(gpu_device, 5)
    refused, ended, idle = _steps(np.random.default_rng(5), [e], e.step, 160, lambda step: None)
    assert refused >= 2 and ended >= 2 and idle >= 10


def test_a_captured_step_with_partial_work(gpu_device):
    eager, graphed = Running(gpu_device, 6), Running(gpu_device, 6)
    rng = np.random.default_rng(6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graphed.set_inputs(rng, np.array([5, 6, 7]))
        graphed.step()                                 # (warm-up on the side stream, then everything back to the start)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    for t in ("cache_lens", "count", "table", "cache", "held", "free"):
        getattr(graphed, t).copy_(getattr(eager, t))

    def both():
        eager.step()
        graph.replay()

    def same(step):
        for t in ("granted", "seqlens", "positions", "slots", "masks", "left", "count", "held", "table", "out", "lse", "path", "path_lens", "next", "cache_lens"):
            assert torch.equal(getattr(eager, t), getattr(graphed, t)), (step, t)
        assert torch.equal(eager.cache.view(torch.int16), graphed.cache.view(torch.int16)), step
    refused, ended, idle = _steps(rng, [eager, graphed], both, 100, same)
    assert refused >= 1 and ended >= 1 and idle >= 10
