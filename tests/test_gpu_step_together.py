"""The calls of a speculative decoding step together, as an engine makes them: step tables, rotary positions with the rows into a paged latent
cache, attention of the tree, verification, accepted rows; several steps, eager and as one captured graph."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import step_reference as R

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32
B, N, HQ, V, PAGE, MOST, LAYERS = 3, 9, 16, 97, 32, 12, 2
SINK, LOCAL, SCALE = 16, 64, 192 ** -0.5


class Engine:
    """Token t of layer l asks with wq[l, t] (512 columns as they are, 64 rotary ones) and leaves the row wk[l, t]."""

    def __init__(self, dev, seed):
        g = torch.Generator(device=dev).manual_seed(seed)
        rnd = lambda *s, dt=BF: torch.randn(*s, generator=g, device=dev).to(dt)
        self.dev = dev
        self.wq, self.wk, self.head = rnd(LAYERS, V, HQ, 576), rnd(LAYERS, V, 1, 576), rnd(HQ * 512, V, dt=torch.float32) / 20
        freq, self.m = loza.loza_ssa_rope_frequencies(64, 10000.0, 4.0, 64)
        self.freq = freq.to(dev)
        i32 = lambda *s: torch.zeros(*s, dtype=I32, device=dev)
        self.cache_lens, self.new_lens, self.parents, self.tokens = i32(B), torch.full((B,), N, dtype=I32, device=dev), i32(B, N), i32(B, N)
        self.free, self.count, self.left = torch.randperm(B * MOST, generator=torch.Generator().manual_seed(seed)).to(I32).to(dev), i32(1) + B * MOST, i32(1)
        self.table = i32(B, MOST) - 1
        self.granted, self.seqlens, self.positions, self.slots = i32(B), i32(B), i32(B, N), i32(B, N)
        self.masks = torch.zeros(B, N, dtype=torch.int64, device=dev)
        self.cache = torch.full((LAYERS, B * MOST, PAGE, 1, 576), float("nan"), dtype=BF, device=dev)
        self.q = torch.empty(B, N, HQ, 576, dtype=BF, device=dev)
        self.out = torch.zeros(LAYERS, B, N, HQ, 512, dtype=BF, device=dev)
        self.lse = torch.empty(B, HQ, N, dtype=torch.float32, device=dev)
        nb = loza.loza_ssa_extend_tree_workspace_bytes(B, HQ, 1, MOST * PAGE, N, 576, 512, SINK, LOCAL)
        self.ws = torch.empty(max(16, nb), dtype=torch.uint8, device=dev)
        self.vws = torch.empty(loza.loza_ssa_verify_tree_workspace_bytes(B, N, V), dtype=torch.uint8, device=dev)
        self.draft = torch.full((B, N, V), 1.0 / V, device=dev)
        self.target = torch.empty(B, N, V, device=dev)
        self.ua, self.un = torch.empty(B, N, device=dev), torch.empty(B, device=dev)
        self.path, self.path_lens, self.next = i32(B, N), i32(B), i32(B)

    def set_inputs(self, rng, first):
        """A tree per sequence whose root is the token `first`; drafts drawn uniformly."""
        par = np.stack([R.random_parents(rng, N) for _ in range(B)])
        tok = rng.integers(0, V, size=(B, N)).astype(np.int32)
        tok[:, 0] = first
        for t, x in ((self.parents, par), (self.tokens, tok), (self.ua, rng.random((B, N), dtype=np.float32)), (self.un, rng.random(B, dtype=np.float32))):
            t.copy_(torch.from_numpy(x))
        return par, tok

    def step(self):
        loza.loza_ssa_step_tables(self.cache_lens, self.new_lens, self.parents, self.free, self.count, self.table, B * MOST, PAGE,
                                  self.granted, self.seqlens, self.positions, self.slots, self.masks, self.left)
        self.count.copy_(self.left)
        tok = self.tokens.long()
        for layer in range(LAYERS):
            x, k, cache = self.wq[layer][tok], self.wk[layer][tok], self.cache[layer]
            self.q[..., :512].copy_(x[..., :512])
            loza.loza_ssa_rope_append(x.view(B * N, HQ, 576)[..., 512:], k.view(B * N, 1, 576), None, self.positions.view(-1), self.slots.view(-1), self.freq,
                                      self.q.view(B * N, HQ, 576)[..., 512:], cache, None, 0, 512, True, self.m)
            loza.loza_ssa_extend_tree(self.q, cache, cache, self.seqlens, self.granted, self.masks, self.out[layer], self.lse,
                                      SINK, LOCAL, 1, SCALE, block_table=self.table, workspace=self.ws)
        logits = sum(self.out[layer].float().view(B * N, HQ * 512) for layer in range(LAYERS)) @ self.head
        self.target.copy_(torch.softmax(logits, -1).view(B, N, V))
        loza.loza_ssa_verify_tree(self.target, self.draft, self.tokens, self.parents, self.granted, self.ua, self.un, self.path, self.path_lens, self.next, self.vws)
        loza.loza_ssa_keep_accepted(self.cache, None, self.slots, self.path, self.path_lens)
        self.cache_lens.add_(self.path_lens)

    def check(self, history, par, tok):
        """The outputs of one step (tokens `history` before it) and the caches after it."""
        path, lens, nxt = (x.cpu().numpy() for x in (self.path, self.path_lens, self.next))
        ref = R.verify_tree(self.target.cpu().numpy(), self.draft.cpu().numpy(), tok, par, np.full(B, N), self.ua.cpu().numpy(), self.un.cpu().numpy())
        assert all(np.array_equal(a, b) for a, b in zip((path, lens, nxt), ref))
        for b in range(B):
            for r in (0, N // 2, N - 1):
                line = [a for a in range(N) if int(R.masks_of(par[b], N)[r]) >> a & 1]
                want = self.decode(history[b] + [int(tok[b, a]) for a in line])
                for layer in range(LAYERS):          # both are within a half ulp and 1e-2 of the exact value
                    assert torch.allclose(self.out[layer, b, r].float(), want[layer].float(), atol=2e-2, rtol=2 ** -7), (b, r, layer)
            history[b] += [int(tok[b, a]) for a in path[b, :lens[b]]]
            assert int(self.cache_lens[b]) == len(history[b])
            at = torch.arange(len(history[b]), device=self.dev)
            for layer in range(LAYERS):
                rows = self.cache[layer][self.table[b].long()[at // PAGE], at % PAGE, 0]
                assert torch.equal(rows, self.rows(layer, history[b])[:, 0]), (b, layer)
        return nxt

    def rows(self, layer, tokens):
        """The cache rows of a token sequence."""
        k = self.wk[layer][torch.tensor(tokens, device=self.dev)]
        y = torch.empty_like(k)
        loza.loza_ssa_rope(k, torch.arange(len(tokens), dtype=I32, device=self.dev), self.freq, y, 512, True, self.m)
        return y

    def decode(self, tokens):
        """What the last of these tokens gets from a contiguous cache of all of them, layer by layer."""
        res = []
        for layer in range(LAYERS):
            kc = self.rows(layer, tokens)[None].contiguous()
            x = self.wq[layer][tokens[-1]][None].clone()
            loza.loza_ssa_rope(x, torch.tensor([len(tokens) - 1], dtype=I32, device=self.dev), self.freq, x, 512, True, self.m)
            out, lse = torch.empty(1, HQ, 512, dtype=BF, device=self.dev), torch.empty(1, HQ, dtype=torch.float32, device=self.dev)
            nb = loza.loza_ssa_decode_workspace_bytes(1, HQ, 1, len(tokens), 512, SINK, LOCAL)
            loza.loza_ssa_decode(x, kc, kc, torch.tensor([len(tokens)], dtype=I32, device=self.dev), out, lse, SINK, LOCAL, SCALE,
                                 torch.empty(max(16, nb), dtype=torch.uint8, device=self.dev))
            res.append(out[0])
        return res


def test_steps_of_a_speculative_decode(gpu_device):
    e, rng = Engine(gpu_device, 1), np.random.default_rng(1)
    history, first = [[] for _ in range(B)], np.array([1, 2, 3])
    for step in range(14):
        e.new_lens.copy_(torch.tensor([N, N, N], dtype=I32))
        par, tok = e.set_inputs(rng, first)
        e.step()
        torch.cuda.synchronize()
        first = e.check(history, par, tok)
    assert min(len(h) for h in history) >= 14 and max(len(h) for h in history) > 14   # (a step keeps one token at least, some keep more)


def test_a_captured_step_is_replayed(gpu_device):
    """One graph of a whole step against the eager engine, with other inputs at every replay and eager work between the replays."""
    eager, graphed = Engine(gpu_device, 2), Engine(gpu_device, 2)
    rng = np.random.default_rng(2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graphed.set_inputs(rng, np.array([5, 6, 7]))
        graphed.step()                                    # (warm-up on the side stream, then everything back to the start)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    for t in ("cache_lens", "count", "table", "cache"):
        getattr(graphed, t).copy_(getattr(eager, t))
    first = np.array([5, 6, 7])
    for step in range(6):
        seed = int(rng.integers(1 << 30))
        for e in (eager, graphed):
            e.set_inputs(np.random.default_rng(seed), first)
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        for t in ("granted", "seqlens", "positions", "slots", "masks", "left", "table", "out", "lse", "path", "path_lens", "next", "cache_lens"):
            a, b = getattr(eager, t), getattr(graphed, t)
            assert torch.equal(a, b) or (a.dtype.is_floating_point and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))), (step, t)
        assert torch.equal(eager.cache.view(torch.int16), graphed.cache.view(torch.int16)), step
        first = eager.next.cpu().numpy()


def test_another_stream(gpu_device):
    """The calls on a stream that is passed, behind work on that stream, while the current stream is busy with something else."""
    s = torch.cuda.Stream()
    e, f = Engine(gpu_device, 3), Engine(gpu_device, 3)
    rng = np.random.default_rng(3)
    par, tok = e.set_inputs(rng, np.array([1, 1, 1]))
    f.set_inputs(np.random.default_rng(3), np.array([1, 1, 1]))
    torch.cuda.synchronize()
    e.step()
    torch.cuda.synchronize()
    busy = torch.randn(2048, 2048, device=gpu_device)
    for _ in range(10):
        busy = busy @ busy * 1e-3
    kw, cache = dict(stream=s), f.cache[0]
    loza.loza_ssa_step_tables(f.cache_lens, f.new_lens, f.parents, f.free, f.count, f.table, B * MOST, PAGE, f.granted, f.seqlens, f.positions, f.slots, f.masks, f.left, **kw)
    x, k = f.wq[0][f.tokens.long()], f.wk[0][f.tokens.long()]
    s.wait_stream(torch.cuda.current_stream())             # (x and k come from there)
    f.q[..., :512].copy_(x[..., :512])
    loza.loza_ssa_rope_append(x.view(B * N, HQ, 576)[..., 512:], k.view(B * N, 1, 576), None, f.positions.view(-1), f.slots.view(-1), f.freq,
                              f.q.view(B * N, HQ, 576)[..., 512:], cache, None, 0, 512, True, f.m, **kw)
    s.wait_stream(torch.cuda.current_stream())
    loza.loza_ssa_extend_tree(f.q, cache, cache, f.seqlens, f.granted, f.masks, f.out[0], f.lse, SINK, LOCAL, 1, SCALE, block_table=f.table, **kw)
    f.target.copy_(e.target)
    s.wait_stream(torch.cuda.current_stream())
    loza.loza_ssa_verify_tree(f.target, f.draft, f.tokens, f.parents, f.granted, f.ua, f.un, f.path, f.path_lens, f.next, f.vws, **kw)
    loza.loza_ssa_keep_accepted(f.cache[:1], None, f.slots, f.path, f.path_lens, **kw)
    s.synchronize()
    torch.cuda.synchronize()
    for t in ("granted", "seqlens", "positions", "slots", "masks", "left", "table", "path", "path_lens", "next"):
        assert torch.equal(getattr(e, t), getattr(f, t)), t
    assert torch.equal(e.out[0], f.out[0]) and torch.equal(e.cache[0].view(torch.int16), f.cache[0].view(torch.int16))
