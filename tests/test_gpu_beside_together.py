"""Steps of a speculative decode with everything around the attention: normed latent rows into a paged cache, attention of the tree, probabilities from logits
under penalties, biases and a grammar, verification, accepted rows, the record of what was said; and after them requests forked and ended and pages behind the
window given back, on a pool that could not hold them. Eager, and as one captured graph."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import beside_reference as N
from tests import step_reference as R
from tests.test_gpu_token_probs import _bits

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32
B, NODES, HQ, V, PAGE, MOST, LAYERS, POOL = 4, 9, 16, 97, 32, 12, 2, 17
SINK, LOCAL, SCALE, EPS = 16, 40, 192 ** -0.5, 1e-6
SINK_PAGES, ROW = 1, 104


class Engine:
    """Token t of layer l asks with wq[l, t] (512 columns as they are, 64 rotary ones) and leaves the row wk[l, t], whose 512 latent columns are normed."""

    def __init__(self, dev, seed):
        g = torch.Generator(device=dev).manual_seed(seed)
        rnd = lambda *s, dt=BF: torch.randn(*s, generator=g, device=dev).to(dt)
        self.dev = dev
        self.wq, self.wk, self.norm = rnd(LAYERS, V, HQ, 576), rnd(LAYERS, V, 1, 576) * 3, [1 + 0.2 * rnd(512, dt=torch.float32) for _ in range(LAYERS)]
        self.head = rnd(HQ * 512, V, dt=torch.float32) / 20
        freq, self.m = loza.loza_ssa_rope_frequencies(64, 10000.0, 4.0, 64)
        self.freq = freq.to(dev)
        i32 = lambda *s: torch.zeros(*s, dtype=I32, device=dev)
        f32 = lambda *s: torch.zeros(*s, dtype=torch.float32, device=dev)
        self.cache_lens, self.held, self.trimmed, self.new_lens, self.ending, self.source = i32(B), i32(B), i32(B), i32(B), i32(B), i32(B) - 1
        self.parents, self.tokens = i32(B, NODES), i32(B, NODES)
        self.free, self.count, self.shared = i32(POOL), i32(1) + POOL, i32(POOL)
        self.free.copy_(torch.randperm(POOL, generator=torch.Generator().manual_seed(seed)))
        self.table = i32(B, MOST) - 1
        self.granted, self.seqlens, self.positions, self.slots, self.left, self.after = i32(B), i32(B), i32(B, NODES), i32(B, NODES), i32(1), i32(B)
        self.masks = torch.zeros(B, NODES, dtype=torch.int64, device=dev)
        self.cache = torch.full((LAYERS, POOL, PAGE, 1, 576), float("nan"), dtype=BF, device=dev)
        self.q = torch.full((B, NODES, HQ, 576), float("nan"), dtype=BF, device=dev)
        self.out, self.lse = torch.zeros(LAYERS, B, NODES, HQ, 512, dtype=BF, device=dev), f32(B, HQ, NODES)
        byte = lambda n: torch.empty(max(16, n), dtype=torch.uint8, device=dev)
        self.ws = byte(loza.loza_ssa_extend_tree_workspace_bytes(B, HQ, 1, MOST * PAGE, NODES, 576, 512, SINK, LOCAL))
        self.vws, self.pws = byte(loza.loza_ssa_verify_tree_workspace_bytes(B, NODES, V)), byte(loza.loza_ssa_token_probs_workspace_bytes(B, NODES, V))
        self.fws = byte(loza.loza_ssa_pages_free_workspace_bytes(POOL))
        self.seen = torch.zeros(B, ROW, dtype=torch.int16, device=dev)
        self.rep, self.fre, self.pre, self.temp = (torch.tensor(x, dtype=torch.float32, device=dev) for x in ([1.0, 1.2, 1.1, 0.9], [0.0, 0.2, 0.0, -0.1], [0.3, 0.0, 0.1, 0.0],
                                                                                                                     [1.0, 0.8, 1.5, 0.0]))
        self.bt, self.bv = i32(B, 3), f32(B, 3)
        self.allowed = i32(B, NODES, (V + 31) // 32)
        self.draft, self.target, self.logits = torch.full((B, NODES, V), 1.0 / V, device=dev), f32(B, NODES, V), f32(B, NODES, V)
        self.ua, self.un = f32(B, NODES), f32(B)
        self.path, self.path_lens, self.next = i32(B, NODES), i32(B), i32(B)
        self.forked, self.lens1, self.held1, self.trimmed1, self.cf, self.ct, self.cr = (i32(B) for _ in range(7))
        self.lens2, self.held2, self.trimmed2, self.count2, self.shared1, self.shared2 = i32(B), i32(B), i32(B), i32(1), i32(POOL), i32(POOL)

    def set_inputs(self, rng, first, new, ending, source):
        par = np.stack([R.random_parents(rng, NODES) for _ in range(B)])
        tok = rng.integers(0, V, size=(B, NODES)).astype(np.int32)
        tok[:, 0] = first
        ok = rng.random((B, NODES, V)) < 0.7
        ok[0] = True
        bt, bv = rng.integers(0, V, size=(B, 3)).astype(np.int32), rng.normal(0, 2, size=(B, 3)).astype(np.float32)
        for t, x in ((self.parents, par), (self.tokens, tok), (self.ua, rng.random((B, NODES), dtype=np.float32)), (self.un, rng.random(B, dtype=np.float32)),
                     (self.allowed, _bits(ok)), (self.bt, bt), (self.bv, bv), (self.new_lens, new), (self.ending, ending), (self.source, source)):
            t.copy_(torch.from_numpy(np.ascontiguousarray(x)))
        return par, tok, ok, bt, bv

    def step(self):
        loza.loza_ssa_step_tables(self.cache_lens, self.new_lens, self.parents, self.free, self.count, self.table, POOL, PAGE, self.granted, self.seqlens,
                                  self.positions, self.slots, self.masks, self.left, held=self.held, held_after=self.after)
        self.count.copy_(self.left)
        self.held.copy_(self.after)
        tok = self.tokens.long()
        for layer in range(LAYERS):
            x, k, cache = self.wq[layer][tok], self.wk[layer][tok], self.cache[layer]
            self.q[..., :512].copy_(x[..., :512])
            loza.loza_ssa_norm_rope_append(x.view(B * NODES, HQ, 576)[..., 512:], None, k.view(B * NODES, 1, 576), self.norm[layer], None, self.positions.view(-1),
                                           self.slots.view(-1), self.freq, self.q.view(B * NODES, HQ, 576)[..., 512:], cache, None, 0, 0, 0, 512, EPS, 0, 512, True, self.m)
            loza.loza_ssa_extend_tree(self.q, cache, cache, self.seqlens, self.granted, self.masks, self.out[layer], self.lse, SINK, LOCAL, 1, SCALE,
                                      block_table=self.table, workspace=self.ws)
        self.logits.copy_((sum(self.out[layer].float().view(B * NODES, HQ * 512) for layer in range(LAYERS)) @ self.head).view(B, NODES, V))
        loza.loza_ssa_token_probs_f32(self.logits, self.target, self.pws, tree_lens=self.granted, tokens=self.tokens, masks=self.masks, seen=self.seen, repetition=self.rep,
                                      frequency=self.fre, presence=self.pre, temperature=self.temp, bias_tokens=self.bt, bias_values=self.bv, allowed=self.allowed)
        loza.loza_ssa_verify_tree(self.target, self.draft, self.tokens, self.parents, self.granted, self.ua, self.un, self.path, self.path_lens, self.next, self.vws)
        loza.loza_ssa_keep_accepted(self.cache, None, self.slots, self.path, self.path_lens)
        loza.loza_ssa_count_tokens(self.tokens, self.path_lens, self.seen, V, path=self.path)
        self.cache_lens.add_(self.path_lens)
        loza.loza_ssa_pages_fork(self.source, self.cache_lens, self.held, self.trimmed, self.free, self.count, self.shared, self.table, POOL, PAGE, SINK, 1, self.forked,
                                 self.lens1, self.held1, self.trimmed1, self.cf, self.ct, self.cr, self.left, self.shared1)
        loza.loza_ssa_pages_copy(self.cache, None, self.cf, self.ct, rows=self.cr)
        self.seen.copy_(torch.where((self.forked != 0)[:, None], self.seen[self.source.long().clamp(0, B - 1)], self.seen))
        loza.loza_ssa_pages_free(self.ending, self.lens1, self.held1, self.trimmed1, self.table, self.shared1, self.free, self.left, POOL, PAGE, SINK, LOCAL, 1,
                                 self.lens2, self.held2, self.trimmed2, self.count2, self.shared2, self.fws)
        self.seen.mul_((self.ending == 0)[:, None].to(torch.int16))
        for a, b in (("cache_lens", "lens2"), ("held", "held2"), ("trimmed", "trimmed2"), ("count", "count2"), ("shared", "shared2")):
            getattr(self, a).copy_(getattr(self, b))

    def rows(self, layer, tokens):
        k = self.wk[layer][torch.tensor(tokens, device=self.dev)]
        y = torch.empty_like(k)
        loza.loza_ssa_norm_rope(k, self.norm[layer], torch.arange(len(tokens), dtype=I32, device=self.dev), self.freq, y, 0, 512, EPS, 512, True, self.m)
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

    def check_pages(self, history):
        """Every page is held as often as `shared` says, or free; the live rows are those of the tokens."""
        table, held, trimmed, lens = (x.cpu().numpy() for x in (self.table, self.held, self.trimmed, self.cache_lens))
        owners = np.zeros(POOL, int)
        for b in range(B):
            for i in range(int(held[b])):
                if i < SINK_PAGES or i >= trimmed[b]:
                    owners[table[b, i]] += 1
        free = self.free[:int(self.count)].tolist()
        assert len(set(free)) == len(free) and all(owners[p] == 0 for p in free) and int((owners > 0).sum()) + len(free) == POOL
        assert np.array_equal(self.shared.cpu().numpy(), np.maximum(owners - 1, 0))
        for b in range(B):
            n = int(lens[b])
            assert n == len(history[b])
            live = [j for j in range(n) if j < SINK or j >= n - LOCAL]
            if live:
                at = torch.tensor(live, device=self.dev)
                for layer in range(LAYERS):
                    got = self.cache[layer][self.table[b].long()[at // PAGE], at % PAGE, 0]
                    assert torch.equal(got, self.rows(layer, history[b])[at, 0]), (b, layer)

    def check_step(self, before, history, par, tok, ok, bt, bv, seen, deep):
        granted, path, lens, nxt = (x.cpu().numpy() for x in (self.granted, self.path, self.path_lens, self.next))
        target, logits = self.target.cpu().numpy(), self.logits.cpu().numpy()
        ref = R.verify_tree(target, self.draft.cpu().numpy(), tok, par, granted, self.ua.cpu().numpy(), self.un.cpu().numpy())
        assert all(np.array_equal(a, b) for a, b in zip((path, lens, nxt), ref))
        rep, fre, pre, temp = (x.cpu().numpy() for x in (self.rep, self.fre, self.pre, self.temp))
        for b in range(B):
            for r in range(int(granted[b])) if deep else ():
                line = [a for a in range(NODES) if int(R.masks_of(par[b], NODES)[r]) >> a & 1]
                want = self.decode(before[b] + [int(tok[b, a]) for a in line])
                for layer in range(LAYERS):            # both are within a half ulp and 1e-2 of the exact value
                    assert torch.allclose(self.out[layer, b, r].float(), want[layer].float(), atol=2e-2, rtol=2 ** -7), (b, r, layer)
                said = (seen[b, :V] & 0x7fff).astype(np.int64)
                np.add.at(said, tok[b, line], 1)
                c = N.changed_logits(logits[b, r], said, (seen[b, :V] != 0) | (said > 0), rep[b], fre[b], pre[b], list(zip(bt[b].tolist(), bv[b])), ok[b, r])
                size = 4 * (np.abs(logits[b, r]).astype(np.float64) * 1.2 + abs(float(fre[b])) * said + abs(float(pre[b])))
                p, bound = N.probabilities(c, float(temp[b]), size)
                assert (np.abs(target[b, r] - p) <= bound).all(), (b, r)
            history[b] += [int(tok[b, a]) for a in path[b, :lens[b]]]
        want = N.count(seen, tok, lens, V, path=path)
        forked, ending, source = (x.cpu().numpy() for x in (self.forked, self.ending, self.source))
        for b in range(B):
            if forked[b]:
                history[b], want[b] = list(history[source[b]]), want[source[b]]
        for b in range(B):
            if ending[b]:
                history[b], want[b] = [], 0
        assert np.array_equal(self.seen.cpu().numpy().view(np.uint16), want)
        return nxt, forked


def _run(rng, engines, run, steps, same):
    history, first = [[] for _ in range(B)], np.array([1, 2, 3, 4])
    seen_forks = seen_ends = seen_trims = shared = 0
    for step in range(steps):
        empty = [b for b in range(B) if not history[b]]
        full = [b for b in range(B) if len(history[b]) + 2 * NODES > MOST * PAGE]
        source, ending = np.full(B, -1, np.int32), np.zeros(B, np.int32)
        new = np.where(rng.random(B) < 0.9, NODES, rng.integers(0, NODES + 1, size=B)).astype(np.int32)
        longest = int(np.argmax([len(h) for h in history]))
        if empty and rng.random() < 0.4 and len(history[longest]) > 3:
            source[empty[0]], new[empty[0]] = longest, 0       # becomes a copy of the longest one
        short = [b for b in range(B) if history[b] and b != longest]
        for b in full or ([int(rng.choice(short))] if short and (int(engines[0].count) < 3 or rng.random() < 0.03) else []):
            ending[b] = 1
        seed = int(rng.integers(1 << 30))
        seen = engines[0].seen.cpu().numpy().view(np.uint16).copy()
        for e in engines:
            inputs = e.set_inputs(np.random.default_rng(seed), first, new, ending, source)
        run()
        torch.cuda.synchronize()
        same(step)
        e = engines[0]
        before = [list(h) for h in history]
        nxt, forked = e.check_step(before, history, *inputs, seen, step % 20 == 0)
        e.check_pages(history)
        first = np.where(nxt >= 0, nxt, first)
        for b in range(B):
            if forked[b]:
                first[b] = first[source[b]]
        seen_forks, seen_ends, seen_trims = seen_forks + int(forked.sum()), seen_ends + int(ending.sum()), seen_trims + int((e.trimmed > 0).any())
        shared = max(shared, int(e.shared.max()))
    return seen_forks, seen_ends, seen_trims, shared


def test_steps_with_everything(gpu_device):
    e = Engine(gpu_device, 5)
    forks, ends, trims, shared = _run(np.random.default_rng(5), [e], e.step, 500, lambda step: None)
    assert forks >= 2 and ends >= 2 and trims >= 2 and shared >= 1


def test_a_captured_step_with_everything(gpu_device):
    eager, graphed = Engine(gpu_device, 6), Engine(gpu_device, 6)
    rng = np.random.default_rng(6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graphed.set_inputs(rng, np.array([5, 6, 7, 8]), np.full(B, NODES, np.int32), np.zeros(B, np.int32), np.full(B, -1, np.int32))
        graphed.step()                                 # (warm-up on the side stream, then everything back to the start)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    state = ("cache_lens", "count", "table", "cache", "held", "free", "trimmed", "shared", "seen", "target", "q")
    for t in state:
        getattr(graphed, t).copy_(getattr(eager, t))

    def both():
        eager.step()
        graph.replay()

    def same(step):
        for t in ("granted", "positions", "slots", "masks", "table", "out", "target", "path", "path_lens", "next", "seen", "cache_lens", "held", "trimmed", "count", "shared", "forked",
                  "cf", "ct", "cr"):
            assert torch.equal(getattr(eager, t), getattr(graphed, t)), (step, t)
        c = int(eager.count)
        assert torch.equal(eager.free[:c], graphed.free[:c]) and torch.equal(eager.cache.view(torch.int16), graphed.cache.view(torch.int16)), step
    forks, ends, trims, shared = _run(rng, [eager, graphed], both, 300, same)
    assert forks >= 1 and ends >= 1 and trims >= 1
