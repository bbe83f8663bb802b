"""The step's calls on tensors whose offsets pass 32 bits: rows at the far end of a large cache, probabilities and heads beyond 2^31 elements. Each
result is compared, bit by bit, with that of a small tensor that holds the same rows."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import step_reference as R

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


def _rand(shape, seed, dev):
    g = torch.Generator(device=dev).manual_seed(seed)
    return torch.randn(shape, generator=g, device=dev).to(BF)


def test_rows_at_the_end_of_a_large_cache(gpu_device):
    """4.3 million latent rows (4.95 GB, 2.5 billion elements): append, tree attention and accepted rows in its last pages."""
    page, n, pages_far, per = 128, 9, 33_600, 6
    rng = np.random.default_rng(1)
    small_table = np.arange(per, dtype=np.int32)[None].copy()
    far_table = (pages_far - 1 - np.arange(per, dtype=np.int32))[None].copy()
    P = 600
    rows, q, k_new = _rand((P, 1, 576), 1, gpu_device), _rand((1, n, 64, 576), 2, gpu_device), _rand((n, 1, 576), 3, gpu_device)
    parents = R.random_parents(rng, n)
    masks = torch.from_numpy(R.masks_of(parents, n)[None].view(np.int64)).to(gpu_device)
    freq = loza.loza_ssa_rope_frequencies(64, 10000.0)[0].to(gpu_device)
    pos = torch.tensor([P + bin(int(m)).count("1") - 1 for m in R.masks_of(parents, n)], dtype=I32, device=gpu_device)
    i32 = lambda *x: torch.tensor(x, dtype=I32, device=gpu_device)
    path = torch.full((1, n), -1, dtype=I32, device=gpu_device)
    path[0, :4] = i32(0, 2, 5, 8)
    results = []
    for pages, table in ((per, small_table), (pages_far, far_table)):
        pool = torch.zeros(pages, page, 1, 576, dtype=BF, device=gpu_device)
        at = torch.arange(P + n)
        slot = torch.from_numpy(table[0][at // page].astype(np.int64) * page + (at % page).numpy()).to(gpu_device)
        assert pages == per or int(slot.min()) * 576 > 2 ** 31
        pool.view(-1, 1, 576)[slot[:P]] = rows
        slots = slot[P:].to(I32)
        loza.loza_ssa_rope_append(None, k_new, None, pos, slots, freq, None, pool, None, 0, 512, True)
        out, lse = torch.empty(1, n, 64, 512, dtype=BF, device=gpu_device), torch.empty(1, 64, n, dtype=torch.float32, device=gpu_device)
        loza.loza_ssa_extend_tree(q, pool, pool, i32(P + n), i32(n), masks, out, lse, 16, 300, 1, 192 ** -0.5,
                                  block_table=torch.from_numpy(np.pad(table, ((0, 0), (0, 2)))).to(gpu_device))
        loza.loza_ssa_keep_accepted(pool[None], None, slots[None].contiguous(), path, i32(4))
        torch.cuda.synchronize()
        results.append((out, lse, pool.view(-1, 1, 576)[slot].clone()))
        del pool
    for a, b in zip(*results):
        assert torch.equal(a, b)
    torch.cuda.empty_cache()


def test_rope_beyond_2_31_elements(gpu_device):
    T, H, d = 60_000, 64, 576                       # 2.2 billion elements
    x = torch.zeros(T, H, d, dtype=BF, device=gpu_device)
    x[-3:] = _rand((3, H, d), 4, gpu_device)
    pos = torch.arange(T, dtype=I32, device=gpu_device)
    freq = loza.loza_ssa_rope_frequencies(64, 10000.0)[0].to(gpu_device)
    out = torch.empty_like(x)
    loza.loza_ssa_rope(x, pos, freq, out, 512, True)
    ref = torch.empty(3, H, d, dtype=BF, device=gpu_device)
    loza.loza_ssa_rope(x[-3:].contiguous(), pos[-3:].contiguous(), freq, ref, 512, True)
    assert torch.equal(out[-3:], ref) and not bool(out[:-3].any())
    del x, out
    torch.cuda.empty_cache()


def test_verification_beyond_2_31_probabilities(gpu_device):
    B, n, V = 9, 64, 4_000_000                      # 2.3 billion
    target = torch.zeros(B, n, V, device=gpu_device)
    rng = np.random.default_rng(2)
    parents, tokens = np.tile(np.arange(-1, n - 1, dtype=np.int32), (B, 1)), rng.integers(0, V, size=(B, n)).astype(np.int32)
    stop = rng.integers(1, n, size=B)               # the chain holds up to node `stop`, whose own token follows
    stop[-1] = n - 1
    last = rng.integers(0, V, size=B)
    for b in range(B):
        for r in range(stop[b] + 1):
            target[b, r, int(tokens[b, r + 1]) if r < stop[b] else int(last[b])] = 1.0
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(gpu_device)
    path, lens, nxt = (torch.empty(*s, dtype=I32, device=gpu_device) for s in ((B, n), (B,), (B,)))
    ws = torch.empty(loza.loza_ssa_verify_tree_workspace_bytes(B, n, V), dtype=torch.uint8, device=gpu_device)
    u = torch.full((B, n), 0.5, device=gpu_device)
    # a child that is not the target's token is rejected (0 < 0 does not hold), and the next token comes from the target
    loza.loza_ssa_verify_tree(target, None, i32(tokens), i32(parents), i32(np.full(B, n)), u, u[:, 0].contiguous(), path, lens, nxt, ws)
    torch.cuda.synchronize()
    accepted = [int(s) + 1 if s == n - 1 or tokens[b, s + 1] != last[b] else None for b, s in enumerate(stop)]
    for b in range(B):
        if accepted[b] is not None:
            assert int(lens[b]) == accepted[b] and int(nxt[b]) == int(last[b]) and path[b, :accepted[b]].tolist() == list(range(accepted[b]))
    del target
    torch.cuda.empty_cache()
