"""Attention of a tree of drafted tokens (loza_ssa_extend_tree) against the oracle, path by path."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import helpers as H
from tests import step_reference as R

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _rand(shape, seed, dev):
    g = torch.Generator(device=dev).manual_seed(seed)
    return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(BF)


def _paginate(cache, page, seed):
    """[B, S, ...] -> pool of scattered pages and the table; the pool holds NaN where no row is."""
    B, S = cache.shape[:2]
    per = -(-S // page)
    perm = torch.randperm(B * per + 3, generator=torch.Generator().manual_seed(seed))[:B * per].view(B, per)
    pool = torch.full((B * per + 3, page, *cache.shape[2:]), float("nan"), dtype=cache.dtype, device=cache.device)
    for b in range(B):
        for i in range(per):
            rows = cache[b, i * page:(i + 1) * page]
            pool[int(perm[b, i]), :rows.shape[0]] = rows
    return pool, perm.to(torch.int32).to(cache.device)


def _call(q, kc, vc, lens, counts, masks, sink, local, block, scale, d_v, page=0, workspace=None):
    dev, (B, n, Hq, _) = q.device, q.shape
    out = torch.full((B, n, Hq, d_v), float("nan"), dtype=BF, device=dev)
    lse = torch.full((B, Hq, n), float("nan"), dtype=torch.float32, device=dev)
    i32 = dict(dtype=torch.int32, device=dev)
    table = None
    k, v = kc, vc
    if page:
        k, table = _paginate(kc, page, 5)
        v = k if vc is kc else _paginate(vc, page, 5)[0]
    loza.loza_ssa_extend_tree(q, k, v, torch.tensor(lens, **i32), torch.tensor(counts, **i32), torch.from_numpy(masks.view(np.int64)).to(dev), out, lse,
                              sink, local, block, scale, block_table=table, workspace=workspace)
    torch.cuda.synchronize()
    return out, lse


def _check(q, kc, vc, lens, counts, masks, out, lse, sink, local, block, scale, label, heads, node_step=1):
    """Every row finite or empty; the nodes 0, step, 2 step .. and the last against the oracle."""
    B, n, Hq, _ = q.shape
    d_v = out.shape[3]
    assert not bool(torch.isnan(out.float()).any()) and not bool(torch.isnan(lse).any()), label
    for b in range(B):
        count = min(counts[b], lens[b])
        empty = [r for r in range(n) if r >= count or int(masks[b, r]) & ((1 << count) - 1) == 0]
        assert bool((out[b, empty] == 0).all()) and bool((lse[b][:, empty] == -float("inf")).all()), label
        nodes = sorted(set(range(0, n, node_step)) | {max(0, count - 1)})
        k = kc[b, :lens[b]].cpu()
        v = k if vc is kc else vc[b, :lens[b]].cpu()
        ref, ref_lse = R.tree_attention(q[b].cpu(), k, v, lens[b], count, masks[b], d_v, sink, local, block, scale, heads, nodes)
        got, got_lse = out[b][nodes][:, heads].double().cpu().numpy(), lse[b][heads][:, nodes].double().cpu().numpy().T
        live = np.isfinite(ref_lse)
        if live.any():
            H._judge(got[live], ref[live], got_lse[live], ref_lse[live], BF, int(live.sum()), f"{label} b{b}")


def _masks(rng, n, counts, kind):
    return np.stack([R.masks_of(R.random_parents(rng, n, kind), c) for c in counts])


# B, Hq, Hkv, d, S_max, n, lens, nodes, sink, local, block, page, kind, step of the nodes compared
CASES = [
    (1, 64, 1, 576, 700, 1, [700], [1], 16, 200, 1, 0, "tree", 1),                       # one node: a decode
    (2, 64, 1, 576, 700, 8, [700, 9], [8, 5], 16, 200, 1, 0, "tree", 1),                 # a short cache, padding
    (3, 64, 1, 576, 512, 13, [500, 13, 0], [13, 13, 4], 0, 100, 1, 64, "tree", 1),       # nothing but the tree; an empty cache
    (2, 64, 1, 576, 1024, 64, [1000, 1024], [64, 41], 1, 3, 128, 128, "tree", 9),        # blocks; a full tree across a page border
    (2, 64, 1, 576, 1024, 64, [1001, 517], [64, 63], 5, 9, 1, 32, "chain", 7),           # a window shorter than the path
    (2, 64, 1, 576, 256, 40, [40, 100], [40, 40], 30, 7, 1, 0, "chain", 3),              # sinks that reach into the path
    (1, 128, 2, 576, 900, 17, [889], [17], 64, 333, 1, 0, "tree", 5),                    # two latents
    (2, 8, 2, 128, 900, 37, [900, 333], [37, 20], 64, 300, 1, 0, "tree", 3),             # separate values, grouped heads
    (2, 6, 2, 128, 900, 33, [801, 64], [33, 33], 1, 2, 64, 64, "star", 4),               # 3 heads a group, siblings
    (1, 32, 32, 128, 4600, 64, [4555], [64], 128, 4096, 1, 128, "tree", 21),             # every head its own keys
    (4, 64, 1, 576, 3000, 64, [2999, 2500, 130, 64], [64, 50, 64, 64], 128, 2048, 1, 0, "tree", 31),
    (9, 64, 1, 576, 1500, 64, [1500 - 37 * b for b in range(9)], [64 - b for b in range(9)], 1, 7, 128, 0, "tree", 63),
    (16, 32, 8, 128, 600, 64, [600 - 11 * b for b in range(16)], [64 - 3 * b for b in range(16)], 16, 256, 1, 0, "tree", 63),
    (4, 32, 8, 128, 1200, 64, [1200, 1100, 64, 999], [64, 61, 64, 30], 64, 1000, 1, 32, "tree", 31),
]


@pytest.mark.parametrize("B,Hq,Hkv,d,S_max,n,lens,counts,sink,local,block,page,kind,step", CASES)
def test_tree_attention(gpu_device, B, Hq, Hkv, d, S_max, n, lens, counts, sink, local, block, page, kind, step):
    rng = np.random.default_rng(n * 1000 + S_max)
    q, kc = _rand((B, n, Hq, d), 1, gpu_device), _rand((B, S_max, Hkv, d), 2, gpu_device)
    vc = kc if d == 576 else _rand((B, S_max, Hkv, d), 3, gpu_device)
    d_v, scale = (512, 192 ** -0.5) if d == 576 else (128, 128 ** -0.5)
    masks = _masks(rng, n, counts, kind)
    for b, L in enumerate(lens):
        kc[b, L:] = float("nan")
        vc[b, L:] = float("nan")
    out, lse = _call(q, kc, vc, lens, counts, masks, sink, local, block, scale, d_v, page)
    heads = sorted({0, 1 % Hq, Hq // 2, Hq - 1})
    _check(q, kc, vc, lens, counts, masks, out, lse, sink, local, block, scale, f"tree n{n} lens{lens[:3]}", heads, step)
    # without scratch memory: the same values in another order of the sums
    out1, lse1 = out, lse
    out, lse = _call(q, kc, vc, lens, counts, masks, sink, local, block, scale, d_v, page, workspace=torch.empty(0, dtype=torch.uint8, device=gpu_device))
    _check(q, kc, vc, lens, counts, masks, out, lse, sink, local, block, scale, f"tree, no scratch memory n{n}", heads, step)
    assert torch.allclose(out.float(), out1.float(), atol=2e-2, rtol=2 ** -7)


@pytest.mark.parametrize("d,Hq,Hkv", [(576, 64, 1), (128, 8, 2)])
def test_masks_that_are_no_trees(gpu_device, d, Hq, Hkv):
    """Empty masks among the nodes, nodes that do not see themselves, bits behind the tree, later nodes, all bits."""
    B, n, lens, counts = 2, 40, [333, 37], [40, 33]
    rng = np.random.default_rng(3)
    q, kc = _rand((B, n, Hq, d), 4, gpu_device), _rand((B, 400, Hkv, d), 5, gpu_device)
    d_v, scale = (512, 192 ** -0.5) if d == 576 else (128, 128 ** -0.5)
    masks = rng.integers(0, 1 << 63, size=(B, n), dtype=np.uint64)
    masks[:, 1::5] = 0
    masks[:, 2] = np.uint64(0xFFFFFFFFFFFFFFFF)
    masks[:, 3] = np.uint64(1 << 39)
    for sink, local, block in ((7, 100, 1), (0, 11, 1), (1, 2, 32)):
        out, lse = _call(q, kc, kc, lens, counts, masks, sink, local, block, scale, d_v)
        _check(q, kc, kc, lens, counts, masks, out, lse, sink, local, block, scale, f"any masks, window {local}", [0, Hq - 1], 1)


# the kernels of larger calls: B, Hq, Hkv, d, S_max, n, sink, local, block, page, values are the keys, (kernel, splits > 1), step of the nodes compared
LARGE = [
    (5, 64, 1, 576, 6144, 33, 128, 5000, 1, 0, True, (loza.KERNEL_TILES, True), 16),
    (2, 64, 1, 576, 4096, 64, 1, 20, 128, 128, True, (loza.KERNEL_TILES, True), 31),
    (5, 128, 2, 576, 4900, 63, 64, 4600, 1, 0, True, (loza.KERNEL_TILES, False), 31),     # weights of one term
    (3, 192, 1, 576, 1500, 61, 1, 7, 128, 0, True, (loza.KERNEL_TILES, False), 30),       # of two throughout; 192 heads: tiles across nodes
    (1, 64, 1, 576, 5000, 7, 128, 4500, 1, 0, True, (loza.KERNEL_ROWS, True), 2),
    (4, 32, 8, 128, 600, 33, 16, 256, 1, 64, False, (loza.KERNEL_ROWS, False), 16),       # pairs of row groups
    (4, 32, 8, 128, 600, 33, 16, 256, 1, 0, True, (loza.KERNEL_ROWS, False), 16),
    (1, 12, 4, 128, 4500, 21, 16, 4300, 1, 0, True, (loza.KERNEL_ROWS, True), 10),
    (8, 32, 8, 128, 4400, 37, 64, 4096, 1, 0, False, (loza.KERNEL_D128, True), 18),
    (4, 48, 8, 128, 4416, 61, 1, 60, 64, 32, False, (loza.KERNEL_D128, True), 20),        # 6 heads a group
    (8, 32, 8, 128, 4400, 40, 64, 4096, 1, 0, True, (loza.KERNEL_D128, True), 39),
    (16, 32, 8, 128, 700, 64, 16, 512, 1, 0, True, (loza.KERNEL_D128, False), 63),
    (20, 32, 8, 128, 320, 60, 2, 20, 1, 32, False, (loza.KERNEL_D128, False), 29),        # so few live keys that weights have two terms
    (40, 16, 8, 128, 300, 64, 0, 200, 1, 0, False, (loza.KERNEL_D128, False), 63),        # half a tile
]


@pytest.mark.parametrize("B,Hq,Hkv,d,S_max,n,sink,local,block,page,alias,kernel,step", LARGE)
def test_tree_attention_by_kernel(gpu_device, B, Hq, Hkv, d, S_max, n, sink, local, block, page, alias, kernel, step):
    got, splits = loza.loza_ssa_extend_tree_kernel(B, Hq, Hkv, S_max, n, d, sink, local, block)
    assert (got, splits > 1) == kernel
    rng = np.random.default_rng(n * 1000 + S_max)
    lens = [S_max, n - 2, S_max - 77, S_max // 2 + 5, 127 + n] + [S_max - 13 * b % 200 for b in range(5, B)]
    counts = [n, n, n - 1, max(1, n // 2), n] + [max(1, n - b) for b in range(5, B)]
    lens, counts = lens[:B], [min(c, x) for c, x in zip(counts[:B], lens)]
    q, kc = _rand((B, n, Hq, d), 11, gpu_device), _rand((B, S_max, Hkv, d), 12, gpu_device)
    vc = kc if alias else _rand((B, S_max, Hkv, d), 13, gpu_device)
    d_v, scale = (512, 192 ** -0.5) if d == 576 else (128, 128 ** -0.5)
    masks = _masks(rng, n, counts, "tree")
    masks[0, n // 3] = 0                                   # a node without a mask, and one that does not see itself
    masks[0, n // 2] &= np.uint64(0xFFFFFFFFFFFFFFFF ^ (1 << (n // 2)))
    for b, L in enumerate(lens):
        kc[b, L:] = float("nan")
        vc[b, L:] = float("nan")
    out, lse = _call(q, kc, vc, lens, counts, masks, sink, local, block, scale, d_v, page)
    heads = sorted({0, Hq // 3, Hq - 1})
    few = list(range(min(B, 5))) + ([B - 1] if B > 5 else [])
    k_few = kc[few]
    _check(q[few], k_few, k_few if alias else vc[few], [lens[b] for b in few], [counts[b] for b in few], masks[few], out[few], lse[few], sink, local, block,
           scale, f"kernel {got} in {splits} n{n}", heads, step)
    again, lse_again = _call(q, kc, vc, lens, counts, masks, sink, local, block, scale, d_v, page)     # the same bits
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse_again.view(torch.int32))


@pytest.mark.parametrize("B,Hq,Hkv,d,S_max,n,sink,local,block,page", [
    (2, 64, 1, 576, 4096, 40, 40, 1000, 1, 32), (1, 64, 1, 576, 4096, 3, 1, 3, 128, 64), (9, 64, 1, 576, 4096, 64, 1, 7, 128, 128),
    (8, 32, 8, 128, 4096, 40, 40, 2000, 1, 32), (16, 32, 8, 128, 2048, 60, 1, 5, 64, 32), (2, 32, 8, 128, 4096, 9, 33, 700, 1, 64)])
def test_pages_without_a_live_key_are_not_read(gpu_device, B, Hq, Hkv, d, S_max, n, sink, local, block, page):
    """Pages between the sink and the first window key hold NaN and their table entries are no pages."""
    rng = np.random.default_rng(page)
    q, kc = _rand((B, n, Hq, d), 14, gpu_device), _rand((B, S_max, Hkv, d), 15, gpu_device)
    vc = kc if d == 576 else _rand((B, S_max, Hkv, d), 16, gpu_device)
    d_v, scale = (512, 192 ** -0.5) if d == 576 else (128, 128 ** -0.5)
    lens, counts = [S_max - 31 * b for b in range(B)], [n - b % 3 for b in range(B)]
    masks = _masks(rng, n, counts, "tree")
    pool, table = _paginate(kc, page, 6)
    vpool = pool if vc is kc else _paginate(vc, page, 6)[0]
    for b in range(B):
        P = lens[b] - counts[b]
        first = max(0, (P // block - local + 1) * block)
        for i in range(-(-sink * block // page), first // page):
            pool[int(table[b, i])] = float("nan")
            vpool[int(table[b, i])] = float("nan")
            table[b, i] = (-1, pool.shape[0] + 7, -2 ** 31)[i % 3]
    out, lse = torch.empty(B, n, Hq, d_v, dtype=BF, device=gpu_device), torch.empty(B, Hq, n, dtype=torch.float32, device=gpu_device)
    i32 = dict(dtype=torch.int32, device=gpu_device)
    loza.loza_ssa_extend_tree(q, pool, vpool, torch.tensor(lens, **i32), torch.tensor(counts, **i32), torch.from_numpy(masks.view(np.int64)).to(gpu_device), out, lse,
                              sink, local, block, scale, block_table=table)
    torch.cuda.synchronize()
    few = sorted({0, B - 1})
    k_few = kc[few]
    _check(q[few], k_few, k_few if vc is kc else vc[few], [lens[b] for b in few], [counts[b] for b in few], masks[few], out[few], lse[few], sink, local, block, scale,
           f"dead pages, page {page}", [0, Hq - 1], max(1, n // 3))


def test_rows_with_large_results(gpu_device):
    """Rows whose weight sits on one key of the tree, or of the cache."""
    B, n, lens, counts = 2, 64, [1500, 1400], [64, 64]
    rng = np.random.default_rng(5)
    q, kc = _rand((B, n, 64, 576), 6, gpu_device), _rand((B, 1500, 1, 576), 7, gpu_device)
    masks = _masks(rng, n, counts, "tree")
    q[0, 5, 3] = 3 * kc[0, lens[0] - 64 + 5, 0]
    q[0, 40, 60] = 3 * kc[0, 1000, 0]
    q[1] *= 4
    out, lse = _call(q, kc, kc, lens, counts, masks, 128, 700, 1, 192 ** -0.5, 512)
    assert out[0, 5, 3].abs().max() >= 2
    _check(q, kc, kc, lens, counts, masks, out, lse, 128, 700, 1, 192 ** -0.5, "large results", [3, 60], 5)


def test_a_chain_is_an_extend(gpu_device):
    B, n, S = 3, 11, 900
    q, kc = _rand((B, n, 64, 576), 8, gpu_device), _rand((B, S, 1, 576), 9, gpu_device)
    lens = [900, 512, 100]
    masks = np.stack([R.masks_of(R.random_parents(None, n, "chain"), n)] * B)
    out, lse = _call(q, kc, kc, lens, [n] * B, masks, 16, 300, 1, 192 ** -0.5, 512)
    ref, ref_lse = torch.empty_like(out), torch.empty_like(lse)
    loza.loza_ssa_extend(q, kc, kc, torch.tensor(lens, dtype=torch.int32, device=gpu_device), ref, ref_lse, 16, 300, 192 ** -0.5)
    torch.cuda.synchronize()
    # either is within a half ulp and 1e-2 of the exact value
    assert torch.allclose(out.float(), ref.float(), atol=2e-2, rtol=2 ** -7) and torch.allclose(lse, ref_lse, atol=4e-5)
