"""Step tables with pages that requests hold beyond what their caches need, against the definition, and engines that run far beyond what their pools hold once."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import step_reference as R
from tests.step_pages import Pool, step_tables_held

pytestmark = pytest.mark.gpu
I32 = torch.int32


def _call(dev):
    def step(cache, new, parents, free, count, held, table, n, num_pages, page):
        B = len(cache)
        up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)
        mk = lambda *s: torch.full(s, -77, dtype=I32, device=dev)
        granted, seqlens, positions, slots, left, after, t = mk(B), mk(B), mk(B, n), mk(B, n), mk(1), mk(B), up(table)
        masks = None if parents is None else torch.full((B, n), -77, dtype=torch.int64, device=dev)
        given = (up(cache), up(new), None if parents is None else up(parents), up(free), torch.tensor([count], dtype=I32, device=dev))
        h = up(held)
        loza.loza_ssa_step_tables(*given, t, num_pages, page, granted, seqlens, positions, slots, masks, left, held=h, held_after=after)
        torch.cuda.synchronize()
        assert np.array_equal(h.cpu().numpy(), held)
        got = [granted, seqlens, positions, slots, masks, left, t, after]
        return [np.zeros((B, n), np.int64) if x is None else x.cpu().numpy() for x in got]
    return step


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("B,n,page,most,free_share", [
    (1, 1, 32, 4, 1.0), (3, 5, 32, 4, 1.0), (7, 64, 32, 9, 0.4), (300, 17, 64, 6, 0.5), (257, 64, 32, 5, 0.9), (2, 63, 128, 3, 0.0), (1030, 3, 32, 4, 0.7)])
def test_held_pages(gpu_device, B, n, page, most, free_share, tree):
    rng = np.random.default_rng(B * 10 + n)
    cache = rng.integers(0, most * page + 1, size=B).astype(np.int32)
    cache[rng.random(B) < 0.5] //= page                         # (some on a page border, many short)
    cache = np.where(rng.random(B) < 0.3, cache // page * page, cache).astype(np.int32)
    held = np.minimum(-(-cache // page) + rng.integers(-1, 4, size=B), most).clip(0).astype(np.int32)
    new = rng.integers(0, n + 1, size=B).astype(np.int32)
    if B > 6:
        new[2], cache[5], held[1], held[4] = -1, -3, -1, most + 1
    num_pages = B * most
    table = rng.permutation(num_pages).astype(np.int32).reshape(B, most)
    if B > 6:
        table[3, :] = num_pages + 5
    free = rng.permutation(num_pages).astype(np.int32)[:int(num_pages * free_share)]
    parents = np.stack([R.random_parents(rng, n) for _ in range(B)]) if tree else None
    for count in {len(free), len(free) // 2, 0}:
        args = (cache, new, parents, free, count, held, table, n, num_pages, page)
        for name, g, r in zip(("granted", "seqlens", "positions", "slots", "masks", "free_left", "block_table", "held_after"), _call(gpu_device)(*args), step_tables_held(*args)):
            assert np.array_equal(g, r), (name, count)


@pytest.mark.parametrize("B,n,page,most,pages,tree", [(3, 9, 32, 12, 36, True), (16, 64, 32, 20, 200, True), (5, 8, 64, 6, 22, True), (4, 40, 32, 9, 30, False)])
def test_no_page_is_lost(gpu_device, B, n, page, most, pages, tree):
    pool = Pool(np.random.default_rng(n), B, most, page, pages, _call(gpu_device))
    for _ in range(300):
        pool.step(n, tree)
    assert pool.ended > 3


def test_arrays_side_by_side(gpu_device):
    """All arrays of a call one behind the other in one buffer: nothing overlaps, and nothing is written beside its place."""
    B, n, page, most, num_pages = 5, 6, 32, 7, 40
    rng = np.random.default_rng(4)
    cache, new = rng.integers(0, 150, size=B).astype(np.int32), rng.integers(0, n + 1, size=B).astype(np.int32)
    held, free = (-(-cache // page) + 1).astype(np.int32), rng.permutation(num_pages).astype(np.int32)[:9]
    table, parents = rng.permutation(num_pages)[:B * most].astype(np.int32).reshape(B, most), np.stack([R.random_parents(rng, n) for _ in range(B)])
    given = [cache, new, parents, free, np.array([9], np.int32), held, table]
    sizes = [x.size for x in given] + [B, B, B * n, B * n, 2 * B * n, 1, B]
    buf = torch.full((sum(sizes) + 2,), -77, dtype=I32, device=gpu_device)
    odd = (sum(sizes[:11]) + 1) % 2                   # (the masks' place has to be a multiple of 8 bytes)
    parts = list(buf[1 - odd:1 - odd + sum(sizes)].split(sizes))
    for t, x in zip(parts, given):
        t.copy_(torch.from_numpy(x.reshape(-1)))
    c, w, p, f, k, h, t, granted, seqlens, pos, slots, masks, left, after = parts
    loza.loza_ssa_step_tables(c, w, p.view(B, n), f, k, t.view(B, most), num_pages, page, granted, seqlens, pos.view(B, n), slots.view(B, n),
                              masks.view(torch.int64).view(B, n), left, held=h, held_after=after)
    torch.cuda.synchronize()
    ref = step_tables_held(cache, new, parents, free, 9, held, table, n, num_pages, page)
    got = (granted, seqlens, pos, slots, masks.view(torch.int64), left, t, after)
    for g, r in zip(got, ref):
        assert np.array_equal(g.cpu().numpy(), r.reshape(-1))
    for g, x in zip(parts, given[:6]):
        assert np.array_equal(g.cpu().numpy(), x.reshape(-1))
    assert int(buf[-1]) == -77 and (odd == 1 or int(buf[0]) == -77)
