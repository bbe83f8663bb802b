"""Step tables with pages that requests hold beyond what their caches need, from the definition (plain integers)."""
import numpy as np

from tests import step_reference as R


def step_tables_held(cache_lens, new_lens, parents, free_pages, free_count, held, table, n, num_pages, page):
    """What loza_ssa_step_tables_held gives: granted, seqlens, positions, slots, masks, free_left, table, held_after."""
    B, most = table.shape
    table, held_after = table.copy(), np.array(held, np.int32)
    granted, seqlens = np.zeros(B, np.int32), np.array(cache_lens, np.int32)
    positions, slots, masks = np.full((B, n), -1, np.int32), np.full((B, n), -1, np.int32), np.zeros((B, n), np.uint64)
    free = min(max(0, int(free_count)), len(free_pages))
    asked, left = 0, free
    for b in range(B):
        c, m, h = int(cache_lens[b]), int(new_lens[b]), int(held[b])
        if c < 0 or m < 0 or m > n or c + m > most * page or h < 0 or h > most:
            continue
        have = max(h, -(-c // page))
        need = max(0, -(-(c + m) // page) - have)
        held_after[b] = have
        first = asked
        asked += need
        if need and asked > free:
            continue
        for i in range(need):
            table[b, have + i] = free_pages[free - 1 - first - i]
        if need:
            left = free - asked
        held_after[b] = have + need
        granted[b], seqlens[b] = m, c + m
        if parents is not None:
            masks[b] = R.masks_of(parents[b], m)
        for t in range(m):
            r, row = (t, c + t) if parents is not None else (n - m + t, c + t)
            pg = int(table[b, row // page])
            slots[b, r] = pg * page + row % page if 0 <= pg < num_pages else -1
            positions[b, r] = row if parents is None else c + bin(int(masks[b, r])).count("1") - 1
    return granted, seqlens, positions, slots, masks.view(np.int64), np.array([left], np.int32), table, held_after


class Pool:
    """The pages of an engine whose requests keep a part of the rows of each step, and end when their caches are full: `step_tables` gives the arrays
    after a step. Every page has one owner, a request or the free list, after every step."""

    def __init__(self, rng, B, most, page, pages, step_tables):
        self.rng, self.page, self.pages, self.step_tables = rng, page, pages, step_tables
        self.free, self.count = rng.permutation(pages).astype(np.int32), pages
        self.cache, self.held, self.table = np.zeros(B, np.int32), np.zeros(B, np.int32), np.full((B, most), -1, np.int32)
        self.refused = self.ended = 0

    def step(self, n, tree):
        B, most = self.table.shape
        full = self.cache + n > most * self.page
        for b in np.flatnonzero(full | (self.rng.random(B) < 0.01)):      # these end
            h = int(self.held[b])
            self.free[self.count:self.count + h] = self.table[b, :h]
            self.count += h
            self.cache[b] = self.held[b] = 0
            self.ended += 1
        new = self.rng.integers(0, n + 1, size=B).astype(np.int32)
        parents = np.stack([R.random_parents(self.rng, n) for _ in range(B)]) if tree else None
        granted, seqlens, positions, slots, masks, left, self.table, self.held = self.step_tables(
            self.cache, new, parents, self.free, self.count, self.held, self.table, n, self.pages, self.page)
        self.count = int(left[0])
        used = [self.table[b, :self.held[b]] for b in range(B)]
        owned = np.concatenate([*used, self.free[:self.count]])
        assert len(owned) == self.pages and np.array_equal(np.sort(owned), np.arange(self.pages))
        for b in range(B):
            mine = slots[b][slots[b] >= 0]
            assert len(mine) == granted[b] == len(set(mine.tolist())) and np.isin(mine // self.page, used[b]).all()
            assert self.held[b] <= -(-int(self.cache[b]) // self.page) + -(-n // self.page) + 1    # (what its rows need, and a step's)
        self.refused += int((granted < new).sum())
        kept = np.where(granted > 0, self.rng.integers(1, n + 1, size=B) % np.maximum(granted, 1) + 1, 0) if tree else granted
        self.cache = (self.cache + kept).astype(np.int32)
