"""The operators around the attention of a decode step, from their definitions (numpy, 64 bits and plain integers): what the tests of
loza_ssa_step_tables, loza_ssa_rope, loza_ssa_extend_tree, loza_ssa_verify_tree and loza_ssa_keep_accepted compare with."""
from __future__ import annotations

import numpy as np
import torch

import oracle


def random_parents(rng, n, kind="tree"):
    if kind == "chain":
        return np.arange(-1, n - 1, dtype=np.int32)
    if kind == "star":
        return np.array([-1] + [0] * (n - 1), dtype=np.int32)
    return np.array([-1] + [int(rng.integers(max(0, r - 7), r)) for r in range(1, n)], dtype=np.int32)


def masks_of(parents, count):
    """uint64 ancestor sets (self included) of the first `count` nodes, 0 behind them."""
    m = np.zeros(len(parents), dtype=np.uint64)
    for r in range(count):
        m[r] = np.uint64(1 << r)
        if 0 <= parents[r] < r:
            m[r] |= m[parents[r]]
    return m


def step_tables(cache_lens, new_lens, parents, free_pages, free_count, table, n, num_pages, page):
    B, most = table.shape
    table = table.copy()
    granted, seqlens = np.zeros(B, np.int32), np.zeros(B, np.int32)
    positions, slots, masks = np.full((B, n), -1, np.int32), np.full((B, n), -1, np.int32), np.zeros((B, n), np.uint64)
    free = min(max(0, int(free_count)), len(free_pages))
    asked, left = 0, free
    for b in range(B):
        c, m = int(cache_lens[b]), int(new_lens[b])
        seqlens[b] = c
        if c < 0 or m < 0 or m > n or c + m > most * page:
            continue
        have = -(-c // page)
        need = -(-(c + m) // page) - have
        first = asked
        asked += need
        if need and asked > free:
            continue
        for i in range(need):
            table[b, have + i] = free_pages[free - 1 - first - i]
        if need:
            left = free - asked
        granted[b], seqlens[b] = m, c + m
        for t in range(m):
            r, row = (t, c + t) if parents is not None else (n - m + t, c + t)
            pg = int(table[b, row // page])
            slots[b, r] = pg * page + row % page if 0 <= pg < num_pages else -1
            positions[b, r] = row
        if parents is not None:
            masks[b] = masks_of(parents[b], m)
            for r in range(m):
                positions[b, r] = c + bin(int(masks[b, r])).count("1") - 1
    return granted, seqlens, positions, slots, masks.view(np.int64), np.array([left], np.int32), table


def rope(x, positions, freq, begin, interleaved, m, inverse=False):
    """x [T, H, d] float64; angles in 80-bit arithmetic. Rows of negative positions come back as NaN (nothing is written there)."""
    y = np.array(x, dtype=np.float64)
    k = len(freq)
    first = begin + (2 * np.arange(k) if interleaved else np.arange(k))
    second = first + (1 if interleaved else k)
    ang = np.asarray(positions, dtype=np.longdouble)[:, None] * np.asarray(freq, dtype=np.longdouble)[None, :]
    co, si = (np.asarray(f(ang), dtype=np.float64)[:, None, :] * m for f in (np.cos, np.sin))
    si = -si if inverse else si
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = a * co - b * si, a * si + b * co
    y[np.asarray(positions) < 0] = np.nan
    return y


def rope_bound(x, begin, rot, interleaved, m, y, bf16):
    """Sine and cosine are off by 2 ulp, and half a unit for the reduced angle and for the product with m each; two products and their sum are
    rounded: less than 8 units of 2^-24 of m (|a| + |b|). One rounding to the result's type."""
    s = np.zeros(x.shape)
    k = rot // 2
    first = begin + (2 * np.arange(k) if interleaved else np.arange(k))
    second = first + (1 if interleaved else k)
    s[..., first] = s[..., second] = np.abs(x[..., first]) + np.abs(x[..., second])
    return 8 * 2.0 ** -24 * abs(m) * s + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(y) * (s > 0) + 1e-38


def verify_tree(target, draft, tokens, parents, tree_lens, u_accept, u_next):
    B, n, V = target.shape
    path, lens, nxt = np.full((B, n), -1, np.int32), np.zeros(B, np.int32), np.full(B, -1, np.int32)
    for b in range(B):
        count = min(max(0, int(tree_lens[b])), n)
        if count == 0:
            continue
        at, walk = 0, [0]
        while True:
            w, s, hit = target[b, at].astype(np.float64), 1.0, -1
            q = None if draft is None else draft[b, at].astype(np.float64)
            for r in range(at + 1, count):
                x = int(tokens[b, r])
                if parents[b, r] != at or not 0 <= x < V:
                    continue
                if float(u_accept[b, r]) * (1.0 if q is None else q[x]) * s < w[x]:
                    hit = r
                    break
                if q is None:
                    s -= w[x]
                    w[x] = 0.0
                else:
                    w = np.maximum(w - s * q, 0.0)
                    s = w.sum()
            if hit < 0:
                break
            at = hit
            walk.append(hit)
        path[b, :len(walk)], lens[b] = walk, len(walk)
        cum = np.cumsum(w)
        if not cum[-1] > 0:
            cum = np.cumsum(target[b, at].astype(np.float64))
        if cum[-1] > 0:
            nxt[b] = int(np.searchsorted(cum, float(u_next[b]) * cum[-1], side="right"))
    return path, lens, nxt


def keep_accepted(rows, slots, path, path_lens):
    """rows [layers, R, ...]; a copy with the accepted rows moved."""
    B, n = slots.shape
    new, R = rows.clone(), rows.shape[1]
    for b in range(B):
        for i in range(min(max(0, int(path_lens[b])), n)):
            f = int(path[b, i])
            if 0 <= f < n and 0 <= slots[b, f] < R and 0 <= slots[b, i] < R:
                new[:, int(slots[b, i])] = rows[:, int(slots[b, f])]
    return new


def tree_attention(q, kc, vc, seqlen, count, masks, d_v, sink, local, block, scale, heads, nodes=None):
    """Nodes (all of them by default) of ONE sequence: q [n, Hq, d], kc, vc [L, Hkv, d] (CPU tensors, vc may be kc). A node's path is laid behind the
    rows before the tree, and the oracle is asked for the last of them. Returns out [nodes, heads, d_v], lse [nodes, heads]."""
    n, Hq, d = q.shape
    P = seqlen - count
    nodes = list(range(n)) if nodes is None else nodes
    out, lse = np.zeros((len(nodes), len(heads), d_v)), np.full((len(nodes), len(heads)), -np.inf)
    for i, r in enumerate(nodes):
        m = int(np.uint64(masks[r])) & ((1 << count) - 1)
        if r >= count or m == 0:
            continue
        rows = list(range(P)) + [P + a for a in range(64) if m >> a & 1]
        at = torch.as_tensor(rows)
        k = kc[at][None]
        v = ("alias", d_v) if vc is kc else vc[at][None]
        z = np.zeros(len(heads), np.int64)
        out[i], lse[i] = oracle.ssa_rows(q[r, heads].contiguous(), k, v, z, np.asarray(heads, np.int64), z + len(rows) - 1, Hq=Hq, n_sink=sink,
                                         window=oracle.INT64_MAX if local is None else local, scale=scale, block=block if block > 1 else None)
    return out, lse
