"""Norms with rotary positions, probabilities from logits, and pages, from their definitions (numpy, 64 bits and plain integers): what the tests of
loza_ssa_norm_rope*, loza_ssa_token_probs, loza_ssa_count_tokens and loza_ssa_pages_* compare with."""
from __future__ import annotations

import numpy as np

from tests import step_reference as R

U = 2.0 ** -24                                     # half a step of fp32


# ---- norms with rotary positions ---------------------------------------------------------------------------

def _pairs(begin, k, interleaved):
    first = begin + (2 * np.arange(k) if interleaved else np.arange(k))
    return first, first + (1 if interleaved else k)


def norm(x, weight, begin, dim, eps):
    """(y, r [T, H, 1]): x float64 with its norm columns normed."""
    y, cols = x.copy(), slice(begin, begin + dim)
    if dim == 0:
        return y, np.ones(x.shape[:2] + (1,))
    r = 1.0 / np.sqrt((x[..., cols] ** 2).mean(-1, keepdims=True) + eps)
    y[..., cols] = x[..., cols] * r * (1.0 if weight is None else weight)
    return y, r


def norm_rope(x, weight, begin, dim, eps, positions, freq, rot_begin, interleaved, m):
    """x [T, H, d] float64 normed and rotated; NaN where the position is negative."""
    return R.rope(norm(x, weight, begin, dim, eps)[0], positions, freq, rot_begin, interleaved, m)


def norm_rope_bound(x, weight, begin, dim, eps, freq, rot_begin, interleaved, m, out, half):
    """The squares of a head are added up in at most 24 steps (8 columns a lane or 16 of one each, 6 exchanges), the product, the mean and eps round once
    each: 27 units of the sum, half of them of its root, one each for root and inverse, two for the products with r and w: less than 18 units of 2^-24 of y. A
    rotation adds 8 of m (|a| + |b|) (step_reference.rope_bound). One rounding to the result's type, `half` of it (2^-8 or 2^-24)."""
    y = np.abs(norm(x, weight, begin, dim, eps)[0])
    first, second = _pairs(rot_begin, len(freq), interleaved)
    bound = 18 * U * y
    bound[..., first] = bound[..., second] = 26 * U * abs(m) * (y[..., first] + y[..., second])
    return bound + half * np.abs(out) + 1e-38


def norm_rope_backward(dout, x, weight, begin, dim, eps, positions, freq, rot_begin, interleaved, m):
    """(dx, dweight) from the formulas; rows of padding are NaN in dx and add nothing to dweight."""
    live = np.asarray(positions) >= 0
    g = R.rope(dout, positions, freq, rot_begin, interleaved, m, inverse=True)
    cols, w = slice(begin, begin + dim), 1.0 if weight is None else weight
    _, r = norm(x, weight, begin, dim, eps)
    gn, xn = g[..., cols], x[..., cols]
    h = gn * w
    dx = g.copy()
    dx[..., cols] = r * (h - xn * r ** 2 * (h * xn).mean(-1, keepdims=True))
    return dx, (gn * xn * r)[live].sum((0, 1))


def norm_rope_backward_bounds(dout, x, weight, begin, dim, eps, positions, freq, rot_begin, interleaved, m, dx, half):
    """G: m (|a| + |b|) for rotated columns, |dout| for others; g is off by 8 units of it at most, h = g w by 9, h x by 10. Their mean is added up in 24 steps
    and rounded twice more: 36 units of A = mean(G |w| |x|). r^2 is off by 31 (r by 15), the product with x by 3 more: x r^2 mean(h x) by 70 units of
    |x| r^2 A. Their difference, and the product with r: 9 + 1 + 16 and 70 + 1 + 16 units. dweight: 8 + 15 + 2 a term, and an addition for every row of a
    workgroup (at most 64 and one 768th of the tokens) and every group of lanes (at most 64)."""
    live = np.asarray(positions) >= 0
    first, second = _pairs(rot_begin, len(freq), interleaved)
    G = np.abs(dout)
    G[..., first] = G[..., second] = abs(m) * (np.abs(dout[..., first]) + np.abs(dout[..., second]))
    cols, w = slice(begin, begin + dim), 1.0 if weight is None else np.abs(weight)
    _, r = norm(x, weight, begin, dim, eps)
    Gn, xn = G[..., cols], np.abs(x[..., cols])
    A = (Gn * w * xn).mean(-1, keepdims=True)
    bound = 8 * U * G
    bound[..., cols] = U * r * (26 * Gn * w + 87 * xn * r ** 2 * A)
    T, H, _ = x.shape
    terms = 25 + 64 + (T / 768 + 64) * H
    return bound + half * np.abs(dx) + 1e-38, terms * U * (Gn * xn * r)[live].sum((0, 1)) + 1e-38


# ---- probabilities from logits ----------------------------------------------------------------------------------

def changed_logits(logits, said, occurs, rep, fre, pre, bias, allowed):
    """One row in fp32, each operation rounded (numpy's float32): what the definition says. bias: a list of (token, value) in order."""
    f = np.float32
    l = np.asarray(logits, dtype=f).copy()
    with np.errstate(all="ignore"):
        l = np.where(occurs, np.where(l > 0, l / f(rep), l * f(rep)), l).astype(f)
        l = np.where(said > 0, (l - f(fre) * said.astype(f)) - f(pre), l).astype(f)
        total = np.zeros(len(l), dtype=f)
        for x, v in bias:
            if 0 <= x < len(l):
                total[x] = total[x] + f(v)
        l = (l + total).astype(f)
    if allowed is not None:
        l[~allowed] = -np.inf
    l[np.isnan(l)] = -np.inf
    return l


def probabilities(l, temperature, size=0.0):
    """From the changed logits of a row, in 64 bits, and their bound. `size`: where a row is not greedy its penalties may be rounded otherwise than in
    changed_logits, within 2^-24 of `size`, four times the sum of the absolute values that went into a logit: the rounded 1 / repetition and its product,
    frequency times the number and presence in one step, the two subtractions. A weight is off by 2^-24 of |l - max| / T three times (the difference, its product with
    1 / T, and that number's own rounding) and by 8 units (the exponential's, scalings and the last product); the sum by the weighted mean of that, and V positive
    terms over at least 256 threads of 8 each, whose reference moves once a unit at most (4 units each time), by V / 256 + 4 V / 2048 + 100."""
    l = l.astype(np.float64)
    top = l.max()
    if top == -np.inf:
        return np.zeros(len(l)), np.zeros(len(l))
    if not 2.0 ** -100 <= temperature <= 2.0 ** 100:
        p = np.zeros(len(l))
        p[int(np.argmax(l))] = 1.0
        return p, np.zeros(len(l))
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.where(l == top, 0.0, l - top) / np.float64(temperature)
    e = np.exp(d)
    p = e / e.sum()
    n = len(l)
    live = np.where(np.isfinite(d), np.abs(d), 0.0)
    own = 3 * live + np.where(np.isfinite(l), size, 0.0) / np.float64(temperature)
    units = own + (e * own).sum() / e.sum() + 8 + n / 256 + 4 * n / 2048 + 100
    return p, units * U * p + 1e-37


def count(seen, tokens, lens, V, path=None, prompt_lens=None, fresh=None):
    """seen [B, row] uint16 after the call."""
    seen = seen.copy()
    B, n = tokens.shape
    for b in range(B):
        if fresh is not None and fresh[b]:
            seen[b] = 0
        for i in range(min(max(0, int(lens[b])), n)):
            at = i if path is None else int(path[b, i])
            if not 0 <= at < n or not 0 <= tokens[b, at] < V:
                continue
            x = int(tokens[b, at])
            if prompt_lens is not None and i < prompt_lens[b]:
                seen[b, x] |= 0x8000
            elif seen[b, x] & 0x7fff != 0x7fff:
                seen[b, x] += 1
    return seen


# ---- pages ----------------------------------------------------------------------------------------------------------

def _valid(count, total):
    return min(max(0, int(count)), total)


def pages_fork(source, lens, held, trimmed, free, free_count, shared, table, page, sink_pages):
    B, most = table.shape
    pages = len(shared)
    out = {"forked": np.zeros(B, np.int32), "lens": lens.copy(), "held": held.copy(), "trimmed": trimmed.copy(), "copy_from": np.full(B, -1, np.int32),
           "copy_to": np.full(B, -1, np.int32), "copy_rows": np.zeros(B, np.int32), "shared": shared.copy(), "table": table.copy()}
    left = _valid(free_count, len(free))
    for b in range(B):
        f = int(source[b])
        if not 0 <= f < B or lens[b] != 0 or held[b] != 0 or not 0 <= lens[f] <= most * page:
            continue
        full, rest = divmod(int(lens[f]), page)
        if rest:
            if left == 0:
                continue
            left -= 1
            out["copy_from"][b], out["copy_to"][b], out["copy_rows"][b] = table[f, full], free[left], rest
            out["table"][b, full] = free[left]
        for i in range(full):
            out["table"][b, i] = table[f, i]
            if (i < sink_pages or i >= trimmed[f]) and 0 <= table[f, i] < pages:
                out["shared"][table[f, i]] += 1
        out["forked"][b], out["lens"][b], out["held"][b], out["trimmed"][b] = 1, lens[f], full + (rest > 0), trimmed[f]
    out["left"] = np.array([left], np.int32)
    return out


def window_begin(i, window, block):
    return max(0, (i // block - window + 1) * block)


def pages_free(ending, lens, held, trimmed, table, shared, free, free_count, page, sink_blocks, window, block):
    """trimmed, shared: None where the call has none."""
    B, most = table.shape
    pages = len(free) if shared is None else len(shared)
    sink = -(-sink_blocks * block // page)
    out = {"lens": lens.copy(), "held": held.copy(), "trimmed": None if trimmed is None else trimmed.copy(), "free": free.copy()}
    given = np.zeros(pages, np.int64)
    for b in range(B):
        if not 0 <= lens[b] <= most * page or not 0 <= held[b] <= most:
            continue
        have = max(int(held[b]), -(-int(lens[b]) // page))
        first = max(sink, 0 if trimmed is None else int(trimmed[b]))
        if ending is not None and ending[b]:
            gone = list(range(min(sink, have))) + list(range(first, have))
            for k in ("lens", "held", "trimmed"):
                if out[k] is not None:
                    out[k][b] = 0
        else:
            upto = first if trimmed is None else max(first, window_begin(int(lens[b]), window, block) // page)
            gone = range(first, min(upto, have))
            if trimmed is not None and upto > sink:
                out["trimmed"][b] = upto
        for i in gone:
            if 0 <= table[b, i] < pages:
                given[table[b, i]] += 1
    extra = np.zeros(pages, np.int64) if shared is None else shared.astype(np.int64)
    back = np.nonzero(given > extra)[0]
    at = _valid(free_count, len(free))
    back = back[: len(free) - at]
    out["free"][at: at + len(back)] = back
    out["count"] = np.array([at + len(back)], np.int32)
    out["shared"] = None if shared is None else np.maximum(extra - given, 0).astype(np.int32)
    return out


def pages_compact(table, free, free_count, shared, pages):
    gone = {int(p) for p in free[: _valid(free_count, len(free))] if 0 <= p < pages}
    used = pages - len(gone)
    movers, holes = [p for p in range(used, pages) if p not in gone], [p for p in range(used) if p in gone]
    name = dict(zip(movers, holes))
    pad = lambda x, n: np.array(list(x) + [-1] * (n - len(x)), dtype=np.int32)
    new = np.zeros(pages, np.int32)
    for p in range(pages):
        if p not in gone:
            new[name.get(p, p)] = 0 if shared is None else shared[p]
    return {"table": np.array([[name.get(int(p), int(p)) for p in row] for row in table], dtype=np.int32), "free": pad(list(range(pages - 1, used - 1, -1)), len(free)),
            "count": np.array([len(gone)], np.int32), "shared": new, "copy_from": pad(movers, pages // 2), "copy_to": pad(holes, pages // 2),
            "copies": np.array([len(movers)], np.int32)}
