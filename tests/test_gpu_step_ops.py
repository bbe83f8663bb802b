"""Step tables, rotary positions, verification and accepted rows on the GPU against their definitions."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import step_reference as R

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _dev(x, dev):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dev)


# ---- tables --------------------------------------------------------------------------------------------

def _tables(dev, cache, new, parents, free, count, table, n, num_pages, page):
    B = len(cache)
    i32 = dict(dtype=torch.int32, device=dev)
    o = {k: torch.full(s, -77, **i32) for k, s in (("granted", (B,)), ("seqlens", (B,)), ("positions", (B, n)), ("slots", (B, n)), ("left", (1,)))}
    masks = torch.full((B, n), -77, dtype=torch.int64, device=dev) if parents is not None else None
    t = _dev(table, dev)
    loza.loza_ssa_step_tables(_dev(cache, dev), _dev(new, dev), None if parents is None else _dev(parents, dev), _dev(free, dev),
                              torch.tensor([count], **i32), t, num_pages, page, o["granted"], o["seqlens"], o["positions"], o["slots"], masks, o["left"])
    torch.cuda.synchronize()
    got = [o["granted"], o["seqlens"], o["positions"], o["slots"], masks, o["left"], t]
    return [None if x is None else x.cpu().numpy() for x in got]


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("B,n,page,most,free_share", [
    (1, 1, 32, 4, 1.0), (3, 5, 32, 4, 1.0), (7, 64, 32, 9, 0.4), (300, 17, 64, 6, 0.5), (257, 64, 32, 5, 0.9), (2, 63, 128, 3, 0.0), (1030, 3, 32, 4, 0.7)])
def test_tables(gpu_device, B, n, page, most, free_share, tree):
    rng = np.random.default_rng(B * 100 + n)
    cache = rng.integers(0, most * page + 1, size=B).astype(np.int32)
    cache[rng.random(B) < 0.3] //= page
    cache[rng.random(B) < 0.3] //= page           # (some on a page border, some empty)
    cache = np.where(rng.random(B) < 0.3, cache // page * page, cache).astype(np.int32)
    new = rng.integers(0, n + 1, size=B).astype(np.int32)
    if B > 6:
        new[2], new[4], cache[5] = -1, n + 1, -3
    num_pages = B * most
    perm = rng.permutation(num_pages).astype(np.int32)
    table = perm.reshape(B, most).copy()
    if B > 6:
        table[3, :] = num_pages + 5                 # pages that do not exist
        table[6, 0] = -9
    total = int(B * most * free_share)
    free = rng.integers(0, num_pages, size=total).astype(np.int32)
    parents = np.stack([R.random_parents(rng, n) for _ in range(B)]) if tree else None
    if tree and n > 4:
        parents[0, 2], parents[0, 3], parents[B - 1, 4] = 2, 60, -5    # no parents: roots of their own
    for count in {total, total // 2, total + 10, -1}:
        got = _tables(gpu_device, cache, new, parents, free, count, table, n, num_pages, page)
        ref = R.step_tables(cache, new, parents, free, count, table, n, num_pages, page)
        for name, g, r in zip(("granted", "seqlens", "positions", "slots", "masks", "free_left", "block_table"), got, ref):
            if g is not None:
                assert np.array_equal(g, r), (name, count)


def test_tables_of_a_long_chunk(gpu_device):
    B, n, page, most = 3, 5000, 128, 100
    rng = np.random.default_rng(1)
    cache, new = np.array([0, 7777, 12799], np.int32), np.array([5000, 4097, 1], np.int32)
    table = rng.permutation(B * most).astype(np.int32).reshape(B, most)
    free = rng.permutation(B * most).astype(np.int32)
    got = _tables(gpu_device, cache, new, None, free, len(free), table, n, B * most, page)
    ref = R.step_tables(cache, new, None, free, len(free), table, n, B * most, page)
    for i in (0, 1, 2, 3, 5, 6):
        assert np.array_equal(got[i], ref[i]), i


# ---- rotary positions ------------------------------------------------------------------------------------

ROPE = [   # T, H, d, begin, rot, interleaved
    (1, 1, 64, 0, 64, True), (5, 3, 576, 512, 64, True), (5, 3, 576, 512, 64, False), (33, 8, 128, 0, 128, False), (2050, 2, 128, 64, 64, True),
    (7, 2, 96, 16, 32, False), (7, 5, 31, 3, 6, False), (7, 5, 31, 3, 6, True), (4, 1, 2, 0, 2, True), (3, 2, 1030, 6, 1024, False), (9, 64, 64, 0, 64, False),
]


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("T,H,d,begin,rot,inter", ROPE)
def test_rope_and_its_gradient(gpu_device, T, H, d, begin, rot, inter, dtype):
    g = torch.Generator(device=gpu_device).manual_seed(T + d)
    freq, m = loza.loza_ssa_rope_frequencies(rot, 10000.0, 32.0, 32768)
    rng = np.random.default_rng(T)
    pos = rng.integers(0, 1 << 20, size=T).astype(np.int32)
    pos[rng.random(T) < 0.2] = -1
    pos[-1] = (1 << 31) - 130
    x = torch.randn(T, H, d, generator=g, device=gpu_device).to(dtype)
    fn = loza.loza_ssa_rope if dtype == BF else loza.loza_ssa_rope_f32
    args = (_dev(pos, gpu_device), freq.to(gpu_device))
    for inverse in (False, True):
        out = torch.full_like(x, 77.0)
        fn(x, *args, out, begin, inter, m, inverse=inverse)
        ref = R.rope(x.double().cpu().numpy(), pos, freq.numpy(), begin, inter, m, inverse)
        got, dead = out.double().cpu().numpy(), pos < 0
        assert (got[dead] == 77.0).all()
        err = np.abs(got - ref)[~dead]
        bound = R.rope_bound(x.double().cpu().numpy(), begin, rot, inter, m, ref, dtype == BF)[~dead]
        assert (err <= bound).all(), float((err - bound).max())
        y = x.clone()                                          # in place: the same bits
        fn(y, *args, y, begin, inter, m, inverse=inverse)
        assert torch.equal(y[~torch.from_numpy(dead).to(gpu_device)], out[~torch.from_numpy(dead).to(gpu_device)])
        assert torch.equal(y[torch.from_numpy(dead).to(gpu_device)], x[torch.from_numpy(dead).to(gpu_device)])


def test_rope_gradient_against_differences(gpu_device):
    """<dout, (f(x + h) - f(x - h)) / 2> = <gradient, h>: f is linear, so only the rounding of fp32 is left."""
    g = torch.Generator(device=gpu_device).manual_seed(2)
    T, H, d = 37, 4, 128
    freq, m = loza.loza_ssa_rope_frequencies(64, 10000.0, 8.0, 4096)
    pos, freq = torch.arange(T, dtype=torch.int32, device=gpu_device) * 911, freq.to(gpu_device)
    x, h, dout = (torch.randn(T, H, d, generator=g, device=gpu_device) for _ in range(3))

    def f(z):
        y = torch.empty_like(z)
        loza.loza_ssa_rope_f32(z, pos, freq, y, 64, False, m)
        return y.double()
    dx = torch.empty_like(dout)
    loza.loza_ssa_rope_f32(dout, pos, freq, dx, 64, False, m, inverse=True)
    left, right = (dout.double() * (f(x + h) - f(x - h)) / 2).sum(), (dx.double() * h.double()).sum()
    assert abs(float(left - right)) < 1e-2     # 18,944 products of size 2, each off by 2^-22 of that: 9e-3 if all erred the same way


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_rope_strides(gpu_device, dtype):
    """Slices of wider rows, transposed heads, a row that is not aligned, a broadcast input."""
    T, H, d = 19, 6, 64
    g = torch.Generator(device=gpu_device).manual_seed(3)
    freq, m = loza.loza_ssa_rope_frequencies(d, 10000.0)
    pos = torch.arange(T, dtype=torch.int32, device=gpu_device) * 31
    fn = loza.loza_ssa_rope if dtype == BF else loza.loza_ssa_rope_f32
    wide = torch.randn(T, H, 576, generator=g, device=gpu_device).to(dtype)
    flipped = torch.randn(H, T, d, generator=g, device=gpu_device).to(dtype).transpose(0, 1)
    odd = torch.randn(T, H, d + 1, generator=g, device=gpu_device).to(dtype)[..., 1:]
    same = torch.randn(T, 1, d, generator=g, device=gpu_device).to(dtype).expand(T, H, d)
    for x in (wide[..., 512:], flipped, odd, same):
        ref = torch.empty(T, H, d, dtype=dtype, device=gpu_device)
        fn(x.contiguous(), pos, freq.to(gpu_device), ref, 0, True, m)
        for make in (lambda: torch.zeros(T, H, 576, dtype=dtype, device=gpu_device)[..., 512:],
                     lambda: torch.zeros(H, T, d, dtype=dtype, device=gpu_device).transpose(0, 1),
                     lambda: torch.zeros(T, H, d + 1, dtype=dtype, device=gpu_device)[..., 1:]):
            out = make()
            fn(x, pos, freq.to(gpu_device), out, 0, True, m)
            assert torch.equal(out, ref)
    before = wide.clone()
    fn(wide[..., 512:], pos, freq.to(gpu_device), wide[..., 512:], 0, True, m)      # in place on a slice: the rest stays
    assert torch.equal(wide[..., :512], before[..., :512]) and not torch.equal(wide, before)


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("T,Hq,Hkv,dq,dk,dv,rot,inter", [(1, 64, 1, 64, 576, 0, 64, True), (70, 64, 1, 64, 576, 0, 64, False), (33, 8, 2, 128, 128, 128, 64, False),
                                                         (9, 0, 3, 0, 40, 24, 8, True), (9, 2, 1, 33, 35, 7, 6, False)])
def test_rope_append(gpu_device, T, Hq, Hkv, dq, dk, dv, rot, inter, dtype):
    g = torch.Generator(device=gpu_device).manual_seed(T)
    rng = np.random.default_rng(T)
    rows = 200
    mk = lambda *s: torch.randn(*s, generator=g, device=gpu_device).to(dtype)
    freq, m = loza.loza_ssa_rope_frequencies(rot, 10000.0, 4.0, 1000)
    pos, slots = rng.integers(0, 1 << 20, size=T).astype(np.int32), rng.permutation(rows)[:T].astype(np.int32)
    if T > 6:
        pos[1], slots[2], slots[3], slots[4] = -1, -1, rows, -(1 << 31)
    q = mk(T, Hq, dq) if Hq else None
    q_out = torch.full((T, Hq, dq), 9.0, dtype=dtype, device=gpu_device) if Hq else None
    k, k_rows = mk(T, Hkv, dk), mk(rows // 4, 4, Hkv, dk)
    v, v_rows = (mk(T, Hkv, dv), mk(rows // 4, 4, Hkv, dv)) if dv else (None, None)
    fn = loza.loza_ssa_rope_append if dtype == BF else loza.loza_ssa_rope_append_f32
    k0, v0 = k_rows.clone(), None if v is None else v_rows.clone()
    fn(q, k, v, _dev(pos, gpu_device), _dev(slots, gpu_device), freq.to(gpu_device), q_out, k_rows, v_rows, dq - rot, dk - rot, inter, m)
    one = loza.loza_ssa_rope if dtype == BF else loza.loza_ssa_rope_f32
    if Hq:
        ref = torch.full_like(q_out, 9.0)
        one(q, _dev(pos, gpu_device), freq.to(gpu_device), ref, dq - rot, inter, m)
        assert torch.equal(q_out, ref)
    ref = torch.full_like(k, 9.0)
    one(k, _dev(pos, gpu_device), freq.to(gpu_device), ref, dk - rot, inter, m)
    k0, k_now = k0.view(rows, Hkv, dk), k_rows.view(rows, Hkv, dk)
    for t in range(T):
        if pos[t] >= 0 and 0 <= slots[t] < rows:
            k0[int(slots[t])] = ref[t]
            if v is not None:
                v0.view(rows, Hkv, dv)[int(slots[t])] = v[t]
    assert torch.equal(k_now, k0) and (v is None or torch.equal(v_rows, v0))


# ---- verification ------------------------------------------------------------------------------------------

def _verify(dev, target, draft, tokens, parents, lens, ua, un, ws=None):
    B, n, V = target.shape
    i32 = dict(dtype=torch.int32, device=dev)
    path, pl, nx = torch.full((B, n), -77, **i32), torch.full((B,), -77, **i32), torch.full((B,), -77, **i32)
    if ws is None:
        ws = torch.full((loza.loza_ssa_verify_tree_workspace_bytes(B, n, V),), 255, dtype=torch.uint8, device=dev)
    f = lambda x: None if x is None else _dev(x, dev)
    loza.loza_ssa_verify_tree(f(target), f(draft), f(tokens), f(parents), f(lens), f(ua), f(un), path, pl, nx, ws)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (path, pl, nx)]


@pytest.mark.parametrize("V", [1, 2, 3, 5, 255, 1023, 4099, 70001])
def test_verify_rows_of_any_alignment(gpu_device, V):
    """Probabilities that start 0 to 3 elements behind an aligned address, target and draft alike or not."""
    rng = np.random.default_rng(V)
    B, n = 2, 6
    target, dr = _probs(rng, B, n, V, 1.0)
    parents = np.stack([R.random_parents(rng, n, "star") for _ in range(B)])
    tokens, lens = rng.integers(0, V, size=(B, n)).astype(np.int32), np.full(B, n, np.int32)
    ua, un = rng.random((B, n), dtype=np.float32), rng.random(B, dtype=np.float32)
    i32 = dict(dtype=torch.int32, device=gpu_device)
    ws = torch.empty(loza.loza_ssa_verify_tree_workspace_bytes(B, n, V), dtype=torch.uint8, device=gpu_device)
    for a, b in ((1, 1), (3, 3), (0, 2), (2, 1)):
        at = lambda x, k: torch.cat([torch.zeros(k), torch.from_numpy(x).flatten()]).to(gpu_device)[k:].view(B, n, V)
        for draft in (dr, None):
            path, pl, nx = torch.full((B, n), -77, **i32), torch.full((B,), -77, **i32), torch.full((B,), -77, **i32)
            t, d = at(target, a), None if draft is None else at(draft, b)
            loza.loza_ssa_verify_tree(t, d, _dev(tokens, gpu_device), _dev(parents, gpu_device), _dev(lens, gpu_device), _dev(ua, gpu_device), _dev(un, gpu_device), path, pl, nx, ws)
            torch.cuda.synchronize()
            for g, r in zip((path, pl, nx), R.verify_tree(target, draft, tokens, parents, lens, ua, un)):
                assert np.array_equal(g.cpu().numpy(), r), (a, b)


def _probs(rng, B, n, V, noise):
    x = rng.standard_normal((B, n, V)) * 2
    soft = lambda z: (np.exp(z - z.max(-1, keepdims=True)) / np.exp(z - z.max(-1, keepdims=True)).sum(-1, keepdims=True)).astype(np.float32)
    return soft(x), soft(x + noise * rng.standard_normal((B, n, V)))


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B,n,V,kind,noise", [(1, 1, 1, "tree", 1), (4, 5, 7, "star", 1), (6, 64, 50, "tree", 1.5), (3, 64, 1000, "chain", 0.2), (2, 9, 32003, "tree", 0.6),
                                              (40, 17, 333, "star", 2), (1, 6, 131072, "tree", 1), (5, 33, 4097, "tree", 0.0),
                                              (2, 40, 70000, "star", 1.5), (9, 30, 66000, "star", 1)])
def test_verify(gpu_device, B, n, V, kind, noise, draft):
    rng = np.random.default_rng(B * n + V)
    target, dr = _probs(rng, B, n, V, noise)
    parents = np.stack([R.random_parents(rng, n, kind) for _ in range(B)])
    tokens = np.zeros((B, n), np.int32)
    for b in range(B):
        for r in range(1, n):
            q = dr[b, parents[b, r]].astype(np.float64)
            tokens[b, r] = rng.choice(V, p=q / q.sum()) if draft or rng.random() < 0.5 else int(np.argsort(-q)[rng.integers(0, min(V, 3))])
    lens = rng.integers(1, n + 1, size=B).astype(np.int32)
    lens[0] = n
    if B > 3:
        lens[1], lens[2] = 0, n + 7
        parents[3, -1], tokens[3, n // 2] = n + 3, V
    ua, un = rng.random((B, n), dtype=np.float32), rng.random(B, dtype=np.float32)
    args = (target, dr if draft else None, tokens, parents, lens, ua, un)
    got, ref = _verify(gpu_device, *args), R.verify_tree(*args)
    for name, g, r in zip(("path", "path_lens", "next_token"), got, ref):
        assert np.array_equal(g, r), name


def test_verify_distribution(gpu_device):
    """The first token after the root is distributed as the target, whatever the drafter: 40,000 trees of 3 siblings over 5 tokens."""
    rng = np.random.default_rng(8)
    B, n, V = 40000, 4, 5
    p, q = np.array([0.4, 0.3, 0.15, 0.1, 0.05], np.float32), np.array([0.1, 0.5, 0.2, 0.1, 0.1], np.float32)
    parents = np.tile(np.array([-1, 0, 0, 0], np.int32), (B, 1))
    tokens = rng.choice(V, p=q.astype(np.float64) / q.astype(np.float64).sum(), size=(B, n)).astype(np.int32)
    target, draft = np.broadcast_to(p, (B, n, V)).copy(), np.broadcast_to(q, (B, n, V)).copy()
    path, lens, nxt = _verify(gpu_device, target, draft, tokens, parents, np.full(B, n, np.int32), rng.random((B, n), dtype=np.float32), rng.random(B, dtype=np.float32))
    first = np.where(lens > 1, tokens[np.arange(B), np.maximum(path[:, 1], 0)], nxt)
    share = np.bincount(first, minlength=V) / B
    assert np.abs(share - p).max() < 5 * 0.5 / B ** 0.5          # five standard deviations of a share
    assert (lens > 1).mean() > 0.5


def test_verify_borders(gpu_device):
    """Probabilities that are dyadic: sums are exact, and a number that equals a border is decided as the definition says."""
    V, n = 8, 3
    p = np.array([4, 2, 1, 1, 4, 4, 0, 0], np.float32) / 16
    q = np.array([8, 2, 0, 2, 2, 0, 1, 1], np.float32) / 16
    cases = []
    for x1 in range(V):
        for x2 in range(V):
            for u in (0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24):
                cases.append((x1, x2, u))
    B = len(cases)
    parents = np.tile(np.array([-1, 0, 0], np.int32), (B, 1))
    tokens = np.array([[0, a, b] for a, b, _ in cases], np.int32)
    u = np.array([c for *_, c in cases], np.float32)
    target, draft = np.broadcast_to(p, (B, n, V)).copy(), np.broadcast_to(q, (B, n, V)).copy()
    for d in (draft, None, target):
        args = (target, d, tokens, parents, np.full(B, n, np.int32), np.stack([u] * n, 1), u[::-1].copy())
        for g, r in zip(_verify(gpu_device, *args), R.verify_tree(*args)):
            assert np.array_equal(g, r)


def test_verify_rows_without_weight(gpu_device):
    B, n, V = 3, 2, 2000
    target = np.zeros((B, n, V), np.float32)
    target[1, :, 1999] = 1.0
    target[2] = np.nan
    parents, tokens = np.tile(np.array([-1, 0], np.int32), (B, 1)), np.full((B, n), 5, np.int32)
    for draft in (None, np.full((B, n, V), 1 / V, np.float32)):
        path, lens, nxt = _verify(gpu_device, target, draft, tokens, parents, np.full(B, n, np.int32), np.zeros((B, n), np.float32), np.zeros(B, np.float32))
        assert lens.tolist() == [1, 1, 1] and nxt.tolist() == [-1, 1999, -1]


# ---- accepted rows -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,row,vrow", [(BF, (1, 576), None), (BF, (8, 128), (8, 128)), (torch.float32, (2, 6), (2, 10)), (BF, (1, 8), None)])
@pytest.mark.parametrize("B,n,layers,pool", [(1, 1, 1, 5), (3, 8, 2, 40), (16, 64, 3, 1100)])
def test_keep_accepted(gpu_device, B, n, layers, pool, dtype, row, vrow):
    rng = np.random.default_rng(n)
    slots = rng.permutation(pool)[:B * n].astype(np.int32).reshape(B, n)
    path, lens = np.full((B, n), -1, np.int32), rng.integers(0, n + 1, size=B).astype(np.int32)
    for b in range(B):
        path[b, :lens[b]] = [0, *sorted(rng.choice(np.arange(1, n), size=lens[b] - 1, replace=False))] if lens[b] else []
    if B > 2:
        lens[1], lens[2] = n + 5, -2
        path[1] = rng.integers(-2, n + 2, size=n)              # not sorted, twice the same, some that do not exist
        slots[1, 0], slots[1, 3] = -1, pool
    mk = lambda r: torch.arange(layers * pool * r[0] * r[1], device=gpu_device).view(layers, pool, *r).remainder(251).to(dtype)
    k, v = mk(row), None if vrow is None else mk(vrow) + 1
    want = [R.keep_accepted(t, slots, path, lens) for t in (k, v) if t is not None]
    loza.loza_ssa_keep_accepted(k, v, _dev(slots, gpu_device), _dev(path, gpu_device), _dev(lens, gpu_device))
    torch.cuda.synchronize()
    assert torch.equal(k, want[0]) and (v is None or torch.equal(v, want[1]))
