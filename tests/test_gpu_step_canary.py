"""The step's calls write nothing outside what they are given: every output between guard zones (as in test_gpu_canary.py), and rows of a
cache that belong to nobody as they were."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import step_reference as R
from tests.test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


def _rand(shape, seed, dev, dtype=BF):
    g = torch.Generator(device=dev).manual_seed(seed)
    return torch.randn(shape, generator=g, device=dev).to(dtype)


@pytest.mark.parametrize("B,Hq,Hkv,d,S_max,n,sink,local,scratch", [
    (2, 64, 1, 576, 3000, 5, 16, 2500, True), (2, 64, 1, 576, 3000, 5, 16, 2500, False), (3, 64, 1, 576, 3000, 47, 16, 2500, True), (5, 192, 1, 576, 500, 43, 16, 100, True),
    (2, 6, 2, 128, 900, 7, 16, 300, True), (4, 28, 4, 128, 4500, 61, 16, 4200, True), (20, 40, 8, 128, 333, 51, 16, 300, True)])
def test_tree_attention_stays_inside_its_buffers(gpu_device, B, Hq, Hkv, d, S_max, n, sink, local, scratch):
    rng = np.random.default_rng(n)
    q, k = _rand((B, n, Hq, d), 1, gpu_device), _rand((B, S_max, Hkv, d), 2, gpu_device)
    d_v = 512 if d == 576 else 128
    G = Guarded(gpu_device)
    out, lse = G.tensor((B, n, Hq, d_v), BF), G.tensor((B, Hq, n), torch.float32)
    nb = loza.loza_ssa_extend_tree_workspace_bytes(B, Hq, Hkv, S_max, n, d, d_v, sink, local) if scratch else 0
    ws = G.tensor((nb,), torch.uint8) if nb else torch.empty(0, dtype=torch.uint8, device=gpu_device)
    lens, counts = [S_max - 3 * b for b in range(B)], [max(1, n - b) for b in range(B)]
    masks = np.stack([R.masks_of(R.random_parents(rng, n), c) for c in counts]).view(np.int64)
    loza.loza_ssa_extend_tree(q, k, k, torch.tensor(lens, dtype=I32, device=gpu_device), torch.tensor(counts, dtype=I32, device=gpu_device),
                              torch.from_numpy(masks).to(gpu_device), out, lse, sink, local, 1, d ** -0.5, workspace=ws)
    G.check(f"tree n{n}")
    assert not bool(torch.isnan(out.float()).any()) and not bool(torch.isnan(lse).any())


def test_step_tables_verify_and_keep_stay_inside_their_buffers(gpu_device):
    rng = np.random.default_rng(4)
    B, n, V, page, most = 5, 61, 1001, 32, 7
    G = Guarded(gpu_device)
    put = lambda x, dt: G.tensor(x.shape, dt).copy_(torch.from_numpy(x))
    cache, new = rng.integers(0, most * page - n, size=B).astype(np.int32), rng.integers(1, n + 1, size=B).astype(np.int32)
    table = put(rng.permutation(B * most).astype(np.int32).reshape(B, most), I32)
    parents = np.stack([R.random_parents(rng, n) for _ in range(B)])
    free = put(rng.permutation(B * most).astype(np.int32), I32)
    for tree in (True, False):
        granted, seqlens, positions, slots, left = (G.tensor(s, I32) for s in ((B,), (B,), (B, n), (B, n), (1,)))
        masks = G.tensor((B, n), torch.int64) if tree else None
        loza.loza_ssa_step_tables(put(cache, I32), put(new, I32), put(parents, I32) if tree else None, free, put(np.array([B * most], np.int32), I32), table, B * most, page,
                                  granted, seqlens, positions, slots, masks, left)
        G.check(f"tables, tree={tree}")
    target = rng.random((B, n, V)).astype(np.float32)
    path, lens, nxt = G.tensor((B, n), I32), G.tensor((B,), I32), G.tensor((B,), I32)
    for draft in (target[:, ::-1].copy(), None):
        loza.loza_ssa_verify_tree(put(target, torch.float32), None if draft is None else put(draft, torch.float32), put(rng.integers(0, V, size=(B, n)).astype(np.int32), I32),
                                  put(parents, I32), put(new, I32), put(rng.random((B, n), dtype=np.float32), torch.float32), put(rng.random(B, dtype=np.float32), torch.float32),
                                  path, lens, nxt, G.tensor((loza.loza_ssa_verify_tree_workspace_bytes(B, n, V),), torch.uint8))
        G.check(f"verify, draft={draft is not None}")
    rows = B * most * page
    k, v = G.tensor((2, rows, 1, 24), BF).zero_(), G.tensor((2, rows, 1, 8), BF).zero_()
    ids = torch.arange(rows, device=gpu_device, dtype=torch.float32).remainder(255).view(1, rows, 1, 1)
    k += ids.to(BF)
    v += ids.to(BF)
    before = k.clone()
    loza.loza_ssa_keep_accepted(k, v, slots, path, lens)
    G.check("keep")
    touched = set(slots.flatten().tolist())
    others = torch.tensor([r for r in range(rows) if r not in touched], device=gpu_device)
    assert torch.equal(k[:, others], before[:, others])


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_rope_stays_inside_its_buffers(gpu_device, dtype):
    T, Hq, Hkv, rows = 37, 5, 2, 50
    fn, app = (loza.loza_ssa_rope, loza.loza_ssa_rope_append) if dtype == BF else (loza.loza_ssa_rope_f32, loza.loza_ssa_rope_append_f32)
    for d, rot in ((64, 64), (33, 6), (96, 32)):
        freq = loza.loza_ssa_rope_frequencies(rot, 10000.0)[0].to(gpu_device)
        G = Guarded(gpu_device)
        pos = torch.arange(T, dtype=I32, device=gpu_device)
        x, out = _rand((T, Hq, d), 5, gpu_device, dtype), G.tensor((T, Hq, d), dtype)
        fn(x, pos, freq, out, d - rot, True, 1.0)
        G.check(f"rope d{d}")
        k, v, kr, vr = _rand((T, Hkv, d), 6, gpu_device, dtype), _rand((T, Hkv, d), 7, gpu_device, dtype), G.tensor((rows, Hkv, d), dtype), G.tensor((rows, Hkv, d), dtype)
        slots = torch.arange(rows - T, rows, dtype=I32, device=gpu_device)
        app(x, k, v, pos, slots, freq, out, kr, vr, d - rot, d - rot, False, 1.0)
        G.check(f"append d{d}")
        assert bool(torch.isnan(kr[:rows - T].float()).all()) and bool(torch.isnan(vr[:rows - T].float()).all())      # (the guard's pattern: not written)
        assert torch.equal(vr[rows - T:], v)
