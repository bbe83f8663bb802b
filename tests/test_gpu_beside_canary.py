"""Norms with rotary positions, token probabilities, records and pages write nothing outside what they are given: every output between guard zones (as in
test_gpu_canary.py)."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import step_reference as R
from tests.test_gpu_canary import Guarded
from tests.test_gpu_pages import Pool
from tests.test_gpu_token_probs import Call, _bits

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,H,d,begin,dim,rot_begin,rot,inter", [(1, 1, 64, 0, 64, 0, 64, True), (1033, 3, 128, 0, 128, 0, 128, False), (37, 1, 576, 0, 512, 512, 64, True), (13, 5, 31, 3, 20, 5, 6, False),
                                                               (2051, 2, 80, 0, 80, 16, 64, True), (3, 2, 1023, 1, 1000, 7, 1016, True)])
def test_norms(gpu_device, T, H, d, begin, dim, rot_begin, rot, inter, dtype):
    g = torch.Generator(device=gpu_device).manual_seed(T)
    rnd = lambda *s: torch.randn(*s, generator=g, device=gpu_device).to(dtype)
    x, dout, w = rnd(T, H, d), rnd(T, H, d), rnd(dim).float()
    freq, m = loza.loza_ssa_rope_frequencies(rot, 10000.0)
    pos, fr = torch.arange(T, dtype=I32, device=gpu_device), freq.to(gpu_device)
    G = Guarded(gpu_device)
    out, dx, dw = G.tensor((T, H, d), dtype), G.tensor((T, H, d), dtype), G.tensor((dim,), F32)
    ws = G.tensor((loza.loza_ssa_norm_rope_backward_workspace_bytes(T, H, d, dim),), torch.uint8)
    f32 = dtype == F32
    (loza.loza_ssa_norm_rope_f32 if f32 else loza.loza_ssa_norm_rope)(x, w, pos, fr, out, begin, dim, 1e-6, rot_begin, inter, m)
    (loza.loza_ssa_norm_rope_backward_f32 if f32 else loza.loza_ssa_norm_rope_backward)(dout, x, w, pos, fr, dx, dw, begin, dim, 1e-6, rot_begin, inter, m, workspace=ws)
    rows, v_rows, q_out = G.tensor((T, 1, H, d), dtype), G.tensor((T, 1, H, 24), dtype), G.tensor((T, H, d), dtype)
    slots = torch.randperm(T, generator=torch.Generator().manual_seed(1)).to(I32).to(gpu_device)
    (loza.loza_ssa_norm_rope_append_f32 if f32 else loza.loza_ssa_norm_rope_append)(x, w, dout, w, rnd(T, H, 24), pos, slots, fr, q_out, rows, v_rows, begin, dim, begin, dim, 1e-6,
                                                                                    rot_begin, rot_begin, inter, m)
    G.check(f"norms {T} {H} {d}")
    for t in (out, dx, dw, rows, v_rows, q_out):
        assert not bool(torch.isnan(t.float()).any())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,n,V", [(1, 1, 1), (2, 3, 509), (3, 2, 2049), (1, 1, 32003), (300, 1, 1537), (4, 33, 20005), (1, 2, 131_085)])
def test_probabilities(gpu_device, B, n, V, dtype):
    c = Call(B, n, V, dtype, B + V)
    c.lens[:] = n
    c.masks = np.stack([R.masks_of(c.parents[b], n) for b in range(B)]).view(np.int64)
    G = Guarded(gpu_device)
    probs, ws = G.tensor((B, n, V), F32), G.tensor((loza.loza_ssa_token_probs_workspace_bytes(B, n, V),), torch.uint8)
    # inputs end where their buffers do: a read beyond them would find the pattern, a NaN
    put = lambda x, dt: G.tensor(x.shape, dt).copy_(torch.from_numpy(np.ascontiguousarray(x)))
    logits = G.tensor((B, n, V), dtype).copy_(c.logits)
    fn = loza.loza_ssa_token_probs if dtype == BF else loza.loza_ssa_token_probs_f32
    fn(logits, probs, ws, tree_lens=put(c.lens, I32), tokens=put(c.tokens, I32), masks=put(c.masks, torch.int64), seen=put(c.seen.view(np.int16), torch.int16),
       repetition=put(c.rep, F32), frequency=put(c.fre, F32), presence=put(c.pre, F32), temperature=put(c.temp, F32), bias_tokens=put(c.bt, I32), bias_values=put(c.bv, F32),
       allowed=put(_bits(c.ok), I32))
    G.check(f"probabilities {B} {n} {V}")
    c.check(probs, None if n * V * B < 200_000 else (0, n - 1))
    assert not bool(torch.isnan(probs).any())


@pytest.mark.parametrize("n", [7, 5001])
def test_records(gpu_device, n):
    B, V = 3, 20_003
    rng = np.random.default_rng(n)
    G = Guarded(gpu_device)
    put = lambda x: G.tensor(x.shape, I32).copy_(torch.from_numpy(x))
    seen = G.tensor((B, 20_008), torch.int16)
    tokens = put(rng.integers(-5, V + 5, size=(B, n)).astype(np.int32))
    for fresh in (np.ones(B, np.int32), np.zeros(B, np.int32)):
        loza.loza_ssa_count_tokens(tokens, put(np.array([n, n + 9, 0], np.int32)), seen, V, path=put(rng.integers(-2, n + 2, size=(B, n)).astype(np.int32)),
                                   prompt_lens=put(np.array([n // 2, 0, 5], np.int32)), fresh=put(fresh))
        G.check(f"records {n}")
    assert not bool(seen[:, V:].any())


@pytest.mark.parametrize("B,page,most", [(1, 32, 3), (40, 32, 300), (300, 64, 5)])
def test_pages(gpu_device, B, page, most):
    rng = np.random.default_rng(B)
    p = Pool(rng, B, page, most)
    G = Guarded(gpu_device)
    put = lambda x: G.tensor(x.shape, I32).copy_(torch.from_numpy(np.ascontiguousarray(x)))
    i32 = lambda *s: G.tensor(s, I32)
    table, free, count, shared = put(p.table), put(p.free), put(np.array([p.count], np.int32)), put(p.shared)
    left, shared1, cf, ct, cr, lens1, held1, trimmed1 = i32(1), i32(p.pages), i32(B), i32(B), i32(B), i32(B), i32(B), i32(B)
    loza.loza_ssa_pages_fork(put(rng.integers(-2, B + 2, size=B).astype(np.int32)), put(p.lens), put(p.held), put(p.trimmed), free, count, shared, table, p.pages, page, 3, 16, i32(B), lens1,
                             held1, trimmed1, cf, ct, cr, left, shared1)
    G.check("fork")
    k, v = G.tensor((2, p.pages, page, 1, 8), BF).zero_(), G.tensor((2, p.pages, page, 2, 72), BF).zero_()
    loza.loza_ssa_pages_copy(k, v, cf, ct, rows=cr)
    G.check("copy")
    count2, shared2 = i32(1), i32(p.pages)
    loza.loza_ssa_pages_free(put((rng.random(B) < 0.4).astype(np.int32)), lens1, held1, trimmed1, table, shared1, free, left, p.pages, page, 3, 5, 16, i32(B), i32(B), i32(B), count2, shared2,
                             G.tensor((loza.loza_ssa_pages_free_workspace_bytes(p.pages),), torch.uint8))
    G.check("free")
    cf2, ct2, n2 = i32(p.pages // 2), i32(p.pages // 2), i32(1)
    loza.loza_ssa_pages_compact(table, free, count2, shared2, p.pages, i32(B, most), i32(p.pages), i32(1), i32(p.pages), cf2, ct2, n2,
                                G.tensor((loza.loza_ssa_pages_compact_workspace_bytes(p.pages),), torch.uint8))
    loza.loza_ssa_pages_copy(k, v, cf2, ct2, count=n2)
    G.check("compact")
    assert not bool(k.any()) and not bool(v.any())
