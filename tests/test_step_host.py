"""The step around the attention, host side: refusals before any HIP call, sizes, and the rotary frequencies. No GPU needed."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from paper_2512_23966_amd import binding as B

ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_ALIGN = -1, -2, -3, -4, -6
A = 4096   # an address that is never read


def _tables(**k):
    a = dict(cache=A, new=2 * A, parents=3 * A, free=4 * A, count=5 * A, table=6 * A, B=2, n=8, num_free=10, num_pages=100, page=64, most=16,
             granted=7 * A, seqlens=8 * A, pos=9 * A, slots=10 * A, masks=11 * A, left=12 * A)
    a.update(k)
    return B.lib().loza_ssa_step_tables(*a.values(), None)


def test_step_tables_refusals():
    for name in ("cache", "new", "count", "table", "granted", "seqlens", "pos", "slots", "left", "free", "parents", "masks"):
        assert _tables(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(B=65537), dict(n=0), dict(n=65), dict(num_free=-1), dict(num_pages=0), dict(page=48), dict(page=16), dict(most=0),
                dict(num_pages=1 << 26), dict(granted=2 * A), dict(seqlens=A), dict(left=5 * A), dict(most=1 << 26)):
        assert _tables(**bad) == ERR_SHAPE, bad
    for name in ("cache", "new", "parents", "free", "count", "table", "granted", "seqlens", "pos", "slots", "left"):
        assert _tables(**{name: A * 20 + 2}) == ERR_ALIGN, name
    assert _tables(masks=A * 20 + 4) == ERR_ALIGN


def _rope(**k):
    a = dict(x=A, pos=2 * A, freq=3 * A, out=4 * A, T=5, H=4, d=64, xt=256, xh=64, ot=256, oh=64, begin=0, rot=64, inter=1, inv=0, m=1.0)
    a.update(k)
    return B.lib().loza_ssa_rope(*a.values(), None)


def test_rope_refusals():
    for name in ("x", "pos", "freq", "out"):
        assert _rope(**{name: None}) == ERR_NULL, name
    for bad in (dict(T=0), dict(H=0), dict(d=0), dict(rot=0), dict(rot=63), dict(rot=66), dict(begin=-2), dict(begin=2), dict(rot=1026, d=4000), dict(m=math.nan),
                dict(m=math.inf), dict(xt=-1), dict(xh=-64), dict(ot=64, oh=64), dict(oh=32), dict(ot=0), dict(oh=64, ot=255),
                dict(out=A, ot=320), dict(ot=1 << 61), dict(xt=1 << 61), dict(T=1 << 31), dict(H=1 << 25, oh=64, ot=1 << 31)):
        assert _rope(**bad) == ERR_SHAPE, bad
    assert _rope(x=A + 1) == ERR_ALIGN and _rope(out=4 * A + 1) == ERR_ALIGN and _rope(pos=2 * A + 2) == ERR_ALIGN and _rope(freq=3 * A + 4) == ERR_ALIGN
    assert B.lib().loza_ssa_rope_f32(A + 2, 2 * A, 3 * A, 4 * A, 5, 4, 64, 256, 64, 256, 64, 0, 64, 1, 0, 1.0, None) == ERR_ALIGN


def _append(fn="loza_ssa_rope_append", **k):
    a = dict(q=A, k=2 * A, v=3 * A, pos=4 * A, slots=5 * A, freq=6 * A, q_out=7 * A, k_rows=8 * A, v_rows=9 * A, T=5, Hq=4, Hkv=2, dq=64, dk=64, dv=64, qt=256, qh=64,
             ot=256, oh=64, kt=128, kh=64, vt=128, vh=64, rows=100, qb=0, kb=0, rot=64, inter=1, m=1.0)
    a.update(k)
    return getattr(B.lib(), fn)(*a.values(), None)


def test_rope_append_refusals():
    for name in ("k", "v", "pos", "slots", "freq", "q_out", "k_rows", "v_rows", "q"):
        assert _append(**{name: None}) == ERR_NULL, name
    for bad in (dict(T=0), dict(Hq=0), dict(Hkv=0), dict(dk=62), dict(dq=62), dict(dv=0), dict(rows=0), dict(rows=1 << 31), dict(kt=-1), dict(vt=-1), dict(oh=10),
                dict(k=8 * A), dict(v=9 * A), dict(kb=1), dict(qb=-1), dict(rot=7), dict(kt=1 << 61), dict(vh=1 << 61), dict(dv=1 << 30)):
        assert _append(**bad) == ERR_SHAPE, bad
    for name in ("q", "k", "v", "q_out", "k_rows", "v_rows"):
        assert _append(**{name: A * 30 + 1}) == ERR_ALIGN, name
        assert _append("loza_ssa_rope_append_f32", **{name: A * 30 + 2}) == ERR_ALIGN, name
    assert _append(slots=A + 2) == ERR_ALIGN


def _tree(**k):
    a = dict(q=A, k=2 * A, v=2 * A, table=None, seqlens=3 * A, lens=4 * A, masks=5 * A, out=6 * A, lse=7 * A, B=2, Hq=64, Hkv=1, S=4096, pages=0, page=0, most=0, n=8,
             d_qk=576, d_v=512, sink=128, local=1024, block=1, scale=0.1, ws=None, ws_bytes=0)
    a.update(k)
    return B.lib().loza_ssa_extend_tree(*a.values(), None)


def test_extend_tree_refusals():
    for name in ("q", "k", "v", "seqlens", "lens", "masks", "out", "lse"):
        assert _tree(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(n=0), dict(n=65), dict(n=8, S=7), dict(Hq=63, Hkv=2), dict(local=0), dict(sink=-1), dict(block=0), dict(scale=0.0), dict(scale=math.nan),
                dict(table=8 * A, pages=10, page=48, most=4), dict(table=8 * A, pages=0, page=64, most=4), dict(table=8 * A, pages=9, page=64, most=0)):
        assert _tree(**bad) == ERR_SHAPE, bad
    assert _tree(v=9 * A) == ERR_UNSUPPORTED and _tree(d_qk=64, d_v=64) == ERR_UNSUPPORTED
    for bad in (dict(lens=A + 2), dict(masks=A + 4), dict(seqlens=A + 2), dict(q=A + 8)):
        assert _tree(**bad) == ERR_ALIGN, bad
    need = loza.loza_ssa_extend_tree_workspace_bytes(2, 64, 1, 65536, 8, 576, 512, 128, 8192)
    kernel, splits = loza.loza_ssa_extend_tree_kernel(2, 64, 1, 65536, 8, 576, 128, 8192)
    rows = 2 * 64 * 8                           # fp32 output, maximum and sums of every row, in blocks of 32 rows where tiles are split
    assert splits > 1 and need == splits * rows * ((512 + 4) * 4 if kernel == loza.KERNEL_ROWS else (512 + 3) * 4)
    assert _tree(S=65536, local=8192, ws=9 * A, ws_bytes=16) == ERR_WORKSPACE
    assert _tree(S=65536, local=8192, ws=9 * A + 8, ws_bytes=need) == ERR_ALIGN
    assert loza.loza_ssa_extend_tree_workspace_bytes(2, 64, 1, 65536, 65, 576, 512, 128, 8192) == 0


def _verify(**k):
    a = dict(target=A, draft=2 * A, tokens=3 * A, parents=4 * A, lens=5 * A, ua=6 * A, un=7 * A, path=8 * A, pl=9 * A, nxt=10 * A, B=2, n=8, V=1000, ws=11 * A, ws_bytes=1 << 30)
    a.update(k)
    return B.lib().loza_ssa_verify_tree(*a.values(), None)


def test_verify_refusals():
    for name in ("target", "tokens", "parents", "lens", "ua", "un", "path", "pl", "nxt"):
        assert _verify(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(B=65536), dict(n=0), dict(n=65), dict(V=0), dict(V=(1 << 30) + 1)):
        assert _verify(**bad) == ERR_SHAPE, bad
    assert _verify(ws=None) == ERR_WORKSPACE and _verify(ws_bytes=loza.loza_ssa_verify_tree_workspace_bytes(2, 8, 1000) - 1) == ERR_WORKSPACE
    for name in ("target", "draft", "tokens", "parents", "lens", "ua", "un", "path", "pl", "nxt"):
        assert _verify(**{name: A * 20 + 2}) == ERR_ALIGN, name
    assert _verify(ws=A + 8) == ERR_ALIGN
    assert loza.loza_ssa_verify_tree_workspace_bytes(0, 8, 1000) == 0 and loza.loza_ssa_verify_tree_workspace_bytes(2, 65, 1000) == 0


@pytest.mark.parametrize("B_", [1, 2, 16, 63, 1024, 65535])
@pytest.mark.parametrize("V", [1, 63, 1000, 32003, 131072, 1 << 30])
def test_verify_workspace_grows_with_neither_batch_nor_vocabulary_beyond_its_slices(B_, V):
    got = loza.loza_ssa_verify_tree_workspace_bytes(B_, 64, V)
    assert 8 * B_ <= got <= 8 * 256 * 8 * B_


def _keep(**k):
    a = dict(k=A, v=2 * A, slots=3 * A, path=4 * A, lens=5 * A, B=2, n=8, layers=3, rows=100, kb=1152, vb=256)
    a.update(k)
    return B.lib().loza_ssa_keep_accepted(*a.values(), None)


def test_keep_refusals():
    for name in ("k", "slots", "path", "lens"):
        assert _keep(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(n=0), dict(n=65), dict(layers=0), dict(B=40000), dict(rows=0), dict(rows=1 << 31), dict(kb=0), dict(kb=24), dict(kb=(1 << 24) + 16), dict(vb=8), dict(v=A)):
        assert _keep(**bad) == ERR_SHAPE, bad
    assert _keep(k=A + 8) == ERR_ALIGN and _keep(v=2 * A + 8) == ERR_ALIGN and _keep(slots=A + 2) == ERR_ALIGN


def test_frequencies():
    freq, m = loza.loza_ssa_rope_frequencies(64, 10000.0)
    assert m == 1.0 and np.allclose(freq.numpy(), 10000.0 ** (-np.arange(0, 64, 2) / 64), rtol=1e-15, atol=0)
    for factor, context, slow, fast in ((32.0, 32768, 1.0, 32.0), (8.0, 4096, 1.0, 32.0), (4.0, 1000, 0.5, 7.0)):
        freq, m = loza.loza_ssa_rope_frequencies(64, 10000.0, factor, context, slow, fast)
        f = 10000.0 ** (-np.arange(0, 64, 2) / 64)
        turns = context * f / (2 * np.pi)
        ramp = np.clip((turns - slow) / (fast - slow), 0, 1)
        assert np.allclose(freq.numpy(), (1 - ramp) * f / factor + ramp * f, rtol=1e-14, atol=0)
        assert m == np.float32(0.1 * math.log(factor) + 1)
        assert (freq.numpy()[turns >= fast] == f[turns >= fast]).all() or np.allclose(freq.numpy()[turns >= fast], f[turns >= fast], rtol=1e-15)
    for bad in (dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=1026), dict(base=1.0), dict(base=math.inf), dict(factor=0.5), dict(factor=2.0, original_context=0),
                dict(factor=2.0, original_context=100, fast_turns=1.0)):
        with pytest.raises(loza.LozaError) as e:
            loza.loza_ssa_rope_frequencies(**{"rot_dim": 64, "base": 10000.0, **bad})
        assert e.value.status == ERR_SHAPE
    out = (ctypes.c_double * 32)()
    assert B.lib().loza_ssa_rope_frequencies(64, 1e4, 1.0, 0, 1.0, 32.0, None, None) == ERR_NULL
    assert out[0] == 0.0


def test_binding_refuses_what_is_not_on_the_gpu():
    z = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(TypeError):
        loza.loza_ssa_step_tables(z[:, 0], z[:, 0], None, z[0], z[0, :1], z, 4, 64, z[:, 0], z[:, 0], z, z, None, z[0, :1])
    x = torch.zeros(2, 3, 8)
    with pytest.raises(TypeError):
        loza.loza_ssa_rope_f32(x, z[:, 0], torch.zeros(2, dtype=torch.float64), x, 0, True)
    with pytest.raises(TypeError):
        loza.loza_ssa_keep_accepted(torch.zeros(1, 8, 1, 8), None, z, z, z[:, 0])
