"""Norms with rotary positions, probabilities from logits, and pages, host side: refusals before any HIP call, and sizes. No GPU needed."""
import math

import pytest
import torch

import paper_2512_23966_amd as loza
from paper_2512_23966_amd import binding as B

ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_ALIGN = -1, -2, -3, -4, -6
A = 1 << 20   # an address that is never read


def _norm(fn="loza_ssa_norm_rope", **k):
    a = dict(x=A, w=2 * A, pos=3 * A, freq=4 * A, out=5 * A, T=5, H=4, d=64, xt=256, xh=64, ot=256, oh=64, begin=0, dim=64, eps=1e-6, rb=0, rot=64, inter=1, m=1.0)
    a.update(k)
    return getattr(B.lib(), fn)(*a.values(), None)


def test_norm_rope_refusals():
    for name in ("x", "pos", "freq", "out"):
        assert _norm(**{name: None}) == ERR_NULL, name
    for bad in (dict(T=0), dict(T=1 << 31), dict(H=0), dict(d=0), dict(d=1025, xh=2000, oh=2000, xt=9000, ot=9000), dict(dim=0), dict(dim=65), dict(begin=-1), dict(begin=1), dict(dim=-1), dict(eps=0.0),
                dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(eps=1e-39), dict(rot=0), dict(rot=63), dict(rot=66), dict(rb=2), dict(rb=-2), dict(m=math.nan), dict(m=math.inf),
                dict(xt=-1), dict(xh=-64), dict(ot=64), dict(oh=32), dict(out=A, ot=320), dict(ot=1 << 61), dict(xt=1 << 61), dict(H=1 << 25, oh=64, ot=1 << 31)):
        assert _norm(**bad) == ERR_SHAPE, bad
    for name, off in (("x", 1), ("out", 1), ("pos", 2), ("freq", 4), ("w", 2)):
        assert _norm(**{name: 9 * A + off}) == ERR_ALIGN, name
    assert _norm("loza_ssa_norm_rope_f32", x=A + 2) == ERR_ALIGN


def _back(fn="loza_ssa_norm_rope_backward", **k):
    a = dict(dout=6 * A, x=A, w=2 * A, pos=3 * A, freq=4 * A, dx=5 * A, dw=7 * A, T=5, H=4, d=64, gt=256, gh=64, xt=256, xh=64, ot=256, oh=64, begin=0, dim=64, eps=1e-6, rb=0, rot=64,
             inter=1, m=1.0, ws=8 * A, nb=5 * 64 * 4)
    a.update(k)
    return getattr(B.lib(), fn)(*a.values(), None)


def test_norm_rope_backward_refusals():
    for name in ("dout", "x", "pos", "freq", "dx"):
        assert _back(**{name: None}) == ERR_NULL, name
    for bad in (dict(T=0), dict(H=0), dict(dim=0), dict(begin=1), dict(eps=0.0), dict(rot=63), dict(gt=-1), dict(gh=1 << 61), dict(ot=64), dict(dx=A, ot=320), dict(dx=6 * A, gt=320),
                dict(d=1025, xh=2000, oh=2000, xt=9000, ot=9000)):
        assert _back(**bad) == ERR_SHAPE, bad
    assert _back(ws=None) == ERR_WORKSPACE and _back(nb=5 * 64 * 4 - 1) == ERR_WORKSPACE and _back(ws=8 * A + 8) == ERR_ALIGN and _back(dw=7 * A + 2) == ERR_ALIGN
    assert _back("loza_ssa_norm_rope_backward_f32", dout=A * 6 + 2) == ERR_ALIGN
    size = loza.loza_ssa_norm_rope_backward_workspace_bytes
    assert size(5, 4, 64, 64) == 5 * 64 * 4 and size(1 << 30, 4, 64, 32) == 768 * 32 * 4
    assert [size(*x) for x in ((0, 4, 64, 64), (5, 0, 64, 64), (5, 4, 1025, 64), (5, 4, 64, 65), (5, 4, 64, 0), (1 << 31, 1, 64, 64))] == [0] * 6


def _append(fn="loza_ssa_norm_rope_append", **k):
    a = dict(q=A, wq=2 * A, k=3 * A, wk=4 * A, v=5 * A, pos=6 * A, slots=7 * A, freq=8 * A, q_out=9 * A, k_rows=10 * A, v_rows=11 * A, T=5, Hq=4, Hkv=2, dq=64, dk=64, dv=64, qt=256, qh=64,
             ot=256, oh=64, kt=128, kh=64, vt=128, vh=64, rows=100, qn=0, qd=64, kn=0, kd=64, eps=1e-6, qb=0, kb=0, rot=64, inter=1, m=1.0)
    a.update(k)
    return getattr(B.lib(), fn)(*a.values(), None)


def test_norm_rope_append_refusals():
    for name in ("k", "v", "pos", "slots", "freq", "q_out", "k_rows", "v_rows", "q"):
        assert _append(**{name: None}) == ERR_NULL, name
    for bad in (dict(T=0), dict(Hq=0), dict(Hkv=0), dict(dk=62), dict(dq=62), dict(dv=0), dict(rows=0), dict(rows=1 << 31), dict(kt=-1), dict(vt=-1), dict(oh=10), dict(k=10 * A), dict(v=11 * A),
                dict(kb=1), dict(qb=-1), dict(rot=7), dict(kt=1 << 61), dict(vh=1 << 61), dict(dv=1 << 30), dict(qd=65), dict(kd=-1), dict(qn=1), dict(kn=-1), dict(eps=0.0), dict(qd=0, eps=math.nan),
                dict(dq=1030, qh=1030, oh=1030), dict(dk=1030, kh=1030)):
        assert _append(**bad) == ERR_SHAPE, bad
    for name in ("q", "k", "v", "q_out", "k_rows", "v_rows"):
        assert _append(**{name: A * 30 + 1}) == ERR_ALIGN, name
        assert _append("loza_ssa_norm_rope_append_f32", **{name: A * 30 + 2}) == ERR_ALIGN, name
    assert _append(slots=A + 2) == ERR_ALIGN and _append(wq=A + 2) == ERR_ALIGN and _append(wk=A + 2) == ERR_ALIGN


def _probs(fn="loza_ssa_token_probs", **k):
    a = dict(logits=A, row=1000, lens=2 * A, tokens=3 * A, masks=4 * A, seen=5 * A, seen_row=1000, rep=6 * A, fre=7 * A, pre=8 * A, temp=9 * A, bt=10 * A, bv=11 * A, n_bias=3, allowed=12 * A, probs=13 * A,
             B=2, n=8, V=1000, ws=14 * A, nb=2 * 8 * 16)
    a.update(k)
    return getattr(B.lib(), fn)(*a.values(), None)


def test_token_probs_refusals():
    for name in ("logits", "probs", "tokens", "masks", "bt", "bv"):
        assert _probs(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(B=65536), dict(n=0), dict(n=65), dict(V=0), dict(V=(1 << 30) + 1), dict(n_bias=-1), dict(n_bias=1025), dict(row=999), dict(row=1 << 60), dict(seen_row=999),
                dict(seen_row=1001), dict(seen_row=1 << 60), dict(probs=A)):
        assert _probs(**bad) == ERR_SHAPE, bad
    assert _probs("loza_ssa_token_probs_f32", probs=A, row=1001) == ERR_SHAPE
    assert _probs(ws=None) == ERR_WORKSPACE and _probs(nb=2 * 8 * 16 - 1) == ERR_WORKSPACE and _probs(ws=14 * A + 8) == ERR_ALIGN
    for name in ("lens", "tokens", "rep", "fre", "pre", "temp", "bt", "bv", "allowed", "probs"):
        assert _probs(**{name: 20 * A + 2}) == ERR_ALIGN, name
    assert _probs(logits=A + 1) == ERR_ALIGN and _probs("loza_ssa_token_probs_f32", logits=A + 2) == ERR_ALIGN and _probs(masks=4 * A + 4) == ERR_ALIGN and _probs(seen=5 * A + 8) == ERR_ALIGN
    size = loza.loza_ssa_token_probs_workspace_bytes
    assert size(2, 8, 1000) == 256 and size(0, 8, 1000) == size(2, 65, 1000) == size(2, 8, 0) == size(65536, 1, 5) == 0
    assert size(65535, 64, 1 << 30) == 0                                    # more rows and slices than a launch takes
    assert 0 < size(1, 1, 1 << 30) <= 8192 * 16


def test_count_tokens_refusals():
    def call(**k):
        a = dict(tokens=A, path=2 * A, lens=3 * A, prompt=4 * A, fresh=5 * A, seen=6 * A, row=1000, B=2, n=8, V=1000)
        a.update(k)
        return B.lib().loza_ssa_count_tokens(*a.values(), None)
    for name in ("tokens", "lens", "seen"):
        assert call(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(B=65536), dict(n=0), dict(n=(1 << 30) + 1), dict(V=0), dict(V=1001), dict(row=1001), dict(row=999), dict(row=1 << 60)):
        assert call(**bad) == ERR_SHAPE, bad
    for name in ("tokens", "path", "lens", "prompt", "fresh"):
        assert call(**{name: 9 * A + 2}) == ERR_ALIGN, name
    assert call(seen=6 * A + 8) == ERR_ALIGN


FORK = ("source", "lens", "held", "trimmed", "free", "count", "shared", "table")
FORKED = ("forked", "lens1", "held1", "trimmed1", "cf", "ct", "cr", "left", "shared1")


def _fork(**k):
    a = {name: (i + 1) * A for i, name in enumerate(FORK)}
    a.update(B=2, num_free=10, num_pages=100, page=64, most=16, sink=1, block=1)
    a.update({name: (i + 20) * A for i, name in enumerate(FORKED)})
    a.update(k)
    return B.lib().loza_ssa_pages_fork(*a.values(), None)


def test_pages_fork_refusals():
    for name in FORK + FORKED:
        assert _fork(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(B=65537), dict(num_free=-1), dict(num_free=1 << 31), dict(num_pages=0), dict(page=48), dict(page=16), dict(most=0), dict(most=1 << 26), dict(sink=-1), dict(block=0),
                *(dict([(name, 2 * A + 4)]) for name in FORKED), dict(shared1=7 * A), dict(lens1=20 * A), dict(table=A)):
        assert _fork(**bad) == ERR_SHAPE, bad
    for name in FORK + FORKED:
        assert _fork(**{name: A * 50 + 2}) == ERR_ALIGN, name


def test_pages_copy_refusals():
    def call(**k):
        a = dict(k=A, v=2 * A, src=3 * A, dst=4 * A, rows=5 * A, count=6 * A, n=3, layers=2, pages=100, page=64, kb=1152, vb=256)
        a.update(k)
        return B.lib().loza_ssa_pages_copy(*a.values(), None)
    for name in ("k", "src", "dst"):
        assert call(**{name: None}) == ERR_NULL, name
    for bad in (dict(n=0), dict(n=1 << 31), dict(layers=0), dict(layers=65536), dict(pages=0), dict(pages=1 << 31), dict(page=0), dict(page=(1 << 20) + 1), dict(kb=8), dict(kb=1160), dict(kb=(1 << 24) + 16),
                dict(vb=0), dict(vb=24), dict(v=A), dict(pages=(1 << 31) - 1, page=1 << 20, kb=1 << 24, layers=65535)):
        assert call(**bad) == ERR_SHAPE, bad
    assert call(k=A + 8) == ERR_ALIGN and call(v=2 * A + 8) == ERR_ALIGN
    for name in ("src", "dst", "rows", "count"):
        assert call(**{name: 9 * A + 2}) == ERR_ALIGN, name


def test_pages_free_refusals():
    ins, outs = ("ending", "lens", "held", "trimmed", "table", "shared", "free", "count"), ("lens1", "held1", "trimmed1", "count1", "shared1")

    def call(**k):
        a = {name: (i + 1) * A for i, name in enumerate(ins)}
        a.update(B=2, num_free=100, num_pages=100, page=64, most=16, sink=1, local=5, block=1)
        a.update({name: (i + 20) * A for i, name in enumerate(outs)})
        a.update(ws=40 * A, nb=416)
        a.update(k)
        return B.lib().loza_ssa_pages_free(*a.values(), None)
    assert loza.loza_ssa_pages_free_workspace_bytes(100) == 416 and loza.loza_ssa_pages_free_workspace_bytes(0) == 0
    for name in ins[1:] + outs:
        assert call(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(B=65537), dict(num_free=99), dict(num_free=1 << 31), dict(num_pages=0), dict(page=48), dict(most=0), dict(sink=-1), dict(local=0), dict(block=0),
                *(dict([(name, 2 * A + 4)]) for name in outs), dict(free=2 * A), dict(shared1=6 * A), dict(ws=5 * A)):
        assert call(**bad) == ERR_SHAPE, bad
    for name in ins + outs:
        assert call(**{name: A * 50 + 2}) == ERR_ALIGN, name
    assert call(ws=None) == ERR_WORKSPACE and call(nb=415) == ERR_WORKSPACE and call(ws=40 * A + 8) == ERR_ALIGN


def test_pages_compact_refusals():
    ins, outs = ("table", "free", "count", "shared"), ("table1", "free1", "count1", "shared1", "cf", "ct", "n")

    def call(**k):
        a = {name: (i + 1) * A for i, name in enumerate(ins)}
        a.update(B=2, num_free=100, num_pages=100, most=16)
        a.update({name: (i + 20) * A for i, name in enumerate(outs)})
        a.update(ws=40 * A, nb=416)
        a.update(k)
        return B.lib().loza_ssa_pages_compact(*a.values(), None)
    assert loza.loza_ssa_pages_compact_workspace_bytes(100) == 416 and loza.loza_ssa_pages_compact_workspace_bytes(1) == 0
    for name in ins + outs:
        assert call(**{name: None}) == ERR_NULL, name
    for bad in (dict(B=0), dict(B=65537), dict(num_free=99), dict(num_free=1 << 31), dict(num_pages=1), dict(num_pages=1 << 31, num_free=1 << 31), dict(most=0),
                *(dict([(name, 2 * A + 4)]) for name in outs), dict(table1=A), dict(shared1=4 * A), dict(ws=A)):
        assert call(**bad) == ERR_SHAPE, bad
    for name in ins + outs:
        assert call(**{name: A * 50 + 2}) == ERR_ALIGN, name
    assert call(ws=None) == ERR_WORKSPACE and call(nb=415) == ERR_WORKSPACE and call(ws=40 * A + 8) == ERR_ALIGN


def test_the_binding_refuses_before_the_library():
    """Tensors that are not on the GPU, and halves of pairs."""
    t, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    f = torch.zeros(32, dtype=torch.float64)
    with pytest.raises(TypeError):
        loza.loza_ssa_norm_rope(t, None, i, f, t, 0, 64, 1e-6, 0, True)
    with pytest.raises(TypeError):
        loza.loza_ssa_norm_rope_backward(t, t, None, i, f, t, None, 0, 64, 1e-6, 0, True)
    with pytest.raises(ValueError):
        loza.loza_ssa_norm_rope_append(t, None, t, None, None, i, i, f, None, t, None, 0, 64, 0, 64, 1e-6, 0, 0, True)
    with pytest.raises((TypeError, ValueError)):
        loza.loza_ssa_token_probs(t, t.float())
    with pytest.raises(TypeError):
        loza.loza_ssa_count_tokens(i.view(1, 4), i[:1], torch.zeros(1, 8, dtype=torch.int16), 8)
    with pytest.raises(TypeError):
        loza.loza_ssa_pages_copy(t.view(1, 4, 2, 1, 64), None, i, i)
    with pytest.raises(ValueError):
        loza.loza_ssa_pages_fork(i, i, i, i, i, i[:1], i, i.view(4, 1), 4, 32, 0, 1, i, i, i, None, i, i, i, i[:1], i)
    with pytest.raises(ValueError):
        loza.loza_ssa_pages_free(None, i, i, None, i.view(4, 1), i, i, i[:1], 4, 32, 0, 1, 1, i, i, None, i[:1], None)
    with pytest.raises(ValueError):
        loza.loza_ssa_pages_compact(i.view(4, 1), i, i[:1], i, 4, i.view(4, 1), i, i[:1], None, i[:2], i[:2], i[:1])
