"""Results of the calls beside the step that lie on other arrays of the call: refused before anything is launched. No GPU needed (the addresses are never read)."""
import pytest

from tests.test_beside_host import A, ERR_SHAPE, B, _append, _back, _norm, _probs

INPUTS = ("logits", "lens", "tokens", "masks", "seen", "rep", "fre", "pre", "temp", "bt", "bv", "allowed")


@pytest.mark.parametrize("fn", ["loza_ssa_token_probs", "loza_ssa_token_probs_f32"])
def test_token_probs(fn):
    at = {name: i * A for i, name in zip((1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12), INPUTS)}
    for name in INPUTS[1:]:
        assert _probs(fn, probs=at[name]) == ERR_SHAPE, name
        assert _probs(fn, ws=at[name]) == ERR_SHAPE, name
    es = 4 if fn.endswith("f32") else 2
    # probabilities that begin inside the logits, or end there; the workspace on the logits' last row, on the probabilities' first and last
    for bad in (dict(probs=A + 16), dict(probs=A + 16 * 1000 * es - 4), dict(probs=A - 16 * 1000 * 4 + 4), dict(ws=A), dict(ws=A + 16 * 1000 * es - 16), dict(ws=13 * A), dict(ws=13 * A + 16 * 4000 - 16),
                dict(ws=13 * A - 240), dict(row=1100, probs=A + (15 * 1100 + 1000) * es - 4), dict(probs=A + 4 * 1000 * es)):
        assert _probs(fn, **bad) == ERR_SHAPE, bad
    if es == 4:                                              # (in place, but for the workspace)
        assert _probs(fn, probs=A, ws=A + 64) == ERR_SHAPE


def test_count_tokens():
    def call(**k):
        a = dict(tokens=A, path=2 * A, lens=3 * A, prompt=4 * A, fresh=5 * A, seen=6 * A, row=1000, B=2, n=8, V=1000)
        a.update(k)
        return B.lib().loza_ssa_count_tokens(*a.values(), None)
    for i in range(1, 6):
        assert call(seen=i * A) == ERR_SHAPE, i
        assert call(seen=i * A - 2 * 1000 * 2 + 16) == ERR_SHAPE, i
    assert call(tokens=6 * A + 2 * 1000 * 2 - 4) == ERR_SHAPE


def test_pages_copy():
    """The pages of keys and values, and the lists, lie apart."""
    def call(**k):
        a = dict(k=100 * A, v=200 * A, src=3 * A, dst=4 * A, rows=5 * A, count=6 * A, n=3, layers=2, pages=100, page=64, kb=1152, vb=256)
        a.update(k)
        return B.lib().loza_ssa_pages_copy(*a.values(), None)
    k_bytes, v_bytes = 2 * 100 * 64 * 1152, 2 * 100 * 64 * 256
    for bad in (dict(v=100 * A + 16), dict(v=100 * A + k_bytes - 16), dict(v=100 * A - v_bytes + 16), dict(v=100 * A + 1152 * 64 * 100)):
        assert call(**bad) == ERR_SHAPE, bad
    for name in ("src", "dst", "rows", "count"):
        for bad in (100 * A, 100 * A + k_bytes - 4, 200 * A, 200 * A + v_bytes - 4):
            assert call(**{name: bad}) == ERR_SHAPE, (name, bad)


def test_norm_rope():
    """Results whose rows lie one behind the other, and dense inputs; strided ones share their buffers (slices of a row of all projections), and are the caller's."""
    for name in ("w", "pos", "freq"):
        assert _norm(**{name: 5 * A}) == ERR_SHAPE, name
    assert _norm(out=A + 16) == ERR_SHAPE and _norm(out=A - 16) == ERR_SHAPE and _norm("loza_ssa_norm_rope_f32", out=A + 16) == ERR_SHAPE
    for name, at in (("dout", 6 * A), ("x", A), ("w", 2 * A), ("pos", 3 * A), ("freq", 4 * A), ("dx", 5 * A), ("dw", 7 * A)):
        assert _back(ws=at) == ERR_SHAPE, name
        assert name == "dw" or _back(dw=at) == ERR_SHAPE, name
        assert name not in ("w", "pos", "freq") or _back(dx=at) == ERR_SHAPE, name
    assert _back(dx=6 * A + 16) == ERR_SHAPE and _back(dx=A + 16) == ERR_SHAPE and _back(dx=A - 16) == ERR_SHAPE
    assert _back(ws=7 * A - 5 * 64 * 4 + 16) == ERR_SHAPE


def test_norm_rope_append():
    for name in ("wq", "wk", "pos", "slots", "freq"):
        for result in (9 * A, 10 * A, 11 * A):
            assert _append(**{name: result}) == ERR_SHAPE, (name, result)
    cache = 100 * 2 * 64 * 2
    for bad in (dict(k_rows=11 * A), dict(v_rows=10 * A + cache - 16), dict(v_rows=10 * A - cache + 16), dict(q_out=10 * A), dict(q_out=11 * A + 16), dict(q_out=A + 16), dict(q=10 * A)):
        assert _append(**bad) == ERR_SHAPE, bad


def test_the_largest_sizes():
    """Numbers of bytes that pass 64 bits: as many as there are."""
    far = 1 << 40
    assert _norm("loza_ssa_norm_rope_f32", T=(1 << 31) - 1, H=1 << 20, d=1024, xt=1 << 30, xh=1024, ot=1 << 30, oh=1024, out=A, x=A + 4 * far) == ERR_SHAPE
    assert _append("loza_ssa_norm_rope_append_f32", rows=(1 << 31) - 1, Hkv=1 << 20, dk=1024, kh=1024, kt=1 << 30, dv=1024, vh=1024, vt=1 << 30, k_rows=10 * A, v_rows=10 * A + 4 * far) == ERR_SHAPE
