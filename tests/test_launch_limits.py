"""Calls of more workgroups than a launch takes (fewer than 2^32 threads in x) are refused before anything is launched: one of more would come back
without an error and with work left out. No GPU needed."""
import pytest

import paper_2512_23966_amd as loza
from paper_2512_23966_amd import binding as B

ERR_SHAPE = -2
A = 4096   # an address that is never read


def _tree(B_, Hq, Hkv, n, d):
    v = A if d == 576 else 2 * A
    return B.lib().loza_ssa_extend_tree(A, A, v, A, A, A, A, A, A, B_, Hq, Hkv, 0, 100, 64, 4, n, d, 512 if d == 576 else 128, 1, 64, 1, 0.1, None, 0, None)


@pytest.mark.parametrize("B_,Hq,Hkv,n,d", [(1 << 24, 1, 1, 1, 576), (1 << 20, 64, 1, 33, 576), (1 << 19, 32, 32, 3, 576), (1 << 23, 1, 1, 1, 128), (1 << 18, 32, 32, 64, 128),
                                           ((1 << 31) - 1, 1 << 30, 1 << 30, 64, 576), ((1 << 31) - 1, (1 << 31) - 1, 1, 64, 128)])
def test_trees(B_, Hq, Hkv, n, d):
    assert _tree(B_, Hq, Hkv, n, d) == ERR_SHAPE
    assert loza.loza_ssa_extend_tree_workspace_bytes(B_, Hq, Hkv, 256, n, d, 512 if d == 576 else 128, 1, 64) == 0
    with pytest.raises(loza.LozaError):
        loza.loza_ssa_extend_tree_kernel(B_, Hq, Hkv, 256, n, d, 1, 64)


@pytest.mark.parametrize("B_,Hq,Hkv,n,d", [((1 << 24) - 1, 1, 1, 1, 576), ((1 << 20) - 1, 64, 1, 32, 576), ((1 << 23) - 1, 1, 1, 64, 128), ((1 << 18) - 1, 32, 32, 64, 128)])
def test_the_most_that_a_tree_call_takes(B_, Hq, Hkv, n, d):
    assert loza.loza_ssa_extend_tree_kernel(B_, Hq, Hkv, 256, n, d, 1, 64)[1] == 1


@pytest.mark.parametrize("B_,Hq,Hkv,q_len,d", [(1 << 24, 1, 1, 1, 576), (1 << 20, 64, 1, 31, 576), (1 << 19, 32, 32, 1, 128), ((1 << 31) - 1, 1 << 30, 1 << 30, 5, 128)])
def test_extends_and_prefills(B_, Hq, Hkv, q_len, d):
    d_v, v = (512, A) if d == 576 else (128, 2 * A)
    L = B.lib()
    assert L.loza_ssa_extend(A, A, v, A, A, A, B_, Hq, Hkv, 64, q_len, d, d_v, 1, 64, 0.1, None) == ERR_SHAPE
    assert L.loza_ssa_extend_paged_blocks(A, A, v, A, A, A, A, B_, Hq, Hkv, 100, 64, 4, q_len, d, d_v, 1, 64, 1, 0.1, None) == ERR_SHAPE
    assert L.loza_ssa_prefill(A, A, v, A, A, B_, Hq, Hkv, q_len, d, d_v, 1, 64, 0.1, None) == ERR_SHAPE


@pytest.mark.parametrize("B_,Hq,Hkv,d", [(1 << 24, 1, 1, 576), (1 << 20, 16, 16, 128), (1 << 22, 64, 1, 128), ((1 << 31) - 1, 1 << 30, 1 << 30, 128)])
def test_decodes(B_, Hq, Hkv, d):
    d_v, v = (512, A) if d == 576 else (128, 2 * A)
    need = loza.loza_ssa_decode_workspace_bytes(B_, Hq, Hkv, 256, d_v, 1, 64)
    assert B.lib().loza_ssa_decode(A, A, v, A, A, A, B_, Hq, Hkv, 256, d, d_v, 1, 64, 0.1, A, need, None) == ERR_SHAPE


@pytest.mark.parametrize("B_,Hq,Hkv,S,d", [(1 << 24, 1, 1, 1, 576), (1 << 19, 64, 1, 32, 576), (1 << 19, 32, 32, 1, 128), ((1 << 31) - 1, 1 << 30, 1 << 30, 5, 128)])
def test_backwards(B_, Hq, Hkv, S, d):
    d_v, v = (512, A) if d == 576 else (128, 2 * A)
    assert B.lib().loza_ssa_backward(A, A, v, A, A, A, A, A, A, B_, Hq, Hkv, S, d, d_v, 1, 64, 0.1, A, 1 << 60, None) == ERR_SHAPE
