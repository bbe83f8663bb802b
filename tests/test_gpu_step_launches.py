"""Calls of more tokens, or more sequences, than one launch takes (its threads in x are fewer than 2^32)."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


@pytest.mark.parametrize("append", [False, True])
def test_rope_of_more_tokens_than_a_launch_takes(gpu_device, append):
    """2^25 + 3 tokens of one narrow head, a thousand rows and positions over and over, against a call of those."""
    T, d = (1 << 25) + 3, 4
    freq = loza.loza_ssa_rope_frequencies(2, 10000.0)[0].to(gpu_device)
    pos = (torch.arange(T, device=gpu_device) % 1000).to(I32)
    pos[12345::1 << 20] = -1
    x = torch.randn(1000, 1, d, generator=torch.Generator(device=gpu_device).manual_seed(1), device=gpu_device).to(BF)
    rows = torch.arange(T, device=gpu_device) % 1000
    y = torch.full((T, 1, d), 7.0, dtype=BF, device=gpu_device)
    if append:
        slots = torch.arange(T - 1, -1, -1, device=gpu_device).to(I32)
        loza.loza_ssa_rope_append(None, x[rows], None, pos, slots, freq, None, y, None, 0, 2, True)
        y = y.flip(0)
    else:
        loza.loza_ssa_rope(x[rows], pos, freq, y, 2, True)
    small = torch.full_like(x, 7.0)
    loza.loza_ssa_rope(x, torch.arange(1000, dtype=I32, device=gpu_device), freq, small, 2, True)
    want = torch.where((pos >= 0)[:, None, None], small[rows], torch.tensor(7.0, dtype=BF, device=gpu_device))
    assert torch.equal(y, want)


def test_f32_backward_of_more_rows_than_a_launch_takes(gpu_device):
    """2^26 + 48 rows (a wave each): 200 short sequences over and over, against a call of those."""
    b, S, H, d, many = 200, 4, 4, 4, (1 << 22) + 3
    g = torch.Generator(device=gpu_device).manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device=gpu_device)
    q, k, v, dout = (r(b, S, H, d) for _ in range(4))
    out, lse = torch.empty_like(q), torch.empty(b, H, S, device=gpu_device)
    loza.loza_ssa_prefill_f32(q, k, v, out, lse, 1, 2, 0.5)
    small = [torch.empty_like(q) for _ in range(3)]
    loza.loza_ssa_backward_f32(q, k, v, out, lse, dout, *small, 1, 2, 0.5)
    at = torch.arange(many, device=gpu_device) % b
    got = [torch.full((many, S, H, d), float("nan"), device=gpu_device) for _ in range(3)]
    loza.loza_ssa_backward_f32(q[at], k[at], v[at], out[at], lse[at], dout[at], *got, 1, 2, 0.5)
    for x, y in zip(got, small):
        assert torch.equal(x, y[at])


@pytest.mark.parametrize("inter", [True, False])
def test_rope_in_place_across_launches(gpu_device, inter):
    """2^24 + 5 tokens with 16-byte rows, out of place into wider rows and in place."""
    T, d = (1 << 24) + 5, 16
    freq = loza.loza_ssa_rope_frequencies(d, 10000.0)[0].to(gpu_device)
    at = torch.arange(T, device=gpu_device) % 1000
    pos = at.to(I32)
    x = torch.randn(1000, 1, d, generator=torch.Generator(device=gpu_device).manual_seed(2), device=gpu_device).to(BF)
    small = torch.empty_like(x)
    loza.loza_ssa_rope(x, torch.arange(1000, dtype=I32, device=gpu_device), freq, small, 0, inter)
    y = x[at]
    wide = torch.full((T, 1, d + 8), 7.0, dtype=BF, device=gpu_device)
    loza.loza_ssa_rope(y, pos, freq, wide[..., 8:], 0, inter)
    assert torch.equal(wide[..., 8:], small[at]) and bool((wide[..., :8] == 7).all())
    loza.loza_ssa_rope(y, pos, freq, y, 0, inter)
    assert torch.equal(y, small[at])
