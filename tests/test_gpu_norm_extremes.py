"""The gradient of norms with rotary positions where the forward call gives 0: heads whose squares add up to more than fp32 holds."""
import pytest
import torch

import paper_2512_23966_amd as loza

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
FORWARD = {BF: loza.loza_ssa_norm_rope, F32: loza.loza_ssa_norm_rope_f32}
BACKWARD = {BF: loza.loza_ssa_norm_rope_backward, F32: loza.loza_ssa_norm_rope_backward_f32}


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_head_too_large_to_be_normed_has_a_gradient_of_zero(gpu_device, dtype, interleaved):
    """Whatever arrives for it, finite: its norm columns get 0 (the result is 0 all around), the others what the rotation gives, and the weight nothing. The heads
    beside it have what they have without it."""
    T, H, d, normed = 6, 3, 96, 64
    g = torch.Generator(device=gpu_device).manual_seed(1)
    x, dout = (torch.randn(T, H, d, generator=g, device=gpu_device).to(dtype) for _ in range(2))
    w = 1 + 0.2 * torch.randn(normed, generator=g, device=gpu_device)
    freq = loza.loza_ssa_rope_frequencies(32, 10000.0)[0].to(gpu_device)
    pos = torch.arange(T, dtype=I32, device=gpu_device)
    tail = (0, normed, 1e-6, normed, interleaved)           # the rotated columns are behind the normed ones
    ref, dref, dwref = torch.empty_like(x), torch.empty_like(x), torch.empty(normed, device=gpu_device)
    FORWARD[dtype](x, w, pos, freq, ref, *tail)
    kept = dout.clone()
    for t, h in ((1, 1), (4, 0), (5, 2)):
        kept[t, h, :normed] = 0
    BACKWARD[dtype](kept, x, w, pos, freq, dref, dwref, *tail)
    for t, h, size, arrives in ((1, 1, 2.0 ** 100, 2.0 ** 40), (4, 0, 2.0 ** 126, 2.0 ** 100), (5, 2, -(2.0 ** 64), 2.0 ** 70)):
        x[t, h, :normed] = size
        dout[t, h, :normed] = arrives
    out, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(normed, device=gpu_device)
    FORWARD[dtype](x, w, pos, freq, out, *tail)
    BACKWARD[dtype](dout, x, w, pos, freq, dx, dw, *tail)
    large = torch.zeros(T, H, dtype=torch.bool, device=gpu_device)
    large[1, 1] = large[4, 0] = large[5, 2] = True
    assert not bool(out[large][:, :normed].any()) and not bool(dx[large][:, :normed].any())
    assert torch.equal(out[~large], ref[~large]) and torch.equal(dx[~large], dref[~large]) and torch.equal(dx[large][:, normed:], dref[large][:, normed:])
    # (one head's 0 in the place of another's 0: the same sums, term by term)
    assert torch.equal(dw, dwref)
