"""Norms with rotary positions and their gradient at the sizes of a training step: results of 16 MB and more (stored past the caches), workgroups that take several
chunks of tokens, every row in earnest."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import beside_reference as N

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
FORWARD = {BF: loza.loza_ssa_norm_rope, F32: loza.loza_ssa_norm_rope_f32}
BACKWARD = {BF: loza.loza_ssa_norm_rope_backward, F32: loza.loza_ssa_norm_rope_backward_f32}
EPS = 1e-6


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("dtype,T", [(BF, 17_003), (F32, 9_001)])      # 1,024 and 2,048 bytes a token of 4 heads: 16 MB are 16,384 and 8,192 tokens
def test_large_results(gpu_device, dtype, T, interleaved):
    H, d = 4, 128
    edge = (16 << 20) // (H * d * (2 if dtype == BF else 4))
    g = torch.Generator(device=gpu_device).manual_seed(T)
    freq, m = loza.loza_ssa_rope_frequencies(d, 10000.0, 32.0, 32768)
    rng = np.random.default_rng(T)
    pos = rng.integers(0, 1 << 20, size=T).astype(np.int32)
    pos[rng.random(T) < 0.1] = -1
    live = pos >= 0
    rnd = lambda *s: torch.randn(*s, generator=g, device=gpu_device)
    x, dout, w = (rnd(T, H, d) * torch.exp(rnd(d))).to(dtype), rnd(T, H, d).to(dtype), 1 + 0.3 * rnd(d)
    at, fr, tail = torch.from_numpy(pos).to(gpu_device), freq.to(gpu_device), (0, d, EPS, 0, interleaved, m)
    on = torch.from_numpy(live).to(gpu_device)
    hx, hw = _np(x), _np(w)

    out = torch.full_like(x, 77.0)
    FORWARD[dtype](x, w, at, fr, out, *tail)
    ref = N.norm_rope(hx, hw, 0, d, EPS, pos, freq.numpy(), 0, interleaved, m)
    bound = N.norm_rope_bound(hx, hw, 0, d, EPS, freq.numpy(), 0, interleaved, m, ref, HALF[dtype])
    got = _np(out)
    assert (got[~live] == 77.0).all() and (np.abs(got - ref)[live] <= bound[live]).all()
    y = x.clone()                                              # in place
    FORWARD[dtype](y, w, at, fr, y, *tail)
    assert torch.equal(y[on], out[on]) and torch.equal(y[~on], x[~on])
    for n in (edge - 1, edge):                                 # either side of the limit: a row's bits do not depend on it
        part = torch.full_like(x[:n], 77.0)
        FORWARD[dtype](x[:n], w, at[:n], fr, part, *tail)
        assert torch.equal(part, out[:n])

    # The weight's gradient of all tokens, and of one in 64: there a head that was lost, or taken twice, is a thousandth of the sum, and its bound 3e-5 of it
    few = torch.from_numpy(rng.random(T) < 1 / 64).to(gpu_device)
    for arrives in (dout, torch.where(few[:, None, None], dout, torch.zeros_like(dout))):
        dx, dw = torch.full_like(x, 77.0), torch.full((d,), float("nan"), device=gpu_device)
        BACKWARD[dtype](arrives, x, w, at, fr, dx, dw, *tail)
        hd = _np(arrives)
        rx, rw = N.norm_rope_backward(hd, hx, hw, 0, d, EPS, pos, freq.numpy(), 0, interleaved, m)
        bx, bw = N.norm_rope_backward_bounds(hd, hx, hw, 0, d, EPS, pos, freq.numpy(), 0, interleaved, m, rx, HALF[dtype])
        got = _np(dx)
        assert (got[~live] == 77.0).all() and (np.abs(got - rx)[live] <= bx[live]).all()
        assert (np.abs(_np(dw) - rw) <= bw).all()
        for src in (arrives, x):                               # in the place of either
            z, again = src.clone(), torch.empty_like(dw)
            BACKWARD[dtype](z if src is arrives else arrives, z if src is x else x, w, at, fr, z, again, *tail)
            assert torch.equal(z[on], dx[on]) and torch.equal(z[~on], src[~on]) and torch.equal(again, dw)
    for n in (edge - 1, edge):
        part = torch.full_like(x[:n], 77.0)
        BACKWARD[dtype](arrives[:n], x[:n], w, at[:n], fr, part, None, *tail)
        assert torch.equal(part, dx[:n])
