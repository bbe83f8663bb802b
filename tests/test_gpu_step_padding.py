"""Rows of a tree call that see nothing (behind the last node, or with an empty mask) give out = 0 and lse = -inf whatever their queries hold: nobody need
have written these (loza_ssa_rope_append leaves the rows of padding as they are). Nor do they change a bit of the rows beside them."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests.test_gpu_step_tree import LARGE, _call, _masks, _rand

pytestmark = pytest.mark.gpu

FEW = [   # few rows: whole, in parts, with three heads a key head, nodes of several sequences short
    (2, 64, 1, 576, 700, 8, 16, 300, 1, 0, True, None, 0),
    (1, 128, 2, 576, 2500, 5, 16, 2300, 1, 64, True, None, 0),
    (2, 6, 2, 128, 900, 33, 1, 8, 64, 64, False, None, 0),
    (1, 4, 4, 128, 900, 3, 16, 700, 1, 0, False, None, 0),
]


@pytest.mark.parametrize("scratch", [True, False])
@pytest.mark.parametrize("B,Hq,Hkv,d,S_max,n,sink,local,block,page,alias,kernel,step", LARGE + FEW)
def test_rows_that_see_nothing(gpu_device, B, Hq, Hkv, d, S_max, n, sink, local, block, page, alias, kernel, step, scratch):
    rng = np.random.default_rng(n)
    lens = [S_max - 13 * b % 200 for b in range(B)]               # (long ones: most tiles lie before the tree and take no mask)
    counts = [max(1, n - 1 - b % 7) for b in range(B)]
    masks = _masks(rng, n, counts, "tree")
    if n > 3:
        masks[::2, n // 3] = 0
    dead = torch.from_numpy(masks == 0).to(gpu_device)            # [B, n]
    q, kc = _rand((B, n, Hq, d), 21, gpu_device), _rand((B, S_max, Hkv, d), 22, gpu_device)
    vc = kc if alias else _rand((B, S_max, Hkv, d), 23, gpu_device)
    d_v, scale = (512, 192 ** -0.5) if d == 576 else (128, 128 ** -0.5)
    ws = None if scratch else torch.empty(0, dtype=torch.uint8, device=gpu_device)

    def call():
        out, lse = _call(q, kc, vc, lens, counts, masks, sink, local, block, scale, d_v, page, workspace=ws)
        lse = lse.transpose(1, 2)                                 # [B, n, Hq]
        assert bool((out[dead] == 0).all()) and bool((lse[dead] == -float("inf")).all())
        return out[~dead].view(torch.int16), lse[~dead].contiguous().view(torch.int32)

    q[dead] = 0
    want = call()
    assert bool(torch.isfinite(want[0].view(torch.bfloat16).float()).all()) and bool(torch.isfinite(want[1].view(torch.float32)).all())
    for fill in (float("nan"), float("inf"), -float("inf"), 3e38, 50.0):
        q[dead] = fill
        got = call()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), fill
    # values that are not finite, at keys that other rows see: these rows see none of them
    for b in range(B):
        vc[b, max(0, lens[b] - counts[b] - 40):lens[b] - counts[b]] = float("inf")
        vc[b, 0] = float("nan")
    call()
