"""Probabilities in the place of fp32 logits where the results are stored past the caches (128 MB and more)."""
import pytest
import torch

from tests.test_gpu_token_probs import F32, Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,V", [(600, 66_001), (3000, 12_003)])
def test_large_rows_in_place(gpu_device, B, V):
    c = Call(B, 1, V, F32, 7)
    ref, x = c.run(), c.logits.clone()
    assert B * V * 4 >= 128 << 20 and torch.equal(c.run(probs=x, logits=x), ref)
    keep = [0, 1, B // 2, B - 1]
    for name in ("seen", "rep", "fre", "pre", "temp", "bt", "bv", "lens", "masks", "tokens", "ok", "logits"):
        setattr(c, name, getattr(c, name)[keep])
    c.B = len(keep)
    c.check(ref[keep])
