"""The attention weight each cached slot receives, where the scores are formed again because they do not fit the
workspace.  Bounds as in test_gpu_decode.py."""
import pytest
import torch

from test_gpu_decode import Problem, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,prefix", [(0, None), (300, None), (40, [100, 7, 50])])
def test_fp32_tiles_that_no_token_sees(d, window, prefix):
    """More (slot tile, head) units than resident CTAs, most of them before every window or of a sequence without new
    tokens: between units that add, a CTA passes by units that do not."""
    p = Problem(8, 2, d, [3000, 6300, 3400], [20, 40, 0], "fp32", 16, seed=51)
    w = torch.zeros((3, 8, 20000), device="cuda")       # 60 tokens x 16 heads x 20000: beyond the kept scores
    p.attend(window, prefix, weight=w)
    _, _, ew, _, _, tw = p.exact(window, prefix)
    check(p, w[:, :, :p.S].cpu(), ew, tw + 1e-30, "key_weight")
    assert not w[2].any() and not w[:, :, p.S:].any()
    for _ in range(3):
        again = torch.zeros_like(w)
        p.attend(window, prefix, weight=again)
        assert torch.equal(again, w)
    assert p.dec.device_status() == 0
