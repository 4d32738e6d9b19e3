"""Conversions refuse one's own memory, whichever of a cache's pointers is in both, and lists of other lengths."""
import pytest
import torch

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth

from test_gpu_decode import i32

pytestmark = pytest.mark.gpu


def caches(L, H=2, S=64, d=128):
    full = [[torch.ones((1, H, S, d), dtype=torch.bfloat16, device="cuda") for _ in range(L)] for _ in "kv"]
    held = [[torch.zeros((1, H, S, d), dtype=torch.uint8, device="cuda") for _ in range(L)] for _ in "kv"]
    held += [[torch.zeros((1, H, S), dtype=torch.uint8, device="cuda") for _ in range(L)] for _ in "kv"]
    return full, held


@pytest.mark.parametrize("L", [1, 3, kvx.KVX_MAX_TARGET_LAYERS])
def test_caches_that_share_memory(L):
    full, held = caches(L)
    dec = kvx.Decoder(synth.ModelGeom(L, 2, 128, 1e4), 4)
    n = i32([64])
    dec.quantise(n, *full, *held)
    dec.dequantise(n, *held, *full)
    for mine, theirs in {(0, 0), (L - 1, 0), (L // 2, L - 1)}:
        for a in range(2):
            for b in range(4):
                both = [list(x) for x in held]
                like = both[b][theirs]
                both[b][theirs] = full[a][mine].view(torch.uint8).view(-1)[:like.numel()].view(like.shape)
                for call in (lambda: dec.quantise(n, *full, *both), lambda: dec.dequantise(n, *both, *full)):
                    with pytest.raises(kvx.KvxError) as e:
                        call()
                    assert e.value.status == kvx.KVX_ERR_INVALID_ARG and "in common" in str(e.value) and dec.launches() == 0
    assert dec.device_status() == 0 and all(bool((x == 1).all()) for y in full for x in y)


def test_lists_of_other_lengths():
    full, held = caches(2)
    dec = kvx.Decoder(synth.ModelGeom(2, 2, 128, 1e4), 4)
    n = i32([64])
    for which in range(6):
        for short in (0, 1):
            lists = [*full, *held]
            lists[which] = lists[which][:short]
            with pytest.raises(ValueError):
                dec.quantise(n, *lists)
            with pytest.raises(ValueError):
                dec.dequantise(n, *lists[2:], *lists[:2])
    with pytest.raises(ValueError):
        dec.quantise(n, *([] for _ in range(6)))
    assert dec.device_status() == 0
