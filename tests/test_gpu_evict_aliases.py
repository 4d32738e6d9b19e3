"""kvx_evict where outputs take an input's place."""
import numpy as np
import pytest
import torch

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth

from test_gpu_decode import evict_definition, i32

pytestmark = pytest.mark.gpu


class Cut:
    """A contiguous cache of L layers, its weights, and what a cut of it gives by definition."""

    def __init__(self, L=10, B=8, H=8, S=600, d=64, keep=200, sinks=4, recent=20, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.keep, self.sinks, self.recent, self.shape = keep, sinks, recent, (L, B, H)
        self.lens = [S, S - 1, keep, keep - 1, keep + 1, 0, 333, S - 50][:B]
        self.w = torch.rand((L, B, H, S), device="cuda", generator=g).pow(6)
        self.k, self.v = (torch.randn((L, B, H, S, d), device="cuda", generator=g).to(dtype) for _ in range(2))
        self.dk, self.dv = (torch.full((L, B, H, keep, d), 9.0, dtype=dtype, device="cuda") for _ in range(2))
        self.kept = torch.full((L, B, H, keep), -7, dtype=torch.int32, device="cuda")
        self.kept_weight = torch.full((L, B, H, keep), -7.0, device="cuda")
        self.dec = kvx.Decoder(synth.ModelGeom(L, H, d, 1e4), H, dtype=kvx.KVX_BF16 if dtype == torch.bfloat16 else kvx.KVX_FP32)

    def evict(self, kv_len, new_len, **kw):
        self.dec.evict(kv_len, self.w, self.keep, list(self.k), list(self.v), list(self.dk), list(self.dv), self.kept, new_len,
                       sinks=self.sinks, recent=self.recent, kept_weight=self.kept_weight, **kw)

    def check(self, new_len):
        assert self.dec.device_status() == 0
        assert new_len.tolist() == [min(n, self.keep) for n in self.lens]
        w, kept = self.w.cpu().numpy(), self.kept.cpu().numpy()
        for l, b, h in np.ndindex(self.shape):
            want = evict_definition(w[l, b, h], self.lens[b], self.keep, self.sinks, self.recent)
            m = len(want)
            assert np.array_equal(kept[l, b, h, :m], want) and (kept[l, b, h, m:] == -1).all()
            at = torch.from_numpy(want).cuda()
            assert torch.equal(self.kept_weight[l, b, h, :m], self.w[l, b, h, at])
            assert torch.equal(self.dk[l, b, h, :m], self.k[l, b, h, at]) and torch.equal(self.dv[l, b, h, :m], self.v[l, b, h, at])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lengths_in_place(dtype):
    """new_len is kv_len, with more (layer, sequence, head) units than the device holds at once."""
    c = Cut(dtype=dtype)
    n = i32(c.lens)
    c.evict(n, n)
    c.check(n)


def test_kept_weights_over_the_weights_are_refused():
    """Units would overwrite weights that others have yet to read."""
    c = Cut(L=2, B=2, H=2, S=400, keep=200)
    n, new_len = i32(c.lens), i32([0] * 2)
    own, w = c.kept_weight, c.w
    flat = torch.zeros(2 * w.numel(), device="cuda")
    inner = flat[w.numel() // 2:w.numel() // 2 + own.numel()].view(own.shape)
    for key_weight, kept_weight in ((w, w), (flat[:w.numel()].view(w.shape), inner), (flat[w.numel() // 2:][:w.numel()].view(w.shape), flat[
            w.numel() // 2 - 1:][:own.numel()].view(own.shape)), (flat[:w.numel()].view(w.shape), flat[w.numel() - 1:][:own.numel()].view(own.shape))):
        c.w, c.kept_weight = key_weight, kept_weight
        with pytest.raises(kvx.KvxError) as e:
            c.evict(n, new_len)
        assert e.value.status == kvx.KVX_ERR_INVALID_ARG and "overlap" in kvx.kvx_last_error()
    # one behind the other, either way round
    both = torch.zeros(w.numel() + own.numel(), device="cuda")
    for first in (0, own.numel()):
        c.w = both[first:first + w.numel()].view(w.shape).copy_(w)
        c.kept_weight = (both[w.numel():] if first == 0 else both[:own.numel()]).view(own.shape)
        c.evict(n, new_len)
        c.check(new_len)
