"""What the binding refuses before it hands out a pointer: tensors that would be misread, of another type, or strided."""
import pytest
import torch

import paper_2608_30963_gb300 as kvx

from test_gpu_decode import Problem, i32

pytestmark = pytest.mark.gpu


class Args:
    """Arguments of the three calls, all of them right; a test replaces one."""

    def __init__(self, dtype="bf16", ps=16):
        p = self.p = Problem(2, 4, 128, [60, 9], [3, 1], dtype, ps, seed=71)
        self.a = dict(q=p.q.cuda(), seq_off=i32(p.off), kv_len=i32(p.L), cache_k=p.cache(p.K), cache_v=p.cache(p.V), out=torch.zeros_like(p.q, device="cuda"),
                      lse=torch.zeros((p.T, 8), device="cuda"), key_weight=torch.zeros((2, 2, p.S), device="cuda"), prefix_len=i32([1, 0]), **p.paged())
        a = self.a
        self.b = dict(q=a["q"], k=a["q"][:, :2].contiguous(), v=a["q"][:, 2:4].contiguous(), seq_off=a["seq_off"], kv_len=a["kv_len"], cache_k=a["cache_k"],
                      cache_v=a["cache_v"], q_out=torch.zeros_like(a["q"]), pos=i32(range(p.T)), **p.paged())
        self.c = dict(kv_len=a["kv_len"], key_weight=torch.rand((2, 2, 2, p.S), device="cuda"), keep=20, src_k=[a["cache_k"]] * 2, src_v=[a["cache_v"]] * 2,
                      dst_k=[p.cache(p.K) for _ in range(2)], dst_v=[p.cache(p.V) for _ in range(2)], kept=torch.zeros((2, 2, 2, 20), dtype=torch.int32, device="cuda"),
                      new_len=i32([0, 0]), kept_weight=torch.zeros((2, 2, 2, 24), device="cuda"))
        if ps:
            self.c.update(page_table=p.table, dst_page_table=p.table, page_size=ps)
        from paper_2608_30963_gb300 import synth
        self.two = kvx.Decoder(synth.ModelGeom(2, 2, 128, 1e4), 8, dtype=p.dec.desc.dtype)

    def calls(self):
        return ((self.p.dec.attend, self.a), (self.p.dec.append, self.b), (self.two.evict, self.c))

    def right(self):
        for f, args in self.calls():
            f(**args)
        assert self.p.dec.device_status() == 0 and self.two.device_status() == 0

    def refused(self, call, name, value):
        f, args = self.calls()[call]
        assert name in args
        with pytest.raises(ValueError):
            f(**dict(args, **{name: value}))


ATTEND, APPEND, EVICT = range(3)


@pytest.mark.parametrize("ps", [0, 16])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_types(dtype, ps):
    """A type of the same size is another type."""
    x = Args(dtype, ps)
    x.right()
    other = torch.float16 if dtype == "bf16" else torch.int32
    like = {torch.int32: torch.float32, torch.float32: torch.int32, torch.bfloat16: other}
    for call, (_, args) in enumerate(x.calls()):
        for name, t in args.items():
            if isinstance(t, torch.Tensor):
                x.refused(call, name, t.view(other if t.dtype == x.p.tdt and name not in ("lse", "key_weight", "kept_weight") else like[t.dtype]))
            elif isinstance(t, list):
                x.refused(call, name, [y.view(other) for y in t])
    x.right()


@pytest.mark.parametrize("ps", [0, 16])
def test_strides(ps):
    """Lengths, offsets, positions, tables and sums are read as arrays without gaps: a view with gaps is another array."""
    x = Args("bf16", ps)
    x.right()
    for call, (_, args) in enumerate(x.calls()):
        for name, t in args.items():
            if isinstance(t, torch.Tensor) and t.dtype != torch.bfloat16:
                gaps = torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype, device="cuda")[..., ::2]
                gaps.copy_(t)
                x.refused(call, name, gaps)
    # one sequence, one element: nothing can have a gap
    one = Problem(2, 4, 128, [60], [1], "bf16", ps, seed=72)
    out = torch.zeros_like(one.q, device="cuda")
    length = torch.tensor([one.L[0], -5], dtype=torch.int32, device="cuda")[::2]
    one.dec.attend(one.q.cuda(), i32(one.off), length, one.cache(one.K), one.cache(one.V), out, **one.paged())
    assert torch.equal(out.cpu(), one.attend()[0])


@pytest.mark.parametrize("ps", [0, 16])
@pytest.mark.parametrize("name", ["src_k", "src_v", "dst_k", "dst_v"])
def test_every_layer_of_an_eviction(name, ps):
    """A later layer that is smaller, wider apart or of another type than the first."""
    x = Args("bf16", ps)
    x.right()
    t = x.c[name][1]
    wide = torch.empty((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype, device="cuda")[..., :t.shape[-1]]
    for bad in (t[:-1], t[:, :, :-1], wide, t.view(torch.float16), t.float(), t.transpose(1, 2), t[:, :, :, :64]):
        x.refused(EVICT, name, [x.c[name][0], bad])
        x.refused(EVICT, name, [bad, x.c[name][1]])
    x.refused(EVICT, name, x.c[name][:1])
    x.right()
    if not ps:      # layers that are all alike views of something wider are taken
        x.c["src_k"] = [torch.cat([t, t], -1)[..., :128] for t in x.c["src_k"]]
        x.c["src_v"] = [torch.cat([t, t], -1)[..., :128] for t in x.c["src_v"]]
        x.right()
