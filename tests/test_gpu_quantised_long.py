"""Few rows over long caches held in 8 bits, where a CTA has tens of thousands of slots of a row: what lies far below the row's largest
weight counts all the same.  Definitions and bounds: test_gpu_quantised.py.

A weight is three e4m3 terms: within 2^-12 of itself, or 2^-23 of the largest contribution (weight times the V row's largest) that its
reference was taken for.  A reference that a large weight has raised stays for at most 32 tiles of 256 slots, so of a row at most 8192
slots lie under each such weight: 8192 * 2^-23 = 2^-10 of it, and as much again for the tile that the next reference is taken from."""
import math

import pytest
import torch

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth

from test_gpu_decode import i32
from test_gpu_quantised import Problem, check, check_lse, value

pytestmark = pytest.mark.gpu
SHAPES = [(128, 7, 1), (128, 4, 4), (128, 8, 4), (256, 2, 3), (256, 8, 2), (256, 8, 4)]      # tiles of 8, 16, 32 rows, each width


def sequences():
    """As many as there are SMs, so that a CTA has a sequence to itself."""
    return torch.cuda.get_device_properties(0).multi_processor_count


def attend(dec, q, code, byte, n, cap=0.0):
    """The same new tokens [new, Hq, d] in many sequences over one another's pages (codes [n, d], bytes [n] of one KV head)."""
    B, page, d = sequences(), 256, code[0].shape[-1]
    table = torch.randperm(-(-n // page), generator=torch.Generator().manual_seed(1)).int()
    pools = []
    for x, fill in [(c, 0x7f) for c in code] + [(b, 255) for b in byte]:
        pad = torch.full((len(table) * page, *x.shape[1:]), fill, dtype=torch.uint8, device="cuda")
        pad[:n] = x
        pool = torch.empty_like(pad).view(len(table), page, *x.shape[1:])
        pool[table.long().cuda()] = pad.view_as(pool)
        pools.append(pool.view(len(table), page, 1, d) if x.dim() == 2 else pool.view(len(table), 1, page))
    new = q.shape[0]
    out, lse = torch.zeros((B * new, *q.shape[1:]), dtype=q.dtype, device="cuda"), torch.zeros((B * new, q.shape[1]), device="cuda")
    dec.attend_quantised(q.repeat(B, 1, 1), i32(range(0, B * new + 1, new)), i32([n] * B), *pools, out, lse=lse,
                         page_table=table.cuda().expand(B, -1).contiguous(), page_size=page)
    assert dec.device_status() == 0 and dec.launches() == 2
    out, lse = out.view(B, new, -1, d), lse.view(B, new, -1)
    assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
    return out[0], lse[0]


@pytest.mark.parametrize("d,G,new", SHAPES)
@pytest.mark.parametrize("n", [131072, 524288])
@pytest.mark.parametrize("first", [0, 300, 70000])
def test_a_tail_far_below_one_large_weight(d, G, new, n, first):
    """One slot's weight is 2^23.6 times each of the others', which are -1 where it is 1 and together a part of it that bf16 sees."""
    code = [torch.zeros((n, d), dtype=torch.uint8, device="cuda"), torch.full((n, d), 0xb8, dtype=torch.uint8, device="cuda")]
    byte = [torch.full((n,), 127, dtype=torch.uint8, device="cuda") for _ in "kv"]
    code[0][first] = code[1][first] = 0x38                   # 1.0
    dec = kvx.Decoder(synth.ModelGeom(1, 1, d, 1e4), G)
    q = torch.full((new, G, d), 23.6 * math.log(2.0) / math.sqrt(d), device="cuda").bfloat16()
    out, lse = attend(dec, q, code, byte, n)
    score = float(q[0, 0].double().sum()) / math.sqrt(d)
    for t in range(new):
        others = n - new + t                                 # besides the large one
        total = math.exp(score) + others
        want, share = (math.exp(score) - others) / total, math.exp(score) / total
        e = 6 * math.sqrt(d) * 2.0 ** -24 * score + 16 * 2.0 ** -24 * score
        tol = 1.05 * (2 * e + 2.0 ** -20 + 2.0 ** -12 + 6 * math.sqrt(n) * 2.0 ** -24) + 2.0 ** -8 * 1.01 * abs(want) + 2 * 2.0 ** -10 * share
        lost = (others - n // 4) * 2.0 ** -23.6 * share      # what it would be off by without them (but for three quarters of a half)
        assert lost > tol or n < 500000
        assert float((out[t].double() - want).abs().max()) <= tol
        assert float((lse[t].double() - math.log(total)).abs().max()) <= e + 2.0 ** -20 + 2.0 ** -22 * math.log(total)


@pytest.mark.parametrize("d,G,new", SHAPES)
@pytest.mark.parametrize("kind", ["even", "rising", "falling", "scales_far_apart", "capped"])
def test_long_ranges(d, G, new, kind):
    """References taken anew again and again: random rows, growing and falling scores, scales far apart."""
    gain = {"rising": lambda x: 0.1 + 4 * x, "falling": lambda x: 4.1 - 4 * x}.get(kind, lambda x: 0 * x + 1)
    n, cap = 41000, 20.0 if kind == "capped" else 0.0
    p = Problem(1, G, d, [n - new], [new], "bf16", 0, seed=3, cap=cap, gain=gain, spread=3.0 if kind == "scales_far_apart" else 0.5)
    eo, el, to, tl = p.exact(weight_eps=2.0 ** -12)
    out, lse = attend(p.dec, p.q.cuda(), [c[0, 0].cuda() for c in p.code], [s[0, 0].cuda() for s in p.byte], n, cap)
    K, V = (value(c, s).double()[0, 0].cuda() for c, s in zip(p.code, p.byte))
    x = (p.q.double().cuda() @ K.T) / math.sqrt(d)
    x = cap * torch.tanh(x / cap) if cap else x
    x = x.masked_fill(torch.arange(n, device="cuda") > torch.arange(n - new, n, device="cuda")[:, None, None], -math.inf)
    part = torch.softmax(x, -1) * V.abs().amax(-1) * 2       # contributions (a row's largest is above half of what its scale allows)
    # each of them above those of 8192 slots at most, and of no more than there are
    floor = (2.0 ** -23 * 2 * part.topk(-(-n // 8192), -1)[0].sum(-1) * 8192).cpu()
    check(out.cpu(), eo, to + floor[..., None], "out")
    check_lse(lse.cpu(), el, tl)


@pytest.mark.parametrize("d,G,new", [(128, 7, 1), (256, 8, 4)])
@pytest.mark.parametrize("byte", [10, 24, 30, 60, 200, 240])
def test_a_tail_under_far_scales(d, G, new, byte):
    """As above, V's rows under scales from 2^-117 to 2^113: references have to stay where their powers are numbers.  Below 2^-100 they do not
    follow the weights down, and the tail may be lost; the large weight's row never is."""
    n = 200000
    code = [torch.zeros((n, d), dtype=torch.uint8, device="cuda"), torch.full((n, d), 0x38, dtype=torch.uint8, device="cuda")]
    scales = [torch.full((n,), x, dtype=torch.uint8, device="cuda") for x in (127, byte)]
    code[0][5] = 0x38
    dec = kvx.Decoder(synth.ModelGeom(1, 1, d, 1e4), G)
    q = torch.full((new, G, d), 23.6 * math.log(2.0) / math.sqrt(d), device="cuda").bfloat16()
    out, lse = attend(dec, q, code, scales, n)
    one = 2.0 ** (byte - 127)
    score = float(q[0, 0].double().sum()) / math.sqrt(d)
    share = math.exp(score) / (math.exp(score) + n)
    tol = 2.0 ** -8 + 2.0 ** -12 + 2 * 2.0 ** -10 * share + (1 - share if byte < 31 else 0.0)
    assert float((out.double() / one - 1.0).abs().max()) <= tol
    assert float((lse.double() - math.log(math.exp(score) + n - new)).abs().max()) <= 1e-4
