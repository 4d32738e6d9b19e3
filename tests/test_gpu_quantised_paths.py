"""Attention over caches held in 8 bits: each of its kernels at its rule's borders, what the workspace holds, and how exact the
weights are where they are split into terms.  Definitions and bounds: test_gpu_quantised.py."""
import math

import pytest
import torch

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth

from test_gpu_decode import i32
from test_gpu_quantised import CODES, Problem, check, check_lse, held, value

pytestmark = pytest.mark.gpu


def run(p, window=0, prefix=None, **kw):
    out, lse = p.attend(window, prefix)
    assert p.dec.device_status() == 0
    eo, el, to, tl = p.exact(window, prefix, **kw)
    check(out, eo, to, "out")
    check_lse(lse, el, tl)
    assert torch.equal(p.attend(window, prefix, lse=False)[0], out), "equal calls give equal bits"
    return out, lse


def wide(p, slots):
    """A page table with room for so many slots: a call that may not fit the workspace."""
    more = -(-slots // p.place.page) - p.place.table.shape[1]
    p.place.table = torch.nn.functional.pad(p.place.table, (0, max(0, more)), value=-1).contiguous()
    return p


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("page", [0, 1, 7, 13, 16])
@pytest.mark.parametrize("G,new", [(7, [1, 1]), (8, [1, 2]), (5, [3, 0]), (8, [4, 4]), (2, [16, 1]), (16, [2, 1]), (32, [1, 1]), (11, [1, 1])])
def test_few_rows(d, page, G, new):
    """Tiles of 8, 16 and 32 rows, and sequences with more tokens than the mean; pages that end anywhere."""
    run(Problem(2, G, d, [519, 70], new, "bf16", page, seed=G + page))


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("L", [1, 2, 127, 128, 129, 255, 256, 257, 511, 512, 513, 769])
def test_few_rows_at_the_ends_of_tiles(d, L):
    run(Problem(1, 4, d, [L - 1], [1], "bf16", 16, seed=L))


@pytest.mark.parametrize("d,H,G", [(128, 2, 6), (256, 1, 4)])
@pytest.mark.parametrize("window,prefix", [(0, None), (1, None), (255, None), (256, [3, 300]), (700, [0, 1000]), (0, [900, 900])])
def test_few_rows_masks(d, H, G, window, prefix):
    run(Problem(H, G, d, [900, 513], [3, 2], "bf16", 16, seed=window), window, prefix)


@pytest.mark.parametrize("d,G,new", [(128, 7, 1), (128, 4, 4), (256, 2, 3), (256, 8, 4), (128, 16, 1)])
def test_few_rows_weights_are_exact_to_three_terms(d, G, new):
    """Three terms leave a weight within 2^-12 of itself or 2^-22 of the row's largest contribution."""
    p = Problem(2, G, d, [3000], [new], "bf16", 16, seed=3)
    out, _ = p.attend()
    eo, _, to, _ = p.exact(weight_eps=2.0 ** -12)
    K, V = (value(c, s).double()[0] for c, s in zip(p.code, p.byte))
    floor = torch.zeros_like(to)
    for t in range(new):
        L = 3000 + t + 1
        for head in range(2 * G):
            w = torch.softmax(p.q[t, head].double() @ K[head // G, :L].T * p.scale, -1)
            floor[t, head] = 2.0 ** -22 * (w * V[head // G, :L].abs().amax(-1)).max() * 448 / 224 * math.sqrt(L) * 6      # (independent roundings)
    assert bool(((out.double() - eo).abs() <= to + floor).all())


@pytest.mark.parametrize("d", [128, 256])
def test_few_rows_one_bf16_term_would_show(d):
    """Two slots whose weights, 1 and about exp(-0.01), nearly cancel: 0.99005 lies 0.0018 from bf16's nearest (multiples of 2^-8), which
    would move the output, their difference over their sum, by 0.0009; three terms may move it by 2^-12."""
    p = Problem(1, 2, d, [1], [1], "bf16", 16, seed=5)
    for i in range(2):
        p.code[i].fill_(0x38)                            # 1.0
        p.byte[i].fill_(127)
    p.code[0][:, :, 0] = 0x00
    p.code[1][:, :, 1] = 0xb8                            # -1.0
    p.q.fill_(-0.01 / (d * p.scale))
    out, _ = p.attend()
    eo, _, to, _ = p.exact(weight_eps=2.0 ** -12)
    check(out, eo, to, "out")
    w = torch.tensor(math.exp(float(p.q[0, 0].double().sum()) * p.scale))
    planted = (1 - float(w.bfloat16())) / (1 + float(w))
    assert abs(planted - float(eo[0, 0, 0])) > 2 * float(to[0, 0, 0])


@pytest.mark.parametrize("d,G,new,gain", [(*s, g) for s in [(128, 7, 1), (128, 4, 4), (256, 2, 3), (256, 8, 4), (128, 16, 1)] for g in (1e4, 1e6, 1e9, 1e20)] +
                         [(*s, g) for s in [(64, 4, 1), (128, 4, 100), (256, 2, 700)] for g in (1e4, 1e6)])
def test_scores_far_from_zero(d, G, new, gain):
    """A row whose largest score is beyond all others by far is that slot's row of V (to the bit where weights are more than one term):
    an error of the score is no error of its weight."""
    p = Problem(2, G, d, [900], [new], "bf16", 16, seed=17, q_gain=gain)
    out, lse = p.attend()
    K, V = (value(c, s).double()[0] for c, s in zip(p.code, p.byte))
    L, alone = p.L[0], 0
    for head in range(2 * G):
        x = p.q[:, head].double() @ K[head // G, :L].T * p.scale
        x = x.masked_fill(torch.arange(L) > torch.arange(L - new, L)[:, None], -math.inf)
        (a, b), (at, _) = (y.unbind(1) for y in x.topk(2, 1))
        mag = (p.q[:, head].double().abs() @ K[head // G, :L].abs().T * p.scale).amax(1)
        # both scores within 6 sqrt(d) roundings of the sum of magnitudes; weights of e^-110 are zero in 32 bits
        one = a - b > 110 + 2 * 6 * math.sqrt(d) * 2.0 ** -24 * mag
        alone += int(one.sum())
        got, want = out[one, head].double(), V[head // G, at[one]]
        # In many rows a weight is one bf16 number over a reference that may lie behind the row's largest score: it is rounded, by 2^-8 of
        # itself at most, and the sum that divides it is not; the result is rounded once more, (1 + 2^-8)^2 - 1 = 2^-7 + 2^-16.
        assert bool(((got - want).abs() <= (2.0 ** -7 + 2.0 ** -16) * want.abs()).all()) if new > 32 else torch.equal(got, want)
        assert bool(((lse[one, head].double() - a[one]).abs() <= (6 * math.sqrt(d) * 2.0 ** -24 * mag + 2.0 ** -22 * a.abs())[one]).all())
    assert alone > new * G and p.dec.device_status() == 0


@pytest.mark.parametrize("d", [128, 256])
def test_few_rows_a_flat_tail(d):
    """One score far above 30000 equal ones that weigh as much together: their terms' roundings all go one way."""
    n = 30000
    p = Problem(1, 2, d, [n], [1], "bf16", 16, seed=4)
    for i in range(2):
        p.code[i].fill_(0x38)                            # 1.0
        p.byte[i].fill_(127)
    p.code[0][:, :, 1:] = 0x00                           # scores: log(n) once, then zero
    p.q.fill_(math.log(n) * math.sqrt(d) / d)
    p.code[1][:, :, 0] = 0xb8                            # -1.0 for the first slot: the sums nearly cancel
    out, lse = p.attend()
    eo, el, to, tl = p.exact(weight_eps=2.0 ** -12)
    check_lse(lse, el, tl)
    w = math.exp(float(p.q[0, 0].double().sum()) * p.scale)                                               # of the first slot, others 1
    assert bool(((out.double() - eo).abs() <= to + (n + 1) * 2.0 ** -22 * w / (w + n)).all())


# rows a (sequence, KV head): up to 128 one row tile, up to six of them converted in place, more of them from the workspace
@pytest.mark.parametrize("d,G,new", [(128, 3, 42), (128, 3, 43), (128, 4, 384), (128, 4, 385), (64, 4, 384), (64, 4, 400), (256, 2, 256), (256, 2, 257), (256, 2, 384), (256, 2, 390), (64, 2, 12),
                                     (128, 33, 4), (128, 5, 7), (64, 64, 3)])
@pytest.mark.parametrize("opt", ["plain", "window_prefix", "capped"])
def test_many_rows(d, G, new, opt):
    p = Problem(1, G, d, [333], [new], "bf16", 16, seed=new, cap=20.0 if opt == "capped" else 0.0)
    run(p, *((150, [70]) if opt == "window_prefix" else (0, None)))


@pytest.mark.parametrize("d,G,new", [(128, 4, 400), (64, 4, 400), (256, 2, 400)])
@pytest.mark.parametrize("layout,page", [("bhsd", 0), ("bshd", 0), ("bhsd", 16), ("bhsd", 7)])
def test_many_rows_with_and_without_the_workspace(d, G, new, layout, page):
    """A call whose cache may not fit the workspace converts in place; both ways, several sequences, one of them without tokens."""
    ctx, tokens = [500, 40, 0, 129], [new, new, new, 0]
    p = Problem(2, G, d, ctx, tokens, "bf16", page, seed=d, layout=layout)
    out, _ = run(p, 300, [65, 2, 9, 1])
    if page:
        far = wide(Problem(2, G, d, ctx, tokens, "bf16", page, seed=d), (16 << 20) // (4 * 2 * d) + 64)
        other, _ = run(far, 300, [65, 2, 9, 1])
        assert float((other.double() - out.double()).abs().max()) <= 2.0 ** -6 * float(out.abs().max())


@pytest.mark.parametrize("new", [400, 40, 3])
def test_bad_pages_and_hidden_rows(new):
    """A page outside the pool reads as zero rows on every path; what no token sees may be anything."""
    p = Problem(1, 4, 128, [600], [new], "bf16", 16, seed=6)
    window = new + 100
    hidden = 600 - window + 1                                               # the first token, in slot 600, sees none before it
    for i in range(2):
        p.code[i][:, :, :hidden], p.byte[i][:, :, :hidden] = 0x7f, 255
    out, lse = p.attend(window)
    eo, el, to, tl = p.exact(window)
    check(out, eo, to, "out")
    check_lse(lse, el, tl)
    table = p.place.table.clone()
    table[0, 35] = -1                                                       # slots 560 .. 575
    got = torch.zeros_like(p.q, device="cuda")
    p.dec.attend_quantised(p.q.cuda(), i32(p.off), i32(p.L), *p.cache(), got, window=window, page_table=table)
    assert p.dec.device_status() == kvx.KVX_DEV_PAGE_INVALID
    for i in range(2):
        p.byte[i][:, :, 560:576] = 0
    eo, _, to, _ = p.exact(window)
    check(got.cpu(), eo, to, "out")


def test_the_workspace_is_shared_by_calls_in_order():
    """Weight sums over a bf16 cache, a prompt and a token over 8-bit ones, again and again on one decoder."""
    p, one = Problem(2, 4, 128, [300], [400], "bf16", 16, seed=8), Problem(2, 4, 128, [700], [1], "bf16", 16, seed=9)
    base, base1 = p.attend()[0], one.attend()[0]
    full = [torch.randn((1, 2, 700, 128), device="cuda").bfloat16() for _ in "kv"]
    q, out, lse = torch.randn((1, 8, 128), device="cuda").bfloat16(), torch.zeros((1, 8, 128), device="cuda").bfloat16(), torch.zeros((1, 8), device="cuda")
    first = torch.zeros((1, 2, 700), device="cuda")
    p.dec.attend(q, i32([0, 1]), i32([700]), *full, out, lse=lse, key_weight=first)
    caches, dev = [x.cache() for x in (p, one)], [x.q.cuda() for x in (p, one)]
    for _ in range(3):
        w, outs = torch.zeros_like(first), [torch.zeros_like(x) for x in dev]
        p.dec.attend(q, i32([0, 1]), i32([700]), *full, out, lse=lse, key_weight=w)
        p.dec.attend_quantised(dev[0], i32(p.off), i32(p.L), *caches[0], outs[0], **p.place.kw())
        p.dec.attend_quantised(dev[1], i32(one.off), i32(one.L), *caches[1], outs[1], **one.place.kw())
        assert torch.equal(w, first) and torch.equal(outs[0].cpu(), base) and torch.equal(outs[1].cpu(), base1)


def test_two_decoders_on_two_streams():
    """Each has a workspace of its own: calls side by side give the bits that they give one after the other."""
    sizes = [(dict(H=2, G=7, d=128, ctx=[5000, 300], new=[1, 1]), dict(H=2, G=4, d=128, ctx=[900, 3], new=[400, 400])),
             (dict(H=2, G=2, d=256, ctx=[3000], new=[6]), dict(H=1, G=4, d=64, ctx=[2000], new=[90]))]
    for pair in sizes:
        ps = [Problem(**kw, seed=29 + i) for i, kw in enumerate(pair)]
        alone = [p.attend()[0] for p in ps]
        args = [(p.q.cuda(), i32(p.off), i32(p.L), *p.cache()) for p in ps]
        outs = [[torch.zeros_like(a[0]) for _ in range(8)] for a in args]
        streams = [torch.cuda.Stream() for _ in ps]
        torch.cuda.synchronize()
        for n in range(8):
            for p, a, o, st in zip(ps, args, outs, streams):
                p.dec.attend_quantised(*a, o[n], stream=st, **p.place.kw())
        torch.cuda.synchronize()
        for p, want, o in zip(ps, alone, outs):
            assert p.dec.device_status() == 0 and all(torch.equal(x.cpu(), want) for x in o)


def test_steps_in_a_graph():
    """Quantise, append, attend (a prompt and a token) and read back as one captured graph, replayed with other lengths."""
    H, G, d, page, pages = 2, 4, 128, 16, 64
    dec = kvx.Decoder(synth.ModelGeom(1, H, d, 1e4), H * G)
    g = torch.Generator(device="cuda").manual_seed(2)
    table = torch.randperm(pages, generator=g, device="cuda").int().view(1, pages)
    full = [torch.randn((pages, page, H, d), device="cuda", generator=g).bfloat16() for _ in "kv"]
    codes = [torch.zeros((pages, page, H, d), dtype=CODES, device="cuda") for _ in "kv"]
    scales = [torch.zeros((pages, H, page), dtype=torch.uint8, device="cuda") for _ in "kv"]
    back = [torch.zeros_like(x) for x in full]
    qkv = torch.randn((400, H * G + 2 * H, d), device="cuda", generator=g).bfloat16()
    rows = qkv[:, :H * G].contiguous(), qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
    length, total, off, off1 = i32([300]), i32([700]), i32([0, 400]), i32([0, 1])
    q_out, out, one = torch.zeros_like(rows[0]), torch.zeros_like(rows[0]), torch.zeros_like(rows[0][:1])
    kw = dict(page_table=table, page_size=page)

    def steps():
        dec.quantise(length, [full[0]], [full[1]], [codes[0]], [codes[1]], [scales[0]], [scales[1]], dst_page_table=table, **kw)
        dec.append_quantised(*rows, off, total, *codes, *scales, q_out, **kw)
        dec.attend_quantised(q_out, off, total, *codes, *scales, out, **kw)
        dec.attend_quantised(q_out[-1:], off1, total, *codes, *scales, one, **kw)
        dec.dequantise(total, [codes[0]], [codes[1]], [scales[0]], [scales[1]], [back[0]], [back[1]], dst_page_table=table, **kw)

    steps()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps()
    for n in (300, 111, 600):
        length.fill_(n)
        total.fill_(n + 400)
        steps()
        want = [x.clone() for x in (q_out, out, one, *back)]
        for x in (q_out, out, one, *back, *codes, *scales):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        s = torch.arange(n + 400, device="cuda")
        p, o = table[0].long()[s // page], s % page
        assert all(torch.equal(a, b) for a, b in zip((q_out, out, one), want[:3]))
        assert all(torch.equal(a[p, o], b[p, o]) for a, b in zip(back, want[3:]))
        assert torch.allclose(one.float(), out[-1:].float(), rtol=2.0 ** -6, atol=2.0 ** -6 * float(out.float().abs().max()))
    assert dec.device_status() == 0


def test_example_goes_on_in_8_bits():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "continue_in_8_bits.py")
    spec = importlib.util.spec_from_file_location("continue_in_8_bits", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    outs, length, share = m.main(context=300, question=20, answer=3, layers=2)
    assert len(outs) == 4 and all(bool(torch.isfinite(x).all()) for x in outs) and int(length) == 323
    assert share == (128 + 1) / 256
