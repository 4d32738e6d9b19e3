"""Queries that hold an infinity, over caches held in 8 bits: scores are infinite, or at the cap where they are capped, on every path.
Definitions and bounds: test_gpu_quantised.py."""
import math

import pytest
import torch

from test_gpu_quantised import Problem, U, check, check_lse, value

pytestmark = pytest.mark.gpu


# whole rows of one CTA, rows split over many, several sequences
SIZES = [(128, 4, [30], [1]), (128, 4, [5000], [1]), (128, 8, [900, 40], [4, 2]), (256, 2, [700, 3], [3, 1]), (256, 5, [6000], [1]), (128, 16, [2500], [2]),
         (64, 4, [3000], [1]), (64, 4, [200, 30], [90, 3]), (128, 4, [200], [90]), (128, 4, [200], [400]), (256, 2, [300], [300])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("d,G,ctx,new", SIZES)
@pytest.mark.parametrize("kind", ["mixed", "below", "two"])
def test_infinite_queries(d, G, ctx, new, cap, dtype, kind):
    """Every token's first head has an infinity in channel 5.  Keys there have either sign (a score of +inf among others: NaN without
    a cap), or all the one that makes every score -inf (without a cap nothing is left); "two": another infinity against it, no score is a number."""
    p = Problem(2, G, d, ctx, new, dtype, 16, seed=d + G + sum(ctx), cap=cap)
    p.q[:, 0, 5] = -math.inf
    p.code[0][..., 5] = (0x3b if kind == "below" else 0x3b | (torch.randint(0, 2, p.code[0].shape[:-1], generator=torch.Generator().manual_seed(1)) << 7).to(torch.uint8))
    p.byte[0].clamp_(max=160)
    if kind == "two":
        p.q[:, 0, 9] = math.inf
        p.code[0][..., 9] = p.code[0][..., 5]
    eo, el, to, tl = p.exact()                           # (of the other heads)
    K, V = (value(c, s).double() for c, s in zip(p.code, p.byte))
    for b, n in enumerate(new):
        L, r = p.L[b], slice(int(p.off[b]), int(p.off[b + 1]))
        x = p.q[r, 0].double() @ K[b, 0, :L].T
        assert bool(x.isnan().all()) if kind == "two" else bool((x.abs() == math.inf).all())
        if cap:
            x = cap * torch.tanh(x / cap)
        hidden = torch.arange(L) > torch.arange(L - n, L)[:, None]
        w = torch.exp(x.masked_fill(hidden, -math.inf) - (x.masked_fill(hidden, -math.inf).amax(1, keepdim=True).clamp(min=-1e300)))
        total, v = w.sum(1, keepdim=True), V[b, 0, :L]
        none = total == 0
        share = torch.where(none, torch.zeros_like(w), w / total)
        e = 24 * U * cap
        eo[r, 0] = share @ v
        to[r, 0] = 1.05 * (2 * e + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0) + 6 * math.sqrt(L) * U) * (share @ v.abs()) + 1.01 * eo[r, 0].abs() * (
            2.0 ** -8 if dtype == "bf16" else U) + 1e-30
        el[r, 0] = torch.logsumexp(x.masked_fill(hidden, -math.inf), 1)
        tl[r, 0] = e + 2.0 ** -20 + 2.0 ** -22 * el[r, 0].abs()
        if cap == 0 and kind == "below":
            assert bool(none.all())
    out, lse = p.attend()
    assert p.dec.device_status() == 0
    # (a score of +inf among others: a weight of inf - inf)
    bad = eo.isnan().any(-1) | el.isnan() | (el == math.inf)
    assert not bad[:, 1:].any() and (bool(bad[:, 0].all()) if kind == "two" else not bad[:, 0].any() if cap or kind == "below" else bool(bad[:, 0].any()))
    assert bool(out[bad].isnan().all()) and bool((lse[bad].isnan()).all())
    check(out[~bad], eo[~bad], to[~bad], "out")
    check_lse(lse[~bad], el[~bad], tl[~bad])


@pytest.mark.parametrize("d,G,ctx,new,page", [(128, 4, [6000], [2], 16), (256, 2, [3000, 40], [3, 2], 7), (128, 8, [700, 5, 0], [4, 2, 3], 0), (64, 4, [900], [60], 16)])
@pytest.mark.parametrize("window,prefix", [(500, None), (300, 900), (0, 70), (1, 0)])
def test_infinite_queries_masks(d, G, ctx, new, page, window, prefix):
    """Each slot that a mask leaves counts once, in whole rows and split ones; tokens that see nothing give zeros.  Capped."""
    cap, blind = 20.0, 1 if prefix is None else 0
    L = [c + n for c, n in zip(ctx, new)]
    L[-1] = max(0, new[-1] - 1) if blind and ctx[-1] == 0 else L[-1]
    p = Problem(2, G, d, ctx, new, "bf16", page, seed=d + window, cap=cap, kv_len=L)
    p.q[:, 1, 5] = math.inf
    p.code[0][..., 5] = 0x3b | (torch.randint(0, 2, p.code[0].shape[:-1], generator=torch.Generator().manual_seed(2)) << 7).to(torch.uint8)
    p.byte[0].clamp_(max=160)
    pre = None if prefix is None else [prefix] * len(new)
    eo, el, to, tl = p.exact(window, pre)
    K, V = (value(c, s).double() for c, s in zip(p.code, p.byte))
    for b, n in enumerate(new):
        r, i, j = slice(int(p.off[b]), int(p.off[b + 1])), torch.arange(L[b] - n, L[b])[:, None], torch.arange(L[b])
        seen = (j <= i) & ((i - j < window) if window else True)
        seen = seen | (j < prefix) if prefix is not None else seen
        x = (cap * torch.sign(p.q[r, 1, 5].double()[:, None] * K[b, 0, :L[b], 5])).masked_fill(~seen, -math.inf)
        w = torch.exp(x - cap)
        share, v, e = w / w.sum(1, keepdim=True).clamp(min=1e-300), V[b, 0, :L[b]], 24 * U * cap
        eo[r, 1] = share @ v
        to[r, 1] = 1.05 * (2 * e + 2.0 ** -20 + 2.0 ** -8 + 6 * math.sqrt(max(L[b], 1)) * U) * (share @ v.abs()) + 2.0 ** -8 * 1.01 * eo[r, 1].abs() + 1e-30
        el[r, 1] = torch.logsumexp(x, 1) if L[b] else -math.inf
        tl[r, 1] = e + 2.0 ** -20 + 2.0 ** -22 * el[r, 1].abs()
    out, lse = p.attend(window, pre)
    check(out, eo, to, "out")
    check_lse(lse, el, tl)
    assert p.dec.device_status() == 0
