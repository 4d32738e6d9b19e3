"""The calls that go on from a cache (kvx_append, kvx_attend, kvx_evict) against their definitions in
64 bits, on the CPU.

Tolerances, set from the arithmetic before any run.  u = 2^-24 is fp32's unit roundoff.
- A score is a sum of d products of exact inputs: within 6 sqrt(d) u times the sum of the products'
  magnitudes (independent roundings, six standard deviations), after the scale; the scaling to log2
  units, the cap and the exponential's argument add a few u of the score.  Call the bound e.
- An attention weight exp(x - lse) is then within a factor 1 + 2e + 2^-20 (its own score, the row's
  sum, the hardware exponential's 2 ulp and the sum's roundings).
- out: sum of the weights' errors times |v|, with weights rounded to bf16 (2^-9) for bf16 caches, and the
  final rounding to the output's type.  lse: e + 2^-20 + 2^-22 |lse|.
- key_weight: the weights' relative bound plus 2^-20 for the sum.
- append: the rotation's sine and cosine are within 1e-6, the result is rounded to its type.
What is copied, and slots, lengths and kept weights, are exact."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Problem:
    """Random new tokens over a random cache; slots past a sequence's length hold NaN."""

    def __init__(self, H, G, d, ctx, new, dtype="bf16", page_size=0, seed=0, cap=0.0, scale=0.0, q_gain=2.0, kv_len=None, layout="bhsd",
                 capacity=None):
        g = torch.Generator().manual_seed(seed)
        self.H, self.G, self.d, self.new, self.page_size = H, G, d, list(new), page_size
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.L = list(kv_len) if kv_len is not None else [c + n for c, n in zip(ctx, new)]
        self.B, self.T, self.S = len(new), sum(new), capacity or max(max(self.L), 1)
        self.cap, self.scale = cap, scale or 1.0 / math.sqrt(d)
        self.off = np.concatenate([[0], np.cumsum(new)])

        def rnd(*shape, gain=1.0):
            return (torch.randn(shape, generator=g) * gain).to(self.tdt)

        self.q = rnd(self.T, H * G, d, gain=q_gain)
        self.K, self.V = rnd(self.B, H, self.S, d), rnd(self.B, H, self.S, d)
        for b, n in enumerate(self.L):
            self.K[b, :, max(n, 0):] = float("nan")
            self.V[b, :, max(n, 0):] = float("nan")
        self.table = None
        if page_size:
            per = -(-self.S // page_size)
            perm = torch.randperm(self.B * per + 3, generator=g)[:self.B * per].view(self.B, per)
            self.num_pages, self.table = self.B * per + 3, perm.int().cuda()
            self.perm = perm
        self.layout = layout
        self.geom = synth.ModelGeom(1, H, d, 1e4)
        self.dec = kvx.Decoder(self.geom, H * G, dtype=kvx.KVX_BF16 if dtype == "bf16" else kvx.KVX_FP32, score_cap=cap, scale=scale)

    def cache(self, x):
        """x [B, H, S, d] as the device cache of this problem's layout."""
        B, H, S, d = x.shape
        if not self.page_size:
            if self.layout == "bshd":       # slots before heads in memory, a strided view
                return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
            return x.cuda()
        ps = self.page_size
        pool = torch.full((self.num_pages, ps, H, d), float("nan"), dtype=x.dtype)
        pad = torch.full((B, H, self.perm.shape[1] * ps, d), float("nan"), dtype=x.dtype)
        pad[:, :, :S] = x
        pool[self.perm.reshape(-1)] = pad.view(B, H, -1, ps, d).permute(0, 2, 3, 1, 4).reshape(-1, ps, H, d)
        return pool.cuda()

    def uncache(self, t, S=None):
        """The device cache as [B, H, S, d]."""
        if not self.page_size:
            return t.cpu()
        p = t.cpu()[self.perm.reshape(-1)].view(self.B, -1, self.page_size, self.H, self.d)
        return p.permute(0, 3, 1, 2, 4).reshape(self.B, self.H, -1, self.d)[:, :, :self.S]

    def paged(self):
        return {"page_table": self.table, "page_size": self.page_size} if self.page_size else {}

    def attend(self, window=0, prefix=None, weight=None, q=None, k=None, v=None, lse=True, out=None, stream=None):
        dev = (self.q if q is None else q).cuda()
        out = torch.full((self.T, self.H * self.G, self.d), 7.0, dtype=self.tdt, device="cuda") if out is None else out
        lse = torch.full((self.T, self.H * self.G), 7.0, device="cuda") if lse else None
        self.dec.attend(dev, i32(self.off), i32(self.L), self.cache(self.K if k is None else k), self.cache(self.V if v is None else v), out,
                        window=window, prefix_len=None if prefix is None else i32(prefix), lse=lse, key_weight=weight, stream=stream,
                        **self.paged())
        torch.cuda.synchronize()
        return out.cpu(), None if lse is None else lse.cpu()

    def exact(self, window=0, prefix=None, K=None, V=None, bad_page=None):
        """out, lse, key weights in 64 bits and the bounds of out, lse and key weights."""
        H, G, d = self.H, self.G, self.d
        K, V = (self.K if K is None else K).double(), (self.V if V is None else V).double()
        out, tol = torch.zeros(self.T, H * G, d, dtype=torch.float64), torch.zeros(self.T, H * G, d, dtype=torch.float64)
        lse, ltol = torch.full((self.T, H * G), -math.inf, dtype=torch.float64), torch.zeros(self.T, H * G, dtype=torch.float64)
        w, wtol = torch.zeros(self.B, H, self.S, dtype=torch.float64), torch.zeros(self.B, H, self.S, dtype=torch.float64)
        for b in range(self.B):
            n, L = self.new[b], min(max(self.L[b], 0), self.S)
            pre = 0 if prefix is None else min(prefix[b], L)
            for t in range(n):
                i = L - n + t
                j = torch.arange(L)
                seen = (j <= i) & ((j > i - window) if window else True) | (j < pre)
                j = j[seen]
                if not len(j):
                    continue
                row = int(self.off[b]) + t
                q = self.q[row].double().view(H, G, d)
                k, v = K[b][:, j], V[b][:, j]
                x = torch.einsum("hgd,hjd->hgj", q, k) * self.scale
                mag = torch.einsum("hgd,hjd->hgj", q.abs(), k.abs()) * self.scale
                if self.cap:
                    x = self.cap * torch.tanh(x / self.cap)
                z = torch.logsumexp(x, -1, keepdim=True)
                e = (6 * math.sqrt(d) * U * mag + 16 * U * x.abs() + (8 * U * self.cap)).amax(-1, keepdim=True)
                p = torch.exp(x - z)
                o = torch.einsum("hgj,hjd->hgd", p, v).reshape(H * G, d)
                ov = torch.einsum("hgj,hjd->hgd", p, v.abs()).reshape(H * G, d)
                bf = self.tdt == torch.bfloat16
                rel = (2 * e + 2.0 ** -20).reshape(H * G, 1) + (2.0 ** -9 if bf else 0.0) + 6 * math.sqrt(len(j)) * U
                out[row], tol[row] = o, 1.05 * rel * ov + (2.0 ** -8 if bf else 2.0 ** -23) * o.abs() + 1e-30
                lse[row], ltol[row] = z.reshape(-1), (e + 2.0 ** -20 + 2.0 ** -22 * z.abs()).reshape(-1)
                w[b][:, j] += p.sum(1)
                wtol[b][:, j] += (p * (2 * e + 2.0 ** -19)).sum(1)
        return out, lse, w, tol, ltol, wtol


def check(p, got, want, tol, what):
    err = (got.double() - want).abs()
    over = err > tol
    assert not bool(over.any()) and bool(torch.isfinite(got).all()), \
        f"{what}: {int(over.sum())} of {over.numel()} beyond the bound, worst {float((err / tol.clamp(min=1e-30)).max()):.3g} times it"


def check_lse(got, want, tol):
    none = want == -math.inf
    assert torch.equal(got == -math.inf, none)
    check(None, got[~none], want[~none], tol[~none], "lse")


# H, G, d, ctx, new, page_size, options
CASES = {
    "one_token_one_slot": (2, 6, 128, [0], [1], 0, {}),
    "one_token_d128": (2, 6, 128, [1000], [1], 16, {}),
    "one_token_d64": (1, 4, 64, [333], [1], 16, {}),
    "one_token_d256": (4, 2, 256, [517], [1], 16, {}),
    "decode_ragged_g7": (4, 7, 128, [700, 0, 63, 64, 65, 2000], [1, 1, 1, 1, 1, 1], 16, {}),
    "decode_empty_sequence": (2, 6, 128, [100, 50, 0, 9], [1, 0, 0, 1], 16, {}),
    "decode_g1": (3, 1, 128, [129, 31], [1, 1], 0, {}),
    "decode_g64": (1, 64, 64, [257], [1], 16, {}),
    "decode_g17": (2, 17, 128, [190], [1], 16, {}),
    "decode_long": (1, 2, 64, [20000], [1], 16, {}),
    "few_tokens": (2, 6, 128, [300, 40], [3, 2], 16, {}),
    "chunk_g7": (4, 7, 128, [300, 17], [65, 130], 16, {}),
    "chunk_from_nothing": (2, 6, 128, [0, 0], [257, 40], 0, {}),
    "chunk_d64": (1, 4, 64, [100, 0, 33], [130, 77, 1], 16, {}),
    "chunk_d256": (2, 2, 256, [200, 9], [140, 64], 16, {}),
    "chunk_odd_pages": (2, 4, 128, [150, 20], [70, 33], 7, {}),
    "chunk_page_1": (1, 4, 128, [50], [40], 1, {}),
    "chunk_page_64": (2, 4, 128, [450, 1], [70, 200], 64, {}),
    "chunk_page_256": (2, 4, 64, [450], [70], 256, {}),
    "chunk_window": (2, 4, 128, [600, 3], [150, 40], 16, {"window": 100}),
    "window_1": (2, 4, 128, [60], [70], 16, {"window": 1}),
    "decode_window": (2, 6, 128, [900, 30], [1, 1], 16, {"window": 65}),
    "prefix_beyond_own": (2, 4, 128, [20, 200], [100, 60], 16, {"prefix": [64, 7]}),
    "prefix_and_window": (1, 4, 128, [700, 40], [80, 1], 16, {"prefix": [33, 41], "window": 90}),
    "prefix_longer_than_cache": (1, 4, 64, [5], [9], 0, {"prefix": [1000]}),
    "capped": (2, 2, 256, [300], [50], 16, {"cap": 50.0}),
    "capped_hard": (2, 4, 128, [300], [50], 16, {"cap": 2.0}),
    "capped_decode": (2, 4, 128, [300], [1], 16, {"cap": 2.0}),
    "long_chunk": (1, 4, 128, [1500], [600], 16, {}),
    "long_chunk_split": (1, 2, 128, [9000], [70], 16, {}),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_attend(name, dtype):
    H, G, d, ctx, new, ps, opt = CASES[name]
    p = Problem(H, G, d, ctx, new, dtype, ps, seed=sum(map(ord, name)), cap=opt.get("cap", 0.0))
    w = torch.full((p.B, H, p.S), 0.25, device="cuda")
    out, lse = p.attend(opt.get("window", 0), opt.get("prefix"), weight=w)
    eo, el, ew, to, tl, tw = p.exact(opt.get("window", 0), opt.get("prefix"))
    check(p, out, eo, to, "out")
    check_lse(lse, el, tl)
    check(p, w.cpu(), ew + 0.25, tw + 2.0 ** -23 * (ew + 0.25), "key_weight")
    again, _ = p.attend(opt.get("window", 0), opt.get("prefix"), lse=False)
    assert torch.equal(again, out), "equal calls give equal bits"
    assert p.dec.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [[5, 1], [200, 3]])
def test_rows_that_see_nothing_are_zero(dtype, new):
    """kv_len below the call's own tokens: the first of them have slots below zero."""
    p = Problem(2, 4, 128, [0, 0], new, dtype, 16, seed=3, kv_len=[new[0] - 4, 0])
    w = torch.zeros((2, 2, p.S), device="cuda")
    out, lse = p.attend(weight=w)
    eo, el, ew, to, tl, tw = p.exact()
    assert bool((el[:4] == -math.inf).all()) and bool((el[new[0]:] == -math.inf).all())
    check(p, out, eo, to, "out")
    check_lse(lse, el, tl)
    check(p, w.cpu(), ew, tw + 1e-30, "key_weight")
    assert not out[:4].any() and not out[new[0]:].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new,bad", [(90, float("nan")), (90, float("inf")), (4, float("nan")), (1, float("inf"))])
def test_hidden_slots_never_reach_a_row(dtype, new, bad):
    """Not finite K and V rows in slots some rows do not see leave those rows as they were."""
    p = Problem(2, 4, 128, [200], [new], dtype, 16, seed=5)
    window = 150
    K, V = p.K.clone(), p.V.clone()
    at = [3, 200 + new // 2] if new > 1 else [3]     # before every window; a token in the middle of the chunk
    for j in at:
        K[:, :, j], V[:, :, j] = bad, bad
    out, lse = p.attend(window, k=K, v=V)
    eo, el, _, to, tl, _ = p.exact(window)
    sees = 200 + torch.arange(new) >= at[-1] if new > 1 else torch.zeros(1, dtype=torch.bool)
    check(p, out[~sees], eo[~sees], to[~sees], "out")
    check_lse(lse[~sees], el[~sees], tl[~sees])
    if new > 1:
        assert bool(torch.isnan(out[sees]).any())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strided_queries_outputs_and_caches(dtype):
    p = Problem(2, 6, 128, [130, 40], [33, 90], dtype, 0, seed=7, layout="bshd")
    eo, el, _, to, tl, _ = p.exact()
    fused = torch.full((p.T, 2 * 6 + 4, 128), float("nan"), dtype=p.tdt, device="cuda")
    fused[:, 2:14] = p.q.cuda()
    wide = torch.full((p.T, 12, 256), 3.0, dtype=p.tdt, device="cuda")
    lse = torch.zeros((p.T, 12), device="cuda")
    p.dec.attend(fused[:, 2:14], i32(p.off), i32(p.L), p.cache(p.K), p.cache(p.V), wide[:, :, 128:], lse=lse)
    torch.cuda.synchronize()
    check(p, wide[:, :, 128:].cpu(), eo, to, "out")
    assert bool((wide[:, :, :128] == 3.0).all())
    check_lse(lse.cpu(), el, tl)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_own_scale_and_large_scores(dtype):
    """A scale of its own, and scores of hundreds: the running maximum carries them."""
    p = Problem(1, 4, 64, [500], [40], dtype, 16, seed=9, scale=1.5, q_gain=8.0)
    out, lse = p.attend()
    eo, el, _, to, tl, _ = p.exact()
    check(p, out, eo, to, "out")
    check_lse(lse, el, tl)


@pytest.mark.parametrize("new", [1, 140])
def test_another_stream(new):
    p = Problem(2, 6, 128, [700], [new], "bf16", 16, seed=11)
    base, _ = p.attend()
    s = torch.cuda.Stream()
    q, k, v = p.q.cuda(), p.cache(p.K), p.cache(p.V)
    off, L, out = i32(p.off), i32(p.L), torch.zeros_like(base, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        p.dec.attend(q, off, L, k, v, out, **p.paged())
    s.synchronize()
    assert torch.equal(out.cpu(), base)


def test_in_a_graph():
    p = Problem(2, 6, 128, [700, 30], [1, 3], "bf16", 16, seed=12)
    w = torch.zeros((2, 2, p.S), device="cuda")
    base, _ = p.attend(weight=w)
    q, k, v = p.q.cuda(), p.cache(p.K), p.cache(p.V)
    off, L, out = i32(p.off), i32(p.L), torch.zeros_like(base, device="cuda")
    w2, lse = torch.zeros_like(w), torch.zeros((p.T, 12), device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.dec.attend(q, off, L, k, v, out, lse=lse, key_weight=w2, **p.paged())
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), base)
    assert torch.allclose(w2, 3 * w, rtol=1e-6, atol=0)


def test_lengths_past_the_cache_and_bad_pages_are_flagged():
    p = Problem(2, 4, 128, [60], [3], "bf16", 16, seed=13)
    q, k, v = p.q.cuda(), p.cache(p.K), p.cache(p.V)
    out = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda")
    table = p.table.clone()
    table[0, 1] = -1
    p.dec.attend(q, i32(p.off), i32(p.L), k, v, out, page_table=table)
    assert p.dec.device_status() == kvx.KVX_DEV_PAGE_INVALID
    table[0, 1] = p.num_pages
    p.dec.attend(q, i32(p.off), i32(p.L), k, v, out, page_table=table)
    assert p.dec.device_status() == kvx.KVX_DEV_PAGE_INVALID
    p.dec.attend(q, i32(p.off), i32([1000]), k, v, out, page_table=p.table)
    assert p.dec.device_status() & kvx.KVX_DEV_SEQ_CLAMPED
    p.dec.append(q, q[:, :2], q[:, :2], i32(p.off), i32([1000]), k, v, torch.empty_like(q), page_table=p.table)
    assert p.dec.device_status() == kvx.KVX_DEV_SEQ_CLAMPED
    p.dec.append(q, q[:, :2], q[:, :2], i32(p.off), i32([30]), k, v, torch.empty_like(q), page_table=table)
    assert p.dec.device_status() == kvx.KVX_DEV_PAGE_INVALID


# ------------------------------------------------------------------ append
GEOMS = {
    "plain": dict(),
    "none": dict(rope_base=0.0),
    "linear": dict(rope_type=1, rope_factor=4.0),
    "llama3": dict(rope_base=5e5, rope_type=2, rope_factor=8.0, rope_original_max_position=512),
    "partial": dict(rotary_dim=32),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("geom", sorted(GEOMS))
@pytest.mark.parametrize("d,G,ctx,new,ps", [(128, 6, [100, 3, 0], [1, 40, 0], 16), (64, 4, [5], [1], 0), (256, 2, [9, 800], [33, 2], 7)])
def test_append(dtype, geom, d, G, ctx, new, ps):
    H = 2
    p = Problem(H, G, d, ctx, new, dtype, ps, seed=21)
    kw = dict(GEOMS[geom])
    g = synth.ModelGeom(1, H, d, kw.pop("rope_base", 1e4), **kw)
    dec = kvx.Decoder(g, H * G, dtype=kvx.KVX_BF16 if dtype == "bf16" else kvx.KVX_FP32)
    gen = torch.Generator().manual_seed(4)
    qkv = torch.randn((p.T, H * G + 2 * H, d), generator=gen).to(p.tdt)
    dev = qkv.cuda()
    pos = torch.randint(0, 100000, (p.T,), generator=gen) if geom != "llama3" else None
    k, v = p.cache(p.K), p.cache(p.V)
    q_out = torch.full((p.T, H * G, d), 5.0, dtype=p.tdt, device="cuda")
    args = (i32(p.off), i32(p.L), k, v)
    kwargs = dict(pos=None if pos is None else i32(pos), **p.paged())
    dec.append(dev[:, :H * G], dev[:, H * G:H * G + H], dev[:, H * G + H:], *args, q_out, **kwargs)
    assert dec.device_status() == 0
    # the definition: pairs (i, i + n/2) of the first n channels turned by pos * f_i
    n = g.rotary_dim or d
    i = np.arange(n // 2)
    f = g.rope_base ** (-2.0 * i / n) if g.rope_base > 0 else np.zeros(n // 2)
    if g.rope_type == 1:
        f = f / g.rope_factor
    if g.rope_type == 2:
        wl, orig = 2 * np.pi / f, g.rope_original_max_position
        m = (orig / wl - g.rope_low_freq_factor) / (g.rope_high_freq_factor - g.rope_low_freq_factor)
        f = np.where(wl < orig / g.rope_high_freq_factor, f, np.where(wl > orig / g.rope_low_freq_factor, f / g.rope_factor,
                                                                      (1 - m) * f / g.rope_factor + m * f))
    at = np.concatenate([np.arange(L - x, L) for L, x in zip(p.L, p.new)]) if pos is None else pos.numpy()
    turn = torch.from_numpy(np.exp(1j * at[:, None] * f[None]))[:, None]

    def rot(x):
        z = torch.complex(x[..., :n // 2].double(), x[..., n // 2:n].double()) * turn
        return torch.cat([z.real, z.imag, x[..., n:].double()], -1)

    eps = 2.0 ** -9 if dtype == "bf16" else U
    for got, want in ((q_out.cpu(), rot(qkv[:, :H * G])),):
        check(p, got, want, 2 * eps * want.abs() + 4e-6 * qkv[:, :H * G].double().abs().amax(-1, keepdim=True), "q")
    K, V = p.K.clone(), p.V.clone()
    newk, newv = rot(qkv[:, H * G:H * G + H]), qkv[:, H * G + H:]
    gk, gv = p.uncache(k), p.uncache(v)
    for b in range(p.B):
        s, t0 = slice(p.L[b] - p.new[b], p.L[b]), int(p.off[b])
        want = newk[t0:t0 + p.new[b]].transpose(0, 1)
        if p.new[b]:
            check(p, gk[b, :, s], want, 2 * eps * want.abs() + 2e-5, "k")
        V[b, :, s] = newv[t0:t0 + p.new[b]].transpose(0, 1)
        K[b, :, s] = gk[b, :, s]
    assert torch.equal(gv.nan_to_num(9.0), V.nan_to_num(9.0)) and torch.equal(gk.nan_to_num(9.0), K.nan_to_num(9.0))
    # in place
    q2 = dev[:, :H * G]
    dec.append(q2, dev[:, H * G:H * G + H], dev[:, H * G + H:], *args, q2, **kwargs)
    assert torch.equal(q2.cpu(), q_out.cpu())


def test_positions_out_of_range_are_flagged():
    p = Problem(1, 2, 64, [4], [2], "bf16", 0, seed=2)
    q = p.q.cuda()
    p.dec.append(q, q[:, :1], q[:, :1], i32(p.off), i32(p.L), p.cache(p.K), p.cache(p.V), torch.empty_like(q), pos=i32([0, 1 << 25]))
    assert p.dec.device_status() == kvx.KVX_DEV_POS_CLAMPED


# ------------------------------------------------------------------ evict
def evict_definition(w, n, keep, sinks, recent):
    if n <= keep:
        return np.arange(n)
    mid = np.arange(sinks, n - recent)
    nan = np.isnan(w[mid])      # NaN ranks below everything, -infinity included
    ranked = mid[np.lexsort((mid, -np.where(nan, 0.0, w[mid]).astype(np.float64), nan))]
    return np.sort(np.concatenate([np.arange(sinks), ranked[:keep - sinks - recent], np.arange(n - recent, n)]))


EVICT = {
    "small": (2, 1, 64, [1000], 256, 4, 32, 0, "pow"),
    "paged": (3, 2, 128, [700, 100, 256, 0, 257], 256, 16, 64, 16, "pow"),
    "odd_pages": (1, 2, 128, [333, 90], 77, 1, 5, 7, "pow"),
    "wide": (1, 2, 256, [300], 100, 0, 0, 16, "pow"),
    "ties": (2, 2, 64, [2500], 1000, 0, 7, 16, "ties"),
    "all_equal": (1, 2, 64, [2500], 1001, 3, 8, 0, "zero"),
    "all_forced": (1, 1, 64, [500], 64, 30, 34, 0, "pow"),
    "keep_one": (1, 1, 64, [500], 1, 0, 0, 0, "pow"),
    "signs_and_nan": (1, 2, 128, [3000], 1500, 0, 0, 16, "odd"),
    "long": (1, 1, 64, [70000], 30011, 4, 100, 16, "pow"),
}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", sorted(EVICT))
def test_evict(name, dtype):
    L, H, d, lens, keep, sinks, recent, ps, kind = EVICT[name]
    rng = np.random.default_rng(len(name))
    S = max(lens) + 9
    p = Problem(H, 1, d, lens, [0] * len(lens), dtype, ps, seed=31, capacity=S)
    kept_lens = [min(n, keep) for n in lens]
    r = Problem(H, 1, d, kept_lens, [0] * len(lens), dtype, ps, seed=32, capacity=keep)
    w = rng.random((L, p.B, H, S), dtype=np.float32) ** 6
    if kind == "ties":
        w = np.round(w * 8) / 8
    elif kind == "zero":
        w[:] = 0.0
    elif kind == "odd":
        w = rng.standard_normal(w.shape).astype(np.float32)
        w[rng.random(w.shape) < 0.2] = np.nan
        w[rng.random(w.shape) < 0.1] = np.inf
        w[rng.random(w.shape) < 0.1] = -np.inf
        w[rng.random(w.shape) < 0.1] = 0.0
        w[rng.random(w.shape) < 0.1] = -0.0
        w[rng.random(w.shape) < 0.1] = 1e-40
    w = w.astype(np.float32)
    dec = kvx.Decoder(synth.ModelGeom(L, H, d, 1e4), H, dtype=p.dec.desc.dtype)
    ks, vs = [], []
    for l in range(L):
        g = torch.Generator().manual_seed(100 + l)
        ks.append(torch.randn(p.K.shape, generator=g).to(p.tdt))
        vs.append(torch.randn(p.K.shape, generator=g).to(p.tdt))
    empty = torch.full(r.K.shape, 9.0, dtype=p.tdt)
    dk, dv = [r.cache(empty) for _ in range(L)], [r.cache(empty) for _ in range(L)]
    kept = torch.full((L, p.B, H, keep), -7, dtype=torch.int32, device="cuda")
    new_len = torch.full((p.B,), -7, dtype=torch.int32, device="cuda")
    kw = torch.full((L, p.B, H, keep + 5), -7.0, device="cuda")
    opt = dict(p.paged(), dst_page_table=r.table) if ps else {}
    dec.evict(i32(lens), torch.from_numpy(w).cuda(), keep, [p.cache(x) for x in ks], [p.cache(x) for x in vs], dk, dv, kept, new_len, sinks=sinks,
              recent=recent, kept_weight=kw, **opt)
    assert dec.device_status() == 0
    assert new_len.tolist() == kept_lens
    kept, kw = kept.cpu().numpy(), kw.cpu().numpy()
    for l in range(L):
        gk, gv = r.uncache(dk[l]), r.uncache(dv[l])
        for b in range(p.B):
            for h in range(H):
                want = evict_definition(w[l, b, h], lens[b], keep, sinks, recent)
                m = len(want)
                assert np.array_equal(kept[l, b, h, :m], want) and (kept[l, b, h, m:] == -1).all()
                assert np.array_equal(kw[l, b, h, :m], w[l, b, h][want], equal_nan=True) and not kw[l, b, h, m:].any()
                assert torch.equal(gk[b, h, :m], ks[l][b, h][want]) and torch.equal(gv[b, h, :m], vs[l][b, h][want])
                assert bool((gk[b, h, m:] == 9.0).all()) and bool((gv[b, h, m:] == 9.0).all())


# ------------------------------------------------------------------ refusals
def test_refusals():
    p = Problem(2, 4, 128, [60], [3], "bf16", 16, seed=13)
    q, k, v = p.q.cuda(), p.cache(p.K), p.cache(p.V)
    out = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda")
    off, L = i32(p.off), i32(p.L)
    ok = dict(page_table=p.table)

    def refused(code, f, *a, **kw):
        with pytest.raises(kvx.KvxError) as e:
            f(*a, **kw)
        assert e.value.status == code and kvx.kvx_last_error()

    bad = kvx.KVX_ERR_INVALID_ARG
    refused(bad, p.dec.attend, q, off, L, k, v, out, window=-1, **ok)
    refused(bad, p.dec.attend, q, off, L, k, v, out, key_weight=torch.zeros((1, 2, 64), device="cuda"), **ok)
    refused(bad, p.dec.attend, q, off, L, k, v, out, page_table=p.table, page_size=0)
    many = torch.zeros(1026, dtype=torch.int32, device="cuda")
    refused(kvx.KVX_ERR_UNSUPPORTED, p.dec.attend, q, many, many, k, v, out, **ok)
    odd = torch.zeros(3 * 8 * 128 + 8, dtype=torch.bfloat16, device="cuda")[4:4 + 3 * 8 * 128].view(3, 8, 128)
    refused(bad, p.dec.attend, odd, off, L, k, v, out, **ok)
    narrow = torch.zeros((3, 8, 132), dtype=torch.bfloat16, device="cuda")[:, :, :128]
    refused(bad, p.dec.attend, narrow, off, L, k, v, out, **ok)
    with pytest.raises(ValueError):
        p.dec.attend(q[:, :4], off, L, k, v, out, **ok)
    with pytest.raises(ValueError):
        p.dec.attend(q.float(), off, L, k, v, out, **ok)
    with pytest.raises(ValueError):                      # lengths and offsets of another width, caches of another shape
        p.dec.attend(q, off.long(), L, k, v, out, **ok)
    with pytest.raises(ValueError):
        p.dec.attend(q, off, L, k[:, :8], v[:, :8], out, **ok)
    with pytest.raises(ValueError):
        p.dec.append(q, q[:, :2], q[:, :2], off, L, k.float(), v.float(), q, **ok)
    kept, n = torch.zeros((1, 1, 2, 8), dtype=torch.int32, device="cuda"), i32([0])
    w = torch.zeros((1, 1, 2, 64), device="cuda")
    args = ([k], [v], [k], [v], kept, n)
    refused(bad, p.dec.evict, L, w, 8, *args, sinks=5, recent=4, page_table=p.table, dst_page_table=p.table)
    refused(bad, p.dec.evict, L, w, 8, *args, sinks=-1, page_table=p.table, dst_page_table=p.table)
    with pytest.raises(ValueError):
        p.dec.evict(L, w, 9, *args, page_table=p.table, dst_page_table=p.table)
    lib, c = kvx.lib(), ctypes
    st = lib.kvx_attend(None, None, None, None, 0, None, None, None)
    assert st == bad
    assert p.dec.device_status() == 0


@pytest.mark.parametrize("ps", [8, 16, 24, 32, 48, 128, 200])
@pytest.mark.parametrize("H,G,d,ctx,new", [(2, 7, 128, [333, 90], [37, 1]), (1, 4, 64, [513], [130]), (2, 2, 256, [200, 40], [1, 66]),
                                           (3, 5, 128, [400, 0, 31], [1, 1, 1])])
def test_page_sizes(ps, H, G, d, ctx, new):
    """Every way rows are brought: groups of eight rows and single rows; the same values whichever."""
    p = Problem(H, G, d, ctx, new, "bf16", ps, seed=41)
    w = torch.zeros((p.B, H, p.S), device="cuda")
    out, lse = p.attend(weight=w)
    eo, el, ew, to, tl, tw = p.exact()
    check(p, out, eo, to, "out")
    check_lse(lse, el, tl)
    check(p, w.cpu(), ew, tw + 1e-30, "key_weight")
    flat = Problem(H, G, d, ctx, new, "bf16", 0, seed=41)
    base, _ = flat.attend(q=p.q, k=p.K, v=p.V)
    assert torch.equal(base, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_sequences(dtype):
    """Sequences of all lengths, most without new tokens: ranges begin and end anywhere."""
    rng = np.random.default_rng(9)
    new = [int(x) for x in rng.choice([0, 0, 1, 1, 2, 9], 200)]
    ctx = [int(x) for x in rng.integers(0, 90, 200)]
    p = Problem(2, 3, 64, ctx, new, dtype, 16, seed=43)
    w = torch.zeros((p.B, 2, p.S), device="cuda")
    out, lse = p.attend(weight=w)
    eo, el, ew, to, tl, tw = p.exact()
    check(p, out, eo, to, "out")
    check_lse(lse, el, tl)
    check(p, w.cpu(), ew, tw + 1e-30, "key_weight")


def test_weights_where_scores_do_not_fit_the_workspace():
    """The same sums from kept scores (few rows, or fp32) and from scores formed again."""
    for dtype, new in (("bf16", 1), ("fp32", 20)):
        p = Problem(1, 8, 64, [700], [new], dtype, 16, seed=44)
        narrow, wide = torch.zeros((1, 1, p.S), device="cuda"), torch.zeros((1, 1, 16 << 20), device="cuda")
        p.attend(weight=narrow)
        p.attend(weight=wide)
        _, _, ew, _, _, tw = p.exact()
        for w in (narrow, wide[:, :, :p.S].contiguous()):
            check(p, w.cpu(), ew, tw + 1e-30, "key_weight")
        assert not wide[:, :, p.S:].any()


# ------------------------------------------------------------------ the steps together
def test_example_goes_on_from_a_handoff():
    """The example's steps: slots kept hold the sinks and the question, weights add up to one a row."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "continue_from_handoff.py")
    spec = importlib.util.spec_from_file_location("continue_from_handoff", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    out, o1, kept, kept_weight, left = m.main(context=300, keep=100, question=20, answer=3, layers=2)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(o1).all()) and int(left) == 103
    kept = kept.cpu()
    assert torch.equal(kept[..., :4], torch.arange(4, dtype=torch.int32).expand(2, 1, 2, 4))
    assert torch.equal(kept[..., -20:], torch.arange(300, 320, dtype=torch.int32).expand(2, 1, 2, 20))
    assert bool((kept[..., 1:] > kept[..., :-1]).all())
    # three decoded tokens, 12 query heads: their weights add 36 a layer to what the kept slots had
    assert bool((kept_weight >= 0).all())
