"""Caches held in 8 bits (kvx_quantise, kvx_dequantise, kvx_append_quantised, kvx_attend_quantised) against their
definitions in 64 bits.

Tolerances, set from the arithmetic before any run.  u = 2^-24 is fp32's unit roundoff.
- quantise and dequantise are exact: scaling by a power of two and one rounding to nearest even.
- append: the rotation's sine and cosine are within 1e-6, so a rotated value is within r = 4e-6 times its head's largest
  magnitude; its code is the one of a value that near: within half a step (2^-4 of it, 2^-10 of the scale where codes are
  subnormal) plus r.  The scale is the smallest for a magnitude within r of the row's largest.
- attend: a cached value is exact, a score is a sum of d exact products: within 6 sqrt(d) u times the sum of their magnitudes
  (independent roundings, six standard deviations) and a few u of the score; the bound is e.  A weight is within a
  factor 1 + 2e + 2^-20 and, for bf16 queries, its rounding where it multiplies V: at most 2^-8 (one bf16 term).  out: the
  weights' errors times |v|, the sums' roundings and the output's own, 2^-8 or 2^-24.  lse: e + 2^-20 + 2^-22 |lse|."""
import math

import numpy as np
import pytest
import torch

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth

from test_gpu_decode import GEOMS, i32

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
CODES = torch.float8_e4m3fn
TYPES = {"bf16": (torch.bfloat16, kvx.KVX_BF16), "fp32": (torch.float32, kvx.KVX_FP32)}


def held(x):
    """Rows [..., d] (float64) as codes (uint8) and scale bytes, by the definition."""
    fine = x.isfinite()
    y = torch.where(fine, x.clamp(-1.875 * 2.0 ** 127, 1.875 * 2.0 ** 127), torch.full_like(x, math.nan))
    top = torch.where(fine, y.abs(), torch.zeros_like(y)).amax(-1)
    s = torch.full(top.shape, 10, dtype=torch.int64)
    for b in range(11, 248):         # the smallest that is large enough
        s = torch.where(top > 448.0 * 2.0 ** (b - 1 - 127), b, s)
    return (y * torch.exp2(127.0 - s.double())[..., None]).float().to(CODES).view(torch.uint8), s.to(torch.uint8)


def value(code, scale):
    """What codes and scale bytes stand for, in 32 bits."""
    return code.view(CODES).float() * (scale.int() << 23).view(torch.float32)[..., None]


class Place:
    """Where rows [B, H, S, ...] lie: contiguous (heads or slots first in memory), or pages in shuffled order."""

    def __init__(self, B, H, S, page, seed=0, layout="bhsd"):
        self.B, self.H, self.S, self.page, self.layout = B, H, S, page, layout
        if page:
            per = max(1, -(-S // page))
            self.pages = B * per + 3
            self.perm = torch.randperm(self.pages, generator=torch.Generator().manual_seed(seed))[:B * per].view(B, per)
            self.table = self.perm.int().cuda()

    def kw(self, name="page_table"):
        return {name: self.table, "page_size": self.page} if self.page else {}

    def put(self, x, fill, scales=False):
        """x [B, H, S, ...] on the device; places that no slot has hold `fill`."""
        if not self.page:
            return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) if self.layout == "bshd" and not scales else x.cuda()
        tail, ps = x.shape[3:], self.page
        pad = torch.full((self.B, self.H, self.perm.shape[1] * ps, *tail), fill, dtype=x.dtype)
        pad[:, :, :self.S] = x
        pool = torch.full((self.pages, ps, self.H, *tail), fill, dtype=x.dtype)
        pool[self.perm.reshape(-1)] = pad.view(self.B, self.H, -1, ps, *tail).transpose(1, 2).transpose(2, 3).reshape(-1, ps, self.H, *tail)
        return (pool.transpose(1, 2).contiguous() if scales else pool).cuda()

    def get(self, t, scales=False):
        t = t.cpu()
        if not self.page:
            return t
        t = t.transpose(1, 2) if scales else t
        x = t[self.perm.reshape(-1)].view(self.B, -1, self.page, self.H, *t.shape[3:])
        return x.transpose(2, 3).transpose(1, 2).reshape(self.B, self.H, -1, *t.shape[3:])[:, :, :self.S]


def special_rows(x):
    """Zeros, values that are not finite, the ends of the range and the borders between scales, in the first slots."""
    big = 3.38e38
    rows = [lambda r: r.zero_(), lambda r: r.mul_(0).add_(-0.0), lambda r: r.fill_(math.nan), lambda r: r.fill_(math.inf),
            lambda r: r[3:4].fill_(math.nan), lambda r: r[5:6].fill_(-math.inf), lambda r: r.fill_(big), lambda r: r.mul_(1e-37),
            lambda r: r.mul_(1e-39), lambda r: r.clamp_(-1, 1)[7:8].fill_(1.75), lambda r: r.clamp_(-1, 1)[7:8].fill_(1.7578125),
            lambda r: r.clamp_(-1, 1)[9:10].fill_(-1.75 * 2.0 ** 119), lambda r: r[2:3].fill_(big), lambda r: r.fill_(2.0 ** -9)]
    for s, f in enumerate(rows):
        if s < x.shape[2]:
            for b in range(x.shape[0]):
                for h in range(x.shape[1]):
                    f(x[b, h, s])
    return x


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("H,d,lens,page,dst_page,layout", [
    (2, 128, [40, 0, 1, 333], 16, 16, "bhsd"), (1, 64, [70, 20], 0, 0, "bhsd"), (3, 256, [33, 14], 7, 7, "bhsd"), (4, 128, [90, 5], 0, 0, "bshd"),
    (2, 64, [500], 64, 0, "bhsd"), (2, 256, [100, 31], 0, 24, "bhsd"), (5, 128, [17] * 9, 16, 16, "bhsd")])
def test_quantise_and_back(dtype, H, d, lens, page, dst_page, layout):
    tdt, kdt = TYPES[dtype]
    L, B, S = 2, len(lens), max(lens) + 3
    g = torch.Generator().manual_seed(d + H)
    src, dst = Place(B, H, S, page, 1, layout), Place(B, H, S, dst_page, 2)
    dec = kvx.Decoder(synth.ModelGeom(L, H, d, 1e4), H, dtype=kdt)
    full = [[special_rows((torch.randn(B, H, S, d, generator=g) * torch.exp(torch.randn(B, H, S, 1, generator=g))).to(tdt)) for _ in range(L)] for _ in "kv"]
    codes = [[dst.put(torch.full((B, H, S, d), 0x55, dtype=torch.uint8), 0x55) for _ in range(L)] for _ in "kv"]
    scales = [[dst.put(torch.full((B, H, S), 0x33, dtype=torch.uint8), 0x33, True) for _ in range(L)] for _ in "kv"]
    tables = {k: v for k, v in (("page_table", src.table if page else None), ("dst_page_table", dst.table if dst_page else None)) if v is not None}
    tables["page_size"] = page or dst_page or 16
    dec.quantise(i32(lens), *[[src.put(x, math.nan) for x in full[i]] for i in range(2)], *codes, *scales, **tables)
    assert dec.device_status() == 0 and dec.launches() == 1
    n = torch.tensor(lens)[:, None]
    live = (torch.arange(S) < n)[:, None].expand(B, H, S)
    for i in range(2):
        for l in range(L):
            c, s = held(full[i][l].double())
            gc, gs = dst.get(codes[i][l]), dst.get(scales[i][l], True)
            assert torch.equal(gs[live], s[live]) and bool((gs[~live] == 0x33).all())
            nan = (c & 0x7f) == 0x7f
            assert torch.equal((gc & 0x7f)[live] == 0x7f, nan[live])
            assert torch.equal(gc.masked_fill(nan, 0)[live], c.masked_fill(nan, 0)[live]) and bool((gc[~live] == 0x55).all())
    # and back, into a cache laid out as the source
    out = [[src.put(torch.full((B, H, S, d), 9.0, dtype=tdt), 9.0) for _ in range(L)] for _ in "kv"]
    back = {"page_size": tables["page_size"]}
    if dst_page:
        back["page_table"] = dst.table
    if page:
        back["dst_page_table"] = src.table
    dec.dequantise(i32(lens), *codes, *scales, *out, **back)
    assert dec.device_status() == 0
    for i in range(2):
        for l in range(L):
            got, want = src.get(out[i][l]), value(dst.get(codes[i][l]), dst.get(scales[i][l], True)).to(tdt)
            assert torch.equal(got.isnan()[live], want.isnan()[live]) and bool((got[~live] == 9.0).all())
            assert torch.equal(got[live].nan_to_num(nan=0.0), want[live].nan_to_num(nan=0.0))


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_as_many_layers_as_a_call_takes(dtype):
    tdt, kdt = TYPES[dtype]
    L, H, d, lens, S = kvx.KVX_MAX_TARGET_LAYERS, 1, 64, [19, 33], 40
    dec = kvx.Decoder(synth.ModelGeom(L, H, d, 1e4), H, dtype=kdt)
    full = [torch.randn((L, 2, H, S, d), generator=torch.Generator().manual_seed(i)).to(tdt).cuda() for i in range(2)]
    codes = [torch.zeros((L, 2, H, S, d), dtype=torch.uint8, device="cuda") for _ in "kv"]
    scales = [torch.zeros((L, 2, H, S), dtype=torch.uint8, device="cuda") for _ in "kv"]
    back = [torch.zeros_like(x) for x in full]
    dec.quantise(i32(lens), *map(list, full), *map(list, codes), *map(list, scales))
    dec.dequantise(i32(lens), *map(list, codes), *map(list, scales), *map(list, back))
    assert dec.device_status() == 0
    live = (torch.arange(S) < torch.tensor(lens)[:, None])[None, :, None].expand(L, 2, H, S)
    for x, c, s, b in zip(full, codes, scales, back):
        wc, ws = held(x.cpu().double())
        assert torch.equal(c.cpu()[live], wc[live]) and torch.equal(s.cpu()[live], ws[live]) and not c.cpu()[~live].any()
        assert torch.equal(b.cpu()[live], value(wc, ws).to(tdt)[live]) and not b.cpu()[~live].any()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_every_code_and_scale(dtype):
    """All 256 codes under scale bytes of every kind, those that are never written too: 0 stands for 0, 255 for infinity."""
    tdt, kdt = TYPES[dtype]
    dec = kvx.Decoder(synth.ModelGeom(1, 1, 256, 1e4), 1, dtype=kdt)
    c = torch.arange(256, dtype=torch.uint8).expand(1, 1, 256, 256).contiguous()
    s = torch.arange(256, dtype=torch.uint8).view(1, 1, 256)
    out = [torch.full((1, 1, 256, 256), 9.0, dtype=tdt, device="cuda") for _ in range(2)]
    dec.dequantise(i32([256]), [c.cuda()], [c.cuda()], [s.cuda()], [s.cuda()], [out[0]], [out[1]])
    want = value(c, s).to(tdt)
    for x in out:
        x = x.cpu()
        assert torch.equal(x.isnan(), want.isnan()) and torch.equal(x[~want.isnan()], want[~want.isnan()])


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("geom", sorted(GEOMS))
@pytest.mark.parametrize("d,H,G,ctx,new,page", [(128, 2, 6, [100, 3, 0], [1, 40, 0], 16), (64, 1, 4, [5], [1], 0), (256, 2, 2, [9, 800], [33, 2], 7),
                                                (64, 3, 1, [0, 0, 7], [1, 9, 50], 24)])
def test_append(dtype, geom, d, H, G, ctx, new, page):
    tdt, kdt = TYPES[dtype]
    kw = dict(GEOMS[geom])
    g = synth.ModelGeom(1, H, d, kw.pop("rope_base", 1e4), **kw)
    dec = kvx.Decoder(g, H * G, dtype=kdt)
    L, T, B = [c + n for c, n in zip(ctx, new)], sum(new), len(new)
    off, S = np.concatenate([[0], np.cumsum(new)]), max(L) + 2
    gen = torch.Generator().manual_seed(4)
    qkv = torch.randn((T, H * G + 2 * H, d), generator=gen).to(tdt)
    pos = torch.randint(0, 100000, (T,), generator=gen) if geom != "llama3" else None
    pl = Place(B, H, S, page, 5)
    codes = [pl.put(torch.full((B, H, S, d), 0x55, dtype=torch.uint8), 0x55) for _ in "kv"]
    scales = [pl.put(torch.full((B, H, S), 0x33, dtype=torch.uint8), 0x33, True) for _ in "kv"]
    dev = qkv.cuda()
    rows = dev[:, :H * G], dev[:, H * G:H * G + H], dev[:, H * G + H:]
    q_out = torch.full((T, H * G, d), 5.0, dtype=tdt, device="cuda")
    args = (i32(off), i32(L), codes[0].view(CODES), codes[1], scales[0].view(torch.float8_e8m0fnu), scales[1])
    kwargs = dict(pos=None if pos is None else i32(pos), **pl.kw())
    dec.append_quantised(*rows, *args, q_out, **kwargs)
    assert dec.device_status() == 0 and dec.launches() == 1
    # the definition of the rotation: pairs (i, i + n/2) of the first n channels turned by pos * f_i
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
    at = np.concatenate([np.arange(a - x, a) for a, x in zip(L, new)]) if pos is None else pos.numpy()
    turn = torch.from_numpy(np.exp(1j * at[:, None] * f[None]))[:, None]

    def rot(x):
        z = torch.complex(x[..., :n // 2].double(), x[..., n // 2:n].double()) * turn
        return torch.cat([z.real, z.imag, x[..., n:].double()], -1)

    eps = 2.0 ** -8 if dtype == "bf16" else U
    want = rot(qkv[:, :H * G])
    r = 4e-6 * qkv[:, :H * G].double().abs().amax(-1, keepdim=True)
    assert bool(((q_out.cpu().double() - want).abs() <= eps * want.abs() + 1.01 * r).all())
    fresh = torch.zeros((B, S), dtype=torch.bool)
    for b in range(B):
        fresh[b, L[b] - new[b]:L[b]] = True
    fresh = fresh[:, None].expand(B, H, S)
    for x, want, exact in ((0, rot(qkv[:, H * G:H * G + H]), False), (1, qkv[:, H * G + H:].double(), True)):
        gc, gs = pl.get(codes[x]), pl.get(scales[x], True)
        assert bool((gc[~fresh] == 0x55).all()) and bool((gs[~fresh] == 0x33).all())
        for b in range(B):
            if not new[b]:
                continue
            s = slice(L[b] - new[b], L[b])
            w = want[off[b]:off[b + 1]].transpose(0, 1)
            c, z = gc[b, :, s], gs[b, :, s]
            if exact:
                wc, wz = held(w)
                assert torch.equal(c, wc) and torch.equal(z, wz)
                continue
            top, scale = w.abs().amax(-1), torch.exp2(z.double() - 127)
            near = 1 + 8e-6
            assert bool((top <= 448 * scale * near).all()) and bool((top * near > 224 * scale).all())
            half = torch.maximum(2.0 ** -4 * w.abs(), 2.0 ** -10 * scale[..., None])
            assert bool(((value(c, z).double() - w).abs() <= half * (1 + 2.0 ** -4 * 1e-3) + 8e-6 * top[..., None]).all())
    # in place
    q2 = dev[:, :H * G]
    dec.append_quantised(q2, rows[1], rows[2], *args, q2, **kwargs)
    assert torch.equal(q2.cpu(), q_out.cpu())


class Problem:
    """New tokens over a cache of random codes; slots past a sequence's length hold NaN codes under infinite scales."""

    def __init__(self, H, G, d, ctx, new, dtype="bf16", page=16, seed=0, cap=0.0, scale=0.0, q_gain=2.0, kv_len=None, layout="bhsd", spread=0.5, gain=None):
        g = torch.Generator().manual_seed(seed)
        self.tdt, kdt = TYPES[dtype]
        self.H, self.G, self.d, self.new = H, G, d, list(new)
        self.L = list(kv_len) if kv_len is not None else [c + n for c, n in zip(ctx, new)]
        self.B, self.T, self.S = len(new), sum(new), max(max(self.L), 1)
        self.cap, self.scale = cap, scale or 1.0 / math.sqrt(d)
        self.off = np.concatenate([[0], np.cumsum(new)])
        self.q = (q_gain * torch.randn(self.T, H * G, d, generator=g)).to(self.tdt)
        rows = [torch.randn(self.B, H, self.S, d, generator=g) * torch.exp(spread * torch.randn(self.B, H, self.S, 1, generator=g)) for _ in "kv"]
        if gain is not None:
            rows[0] = rows[0] * gain(torch.arange(self.S).double() / max(1, self.S - 1)).float()[:, None]
        self.code, self.byte = map(list, zip(*(held(x.double()) for x in rows)))
        for b, n in enumerate(self.L):
            for i in range(2):
                self.code[i][b, :, max(n, 0):] = 0x7f
                self.byte[i][b, :, max(n, 0):] = 255
        self.place = Place(self.B, H, self.S, page, seed, layout)
        self.dec = kvx.Decoder(synth.ModelGeom(1, H, d, 1e4), H * G, dtype=kdt, score_cap=cap, scale=scale)

    def cache(self):
        return [*(self.place.put(c, 0x7f) for c in self.code), *(self.place.put(s, 255, True) for s in self.byte)]

    def attend(self, window=0, prefix=None, lse=True, **kw):
        out = torch.full((self.T, self.H * self.G, self.d), 7.0, dtype=self.tdt, device="cuda")
        lse = torch.full((self.T, self.H * self.G), 7.0, device="cuda") if lse else None
        self.dec.attend_quantised(self.q.cuda(), i32(self.off), i32(self.L), *self.cache(), out, window=window,
                                  prefix_len=None if prefix is None else i32(prefix), lse=lse, **self.place.kw(), **kw)
        torch.cuda.synchronize()
        return out.cpu(), None if lse is None else lse.cpu()

    def exact(self, window=0, prefix=None, weight_eps=None):
        """out, lse in 64 bits and their bounds (on the device: the sums are long)."""
        H, G, d, bf = self.H, self.G, self.d, self.tdt == torch.bfloat16
        eps = (2.0 ** -8 if bf else 0.0) if weight_eps is None else weight_eps
        K, V = (value(c, s).double() for c, s in zip(self.code, self.byte))
        out, tol = torch.zeros(self.T, H * G, d, dtype=torch.float64), torch.zeros(self.T, H * G, d, dtype=torch.float64)
        lse, ltol = torch.full((self.T, H * G), -math.inf, dtype=torch.float64), torch.zeros(self.T, H * G, dtype=torch.float64)
        for b in range(self.B):
            n, L = self.new[b], min(max(self.L[b], 0), self.S)
            if not n or not L:
                continue
            i, j = torch.arange(L - n, L).cuda()[:, None], torch.arange(L).cuda()
            seen = (j <= i) & ((i - j < window) if window else True)
            if prefix is not None:
                seen = seen | (j < prefix[b])
            none = ~seen.any(1)
            for head in range(H * G):
                q, k, v = self.q[self.off[b]:self.off[b + 1], head].double().cuda(), K[b, head // G, :L].cuda(), V[b, head // G, :L].cuda()
                if not bool(torch.isfinite(k).all() and torch.isfinite(v).all()):   # hidden rows only: where they are seen nothing is compared
                    k, v = k.nan_to_num(0.0, 0.0, 0.0), v.nan_to_num(0.0, 0.0, 0.0)
                x, mag = q @ k.T * self.scale, q.abs() @ k.abs().T * self.scale
                if self.cap:
                    x = self.cap * torch.tanh(x / self.cap)
                e = (6 * math.sqrt(d) * U * mag + 16 * U * x.abs() + 8 * U * self.cap).masked_fill(~seen, 0.0).amax(1, keepdim=True)
                x = x.masked_fill(~seen, -math.inf)
                z = torch.logsumexp(x, 1, keepdim=True)
                p = torch.exp(x - torch.where(none[:, None], torch.zeros_like(z), z))
                o, mass = p @ v, p @ v.abs()
                rel = 2 * e + 2.0 ** -20 + eps + 6 * seen.sum(1, keepdim=True).double().sqrt() * U
                r = slice(int(self.off[b]), int(self.off[b + 1]))
                out[r, head], tol[r, head] = o.cpu(), (1.05 * rel * mass + (2.0 ** -8 if bf else U) * 1.01 * o.abs() + 1e-30).cpu()
                lse[r, head], ltol[r, head] = z[:, 0].cpu(), (e + 2.0 ** -20 + 2.0 ** -22 * z.abs())[:, 0].cpu()
        return out, lse, tol, ltol


def check(got, want, tol, what):
    err = (got.double() - want).abs()
    assert bool(torch.isfinite(got).all()) and bool((err <= tol).all()), \
        f"{what}: {int((err > tol).sum())} of {err.numel()} beyond the bound, worst {float((err / tol.clamp(min=1e-30)).max()):.3g} times it"


def check_lse(got, want, tol):
    none = want == -math.inf
    assert torch.equal(got == -math.inf, none)
    check(got[~none], want[~none], tol[~none], "lse")


# H, G, d, ctx, new, page, options
CASES = {
    "one_token_one_slot": (2, 6, 128, [0], [1], 0, {}),
    "one_token_d128": (2, 6, 128, [1000], [1], 16, {}),
    "one_token_d64": (1, 4, 64, [333], [1], 16, {}),
    "one_token_d256": (4, 2, 256, [517], [1], 16, {}),
    "decode_ragged_g7": (4, 7, 128, [700, 0, 63, 64, 65, 2000, 127, 128], [1] * 8, 16, {}),
    "decode_empty_sequence": (2, 6, 128, [100, 50, 0, 9], [1, 0, 0, 1], 16, {}),
    "decode_g1": (3, 1, 128, [129, 31], [1, 1], 0, {}),
    "decode_g5_d256": (1, 5, 256, [1500, 31], [1, 1], 64, {}),
    "decode_g8_d64": (2, 8, 64, [1500, 31], [1, 1], 24, {}),
    "decode_g16": (1, 16, 128, [400], [1], 16, {}),
    "decode_g17": (2, 17, 128, [190], [1], 16, {}),
    "decode_g64": (1, 64, 64, [257], [1], 16, {}),
    "decode_long": (1, 2, 64, [20000], [1], 16, {}),
    "decode_long_d128": (2, 7, 128, [30000, 11], [1, 1], 16, {}),
    "few_tokens": (2, 6, 128, [300, 40], [3, 2], 16, {}),
    "four_tokens_g8": (2, 8, 128, [1300, 40, 0], [4, 4, 3], 16, {}),
    "four_tokens_d256": (2, 2, 256, [1300, 40], [4, 1], 16, {}),
    "chunk_g7": (4, 7, 128, [300, 17], [65, 130], 16, {}),
    "chunk_from_nothing": (2, 6, 128, [0, 0], [257, 40], 0, {}),
    "chunk_d64": (1, 4, 64, [100, 0, 33], [130, 77, 1], 16, {}),
    "chunk_d256": (2, 2, 256, [200, 9], [140, 64], 16, {}),
    "chunk_odd_pages": (2, 4, 128, [150, 20], [70, 33], 7, {}),
    "chunk_page_1": (1, 4, 128, [50], [40], 1, {}),
    "chunk_page_256": (2, 4, 64, [450], [70], 256, {}),
    "chunk_window": (2, 4, 128, [600, 3], [150, 40], 16, {"window": 100}),
    "window_1": (2, 4, 128, [60], [70], 16, {"window": 1}),
    "decode_window": (2, 6, 128, [900, 30], [1, 1], 16, {"window": 65}),
    "decode_prefix_window": (2, 6, 128, [1900, 30], [2, 1], 16, {"window": 65, "prefix": [200, 7]}),
    "prefix_beyond_own": (2, 4, 128, [20, 200], [100, 60], 16, {"prefix": [64, 7]}),
    "prefix_and_window": (1, 4, 128, [700, 40], [80, 1], 16, {"prefix": [33, 41], "window": 90}),
    "prefix_longer_than_cache": (1, 4, 64, [5], [9], 0, {"prefix": [1000]}),
    "capped": (2, 2, 256, [300], [50], 16, {"cap": 50.0}),
    "capped_hard": (2, 4, 128, [300], [50], 16, {"cap": 2.0}),
    "capped_decode": (2, 4, 128, [300], [1], 16, {"cap": 2.0}),
    "capped_decode_d64": (2, 4, 64, [300], [2], 16, {"cap": 20.0}),
    "long_chunk": (1, 4, 128, [1500], [600], 16, {}),
    "long_chunk_split": (1, 2, 128, [9000], [70], 16, {}),
}


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("name", sorted(CASES))
def test_attend(name, dtype):
    H, G, d, ctx, new, page, opt = CASES[name]
    p = Problem(H, G, d, ctx, new, dtype, page, seed=sum(map(ord, name)), cap=opt.get("cap", 0.0))
    args = (opt.get("window", 0), opt.get("prefix"))
    out, lse = p.attend(*args)
    assert p.dec.device_status() == 0
    eo, el, to, tl = p.exact(*args)
    check(out, eo, to, "out")
    check_lse(lse, el, tl)
    again, _ = p.attend(*args, lse=False)
    assert torch.equal(again, out), "equal calls give equal bits"


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("d,G,new", [(128, 7, 1), (64, 4, 1), (256, 2, 2), (128, 4, 100), (256, 2, 130)])
@pytest.mark.parametrize("kind", ["rising", "falling", "scales_far_apart", "large_scores"])
def test_attend_growth(dtype, d, G, new, kind):
    """Maxima that grow inside a range, scales that lie far apart, scores of hundreds."""
    gain = {"rising": lambda x: 0.1 + 6 * x, "falling": lambda x: 6.1 - 6 * x, "scales_far_apart": lambda x: 0 * x + 1, "large_scores": lambda x: 0 * x + 8}[kind]
    p = Problem(2, G, d, [2500, 300], [new, new], dtype, 16, seed=17, gain=gain, spread=4.0 if kind == "scales_far_apart" else 0.3)
    out, lse = p.attend()
    eo, el, to, tl = p.exact()
    check(out, eo, to, "out")
    check_lse(lse, el, tl)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("new", [[5, 1], [200, 3], [1, 1]])
def test_rows_that_see_nothing_are_zero(dtype, new):
    p = Problem(2, 4, 128, [0, 0], new, dtype, 16, seed=3, kv_len=[max(0, new[0] - 4), 0])
    out, lse = p.attend()
    eo, el, to, tl = p.exact()
    blind = min(4, new[0])
    assert bool((el[:blind] == -math.inf).all()) and bool((el[new[0]:] == -math.inf).all())
    check(out, eo, to, "out")
    check_lse(lse, el, tl)
    assert not out[:blind].any() and not out[new[0]:].any()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new", [90, 4, 1])
@pytest.mark.parametrize("code,byte", [(0x7f, 130), (0x01, 255), (0x7e, 254)])
def test_hidden_slots_never_reach_a_row(dtype, d, new, code, byte):
    """Rows of K and V that some tokens do not see may hold NaN codes, infinite and huge scales."""
    p = Problem(2, 4, d, [200], [new], dtype, 16, seed=5)
    window = 150
    at = [3, 200 + new // 2] if new > 1 else [3]     # before every window; a token in the middle of the chunk
    for j in at:
        for i in range(2):
            p.code[i][:, :, j], p.byte[i][:, :, j] = code, byte
    out, lse = p.attend(window)
    eo, el, to, tl = p.exact(window)
    sees = 200 + torch.arange(new) >= at[-1] if new > 1 else torch.zeros(1, dtype=torch.bool)
    check(out[~sees], eo[~sees], to[~sees], "out")
    check_lse(lse[~sees], el[~sees], tl[~sees])


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("new", [1, 90])
def test_values_that_are_not_finite(dtype, new):
    """A NaN in V reaches its own channel of the tokens that see it, a NaN in K every channel."""
    p = Problem(2, 4, 128, [200], [new], dtype, 16, seed=6)
    p.code[1][:, :, 50, 9] = 0x7f
    out, lse = p.attend()
    assert bool(out[:, :, 9].isnan().all()) and bool(torch.isfinite(lse).all())
    others = torch.arange(128) != 9
    eo, el, to, tl = p.exact()
    check(out[..., others], eo[..., others], to[..., others], "out")
    p.code[0][:, :, 50, 3] = 0xff
    out, _ = p.attend()
    assert bool(out.isnan().all())


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("new", [[33, 90], [1, 2]])
def test_strided_queries_outputs_and_caches(dtype, new):
    p = Problem(2, 6, 128, [130, 40], new, dtype, 0, seed=7, layout="bshd")
    eo, el, to, tl = p.exact()
    fused = torch.full((p.T, 2 * 6 + 4, 128), math.nan, dtype=p.tdt, device="cuda")
    fused[:, 2:14] = p.q.cuda()
    wide = torch.full((p.T, 12, 256), 3.0, dtype=p.tdt, device="cuda")
    lse = torch.zeros((p.T, 12), device="cuda")
    ck, cv, ks, vs = p.cache()
    wider = [torch.full((p.B, 3, p.S + 5), 255, dtype=torch.uint8, device="cuda") for _ in "kv"]     # scales with strides of their own
    for w, s in zip(wider, (ks, vs)):
        w[:, 1:, 2:2 + p.S] = s
    p.dec.attend_quantised(fused[:, 2:14], i32(p.off), i32(p.L), ck, cv, *(w[:, 1:, 2:2 + p.S] for w in wider), wide[:, :, 128:], lse=lse)
    torch.cuda.synchronize()
    check(wide[:, :, 128:].cpu(), eo, to, "out")
    assert bool((wide[:, :, :128] == 3.0).all())
    check_lse(lse.cpu(), el, tl)


@pytest.mark.parametrize("new", [1, 140])
def test_another_stream_and_a_graph(new):
    p = Problem(2, 6, 128, [700], [new], "bf16", 16, seed=11)
    base, _ = p.attend()
    cache, q, off, L, out = p.cache(), p.q.cuda(), i32(p.off), i32(p.L), torch.zeros_like(base, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        p.dec.attend_quantised(q, off, L, *cache, out, **p.place.kw())
    s.synchronize()
    assert torch.equal(out.cpu(), base)
    out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.dec.attend_quantised(q, off, L, *cache, out, **p.place.kw())
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), base)


@pytest.mark.parametrize("page", [8, 16, 24, 32, 48, 128, 200])
@pytest.mark.parametrize("H,G,d,ctx,new", [(2, 7, 128, [333, 90], [37, 1]), (1, 4, 64, [513], [130]), (2, 2, 256, [200, 40], [1, 66]),
                                           (3, 5, 128, [400, 0, 31], [1, 1, 1]), (2, 8, 64, [700, 3], [2, 1]), (1, 4, 256, [700, 3], [1, 2])])
def test_page_sizes(page, H, G, d, ctx, new):
    p, flat = Problem(H, G, d, ctx, new, "bf16", page, seed=41), Problem(H, G, d, ctx, new, "bf16", 0, seed=41)
    out, lse = p.attend()
    eo, el, to, tl = p.exact()
    check(out, eo, to, "out")
    check_lse(lse, el, tl)
    assert torch.equal(flat.attend()[0], out)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("most", [1, 9])
def test_many_sequences(dtype, most):
    rng = np.random.default_rng(9)
    new = [int(x) for x in rng.choice([0, 0, 1, 1, min(2, most), most], 200)]
    p = Problem(2, 3, 64, [int(x) for x in rng.integers(0, 190, 200)], new, dtype, 16, seed=43)
    out, lse = p.attend()
    eo, el, to, tl = p.exact()
    check(out, eo, to, "out")
    check_lse(lse, el, tl)


def test_pages_beyond_32_bits():
    """Pages whose rows lie behind the first 2^32 bytes of a pool."""
    H, d, page, n = 4, 256, 64, 200
    pages = (1 << 32) // (H * d * page) + 8
    codes = [torch.zeros((pages, page, H, d), dtype=torch.uint8, device="cuda") for _ in "kv"]
    scales = [torch.zeros((pages, H, page), dtype=torch.uint8, device="cuda") for _ in "kv"]
    table = torch.arange(pages - 1, pages - 6, -1, dtype=torch.int32, device="cuda").view(1, 5)
    dec = kvx.Decoder(synth.ModelGeom(1, H, d, 0.0), H)
    x = [torch.randn((1, H, n, d), device="cuda").bfloat16() for _ in "kv"]
    dec.quantise(i32([n]), [x[0]], [x[1]], [codes[0]], [codes[1]], [scales[0]], [scales[1]], dst_page_table=table, page_size=page)
    back = [torch.zeros_like(t) for t in x]
    dec.dequantise(i32([n]), [codes[0]], [codes[1]], [scales[0]], [scales[1]], [back[0]], [back[1]], page_table=table, page_size=page)
    new = torch.randn((1, H, d), device="cuda").bfloat16()
    q = torch.randn((1, H, d), device="cuda").bfloat16()
    dec.append_quantised(q, new, new, i32([0, 1]), i32([n + 1]), *codes, *scales, torch.empty_like(q), page_table=table, page_size=page)
    out = torch.zeros_like(q)
    dec.attend_quantised(q, i32([0, 1]), i32([n + 1]), *codes, *scales, out, page_table=table, page_size=page)
    assert dec.device_status() == 0
    for a, b in zip(back, x):
        c, s = held(b.double().cpu())
        assert torch.equal(a.cpu(), value(c, s).bfloat16())
    c, s = held(new.double().cpu())
    K, V = (torch.cat([t.double().cpu()[0], value(c, s).double().transpose(0, 1)], 1) for t in back)
    w = torch.softmax(torch.einsum("hd,hjd->hj", q[0].double().cpu(), K) / 16, -1)
    want = torch.einsum("hj,hjd->hd", w, V)
    assert bool(((out[0].double().cpu() - want).abs() <= 2.0 ** -8 * (want.abs() + torch.einsum("hj,hjd->hd", w, V.abs())) + 1e-5).all())


def test_lengths_past_the_cache_and_bad_pages_are_flagged():
    p = Problem(2, 4, 128, [60], [3], "bf16", 16, seed=13)
    cache, q, off = p.cache(), p.q.cuda(), i32(p.off)
    out, k = torch.zeros_like(q), q[:, :2]
    full = [torch.zeros((1, 2, 63, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    one = [[t] for t in cache]
    for bad in (-1, p.place.pages):
        table = p.place.table.clone()
        table[0, 1] = bad
        for call in (lambda: p.dec.attend_quantised(q, off, i32(p.L), *cache, out, page_table=table),
                     lambda: p.dec.append_quantised(q, k, k, off, i32([30]), *cache, torch.empty_like(q), page_table=table),
                     lambda: p.dec.dequantise(i32([40]), *one, [full[0]], [full[1]], page_table=table),
                     lambda: p.dec.quantise(i32([40]), [full[0]], [full[1]], *one, dst_page_table=table)):
            call()
            assert p.dec.device_status() == kvx.KVX_DEV_PAGE_INVALID
    table = p.place.table
    p.dec.attend_quantised(q, off, i32([1000]), *cache, out, page_table=table)
    assert p.dec.device_status() & kvx.KVX_DEV_SEQ_CLAMPED
    p.dec.append_quantised(q, k, k, off, i32([1000]), *cache, torch.empty_like(q), page_table=table)
    assert p.dec.device_status() == kvx.KVX_DEV_SEQ_CLAMPED
    for n in (1000, -1, 64):          # the contiguous cache has 63 slots
        p.dec.dequantise(i32([n]), *one, [full[0]], [full[1]], page_table=table)
        assert p.dec.device_status() == kvx.KVX_DEV_SEQ_CLAMPED


def test_no_tokens_and_empty_lengths():
    p = Problem(2, 4, 128, [60], [3], "bf16", 16, seed=13)
    cache, q = p.cache(), p.q.cuda()[:0]
    before = [c.clone() for c in cache]
    p.dec.append_quantised(q, q[:, :2], q[:, :2], i32([0, 0]), i32([60]), *cache, q, page_table=p.place.table)
    p.dec.attend_quantised(q, i32([0, 0]), i32([60]), *cache, q, page_table=p.place.table)
    full = [torch.full((1, 2, 63, 128), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    p.dec.dequantise(i32([0]), *[[t] for t in cache], [full[0]], [full[1]], page_table=p.place.table)
    p.dec.quantise(i32([0]), [full[0]], [full[1]], *[[t] for t in cache], dst_page_table=p.place.table)
    assert p.dec.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(before, cache)) and all(bool((x == 9.0).all()) for x in full)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_the_steps_together(dtype):
    """A cache quantised, tokens appended, attended over and read back: attention over the values read back agrees."""
    tdt, kdt = TYPES[dtype]
    H, G, d, n, page = 2, 6, 128, 300, 16
    dec = kvx.Decoder(synth.ModelGeom(2, H, d, 1e4), H * G, dtype=kdt)
    g = torch.Generator(device="cuda").manual_seed(1)
    pages = -(-(n + 20) // page)
    table = torch.randperm(pages, generator=g, device="cuda").int().view(1, pages)
    full = [[torch.randn((pages, page, H, d), device="cuda", generator=g).to(tdt) for _ in range(2)] for _ in "kv"]
    codes = [[torch.zeros((pages, page, H, d), dtype=CODES, device="cuda") for _ in range(2)] for _ in "kv"]
    scales = [[torch.zeros((pages, H, page), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2)] for _ in "kv"]
    dec.quantise(i32([n]), *full, *codes, *scales, page_table=table, dst_page_table=table, page_size=page)
    length = n
    for new in (19, 1):
        length += new
        off, L = i32([0, new]), i32([length])
        for l in range(2):
            qkv = torch.randn((new, H * G + 2 * H, d), device="cuda", generator=g).to(tdt)
            q = qkv[:, :H * G]
            c = [x[l] for x in (*codes, *scales)]
            dec.append_quantised(q, qkv[:, H * G:H * G + H], qkv[:, H * G + H:], off, L, *c, q, page_table=table, page_size=page)
            out, ref = (torch.zeros((new, H * G, d), dtype=tdt, device="cuda") for _ in range(2))
            lse, lref = (torch.zeros((new, H * G), device="cuda") for _ in range(2))
            dec.attend_quantised(q, off, L, *c, out, lse=lse, page_table=table, page_size=page)
            back = [[torch.zeros_like(full[0][0])] for _ in "kv"]
            dec.dequantise(L, *[[x] for x in c], *back, page_table=table, dst_page_table=table, page_size=page)
            dec.attend(q, off, L, back[0][0], back[1][0], ref, lse=lref, page_table=table, page_size=page)
            err = (out.double() - ref.double()).abs()
            assert float(err.max()) <= (2.0 ** -6 if dtype == "bf16" else 1e-5) * float(ref.abs().max())
            assert torch.allclose(lse, lref, rtol=1e-6, atol=1e-5)
    assert dec.device_status() == 0


def test_refusals():
    p = Problem(2, 4, 128, [60], [3], "bf16", 16, seed=13)
    ck, cv, ks, vs = cache = p.cache()
    q, off, L, table = p.q.cuda(), i32(p.off), i32(p.L), p.place.table
    k, out = q[:, :2], torch.zeros_like(q)
    full = [torch.zeros((1, 2, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    attend = lambda *c, **kw: p.dec.attend_quantised(q, off, L, *c, out, **{"page_table": table, **kw})
    append = lambda *c, **kw: p.dec.append_quantised(q, k, k, off, L, *c, torch.empty_like(q), **{"page_table": table, **kw})
    quantise = lambda *c, **kw: p.dec.quantise(L, [full[0]], [full[1]], *[[x] for x in c], **{"dst_page_table": table, **kw})
    back = lambda *c, **kw: p.dec.dequantise(L, *[[x] for x in c], [full[0]], [full[1]], **{"page_table": table, **kw})
    for call in (attend, append, quantise, back):
        call(*cache)
        for bad in ((ck[:, :8], cv[:, :8], ks, vs), (ck, cv[:-1], ks, vs), (ck.view(torch.int8), cv, ks, vs), (ck, cv, ks[:, :1], vs), (ck, cv, ks, vs[:-1]),
                    (ck, cv, ks.view(torch.int8), vs), (ck[:, :, :1], cv[:, :, :1], ks[:, :1], vs[:, :1]), (ck, cv, ks[:, :, ::2], vs[:, :, ::2]),
                    (ck[..., :64], cv[..., :64], ks, vs), (ck, cv, ks.transpose(1, 2), vs.transpose(1, 2))):
            with pytest.raises(ValueError):
                call(*bad)
        with pytest.raises(kvx.KvxError):
            call(*cache, page_size=0)
    with pytest.raises(ValueError):
        p.dec.quantise(L, [full[0].float()], [full[1].float()], [ck], [cv], [ks], [vs], dst_page_table=table)
    with pytest.raises(ValueError):
        p.dec.quantise(L, [full[0]] * 2, [full[1]] * 2, [ck], [cv], [ks], [vs], dst_page_table=table)
    with pytest.raises(ValueError):
        p.dec.quantise(L.long(), [full[0]], [full[1]], [ck], [cv], [ks], [vs], dst_page_table=table)
    with pytest.raises(kvx.KvxError) as e:               # one layer in the model
        p.dec.quantise(L, [full[0]] * 2, [full[1]] * 2, [ck] * 2, [cv] * 2, [ks] * 2, [vs] * 2, dst_page_table=table)
    assert e.value.status == kvx.KVX_ERR_INVALID_ARG
    with pytest.raises(kvx.KvxError):
        attend(*cache, window=-1)
    many = torch.zeros(1026, dtype=torch.int32, device="cuda")
    for call in (lambda: p.dec.attend_quantised(q, many, many, *cache, out, page_table=table),
                 lambda: p.dec.quantise(many, [full[0]], [full[1]], [ck], [cv], [ks], [vs], dst_page_table=table)):
        with pytest.raises(kvx.KvxError) as e:
            call()
        assert e.value.status == kvx.KVX_ERR_UNSUPPORTED
    # codes that are not 16-byte aligned, strides that are not multiples of 16
    raw = torch.zeros(1 * 2 * 80 * 128 + 8, dtype=torch.uint8, device="cuda")
    odd = raw[8:8 + 2 * 64 * 128].view(1, 2, 64, 128)
    flat = torch.zeros((1, 2, 64), dtype=torch.uint8, device="cuda")
    wide = torch.zeros((1, 2, 64, 136), dtype=torch.uint8, device="cuda")[..., :128]
    for c in (odd, wide):
        with pytest.raises(kvx.KvxError) as e:
            p.dec.attend_quantised(q, off, L, c, c, flat, flat, out)
        assert e.value.status == kvx.KVX_ERR_INVALID_ARG
    # a cache over itself
    same = torch.zeros((1, 2, 64, 128), dtype=torch.bfloat16, device="cuda")
    small = same.view(torch.uint8).view(-1)[:2 * 64 * 128].view(1, 2, 64, 128)
    with pytest.raises(kvx.KvxError) as e:
        p.dec.quantise(L, [same], [full[1]], [small], [small.clone()], [flat], [flat])
    assert e.value.status == kvx.KVX_ERR_INVALID_ARG
    # weight sums: not over 8 bits
    import ctypes
    opts = kvx.kvx_attend_opts(0, None, 1, 1, 64)
    rows = kvx.kvx_rows(q.data_ptr(), q.stride(0), q.stride(1))
    tok = kvx.kvx_new_tokens(1, 3, off.data_ptr(), L.data_ptr(), None)
    c, _keep = p.dec._code_layers([ck], [cv], [ks], [vs], 1, table, 16, 0)
    assert kvx.lib().kvx_attend_quantised(p.dec.handle, ctypes.byref(tok), ctypes.byref(rows), c, 0, ctypes.byref(opts), ctypes.byref(rows),
                                          None) == kvx.KVX_ERR_UNSUPPORTED
    assert p.dec.device_status() == 0


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("d,G,n", [(128, 1, 256), (128, 6, 100), (64, 4, 256), (256, 2, 256), (128, 4, 3), (64, 2, 2), (256, 4, 1)])
def test_a_single_seen_row_comes_back_exactly(dtype, d, G, n):
    """Every code under every scale byte that is written (values up to 2^120): tokens that see their own slot alone return its V row."""
    p = Problem(2, G, d, [0], [n], dtype, 16, seed=8)
    g = torch.Generator().manual_seed(n)
    p.code[0].zero_()                                    # scores of zero: weights of one
    p.code[1] = torch.stack([torch.stack([torch.randint(0, 256, (d,), generator=g, dtype=torch.uint8) for _ in range(n)]) for _ in range(2)])[None]
    p.byte[1] = torch.randint(10, 239, (1, 2, n), generator=g, dtype=torch.int64).to(torch.uint8)
    out, lse = p.attend(window=1)
    assert not lse.any()
    want = value(p.code[1], p.byte[1])[0].transpose(0, 1).repeat_interleave(G, 1).to(p.tdt)       # [n, Hq, d]
    assert torch.equal(out.isnan(), want.isnan())
    fine = ~want.isnan()
    tol = 2.0 ** -20 if dtype == "fp32" else 0.0         # (rows summed again have a weight within 2^-20 of one)
    assert bool(((out[fine].double() - want[fine].double()).abs() <= tol * want[fine].double().abs()).all())
