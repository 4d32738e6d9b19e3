"""kvx_attend over bf16 caches where the running maximum of a row grows inside a CTA's range, so that its
output sums are rescaled between products, against the definition in 64 bits.

The bounds are those of test_gpu_decode.py with the weights' rounding as the arithmetic has it: bf16 has 8
significant bits, so a weight is within 2^-8 of itself where it is multiplied as one bf16 term and within
2^-16 as two (high part and the rest, each rounded); the output's own rounding is 2^-8.
"""
import math

import pytest
import torch

import paper_2608_30963_gb300 as kvx
from paper_2608_30963_gb300 import synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
PAGE = 16


class Call:
    """New tokens over a paged bf16 cache whose keys' gain rises with the slot; in prompts every fourth query
    is zero, so that its scores never grow, beside rows whose scores do."""

    def __init__(self, H, G, d, ctx, new, top_gain, seed, window=0, scale=0.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.H, self.G, self.d, self.ctx, self.new, self.window = H, G, d, ctx, new, window
        self.L = [c + n for c, n in zip(ctx, new)]
        self.scale = scale or 1.0 / math.sqrt(d)
        T, S = sum(new), max(self.L)

        def rnd(*shape):
            return torch.randn(shape, device="cuda", generator=g)

        q = 2.0 * rnd(T, H * G, d)
        if T >= 16:
            q[::4] = 0.0
        self.q = q.bfloat16()
        gain = 0.25 + top_gain * torch.arange(S, device="cuda") / max(S - 1, 1)
        self.K, self.V = (rnd(len(new), H, S, d) * gain[:, None]).bfloat16(), rnd(len(new), H, S, d).bfloat16()
        per = -(-S // PAGE)
        perm = torch.randperm(len(new) * per, generator=torch.Generator().manual_seed(seed)).cuda()
        self.table = perm.view(len(new), per).int()

        def pool(x):
            pad = torch.zeros(len(new), H, per * PAGE, d, dtype=x.dtype, device="cuda")
            pad[:, :, :S] = x
            out = torch.zeros(len(new) * per, PAGE, H, d, dtype=x.dtype, device="cuda")
            out[perm] = pad.view(len(new), H, per, PAGE, d).permute(0, 2, 3, 1, 4).reshape(-1, PAGE, H, d)
            return out

        self.ck, self.cv = pool(self.K), pool(self.V)
        self.off = torch.tensor([0] + list(torch.tensor(new).cumsum(0)), dtype=torch.int32, device="cuda")
        self.len = torch.tensor(self.L, dtype=torch.int32, device="cuda")
        self.dec = kvx.Decoder(synth.ModelGeom(1, H, d, 1e4), H * G, scale=scale)

    def run(self, weight=None):
        out, lse = torch.full_like(self.q, 7.0), torch.full(self.q.shape[:2], 7.0, device="cuda")
        self.dec.attend(self.q, self.off, self.len, self.ck, self.cv, out, window=self.window, lse=lse, key_weight=weight,
                        page_table=self.table, page_size=PAGE)
        assert self.dec.device_status() == 0
        return out, lse

    def check(self, out, lse, weight_eps):
        """out and lse within the bounds; weight_eps(slots seen by each token): the weights' rounding.  Returns by how much the definition
        with its weights rounded to one bf16 term would be beyond the bound (a mistake planted here, in 64 bits)."""
        t0, planted = 0, 0.0
        for b, (n, L) in enumerate(zip(self.new, self.L)):
            i = torch.arange(L - n, L, device="cuda")[:, None]
            j = torch.arange(L, device="cuda")
            seen = (j <= i) & ((i - j < self.window) if self.window else True)
            count = seen.sum(1)
            eps = weight_eps(count)[:, None]
            for head in range(self.H * self.G):
                k, v = self.K[b, head // self.G, :L].double(), self.V[b, head // self.G, :L].double()
                q = self.q[t0:t0 + n, head].double()
                x = (q @ k.T * self.scale).masked_fill(~seen, -math.inf)
                mag = q.abs() @ k.abs().T * self.scale
                e = (6 * math.sqrt(self.d) * U * mag + 16 * U * x.abs()).masked_fill(~seen, 0.0).amax(1, keepdim=True)
                z = torch.logsumexp(x, 1, keepdim=True)
                p = torch.exp(x - z)
                want, mass = p @ v, p @ v.abs()
                rel = 2 * e + 2.0 ** -20 + eps + 6 * count[:, None].double().sqrt() * U
                tol = 1.05 * rel * mass + 1.01 * 2.0 ** -8 * want.abs() + 1e-30
                err = (out[t0:t0 + n, head].double() - want).abs()
                assert bool((err <= tol).all()), f"out, sequence {b}, head {head}: {float((err / tol).max()):.3g} times the bound"
                rounded = torch.exp(x - x.amax(1, keepdim=True)).bfloat16().double() * torch.exp(x.amax(1, keepdim=True) - z)
                planted = max(planted, float(((rounded @ v - want).abs() / tol).max()))
                lerr, ltol = (lse[t0:t0 + n, head].double() - z[:, 0]).abs(), e[:, 0] + 2.0 ** -20 + 2.0 ** -22 * z[:, 0].abs()
                assert bool((lerr <= ltol).all()), f"lse, sequence {b}, head {head}"
            t0 += n
        return planted

    def repeats(self, out, lse, times=4):
        for _ in range(times):
            o, z = self.run()
            assert torch.equal(o, out) and torch.equal(z, lse), "equal calls give equal bits"


def one_term(count):
    return torch.full(count.shape, 2.0 ** -8, device="cuda", dtype=torch.float64)


def two_terms(count):
    return torch.full(count.shape, 2.0 ** -16, device="cuda", dtype=torch.float64)


# H, G, new tokens of each sequence, their slots before: ranges of several slot tiles a CTA
PROMPTS = {
    "prompt": (4, 2, [512], [3584]),
    "prompt_odd": (2, 8, [301], [5003]),
    "ragged": (4, 2, [260, 70, 1, 500], [2000, 4100, 1500, 77]),
}
TOKENS = {
    "token": (4, 2, [1], [20001]),
    "tokens": (2, 8, [1, 1, 1, 1, 3], [9000, 700, 12345, 33, 4097]),
}


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("gain", [3.0, 24.0])
@pytest.mark.parametrize("name", sorted(PROMPTS))
def test_prompts_whose_maxima_grow(name, gain, d):
    """Maxima that grow by more than 2^8 in many tiles, at a range's start and in its middle."""
    H, G, new, ctx = PROMPTS[name]
    c = Call(H, G, d, ctx, new, gain, seed=d)
    out, lse = c.run()
    c.check(out, lse, one_term)
    c.repeats(out, lse)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [65, 700])
@pytest.mark.parametrize("gain", [0.0, 24.0])
def test_windows_leave_rows_nothing_in_their_first_tiles(window, gain, d):
    """Rows that see nothing in the tiles a row tile begins with, and something later, with and without scores that grow."""
    c = Call(4, 2, d, [2500, 3], [512, 900], gain, seed=d + 1, window=window)
    out, lse = c.run()
    c.check(out, lse, one_term)
    c.repeats(out, lse)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 1000])
@pytest.mark.parametrize("name", sorted(TOKENS))
def test_single_tokens_whose_maxima_grow(name, window, d):
    H, G, new, ctx = TOKENS[name]
    for gain in (3.0, 24.0):
        c = Call(H, G, d, ctx, new, gain, seed=d + 2, window=window)
        out, lse = c.run()
        c.check(out, lse, two_terms)
        c.repeats(out, lse)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("G,new,ctx", [(7, [301], [5003]), (6, [200, 90], [3000, 2100]), (7, [1], [20001]), (6, [1, 9], [9000, 4097])])
def test_bits_do_not_depend_on_what_ran_before(G, new, ctx, d):
    """Query heads that do not fill a row tile: its last rows hold what an earlier kernel left in shared memory."""
    c = Call(2, G, d, ctx, new, 3.0, seed=d + 3)
    full = Call(2, 8, d, ctx, [max(n, 200) if max(new) > 9 else n for n in new], 3.0, seed=d + 4)   # heads that fill it
    base = None
    for gain in (0.0, 1.0, 300.0, 1.0):
        full.q.copy_((gain * torch.randn(full.q.shape, device="cuda")).bfloat16())
        full.run()
        out, lse = c.run()
        base = base or (out, lse)
        assert torch.equal(out, base[0]) and torch.equal(lse, base[1])
    c.check(out, lse, one_term)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("G,new,ctx", [(2, [70, 300], [3000, 3000]), (7, [30, 40, 50], [4000, 100, 2000]), (7, [1, 1, 1], [9000, 300, 4000])])
def test_bits_do_not_depend_on_the_next_sequence(G, new, ctx, d):
    """Row tiles that end inside a sequence's last tokens hold the next sequence's queries, too."""
    c = Call(2, G, d, ctx, new, 3.0, seed=d + 5)
    out, lse = c.run()
    n = new[0]
    for gain in (0.0, 300.0, float("inf"), float("nan")):
        c.q[n:] = gain * torch.randn_like(c.q[n:])
        o, z = c.run()
        assert torch.equal(o[:n], out[:n]) and torch.equal(z[:n], lse[:n])
