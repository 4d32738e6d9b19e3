"""Cases of the operators that hold a target model's cache in 8 bits.

A cache that a handoff has left is quantised (quantise: every layer in one call), new tokens are rotated and quantised as
they are written (append), attend to everything cached (attend), and a cache is read back into its model's own type
(dequantise).  A row (slot, KV head) of K or V is d codes in e4m3 and one scale, a power of two held in a byte
(its exponent):  amax <= 448 2^e for the smallest such e, code = e4m3(x / 2^e), value = code 2^e.  Caches are
contiguous [B, H, S, d] with scales [B, H, S], or pools of pages [pages, page, H, d] in shuffled order with scales
[pages, H, page].

Fields of a case:
  op       "append", "attend", "quantise" or "dequantise"
  model    MODELS: KV heads, query heads, head width, RoPE base
  dtype    "bf16" or "fp32": the model's own type, of queries, new keys and values, outputs, and of the caches that are
           quantised or read back
  ctx      cached tokens of each sequence before the new ones, comma separated
  new      new tokens of each sequence, comma separated (append, attend)
  page     tokens a page; 0: a contiguous cache
  cap      scores capped as cap * tanh(s / cap); 0: none
  window   a new token sees the last so many slots up to its own; 0: all
  prefix   the first so many slots are seen by every new token (0: none)
  layers   (quantise, dequantise) layers in one call
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False     # False: the plain forms below; True: the library's operators

#        KV heads, query heads, head width, RoPE base: the widths and KV heads of the library's own target models
MODELS = {
    "tiny": (1, 4, 64, 1e4),
    "1p5b": (2, 12, 128, 1e6),
    "7b": (4, 28, 128, 1e6),
    "gemma2b": (4, 8, 256, 1e4),
    "70b": (8, 64, 128, 5e5),
}
CODES, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _case(name, op, model, ctx, new=(), dtype="bf16", page=16, cap=0.0, window=0, prefix=0, layers=1):
    c = {"op": op, "model": model, "dtype": dtype, "ctx": ",".join(str(n) for n in ctx),
         "new": ",".join(str(n) for n in new), "page": page, "cap": cap, "window": window, "prefix": prefix, "layers": layers}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step's token of one conversation: all launch and memory latency
        _case("append_1_token", "append", "1p5b", [1000], [1]),
        # a serving batch's prompts after their contexts, ragged, one of them a single token
        _case("append_b8_chunks", "append", "7b", [4096, 517, 33, 8192, 1000, 2049, 12000, 1], [2048, 700, 64, 1024, 31, 1500, 4096, 1]),
        # a short float32 cache of one layer, contiguous: the smallest call over a cache
        _case("quantise_1k_fp32", "quantise", "tiny", [1000], dtype="fp32", page=0),
        # what a handoff has left of a serving batch, every layer
        _case("quantise_28_layers_b4_16k", "quantise", "1p5b", [16384, 12001, 9000, 16000], layers=28),
        # wide heads of a few layers, ragged
        _case("dequantise_3_layers_ragged", "dequantise", "gemma2b", [1500, 1, 613], page=64, layers=3),
        # a batch's caches read back for a step that wants the model's own type
        _case("dequantise_28_layers_b4_16k", "dequantise", "1p5b", [16384, 12001, 9000, 16000], layers=28),
        # one decode step of one conversation over a short context: latency
        _case("attend_1_token_1k", "attend", "1p5b", [1000], [1]),
        # a decode step of a long-context serving batch: the cache is read once
        _case("attend_decode_b8_32k", "attend", "7b", [27649, 16385, 32767, 20011, 31007, 18000, 24576, 29999], [1] * 8),
        # a few drafted tokens checked in one step, wide groups of query heads
        _case("attend_4_tokens_b4_16k", "attend", "70b", [16384, 12001, 9000, 16000], [4, 4, 3, 4]),
        # a question over a context, capped scores and a sliding window, contiguous cache
        _case("attend_512_over_8k_capped", "attend", "gemma2b", [8192 - 512], [512], page=0, cap=50.0, window=4096),
        # the largest: a long prompt read on top of a long context
        _case("attend_4k_over_32k", "attend", "7b", [28672], [4096]),
        # float32 queries at an ordinary prompt length, a prefix that every new token sees
        _case("attend_100_over_1k_fp32", "attend", "1p5b", [1000], [100], dtype="fp32", page=0, window=300, prefix=50),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "quantise", "dequantise", "attend", "attend", "attend", "attend"])
    model = rng.choice(sorted(MODELS))
    H, Hq, d, _ = MODELS[model]
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    batch = rng.choice([1, 1, 2, 3, 5, 8])
    page = rng.choice([0, 16, 16, 64, 24])
    if op in ("quantise", "dequantise"):
        layers = rng.choice([1, 2, 7, 26, 28])
        top = max(256, min(32768, (28 * 4 * 13000 * 2 * 128 * 2) // (layers * batch * H * d * (2 if dtype == "bf16" else 4))))
        return _case(None, op, model, [max(1, int(_log_int(rng, 64, top) * rng.uniform(0.5, 1.0))) for _ in range(batch)], dtype=dtype,
                     page=page, layers=layers)
    ctx = [max(0, int(_log_int(rng, 1, 32768) * rng.uniform(0.5, 1.0)) - 1) for _ in range(batch)]
    if op == "append":
        return _case(None, op, model, ctx, [_log_int(rng, 1, 4096) for _ in range(batch)], dtype=dtype, page=page)
    top = rng.choice([1, 1, 1, 4, 16, 64, 512, 4096])
    new = [_log_int(rng, 1, top) for _ in range(batch)]
    # float32 runs at a fraction of the rate of bf16 on the tensor cores: shorter lengths
    most = 28 * 4096 * 32768 // (32 if dtype == "fp32" else 1)
    while Hq * d * batch * max(new) * (max(ctx) + max(new)) > most * 128:
        ctx, new = [n // 2 for n in ctx], [max(1, n // 2) for n in new]
    return _case(None, op, model, ctx, new, dtype=dtype, page=page, cap=rng.choice([0.0, 0.0, 20.0, 50.0]),
                 window=rng.choice([0, 0, 0, _log_int(rng, 16, 8192)]), prefix=rng.choice([0, 0, 0, rng.randint(1, 200)]))


# ------------------------------------------------------------------ inputs
def _lens(case):
    ctx = [int(x) for x in case["ctx"].split(",")]
    new = [int(x) for x in case["new"].split(",")] if case["new"] else [0] * len(ctx)
    return ctx, new


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def _table(lens, page, rng):
    per = [max(1, -(-n // page)) for n in lens]
    perm, table, k = rng.permutation(sum(per)), np.zeros((len(lens), max(per))), 0
    for b, n in enumerate(per):
        table[b, :n] = perm[k:k + n]
        k += n
    return _i32(table), sum(per)


def _zeros(case, layers, lens, pages, tdt):
    """A cache's K and V of zeros (with their scales where tdt is the codes' type)."""
    H, _, d, _ = MODELS[case["model"]]
    p = case["page"]
    rows = (layers, pages, p, H, d) if p else (layers, len(lens), H, max(lens), d)
    scales = (layers, pages, H, p) if p else rows[:-1]
    x = {n: torch.zeros(rows, device="cuda", dtype=torch.uint8 if tdt == CODES else tdt) for n in "kv"}
    if tdt == CODES:
        x = {n: t.view(CODES) for n, t in x.items()}
        x.update({n + "_scale": torch.zeros(scales, device="cuda", dtype=torch.uint8).view(SCALES) for n in "kv"})
    return x


def prepare(case, seed):
    H, Hq, d, base = MODELS[case["model"]]
    ctx, new = _lens(case)
    total, page, op = [c + n for c, n in zip(ctx, new)], case["page"], case["op"]
    rng = np.random.default_rng([seed, 37])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    tdt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    st = {"case": case, "B": len(ctx), "H": H, "Hq": Hq, "d": d, "tdt": tdt, "page": page, "S": max(total), "kv_len": _i32(total)}
    st["table"], pages = _table(total, page, rng) if page else (None, 0)
    # keys have channels that are larger than others, values less so; rows differ in size
    gain = {"k": 1.0, "v": 0.3}
    gain = {n: torch.exp(g * torch.randn((H, 1, d), device="cuda", generator=gen)) for n, g in gain.items()}
    gain["k"] = gain["k"] / gain["k"].square().mean(-1, keepdim=True).sqrt()

    def rows(cache, name):
        """Random rows for each layer of a cache."""
        for x in cache:
            r = torch.randn(x.shape, device="cuda", generator=gen) * (gain[name].squeeze(1) if page else gain[name])
            yield r * torch.exp(0.3 * torch.randn(x.shape[:-1] + (1,), device="cuda", generator=gen))

    if op == "quantise":
        st["src"] = _zeros(case, case["layers"], total, pages, tdt)
        for n in "kv":
            for l, r in enumerate(rows(st["src"][n], n)):
                st["src"][n][l] = r.to(tdt)
    else:
        st["cache"] = _zeros(case, case["layers"], total, pages, CODES)
        if op != "append":
            for n in "kv":
                for l, r in enumerate(rows(st["cache"][n], n)):
                    code, e = _quantised(r)
                    st["cache"][n].view(torch.uint8)[l] = code.to(CODES).view(torch.uint8)
                    s = st["cache"][n + "_scale"].view(torch.uint8)[l]
                    s.copy_(((e + 127).transpose(1, 2) if page else e + 127))
    if op in ("quantise", "dequantise"):
        st["dst_table"], pages = _table(total, page, rng) if page else (None, 0)
        st["dst"] = _zeros(case, case["layers"], total, pages, CODES if op == "quantise" else tdt)
    else:
        T = sum(new)
        off = np.concatenate([[0], np.cumsum(new)])
        st.update(T=T, seq_off=_i32(off), n_max=max(new))
        # the projections' output for the new tokens: queries, keys and values of a token side by side
        qkv = torch.randn((T, Hq + 2 * H, d), device="cuda", generator=gen)
        qkv[:, :Hq] *= 2.0       # scores with a spread of about two: some tokens stand out
        qkv[:, Hq:Hq + H] *= gain["k"].squeeze(1)
        qkv[:, Hq + H:] *= gain["v"].squeeze(1)
        qkv = qkv.to(tdt)
        st["q"], st["new_k"], st["new_v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        if op == "append":
            st["q_out"] = torch.zeros((T, Hq, d), dtype=tdt, device="cuda")
            # the plain form's table of rotations, worked out once as a program does, in 64 bits
            f = torch.pow(torch.tensor(base, dtype=torch.float64, device="cuda"),
                          -2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
            a = torch.arange(st["S"], dtype=torch.float64, device="cuda")[:, None] * f
            st["cos"], st["sin"] = a.cos().float(), a.sin().float()
        else:
            st["q"] = st["q"].contiguous()
            st["out"] = torch.zeros((T, Hq, d), dtype=tdt, device="cuda")
            st["lse"] = torch.zeros((T, Hq), device="cuda")
            st["prefix_len"] = _i32([case["prefix"]] * st["B"]) if case["prefix"] else None
    if own:
        import paper_2608_30963_gb300 as kvx
        from paper_2608_30963_gb300 import synth
        st["dec"] = kvx.Decoder(synth.ModelGeom(case["layers"], H, d, base), Hq,
                                dtype=kvx.KVX_BF16 if case["dtype"] == "bf16" else kvx.KVX_FP32, score_cap=case["cap"])
    return st


# ------------------------------------------------------------------ the plain forms
def _quantised(x):
    """Codes (as 32-bit values not yet rounded to e4m3) and exponents of rows [..., d]."""
    m, e = torch.frexp(x.abs().amax(-1).clamp(min=1e-38))
    e = (e - 9 + (m > 0.875)).clamp(-117, 120)
    return x * ((127 - e) << 23).view(torch.float32)[..., None], e


def _power(scale):
    """Scales as 32-bit numbers."""
    return (scale.view(torch.uint8).int() << 23).view(torch.float32)


def _tokens(st):
    """Packed index of token i of each sequence [B, n_max] (clamped), whether it exists, its slot."""
    off = st["seq_off"].long()
    i = torch.arange(st["n_max"], device="cuda")
    n = (off[1:] - off[:-1])[:, None]
    return (off[:-1, None] + i).clamp(max=max(0, st["T"] - 1)), i < n, st["kv_len"].long()[:, None] - n + i


def _page_of(st, table, s):
    """Page and place in it of slots s (one row of them for every sequence, [S] or [B, S])."""
    p = (s // st["page"]).clamp(max=table.shape[1] - 1)
    return (table.long()[:, p] if p.dim() == 1 else table.long().gather(1, p)), s % st["page"]


def _values(st, cache, name, table, l):
    """Rows of layer l of an 8-bit cache in 32 bits, [B, H, S, d]."""
    code, scale = cache[name][l], cache[name + "_scale"][l]
    if table is None:
        return code.float() * _power(scale)[..., None]
    p, o = _page_of(st, table, torch.arange(st["S"], device="cuda"))
    o = o.expand_as(p)
    return (code.view(torch.uint8)[p, o].view(CODES).float() * _power(scale)[p, :, o][..., None]).transpose(1, 2)


def _append(st):
    d, page = st["d"], st["page"]
    at, real, slot = _tokens(st)
    b = torch.arange(st["B"], device="cuda")[:, None].expand_as(real)[real]
    p = _page_of(st, st["table"], slot.clamp(min=0))[0][real] if page else None
    at, slot = at[real], slot[real]
    cos, sin = st["cos"][slot][:, None], st["sin"][slot][:, None]

    def rotated(x):
        lo, hi = x[at].float().split(d // 2, dim=-1)
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)

    st["q_out"][at] = rotated(st["q"]).to(st["tdt"])
    for n, x in (("k", rotated(st["new_k"])), ("v", st["new_v"][at].float())):
        code, e = _quantised(x)
        code, e = code.to(CODES).view(torch.uint8), (e + 127).to(torch.uint8)
        codes, scales = st["cache"][n][0].view(torch.uint8), st["cache"][n + "_scale"][0].view(torch.uint8)
        if page:
            codes[p, slot % page] = code
            scales[p, :, slot % page] = e
        else:
            codes[b, :, slot] = code
            scales[b, :, slot] = e
    return {"q": st["q_out"], **st["cache"]}


def _attend(st):
    case, B, H, Hq, d = st["case"], st["B"], st["H"], st["Hq"], st["d"]
    G, n, S = Hq // H, st["n_max"], st["S"]
    at, real, slot = _tokens(st)
    q = st["q"][at].float().view(B, n, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, d)
    s = torch.matmul(q, _values(st, st["cache"], "k", st["table"], 0).transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    if case["cap"]:
        s = s.div_(case["cap"]).tanh_().mul_(case["cap"])
    j, i = torch.arange(S, device="cuda"), slot[:, :, None]
    seen = j <= i
    if case["window"]:
        seen = seen & (i - j < case["window"])
    if case["prefix"]:
        seen = seen | ((j < st["prefix_len"][:, None, None]) & (j < st["kv_len"][:, None, None]))
    seen = (seen & real[:, :, None])[:, None, None]
    s = s.view(B, H, G, n, S).masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    safe = torch.where(top > -math.inf, top, torch.zeros_like(top))
    p = s.sub_(safe).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    o = torch.matmul(p.view(B, H, G * n, S), _values(st, st["cache"], "v", st["table"], 0)).view(B, H, G, n, d)
    st["out"][at[real]] = o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, d)[real].to(st["tdt"])
    st["lse"][at[real]] = (safe + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, Hq)[real]
    return {"out": st["out"], "lse": st["lse"]}


def _live(st):
    """Sequences and slots of the cached tokens."""
    return torch.nonzero(torch.arange(st["S"], device="cuda") < st["kv_len"][:, None], as_tuple=True)


def _quantise(st):
    b, s = _live(st)
    if st["page"]:
        (p, o), (P, O) = ((t[b, s], i[s]) for t, i in (_page_of(st, x, torch.arange(st["S"], device="cuda")) for x in (st["table"], st["dst_table"])))
    for n in "kv":
        x = st["src"][n][:, p, o] if st["page"] else st["src"][n][:, b, :, s].transpose(0, 1)     # [L, tokens, H, d]
        code, e = _quantised(x.float())
        code, e = code.to(CODES).view(torch.uint8), (e + 127).to(torch.uint8)
        codes, scales = st["dst"][n].view(torch.uint8), st["dst"][n + "_scale"].view(torch.uint8)
        if st["page"]:
            codes[:, P, O] = code
            scales[:, P, :, O] = e.transpose(0, 1)
        else:
            codes[:, b, :, s] = code.transpose(0, 1)
            scales[:, b, :, s] = e.transpose(0, 1)
    return st["dst"]


def _dequantise(st):
    b, s = _live(st)
    if st["page"]:
        P, O = _page_of(st, st["dst_table"], torch.arange(st["S"], device="cuda"))
        P, O = P[b, s], O[s]
    for n in "kv":
        for l in range(st["case"]["layers"]):
            x = _values(st, st["cache"], n, st["table"], l)[b, :, s].to(st["tdt"])
            if st["page"]:
                st["dst"][n][l, P, O] = x
            else:
                st["dst"][n][l, b, :, s] = x
    return st["dst"]


def _library(st):
    case, dec, op = st["case"], st["dec"], st["case"]["op"]
    pages = {"page_table": st["table"], "page_size": st["page"]} if st["page"] else {}
    if op == "append":
        c = {n: x[0] for n, x in st["cache"].items()}
        dec.append_quantised(st["q"], st["new_k"], st["new_v"], st["seq_off"], st["kv_len"], c["k"], c["v"], c["k_scale"], c["v_scale"],
                             st["q_out"], **pages)
        return {"q": st["q_out"], **st["cache"]}
    if op == "attend":
        c = {n: x[0] for n, x in st["cache"].items()}
        dec.attend_quantised(st["q"], st["seq_off"], st["kv_len"], c["k"], c["v"], c["k_scale"], c["v_scale"], st["out"],
                             window=case["window"], prefix_len=st["prefix_len"], lse=st["lse"], **pages)
        return {"out": st["out"], "lse": st["lse"]}
    if pages:
        pages["dst_page_table"] = st["dst_table"]
    d = {n: list(x) for n, x in st["dst"].items()}
    if op == "quantise":
        s = st["src"]
        dec.quantise(st["kv_len"], list(s["k"]), list(s["v"]), d["k"], d["v"], d["k_scale"], d["v_scale"], **pages)
    else:
        s = {n: list(x) for n, x in st["cache"].items()}
        dec.dequantise(st["kv_len"], s["k"], s["v"], s["k_scale"], s["v_scale"], d["k"], d["v"], **pages)
    return st["dst"]


def run(state):
    """Codes and scales come as the numbers that they are (e4m3 numbers, powers of two)."""
    if own:
        return _library(state)
    return {"append": _append, "attend": _attend, "quantise": _quantise, "dequantise": _dequantise}[state["case"]["op"]](state)


# ------------------------------------------------------------------ the work of a pass
def _seen(case, b):
    """(query, slot) pairs of sequence b that are seen, and the slots that any query sees."""
    ctx, new = _lens(case)
    n, L = new[b], ctx[b] + new[b]
    i = np.arange(L - n, L)
    lo = np.maximum(0, i - case["window"] + 1) if case["window"] else np.zeros(n, np.int64)
    p = min(case["prefix"], L)
    pairs = int(((i + 1 - lo) + np.minimum(p, lo) + np.maximum(0, p - i - 1)).sum())
    return pairs, min(L, (L - int(lo[0])) + min(p, int(lo[0])))


def work(case):
    H, Hq, d, _ = MODELS[case["model"]]
    size = 2 if case["dtype"] == "bf16" else 4
    ctx, new = _lens(case)
    if case["op"] == "append":      # q, k, v read, q and the cache's rows written; six operations a rotated pair, two a code
        T = sum(new)
        return {"bytes": T * ((2 * Hq + 2 * H) * d * size + 2 * H * (d + 1)), "flops": T * (3 * (Hq + H) * d + 4 * H * d)}
    if case["op"] != "attend":      # rows of one type read, of the other written
        rows = 2 * case["layers"] * H * sum(ctx)
        return {"bytes": rows * (d * size + d + 1), "flops": rows * d * (2 if case["op"] == "quantise" else 1)}
    pairs = [_seen(case, b) for b in range(len(ctx))]
    rows = sum(r for _, r in pairs) * H
    return {"bytes": 2 * rows * (d + 1) + 2 * sum(new) * Hq * d * size + 4 * sum(new) * Hq,
            "flops": 4 * d * Hq * sum(p for p, _ in pairs)}


# ------------------------------------------------------------------ the definition in 64 bits
def _at(case, table, b, s):
    """Index of slots s of sequence b in a layer's rows, and in its scales."""
    if not case["page"]:
        return (b, slice(None), s), (b, slice(None), s)
    p, o = table[b].long()[s // case["page"]], s % case["page"]
    return (p, o), (p, slice(None), o)


def _held(x):
    """Rows as a cache holds them, before the codes' rounding to 8 bits (both sides are off by that rounding alone)."""
    top = x.abs().amax(-1)
    e = torch.floor(torch.log2(top.clamp(min=1e-300))) - 8
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e).clamp(-117, 120)
    return x / torch.exp2(e)[..., None], torch.exp2(e)


def _exact_append(st, case):
    H, Hq, d, base = MODELS[case["model"]]
    theta = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    ctx, new = _lens(case)
    q_out = torch.zeros((st["T"], Hq, d), dtype=torch.float64, device="cuda")
    cache = {n: x.double() for n, x in st["cache"].items()}
    t0 = 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        s = torch.arange(c, c + n, device="cuda")
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s.double()[:, None] * theta)[:, None]

        def rot(x):
            y = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double()) * turn
            return torch.cat([y.real, y.imag], dim=-1)

        q_out[t0:t0 + n] = rot(st["q"][t0:t0 + n])
        rows, scales = _at(case, st["table"], b, s)
        for name, x in (("k", rot(st["new_k"][t0:t0 + n])), ("v", st["new_v"][t0:t0 + n].double())):
            code, scale = _held(x)                        # [n, H, d], [n, H]
            if case["page"]:
                cache[name][0][rows], cache[name + "_scale"][0][scales] = code, scale
            else:
                cache[name][0][rows], cache[name + "_scale"][0][scales] = code.transpose(0, 1), scale.transpose(0, 1)
        t0 += n
    return {"q": q_out, **cache}


def _exact_move(st, case):
    ctx, _ = _lens(case)
    to = {n: x.double() for n, x in st["dst"].items()}
    for b, n in enumerate(ctx):
        s = torch.arange(n, device="cuda")
        rows, scales = _at(case, st["table"], b, s)
        Rows, Scales = _at(case, st["dst_table"], b, s)
        for l in range(case["layers"]):
            for name in "kv":
                if case["op"] == "quantise":
                    code, scale = _held(st["src"][name][l][rows].double())
                    to[name][l][Rows], to[name + "_scale"][l][Scales] = code, scale
                else:
                    code, scale = st["cache"][name][l].double()[rows], st["cache"][name + "_scale"][l].double()[scales]
                    to[name][l][Rows] = code * scale[..., None]
    return to


def _exact_attend(st, case):
    H, Hq, d, _ = MODELS[case["model"]]
    ctx, new = _lens(case)
    out = torch.zeros((st["T"], Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((st["T"], Hq), dtype=torch.float64, device="cuda")
    t0 = 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        L = c + n
        rows, scales = _at(case, st["table"], b, torch.arange(L, device="cuda"))
        K, V = (st["cache"][x][0].double()[rows] * st["cache"][x + "_scale"][0].double()[scales][..., None] for x in "kv")
        if case["page"]:
            K, V = K.transpose(0, 1), V.transpose(0, 1)
        s, i = torch.arange(L, device="cuda"), torch.arange(c, L, device="cuda")[:, None]
        hidden = s > i
        if case["window"]:
            hidden |= s <= i - case["window"]
        if case["prefix"]:
            hidden &= s >= case["prefix"]
        for head in range(Hq):
            k, v = K[head // (Hq // H)], V[head // (Hq // H)]
            for r in range(0, n, 1024):
                x = st["q"][t0 + r:t0 + min(n, r + 1024), head].double() @ k.T / d ** 0.5
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                x[hidden[r:r + 1024]] = -math.inf
                z = torch.logsumexp(x, dim=1)
                x = torch.exp(x - z[:, None])
                out[t0 + r:t0 + r + len(x), head], lse[t0 + r:t0 + r + len(x), head] = x @ v, z
        t0 += n
    return {"out": out, "lse": lse}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(dict(case), seed)
    finally:
        own = was
    return {"append": _exact_append, "attend": _exact_attend, "quantise": _exact_move, "dequantise": _exact_move}[case["op"]](st, case)
