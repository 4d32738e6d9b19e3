"""Cases of the operators that carry a target model on from a handed-over cache.

A handoff leaves a translated KV cache; the frozen target model then goes on from it.  Its new
tokens are rotated and written into the cache (append), attend to everything cached (attend), the
attention weight that each cached token receives is summed (weigh: the same attention with the sums
as a second output), and a cache that has grown too long is cut down to the tokens that received
the most (evict).  Caches are the ones a translation writes: contiguous [B, H, S, d] or pools of
16-token pages [pages, 16, H, d] in shuffled order.

Fields of a case:
  op       "append", "attend", "weigh" (attend, adding to the weight sums) or "evict"
  model    MODELS: KV heads, query heads, head width, RoPE base
  dtype    "bf16" or "fp32": caches, queries and outputs
  ctx      cached tokens of each sequence before the new ones, comma separated
  new      new tokens of each sequence, comma separated (append, attend, weigh)
  paged    paged cache, else contiguous
  cap      scores capped as cap * tanh(s / cap); 0: none
  window   a new token sees the last so many slots up to its own; 0: all
  prefix   the first so many slots are seen by every new token (0: none)
  layers, keep, sinks, recent   (evict) layers in one call; slots kept of each sequence, KV head and
           layer, of them the first `sinks` and the last `recent` in any case
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
PAGE = 16


def _case(name, op, model, ctx, new=(), dtype="bf16", paged=True, cap=0.0, window=0, prefix=0, layers=1, keep=0, sinks=0,
          recent=0):
    c = {"op": op, "model": model, "dtype": dtype, "ctx": ",".join(str(n) for n in ctx),
         "new": ",".join(str(n) for n in new), "paged": paged, "cap": cap, "window": window, "prefix": prefix,
         "layers": layers, "keep": keep, "sinks": sinks, "recent": recent}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step's token of one conversation: all launch and memory latency
        _case("append_1_token", "append", "1p5b", [1000], [1]),
        # a serving batch's prompts after their handed-over contexts, ragged, into a paged cache
        _case("append_b8_chunks", "append", "7b", [8192, 517, 33, 4096, 1000, 2049, 16000, 1], [1024, 517, 64, 2048, 31, 1500, 4096, 1]),
        # one decode step of one conversation over a short handed-over context: latency
        _case("attend_1_token_1k", "attend", "1p5b", [1000], [1]),
        # a decode step of a long-context serving batch: the cache is read once
        _case("attend_decode_b8_32k", "attend", "7b", [27649, 16385, 32767, 20011, 31007, 18000, 24576, 29999], [1] * 8),
        # a question of a few hundred tokens over a handed-over context, capped scores and a sliding
        # window as the 256-wide target's layers have them, contiguous cache
        _case("attend_512_over_8k_capped", "attend", "gemma2b", [8192 - 512], [512], paged=False, cap=50.0, window=4096),
        # the largest: a long prompt read on top of a long handed-over context
        _case("attend_4k_over_32k", "attend", "7b", [28672], [4096]),
        # a ragged batch, a prefix that every new token sees, small heads
        _case("attend_b4_ragged_prefix", "attend", "tiny", [0, 700, 2100, 5], [130, 517, 3, 1000], prefix=64, window=256),
        # float32 caches at an ordinary prompt length
        _case("attend_100_over_1k_fp32", "attend", "1p5b", [1000], [100], dtype="fp32", paged=False),
        # decode steps that keep account of the weight each cached token receives
        _case("weigh_decode_b4_16k", "weigh", "7b", [16384, 12001, 9000, 16000], [1] * 4),
        # the observation chunk before an eviction: a prompt's end over a long context
        _case("weigh_256_over_16k", "weigh", "7b", [16128], [256]),
        # a small float32 cache cut down
        _case("evict_1k_to_256_fp32", "evict", "tiny", [1000], dtype="fp32", paged=False, layers=2, keep=256, sinks=4, recent=32),
        # every layer of a serving batch cut down to a quarter
        _case("evict_28_layers_b4_16k", "evict", "1p5b", [16384, 12001, 9000, 16000], layers=28, keep=4096, sinks=16, recent=512),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "weigh", "weigh", "evict"])
    model = rng.choice(sorted(MODELS))
    H, Hq, d, _ = MODELS[model]
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    batch = rng.choice([1, 1, 2, 3, 5, 8])
    paged = rng.random() < 0.7
    if op == "evict":
        layers = rng.choice([1, 2, 7, 26, 28])
        top = max(256, min(32768, (28 * 4 * 16384 * 2 * 128 * 2) // (layers * batch * H * d * (2 if dtype == "bf16" else 4))))
        ctx = [max(1, int(_log_int(rng, 64, top) * rng.uniform(0.5, 1.0))) for _ in range(batch)]
        keep = max(1, int(max(ctx) * rng.uniform(0.1, 0.9)))
        sinks = rng.randint(0, min(16, keep))
        return _case(None, op, model, ctx, dtype=dtype, paged=paged, layers=layers, keep=keep, sinks=sinks,
                     recent=rng.randint(0, (keep - sinks) // 2))
    ctx = [max(0, int(_log_int(rng, 1, 32768) * rng.uniform(0.5, 1.0)) - 1) for _ in range(batch)]
    if op == "append":
        return _case(None, op, model, ctx, [_log_int(rng, 1, 4096) for _ in range(batch)], dtype=dtype, paged=paged)
    top = rng.choice([1, 1, 8, 64, 512, 4096])
    new = [_log_int(rng, 1, top) for _ in range(batch)]
    # float32 runs at a fraction of the rate of bf16 on the tensor cores: shorter lengths
    most = 28 * 4096 * 32768 // (32 if dtype == "fp32" else 1)
    while Hq * d * batch * max(new) * (max(ctx) + max(new)) > most * 128:
        ctx, new = [n // 2 for n in ctx], [max(1, n // 2) for n in new]
    return _case(None, op, model, ctx, new, dtype=dtype, paged=paged, cap=rng.choice([0.0, 0.0, 20.0, 50.0]),
                 window=rng.choice([0, 0, 0, _log_int(rng, 16, 8192)]), prefix=rng.choice([0, 0, 0, rng.randint(1, 200)]))


# ------------------------------------------------------------------ inputs
def _lens(case):
    ctx = [int(x) for x in case["ctx"].split(",")]
    new = [int(x) for x in case["new"].split(",")] if case["new"] else [0] * len(ctx)
    return ctx, new


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def _table(lens, rng):
    per = [max(1, -(-n // PAGE)) for n in lens]
    perm, table, k = rng.permutation(sum(per)), np.zeros((len(lens), max(per))), 0
    for b, n in enumerate(per):
        table[b, :n] = perm[k:k + n]
        k += n
    return _i32(table), sum(per)


def _cache(case, gen, layers, lens, pages, tdt, fill):
    H, _, d, _ = MODELS[case["model"]]
    shape = (layers, pages, PAGE, H, d) if case["paged"] else (layers, len(lens), H, max(lens), d)
    if fill:
        return [torch.randn(shape, device="cuda", generator=gen, dtype=torch.float32 if tdt == torch.float32 else tdt)
                for _ in range(2)]
    return [torch.zeros(shape, device="cuda", dtype=tdt) for _ in range(2)]


def prepare(case, seed):
    H, Hq, d, base = MODELS[case["model"]]
    ctx, new = _lens(case)
    total = [c + n for c, n in zip(ctx, new)]
    rng = np.random.default_rng([seed, 21])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    tdt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    st = {"case": case, "B": len(ctx), "H": H, "Hq": Hq, "d": d, "tdt": tdt, "S": max(total), "kv_len": _i32(total)}
    st["table"], pages = _table(total, rng) if case["paged"] else (None, 0)
    st["k"], st["v"] = _cache(case, gen, case["layers"], total, pages, tdt, True)
    if case["op"] == "evict":
        st["keep"] = min(case["keep"], st["S"])
        kept = [min(n, st["keep"]) for n in total]
        st["dst_table"], pages = _table(kept, rng) if case["paged"] else (None, 0)
        st["dst_k"], st["dst_v"] = _cache(case, gen, case["layers"], kept, pages, tdt, False)
        # sums of attention weights: a few tokens with most of it, a long tail, some equal values
        w = torch.rand((case["layers"], st["B"], H, st["S"]), device="cuda", generator=gen).pow(6)
        st["weight"] = torch.where(w < 1e-4, torch.zeros_like(w), (w * 4096).round() / 4096 + (w > 0.01) * w)
        st["kept"] = torch.full((case["layers"], st["B"], H, st["keep"]), -2, dtype=torch.int32, device="cuda")
        st["kept_weight"] = torch.zeros((case["layers"], st["B"], H, st["keep"]), device="cuda")
        st["new_len"] = torch.zeros(st["B"], dtype=torch.int32, device="cuda")
    else:
        T = sum(new)
        off = np.concatenate([[0], np.cumsum(new)])
        st.update(T=T, seq_off=_i32(off), n_max=max(new))
        # the projections' output for the new tokens: queries, keys and values of a token side by side
        qkv = torch.randn((T, Hq + 2 * H, d), device="cuda", generator=gen)
        qkv[:, :Hq] *= 2.0       # scores with a spread of about two: some tokens stand out
        qkv = qkv.to(tdt)
        st["q"], st["new_k"], st["new_v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        if case["op"] == "append":
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
            st["weight"] = torch.zeros((st["B"], H, st["S"]), device="cuda") if case["op"] == "weigh" else None
    if own:
        import paper_2608_30963_gb300 as kvx
        from paper_2608_30963_gb300 import synth
        st["dec"] = kvx.Decoder(synth.ModelGeom(case["layers"], H, d, base), Hq,
                                dtype=kvx.KVX_BF16 if case["dtype"] == "bf16" else kvx.KVX_FP32, score_cap=case["cap"])
    return st


# ------------------------------------------------------------------ the plain forms
def _tokens(st):
    """Packed index of token i of each sequence [B, n_max] (clamped), whether it exists, its slot."""
    off = st["seq_off"].long()
    i = torch.arange(st["n_max"], device="cuda")
    n = (off[1:] - off[:-1])[:, None]
    return (off[:-1, None] + i).clamp(max=max(0, st["T"] - 1)), i < n, st["kv_len"].long()[:, None] - n + i


def _place(st):
    """Row of each slot [B, S] in a paged cache's pool, rows past the table clamped to its last page."""
    s = torch.arange(st["S"], device="cuda")
    return st["table"].long()[:, (s // PAGE).clamp(max=st["table"].shape[1] - 1)] * PAGE + s % PAGE


def _rows(st, cache):
    """One layer's cached rows in 32 bits, [B, H, S, d]."""
    if st["table"] is None:
        return cache[0].float()
    return cache[0].reshape(-1, st["H"], st["d"])[_place(st)].permute(0, 2, 1, 3).float()


def _append(st):
    B, H, d = st["B"], st["H"], st["d"]
    at, real, slot = _tokens(st)
    at, b, slot = at[real], torch.arange(B, device="cuda")[:, None].expand_as(real)[real], slot[real]
    cos, sin = st["cos"][slot][:, None], st["sin"][slot][:, None]

    def rotated(x):
        lo, hi = x[at].float().split(d // 2, dim=-1)
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).to(st["tdt"])

    st["q_out"][at] = rotated(st["q"])
    for cache, rows in ((st["k"], rotated(st["new_k"])), (st["v"], st["new_v"][at])):
        if st["table"] is None:
            cache[0][b, :, slot] = rows
        else:
            cache[0].view(-1, H, d)[_place(st)[b, slot]] = rows
    return {"q": st["q_out"], "k": st["k"], "v": st["v"]}


def _attend(st):
    case, B, H, Hq, d = st["case"], st["B"], st["H"], st["Hq"], st["d"]
    G, n, S = Hq // H, st["n_max"], st["S"]
    at, real, slot = _tokens(st)
    q = st["q"][at].float().view(B, n, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, d)
    s = torch.matmul(q, _rows(st, st["k"]).transpose(2, 3)).mul_(1.0 / math.sqrt(d))
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
    o = torch.matmul(p.view(B, H, G * n, S), _rows(st, st["v"])).view(B, H, G, n, d)
    st["out"][at[real]] = o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, d)[real].to(st["tdt"])
    st["lse"][at[real]] = (safe + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, Hq)[real]
    if st["weight"] is None:
        return {"out": st["out"], "lse": st["lse"]}
    st["weight"] += p.sum((2, 3))
    return {"out": st["out"], "lse": st["lse"], "weight": st["weight"]}


def _evict(st):
    case, B, H, S, keep = st["case"], st["B"], st["H"], st["S"], st["keep"]
    L, n = case["layers"], st["kv_len"].long()[:, None, None]
    j = torch.arange(S, device="cuda")
    forced = (j < case["sinks"]) | (j >= n - case["recent"])
    w = st["weight"].masked_fill(forced, math.inf).masked_fill(j >= n, -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]    # ties: the lowest slot first
    new = torch.clamp(n, max=keep)
    r = torch.arange(keep, device="cuda")
    live = (r < new).expand(L, B, H, keep)
    kept = torch.sort(order.masked_fill(~live, S), dim=-1).values
    st["kept"].copy_(kept.masked_fill(~live, -1))
    st["new_len"].copy_(new.view(B))
    st["kept_weight"].copy_(torch.gather(st["weight"], 3, kept.clamp(max=S - 1)).masked_fill(~live, 0.0))
    l, b, h, r = torch.nonzero(live, as_tuple=True)
    s = kept[live]
    for src, dst in ((st["k"], st["dst_k"]), (st["v"], st["dst_v"])):
        if st["table"] is None:
            dst[l, b, h, r] = src[l, b, h, s]
        else:
            dst[l, st["dst_table"].long()[b, r // PAGE], r % PAGE, h] = src[l, st["table"].long()[b, s // PAGE], s % PAGE, h]
    return {k: st[k] for k in ("kept", "new_len", "kept_weight", "dst_k", "dst_v")}


def _library(st):
    case, dec = st["case"], st["dec"]
    pages = {"page_table": st["table"], "page_size": PAGE} if st["table"] is not None else {}
    if case["op"] == "append":
        dec.append(st["q"], st["new_k"], st["new_v"], st["seq_off"], st["kv_len"], st["k"][0], st["v"][0], st["q_out"], **pages)
        return {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    if case["op"] == "evict":
        if pages:
            pages["dst_page_table"] = st["dst_table"]
        dec.evict(st["kv_len"], st["weight"], st["keep"], list(st["k"]), list(st["v"]), list(st["dst_k"]), list(st["dst_v"]),
                  st["kept"], st["new_len"], sinks=case["sinks"], recent=case["recent"], kept_weight=st["kept_weight"], **pages)
        return {k: st[k] for k in ("kept", "new_len", "kept_weight", "dst_k", "dst_v")}
    dec.attend(st["q"], st["seq_off"], st["kv_len"], st["k"][0], st["v"][0], st["out"], window=case["window"],
               prefix_len=st["prefix_len"], lse=st["lse"], key_weight=st["weight"], **pages)
    return {k: st[k] for k in ("out", "lse", "weight") if st[k] is not None}


def run(state):
    if own:
        return _library(state)
    return {"append": _append, "attend": _attend, "weigh": _attend, "evict": _evict}[state["case"]["op"]](state)


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
    if case["op"] == "append":      # q, k, v read, q and the cache rows written; a rotation is six operations a pair
        T = sum(new)
        return {"bytes": 2 * T * (Hq + 2 * H) * d * size, "flops": 3 * T * (Hq + H) * d}
    if case["op"] == "evict":       # weights read, kept rows read and written, their slots and weights written
        kept = case["layers"] * H * sum(min(n, case["keep"]) for n in ctx)
        slots = case["layers"] * H * sum(ctx)
        return {"bytes": 4 * slots + kept * (4 * d * size + 8), "flops": 2 * slots}
    pairs = [_seen(case, b) for b in range(len(ctx))]
    rows = sum(r for _, r in pairs) * H
    extra = 8 * rows if case["op"] == "weigh" else 0      # the sums are read and written
    return {"bytes": 2 * rows * d * size + 2 * sum(new) * Hq * d * size + 4 * sum(new) * Hq + extra,
            "flops": 4 * d * Hq * sum(p for p, _ in pairs)}


# ------------------------------------------------------------------ the definition in 64 bits
def _slot_row(st, table, b, s):
    """Index of slots s of sequence b in a layer's cache, as (first, second) coordinates."""
    return (table[b].long()[s // PAGE], s % PAGE)


def _exact_append(st, case):
    H, Hq, d, base = MODELS[case["model"]]
    theta = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    ctx, new = _lens(case)
    q_out = torch.zeros((st["T"], Hq, d), dtype=torch.float64, device="cuda")
    caches = {"k": st["k"].double(), "v": st["v"].double()}
    t0 = 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        s = torch.arange(c, c + n, device="cuda")
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s.double()[:, None] * theta)[:, None]

        def rot(x):
            y = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double()) * turn
            return torch.cat([y.real, y.imag], dim=-1)

        q_out[t0:t0 + n] = rot(st["q"][t0:t0 + n])
        for name, rows in (("k", rot(st["new_k"][t0:t0 + n])), ("v", st["new_v"][t0:t0 + n].double())):
            if case["paged"]:
                caches[name][0][_slot_row(st, st["table"], b, s)] = rows
            else:
                caches[name][0, b, :, c:c + n] = rows.transpose(0, 1)
        t0 += n
    return {"q": q_out, "k": caches["k"], "v": caches["v"]}


def _exact_attend(st, case):
    H, Hq, d, _ = MODELS[case["model"]]
    ctx, new = _lens(case)
    out = torch.zeros((st["T"], Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((st["T"], Hq), dtype=torch.float64, device="cuda")
    weight = torch.zeros((st["B"], H, st["S"]), dtype=torch.float64, device="cuda")
    t0 = 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        L = c + n
        s = torch.arange(L, device="cuda")
        K, V = ((x[0][_slot_row(st, st["table"], b, s)].transpose(0, 1) if case["paged"] else x[0, b, :, :L]) for x in (st["k"], st["v"]))
        i = torch.arange(c, L, device="cuda")[:, None]
        hidden = s > i
        if case["window"]:
            hidden |= s <= i - case["window"]
        if case["prefix"]:
            hidden &= s >= case["prefix"]
        for head in range(Hq):
            k, v = K[head // (Hq // H)].double(), V[head // (Hq // H)].double()
            for r in range(0, n, 1024):
                x = st["q"][t0 + r:t0 + min(n, r + 1024), head].double() @ k.T / d ** 0.5
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                x[hidden[r:r + 1024]] = -math.inf
                z = torch.logsumexp(x, dim=1)
                x = torch.exp(x - z[:, None])
                out[t0 + r:t0 + r + len(x), head], lse[t0 + r:t0 + r + len(x), head] = x @ v, z
                weight[b, head // (Hq // H), :L] += x.sum(0)
        t0 += n
    return {"out": out, "lse": lse, "weight": weight} if case["op"] == "weigh" else {"out": out, "lse": lse}


def _exact_evict(st, case):
    ctx, _ = _lens(case)
    w = st["weight"].double().cpu().numpy()
    kept_weight = np.zeros(tuple(st["kept_weight"].shape))
    moved = {"k": st["dst_k"].double(), "v": st["dst_v"].double()}
    for l in range(w.shape[0]):
        for b, n in enumerate(ctx):
            m = min(n, st["keep"])
            rest = np.arange(min(case["sinks"], n), max(min(case["sinks"], n), n - case["recent"]))
            for h in range(w.shape[2]):
                ranked = rest[np.lexsort((rest, -w[l, b, h, rest]))]
                chosen = np.setdiff1d(np.arange(n), ranked[max(0, m - (n - len(rest))):])
                kept_weight[l, b, h, :m] = w[l, b, h, chosen]
                s, r = torch.from_numpy(chosen).cuda(), torch.arange(m, device="cuda")
                for name in ("k", "v"):
                    if case["paged"]:
                        p, o = _slot_row(st, st["table"], b, s)
                        P, O = _slot_row(st, st["dst_table"], b, r)
                        moved[name][l, P, O, h] = st[name][l, p, o, h].double()
                    else:
                        moved[name][l, b, h, :m] = st[name][l, b, h, s].double()
    return {"kept": None, "new_len": None, "kept_weight": torch.from_numpy(kept_weight), "dst_k": moved["k"], "dst_v": moved["v"]}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(dict(case), seed)
    finally:
        own = was
    return {"append": _exact_append, "attend": _exact_attend, "weigh": _exact_attend, "evict": _exact_evict}[case["op"]](st, case)
