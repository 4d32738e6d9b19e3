"""A target model goes on from a handed-over cache.

The steps a serving process makes after a handoff, for the cache's part of every target layer:
translate the source model's cache into the target's paged cache; write a question's tokens behind
the context and attend to both, summing the weight each cached token receives; cut the cache down to
the tokens that received the most; decode token by token from what is left.  The model's own
projections and MLPs are not part of the library: random queries, keys and values stand in for them.

    python examples/continue_from_handoff.py [context tokens] [kept tokens]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_30963_gb300 as kvx  # noqa: E402
from paper_2608_30963_gb300 import synth  # noqa: E402

PAGE = 16


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def pages(tokens):
    """A page table for one sequence: every page of a pool, in order."""
    n = -(-tokens // PAGE)
    return torch.arange(n, dtype=torch.int32, device="cuda").view(1, n), n


def main(context=2000, keep=500, question=48, answer=8, layers=4, q_heads=12):
    torch.manual_seed(0)
    src, dst = synth.ModelGeom(layers, 4, 128, 1e6), synth.ModelGeom(layers, 2, 128, 1e6)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    H, d = dst.num_kv_heads, dst.head_dim

    # the handoff: the source model's cache of the context, translated into pages of the target's
    tr = kvx.Translator(src, dst, torch.randn(layers, H, 256, d, **bf16) / 16, torch.randn(layers, H, 256, d, **bf16) / 16)
    src_k, src_v = ([torch.randn(1, 4, context, 128, **bf16) for _ in range(layers)] for _ in range(2))
    table, n = pages(context + question)
    k, v = ([torch.zeros(n, PAGE, H, d, **bf16) for _ in range(layers)] for _ in range(2))
    tr.translate(src_k, src_v, i32(context), i32(0, context), context, k, v, page_table=table, page_size=PAGE)

    # the question: its tokens behind the context, one call a layer for the write and one for the attention
    dec = kvx.Decoder(dst, q_heads)
    off, length = i32(0, question), i32(context + question)
    weight = torch.zeros(layers, 1, H, context + question, device="cuda")
    lse = torch.empty(question, q_heads, device="cuda")
    out = torch.empty(question, q_heads, d, **bf16)
    for layer in range(layers):
        qkv = torch.randn(question, q_heads + 2 * H, d, **bf16)       # the layer's fused projection
        q = qkv[:, :q_heads]
        dec.append(q, qkv[:, q_heads:q_heads + H], qkv[:, q_heads + H:], off, length, k[layer], v[layer], q, page_table=table)
        dec.attend(q, off, length, k[layer], v[layer], out, lse=lse, key_weight=weight[layer], page_table=table)

    # the cache cut down: attention sinks and the question stay, of the rest what received the most weight
    small, m = pages(keep + answer)
    sk, sv = ([torch.zeros(m, PAGE, H, d, **bf16) for _ in range(layers)] for _ in range(2))
    kept = torch.empty(layers, 1, H, keep, dtype=torch.int32, device="cuda")
    kept_weight = torch.zeros(layers, 1, H, keep + answer, device="cuda")
    left = i32(0)
    dec.evict(length, weight, keep, k, v, sk, sv, kept, left, sinks=4, recent=question, kept_weight=kept_weight, page_table=table,
              dst_page_table=small)

    # the answer, a token at a time: slots go on from the cut cache, positions from the whole text
    one, o1 = i32(0, 1), torch.empty(1, q_heads, d, **bf16)
    for step in range(answer):
        left += 1
        for layer in range(layers):
            qkv = torch.randn(1, q_heads + 2 * H, d, **bf16)
            q = qkv[:, :q_heads]
            dec.append(q, qkv[:, q_heads:q_heads + H], qkv[:, q_heads + H:], one, left, sk[layer], sv[layer], q,
                       pos=i32(context + question + step), page_table=small)
            dec.attend(q, one, left, sk[layer], sv[layer], o1, lse=lse[:1], key_weight=kept_weight[layer], page_table=small)
    torch.cuda.synchronize()
    assert tr.device_status() == 0 and dec.device_status() == 0
    share = float(kept_weight[..., :keep].sum() / (weight.sum() + answer * layers * q_heads))
    print(f"{context} handed-over tokens and a question of {question}: {keep} of {context + question} slots kept, "
          f"{answer} tokens decoded from {int(left)} slots; the kept slots hold {100 * share:.0f}% of the attention weight")
    return out, o1, kept, kept_weight, left


if __name__ == "__main__":
    main(*(int(x) for x in sys.argv[1:3]))
