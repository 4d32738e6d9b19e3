"""A target model goes on from a handed-over cache that it holds in 8 bits.

The steps a serving process makes where caches fill its memory: translate the source model's cache into the target's
paged cache; quantise every layer of it into pages of codes and scales, a little over half the bytes, and let the first one go;
write a question's tokens behind the context and attend to both; decode token by token.  The model's own projections and MLPs
are not part of the library: random queries, keys and values stand in for them.

    python examples/continue_in_8_bits.py [context tokens]
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


def main(context=2000, question=48, answer=8, layers=4, q_heads=12):
    torch.manual_seed(0)
    src, dst = synth.ModelGeom(layers, 4, 128, 1e6), synth.ModelGeom(layers, 2, 128, 1e6)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    H, d = dst.num_kv_heads, dst.head_dim

    # the handoff: the source model's cache of the context, translated into pages of the target's
    tr = kvx.Translator(src, dst, torch.randn(layers, H, 256, d, **bf16) / 16, torch.randn(layers, H, 256, d, **bf16) / 16)
    src_k, src_v = ([torch.randn(1, 4, context, 128, **bf16) for _ in range(layers)] for _ in range(2))
    pages = -(-(context + question + answer) // PAGE)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    k, v = ([torch.zeros(pages, PAGE, H, d, **bf16) for _ in range(layers)] for _ in range(2))
    tr.translate(src_k, src_v, i32(context), i32(0, context), context, k, v, page_table=table, page_size=PAGE)

    # every layer into 8 bits: codes of a byte, and a scale of a byte for each row
    dec = kvx.Decoder(dst, q_heads)
    ck, cv = ([torch.zeros(pages, PAGE, H, d, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(layers)] for _ in range(2))
    ks, vs = ([torch.zeros(pages, H, PAGE, dtype=torch.uint8, device="cuda") for _ in range(layers)] for _ in range(2))
    dec.quantise(i32(context), k, v, ck, cv, ks, vs, page_table=table, dst_page_table=table, page_size=PAGE)
    torch.cuda.synchronize()
    before, after = (sum(t.numel() * t.element_size() for x in some for t in x) for some in ((k, v), (ck, cv, ks, vs)))
    del k, v

    # the question, then the answer a token at a time: one call a layer for the write and one for the attention
    length, outs = i32(context), []
    for n in [question] + [1] * answer:
        length += n
        off, out = i32(0, n), torch.empty(n, q_heads, d, **bf16)
        for layer in range(layers):
            qkv = torch.randn(n, q_heads + 2 * H, d, **bf16)       # the layer's fused projection
            q = qkv[:, :q_heads]
            cache = ck[layer], cv[layer], ks[layer], vs[layer]
            dec.append_quantised(q, qkv[:, q_heads:q_heads + H], qkv[:, q_heads + H:], off, length, *cache, q, page_table=table)
            dec.attend_quantised(q, off, length, *cache, out, page_table=table)
        outs.append(out)
    torch.cuda.synchronize()
    assert tr.device_status() == 0 and dec.device_status() == 0
    print(f"{context} handed-over tokens in {after / before:.3f} of their bytes, a question of {question} and {answer} tokens on top of them")
    return outs, length, after / before


if __name__ == "__main__":
    main(*(int(x) for x in sys.argv[1:2]))
