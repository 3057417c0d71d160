"""The attention half of a transformer block, one token of every sequence at a time.

    python examples/w4a16_step.py

The path that a served model runs when it generates: the norm before the block, a
projection with MXFP4 weights and 16-bit activations, rotary positions, the new keys
and values quantized into a paged cache, attention over it, and the output projection
added to the residual stream.  Random weights and tokens stand in for a model's.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_21446_amd as kq  # noqa: E402

HEADS, KV_HEADS, D = 9, 3, 128  # query heads, heads of the cache, columns of each


def inputs(batch=5, pages=64, page_size=16, format="mxfp4", seed=0):
    """Weights, and a cache whose pages the sequences take as they grow (here each has its own from the start)."""
    g = torch.Generator().manual_seed(seed)
    w = lambda n, k: kq.mxfp4((torch.randn((n, k), generator=g) / math.sqrt(k)).to(torch.bfloat16).cuda())  # noqa: E731
    width = HEADS * D
    each = pages // batch
    order = torch.randperm(pages, generator=g)[: batch * each].reshape(batch, each)
    return {"norm": (1 + 0.1 * torch.randn(width, generator=g)).to(torch.bfloat16).cuda(), "qkv": w((HEADS + 2 * KV_HEADS) * D, width),
            "out": w(width, width), "cache": kq.kv_cache(pages, page_size, KV_HEADS, D, format=format),
            "table": order.to(torch.int32).cuda(), "lengths": torch.zeros(batch, dtype=torch.int32, device="cuda")}


def step(stream, p):
    """stream + attention(norm(stream)) for one token [batch, width] of every sequence; the cache and the lengths grow by
    one token.  Returns the new stream and what lies between."""
    batch, size = stream.shape[0], p["cache"].page_size
    h, y = kq.block_norm(stream, weight=p["norm"], norm="rms")
    qkv = kq.w4a16_linear(y, *p["qkv"]).view(batch, HEADS + 2 * KV_HEADS, D)
    at = p["lengths"].clone()  # the new token's position
    raw = qkv.clone()
    kq.rope(qkv[:, :HEADS + KV_HEADS], at, D, pairing="halves", out=qkv[:, :HEADS + KV_HEADS])
    page = p["table"].gather(1, (at // size).long().unsqueeze(1)).squeeze(1)
    kq.kv_cache_write(p["cache"], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:], page.long() * size + at % size)
    p["lengths"] += 1
    a = kq.paged_attention(qkv[:, :HEADS], p["cache"], p["table"], p["lengths"])
    out = kq.w4a16_linear(a.view(batch, HEADS * D), *p["out"], residual=h)
    return out, {"h": h, "y": y, "raw": raw, "qkv": qkv, "at": at, "a": a}


def main():
    p = inputs()
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(40):
        out, _ = step(torch.randn((5, HEADS * D), generator=g, device="cuda").to(torch.bfloat16), p)
    print("step", i, tuple(out.shape), "rms", float(out.float().square().mean().sqrt()), "tokens", p["lengths"].tolist())


if __name__ == "__main__":
    main()
