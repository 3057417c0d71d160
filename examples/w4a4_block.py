"""The feed-forward half of a transformer block in W4A4, dense and with experts.

    python examples/w4a4_block.py

Both run the path a served model runs: the residual stream's update and AdaLN in
one call, the online Kronecker quantizer, MXFP4 linear layers with their
activation, gate and residual in the epilogue.  Random weights and tokens stand
in for a model's.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_21446_amd as kq  # noqa: E402


class Layer:
    """A linear layer prepared once: the factors of its activations' transform, packed, and its weight W T^-T in MXFP4
    (one weight, or one for each expert under shared factors)."""

    def __init__(self, weight, generator):
        eye = lambda n: torch.eye(n) + 0.1 * torch.randn((1, n, n), generator=generator)  # noqa: E731
        A, B = eye(4), eye(8)
        self.A, self.B = A.cuda(), B.cuda()
        self.kpack = kq.pack_factors(self.A, self.B)
        done = [kq.weight_transform(w, A, B)[1:] for w in (weight if weight.dim() == 3 else [weight])]
        self.codes, self.scales = (torch.stack(t) if weight.dim() == 3 else t[0] for t in zip(*done))

    def quantize(self, x):
        return kq.quantize_packed(x, self.A, self.B, self.kpack)[:2]


def dense(stream, attention, mod, up, down, up_bias, down_bias):
    """stream + gate attention, AdaLN, MLP, gated onto the stream.  mod [B, 4 d]: the attention's gate, scale, shift, the
    MLP's gate.  Returns the new stream and what lies between."""
    gate, scale, shift, gate_mlp = mod.chunk(4, dim=1)
    h, y = kq.block_norm(attention, stream, gate=gate, scale=scale, shift=shift, norm="layer")
    yq = up.quantize(y)
    u = kq.mxfp4_linear(*yq, up.codes, up.scales, bias=up_bias, act="gelu_tanh")
    uq = down.quantize(u)
    out = kq.mxfp4_linear(*uq, down.codes, down.scales, bias=down_bias, gate=gate_mlp, residual=h)
    return out, {"h": h, "y": y, "yq": yq, "u": u, "uq": uq}


def route(logits, k):
    """Each token's k experts and weights, as rows sorted by expert: offsets [E + 1], the token of each row, its weight."""
    weight, expert = torch.topk(torch.softmax(logits, -1), k, dim=-1)
    order = torch.argsort(expert.reshape(-1), stable=True)
    count = torch.bincount(expert.reshape(-1), minlength=logits.shape[1])
    offsets = torch.nn.functional.pad(count.cumsum(0), (1, 0)).to(torch.int32)
    return offsets, (order // k).to(torch.int32), weight.reshape(-1)[order].contiguous()


def experts(stream, attention, weight, post_weight, router, up, down, k):
    """stream + norm(attention), RMSNorm, k experts a token (SwiGLU), added to the stream."""
    h, y = kq.block_norm(attention, stream, weight=weight, post_weight=post_weight, norm="rms", post_norm="rms")
    offsets, rows, row_weight = route(y.float() @ router, k)
    yq = up.quantize(y)
    u = kq.mxfp4_grouped_linear(*yq, up.codes, up.scales, offsets, rows=rows, act="swiglu")
    uq = down.quantize(u)
    v = kq.mxfp4_grouped_linear(*uq, down.codes, down.scales, offsets, row_scale=row_weight, out_dtype=torch.float32)
    out = h.float().index_add_(0, rows.long(), v).to(h.dtype)
    return out, {"h": h, "y": y, "offsets": offsets, "rows": rows, "row_weight": row_weight, "yq": yq, "u": u, "uq": uq, "v": v}


def inputs(tokens=512, batches=2, d=1152, wide=4608, n_experts=8, expert_wide=640, seed=0):
    """Everything both blocks need."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    bf16 = lambda t: t.to(torch.bfloat16).cuda()  # noqa: E731
    w = lambda *s: bf16(r(*s) / math.sqrt(s[-1]))  # noqa: E731
    return {"stream": bf16(r(tokens, d)), "attention": bf16(r(tokens, d)), "mod": bf16(0.3 * r(batches, 4 * d)),
            "up": Layer(w(wide, d), g), "down": Layer(w(d, wide), g), "up_bias": bf16(0.1 * r(wide)), "down_bias": bf16(0.1 * r(d)),
            "weight": bf16(1 + 0.1 * r(d)), "post_weight": bf16(0.5 + 0.1 * r(d)), "router": (r(d, n_experts) / math.sqrt(d)).cuda(),
            "expert_up": Layer(w(n_experts, 2 * expert_wide, d), g), "expert_down": Layer(w(n_experts, d, expert_wide), g)}


def main():
    p = inputs()
    out, _ = dense(p["stream"], p["attention"], p["mod"], p["up"], p["down"], p["up_bias"], p["down_bias"])
    print("dense  ", tuple(out.shape), "rms", float(out.float().square().mean().sqrt()))
    out, mid = experts(p["stream"], p["attention"], p["weight"], p["post_weight"], p["router"], p["expert_up"], p["expert_down"], 2)
    print("experts", tuple(out.shape), "rms", float(out.float().square().mean().sqrt()), "rows", mid["offsets"].diff().tolist())


if __name__ == "__main__":
    main()
