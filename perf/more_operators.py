"""The operators of one step of token generation around a W4A4 model, what they are
measured on, and their plain forms.

Four kinds of calls:

  rope    rotary positions with one to four axes (text; row and column of an
          image; time, row and column of a video), and their gradient;
  cache   the keys and values of new tokens quantized as they are written into a
          paged cache, and tokens of it read back;
  attn    attention of one new token of every sequence over that cache;
  linear  act(x deq(B)^T + bias), gated and added to the residual, for a few rows
          of 16- or 32-bit activations and an MXFP4 weight.

Sizes are layer shapes that the benchmark and the tests use (1152 to 12288
features, up to 18432 tokens) and generic head layouts.  Where ``own`` is true
the calls are the package's; otherwise they are elementary torch operations in
32 bits (angles in 64) on the same inputs.
"""
import math
import random

import torch

own = False

BF16, FP32 = "bf16", "fp32"
_DTYPE = {BF16: torch.bfloat16, FP32: torch.float32, "int32": torch.int32, "int64": torch.int64}
_BITS = {"bf16": 16, "mxfp8": 8, "mxfp4": 4}  # of a cache's element
BATCHES = 2  # of a gate: the rows of a call are those of two sequences


def _rope(name, T, H, D, axes, pairing, theta, pos, x, back=False):
    return {"name": name, "op": "rope", "T": T, "H": H, "D": D, "axes": axes, "pairing": pairing, "theta": theta, "pos": pos,
            "x": x, "back": back}


def _cache(name, form, B, T, R, L, H, D, page, x):
    return {"name": name, "op": "cache", "form": form, "B": B, "T": T, "R": R, "L": L, "H": H, "D": D, "page": page, "x": x}


def _attn(name, form, B, L, ragged, H, G, D, page, window, q, lse=False):
    return {"name": name, "op": "attn", "form": form, "B": B, "L": L, "ragged": ragged, "H": H, "G": G, "D": D, "page": page,
            "window": window, "q": q, "lse": lse}


def _linear(name, M, K, N, act, bias, residual, x, out):
    return {"name": name, "op": "linear", "M": M, "K": K, "N": N, "act": act, "bias": bias, "residual": residual, "x": x, "out": out}


def listed():
    return [
        # queries and keys of one new token far into a text, a slice of the fused projection's row
        _rope("rope_text_1x40x128", 1, 40, 128, "128", "halves", 500000.0, "int64", BF16),
        # queries and keys of one image's tokens: a text axis, row and column, slices of the fused projection
        _rope("rope_image_4608x48x128", 4608, 48, 128, "16,56,56", "pairs", 10000.0, "int32", BF16),
        # gradients through the positions of a video's tokens: scaled time, row and column
        _rope("rope_bwd_video_18000x16x72", 18000, 16, 72, "24,24,24", "pairs", 10000.0, FP32, FP32, True),
        # one new token of 32 sequences; the page that each is in, read back as for a fork
        _cache("cache_mxfp4_32x8x128", "mxfp4", 32, 1, 16, 4000, 8, 128, 16, BF16),
        # a prompt of an odd number of tokens behind a long prefix, all read back for the prompt's own attention
        _cache("cache_mxfp8_8191x8x128", "mxfp8", 1, 8191, 32768, 32768, 8, 128, 64, BF16),
        # one conversation: the fewest workgroups, latency counts
        _attn("attn_bf16_1x1000x32", "bf16", 1, 1000, False, 8, 4, 128, 16, 0, BF16),
        # a serving batch of ragged sequences, one of them empty
        _attn("attn_mxfp4_64x8192x32", "mxfp4", 64, 8192, True, 8, 4, 128, 32, 0, BF16),
        # four long documents, joined with another part's result by the caller
        _attn("attn_mxfp8_4x131072x32", "mxfp8", 4, 131072, False, 8, 4, 128, 128, 0, BF16, True),
        # heads of their own keys, a sliding window, all in 32 bits
        _attn("attn_mxfp4_window_7x5000x18", "mxfp4", 7, 5000, True, 18, 1, 64, 64, 1500, FP32),
        # one token through a projection: launch latency and the weight's read
        _linear("w4a16_1x4096x4096", 1, 4096, 4096, "none", False, False, BF16, BF16),
        # a speculative step of seven tokens through a gated up projection
        _linear("w4a16_swiglu_7x2240x11200", 7, 2240, 11200, "swiglu", True, False, BF16, BF16),
        # sixteen sequences' tokens through a down projection, gated and added to a stream in 32 bits
        _linear("w4a16_gate_16x12288x4096", 16, 12288, 4096, "none", True, True, FP32, FP32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = {"rope": _draw_rope, "cache": _draw_cache, "attn": _draw_attn, "linear": _draw_linear}[
        rng.choice(["rope", "cache", "attn", "attn", "linear", "linear"])](rng)
    return {k: v for k, v in case.items() if k != "name"}


def _draw_rope(rng):
    D = rng.choice([64, 72, 80, 96, 128, 128, 160, 256])
    axes = rng.choice([[D], [D // 2], [D // 4 // 2 * 2, D // 8 // 2 * 2], [D // 4 // 2 * 2] * 3, [D // 8 // 2 * 2] * 4])
    H = rng.randint(1, 64)
    T = _log_int(rng, 1, max(1, min(18432, 18000 * 1152 // (H * D))))
    return _rope("", T, H, D, ",".join(map(str, axes)), rng.choice(["pairs", "halves"]), rng.choice([256.0, 10000.0, 500000.0]),
                 rng.choice(["int32", "int64", FP32]), rng.choice([BF16, BF16, FP32]), rng.random() < 0.4)


def _draw_cache(rng):
    H, D, page = rng.choice([1, 2, 4, 8, 18]), rng.choice([64, 96, 128, 128, 256]), rng.choice([16, 32, 64, 128])
    form, B, x = rng.choice(["bf16", "mxfp8", "mxfp4", "mxfp4"]), _log_int(rng, 1, 64), rng.choice([BF16, BF16, FP32])
    L = _log_int(rng, 1, max(2, min(32768, 32768 * 1024 // (H * D * B))))
    T = _log_int(rng, 1, max(1, L // 4))
    return _cache("", form, B, T, rng.randint(T, L) if L > T else T, max(L, T), H, D, page, x)


def _draw_attn(rng):
    H, G, D = rng.choice([1, 2, 4, 8, 18]), rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([64, 96, 128, 128, 256])
    form, B = rng.choice(["bf16", "mxfp8", "mxfp4", "mxfp4"]), _log_int(rng, 1, 64)
    L = _log_int(rng, 1, min(131072, 4 * 131072 * 1024 * 4 * 8 // (B * H * D * max(G, 4) * max(8, _BITS[form]))))
    window = rng.choice([0, 0, 0, _log_int(rng, 1, max(2, L))])
    return _attn("", form, B, L, rng.random() < 0.7, H, G, D, rng.choice([16, 32, 64, 128]),
                 window, rng.choice([BF16, BF16, BF16, FP32]), rng.random() < 0.3)


def _draw_linear(rng):
    K, N, M = 32 * _log_int(rng, 8, 384), _log_int(rng, 64, 12288), _log_int(rng, 1, 16)
    residual = M % BATCHES == 0 and rng.random() < 0.4
    act = "none" if residual else rng.choice(["none", "gelu", "gelu_tanh", "silu", "relu", "swiglu"])
    return _linear("", M, K, N + N % 2 if act == "swiglu" else N, act, rng.random() < 0.6, residual, rng.choice([BF16, BF16, FP32]),
                   rng.choice([BF16, BF16, FP32]))


# ------------------------------------------------------------------ inputs

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1009 + salt)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _axes(case):
    return [int(d) for d in case["axes"].split(",")]


def _prepare_rope(case, seed):
    T, H, D, n = case["T"], case["H"], case["D"], len(_axes(case))
    g, dtype = _gen(seed, 1), _DTYPE[case["x"]]
    # rows of a fused projection: queries and keys, then as many values' heads as keys'; a gradient is an array of its own
    x = _randn(g, T, H if case["back"] else H + (H + 4) // 5, D).to(dtype)
    if n == 1:  # a text, from somewhere in it on
        pos = torch.arange(T, device="cuda").unsqueeze(1) + torch.randint(0, 1000000, (1,), generator=g, device="cuda")
    else:  # the last two axes a grid, those before it the number of the grid
        side = max(1, round(T ** (1.0 / min(n, 3))))
        i = torch.arange(T, device="cuda")
        pos = torch.stack([i // (side * side)] * (n - 2) + [i // side % side, i % side], 1)
        pos = pos + torch.randint(0, 64, (1, n), generator=g, device="cuda")
    pos = (pos * 0.75).float() if case["pos"] == FP32 else pos.to(_DTYPE[case["pos"]])
    return {"case": case, "x": x[:, :H], "positions": pos.contiguous()}


def _scale_bytes(amax, most):
    """E8M0 bytes of blocks: the binade of the largest magnitude over that of the format's largest."""
    e = torch.frexp(amax)[1] - 1 - most + 127
    return torch.where(amax > 0, e.clamp(0, 254), torch.zeros_like(e)).to(torch.uint8)


def _encoded(x, form):
    """Values [.., D] in 32 bits as a cache holds them: elements, and their scales [.., D / 32]."""
    if form == "bf16":
        return x.to(torch.bfloat16), None
    v = x.reshape(*x.shape[:-1], -1, 32)
    s = _scale_bytes(v.abs().amax(-1), 2 if form == "mxfp4" else 8)
    v = v * torch.exp2(127.0 - s.float()).unsqueeze(-1)
    if form == "mxfp8":
        return v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).reshape(x.shape), s
    m = v.abs()  # the border between two magnitudes goes to the one with an even code
    code = (m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
    code = (code + 8 * (v < 0)).to(torch.uint8).reshape(*x.shape[:-1], -1, 2)
    return code[..., 0] | (code[..., 1] << 4), s


def _lengths(case):
    """The sequences' lengths: all L, or the first L, the others up to it, and the last of four or more empty."""
    B, L = case["B"], case["L"]
    if not case["ragged"]:
        return [L] * B
    rng = random.Random(B * 1000003 + L)
    n = [L] + [_log_int(rng, 1, L) if rng.random() < 0.5 else rng.randint(1, L) for _ in range(B - 1)]
    return n[:-1] + [0] if B >= 4 else n


def _pages(g, case, spare):
    """A cache of random tokens, and the sequences' pages in it in no order."""
    B, L, H, D, page, form = (case[n] for n in ("B", "L", "H", "D", "page", "form"))
    each = -(-L // page)
    n = B * each + spare
    table = torch.randperm(n, generator=g, device="cuda")[: B * each].reshape(B, each).to(torch.int32)
    channel = 1.0 + 3.0 * (torch.rand(H, 1, D, generator=g, device="cuda") < 0.03)  # a few channels of the keys are large
    k, ks = _encoded(_randn(g, n, H, page, D) * channel, form)
    v, vs = _encoded(_randn(g, n, H, page, D) + 0.3 * _randn(g, H, 1, D), form)
    return {"k": k, "k_scales": ks, "v": v, "v_scales": vs}, table


def _prepare_cache(case, seed):
    B, T, R, L, H, D, page = (case[n] for n in ("B", "T", "R", "L", "H", "D", "page"))
    g = _gen(seed, 2)
    cache, table = _pages(g, case, 3)
    at = torch.arange(L, device="cuda")
    slots = table[:, at // page].long() * page + at % page
    kv = _randn(g, B * T, 2, H, D)
    kv[:, 0] *= 1.0 + 3.0 * (torch.rand(H, D, generator=g, device="cuda") < 0.03)
    kv = kv.to(_DTYPE[case["x"]])  # keys and values are slices of one projection
    # the sequences' last T tokens are new, their last R are read
    return {"case": case, "cache": cache, "new_k": kv[:, 0], "new_v": kv[:, 1], "slots": slots[:, L - T:].reshape(-1).contiguous(),
            "read": slots[:, L - R:].reshape(-1).contiguous()}


def _prepare_attn(case, seed):
    B, H, G, D = (case[n] for n in ("B", "H", "G", "D"))
    g = _gen(seed, 3)
    cache, table = _pages(g, case, 1)
    q = (1.5 * _randn(g, B, H * G, D)).to(_DTYPE[case["q"]])
    return {"case": case, "cache": cache, "table": table, "q": q,
            "lengths": torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")}


def _prepare_linear(case, seed):
    M, K, N = case["M"], case["K"], case["N"]
    g, st = _gen(seed, 4), {"case": case}
    x = _randn(g, M, K) * _randn(g, M, K).abs().clamp_min(0.2).rsqrt()  # heavy-tailed, a few channels large
    x[:, torch.randperm(K, generator=g, device="cuda")[: max(1, round(0.005 * K))]] *= 20.0
    st["x"] = x.to(_DTYPE[case["x"]])
    st["codes"], st["scales"] = _encoded(_randn(g, N, K) / math.sqrt(K), "mxfp4")
    if case["bias"]:
        st["bias"] = 0.2 * _randn(g, N)
    if case["residual"]:
        st["gate"] = 0.5 * _randn(g, BATCHES, N)
        st["residual"] = _randn(g, M, N).to(_DTYPE[case["out"]])
    return st


def prepare(case, seed):
    return {"rope": _prepare_rope, "cache": _prepare_cache, "attn": _prepare_attn, "linear": _prepare_linear}[case["op"]](case, seed)


# ------------------------------------------------------------------ the calls

def _run_own(st):
    import paper_2607_21446_amd as kq
    case = st["case"]
    if case["op"] == "rope":
        call = kq.rope_backward if case["back"] else kq.rope
        return call(st["x"], st["positions"], _axes(case), theta=case["theta"], pairing=case["pairing"])
    if case["op"] == "linear":
        return kq.w4a16_linear(st["x"], st["codes"], st["scales"], bias=st.get("bias"), act=None if case["act"] == "none" else case["act"],
                               gate=st.get("gate"), residual=st.get("residual"), out_dtype=_DTYPE[case["out"]])
    cache = kq.KVCache(**st["cache"])
    if case["op"] == "cache":
        kq.kv_cache_write(cache, st["new_k"], st["new_v"], st["slots"])
        return kq.kv_cache_read(cache, st["read"])
    return kq.paged_attention(st["q"], cache, st["table"], st["lengths"], window=case["window"] or None, want_lse=case["lse"])


def run(st):
    if own:
        return _run_own(st)
    return {"rope": _plain_rope, "cache": _plain_cache, "attn": _plain_attn, "linear": _plain_linear}[st["case"]["op"]](st)


# ------------------------------------------------------------------ plain forms, in 32 bits

def _angles(positions, axes, theta):
    """Angles of a row's pairs in 64 bits, section by section."""
    return torch.cat([positions[:, a:a + 1].double() * theta ** (-torch.arange(0, d, 2, device=positions.device).double() / d)
                      for a, d in enumerate(axes)], 1)


def _plain_rope(st):
    case, x = st["case"], st["x"].float()
    axes = _axes(case)
    n = sum(axes)
    angle = _angles(st["positions"], axes, case["theta"])
    c, s = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    s = -s if case["back"] else s
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if case["pairing"] == "pairs" else (x[..., : n // 2], x[..., n // 2: n])
    turned = [a * c - b * s, b * c + a * s]
    turned = torch.stack(turned, -1).flatten(-2) if case["pairing"] == "pairs" else torch.cat(turned, -1)
    return torch.cat([turned, x[..., n:]], -1).to(st["x"].dtype)


def _values(codes, scales):
    """What a cache's or a weight's elements stand for, in 32 bits."""
    if scales is None:
        return codes.float()
    if codes.shape[-1] == 32 * scales.shape[-1]:
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
        v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1)
    return (v.reshape(*scales.shape, 32) * torch.exp2(scales.float() - 127.0).unsqueeze(-1)).flatten(-2)


def _written(elements, scales, new, slots, form, page):
    e, s = _encoded(new.float(), form)
    elements[slots // page, :, slots % page] = e
    if s is not None:
        scales[slots // page, :, slots % page] = s


def _plain_cache(st):
    c, form, page = st["cache"], st["case"]["form"], st["case"]["page"]
    _written(c["k"], c["k_scales"], st["new_k"], st["slots"], form, page)
    _written(c["v"], c["v_scales"], st["new_v"], st["slots"], form, page)
    p, o = st["read"] // page, st["read"] % page
    at = lambda t: None if t is None else t[p, :, o]  # noqa: E731
    return tuple(_values(at(c[n]), at(c[n + "_scales"])).to(torch.bfloat16) for n in ("k", "v"))


def _plain_attn(st):
    """Every sequence padded to the longest."""
    case, c, B = st["case"], st["cache"], st["case"]["B"]
    H, G, D, t = case["H"], case["G"], case["D"], st["table"].long()
    of = lambda n: None if n is None else n[t].transpose(1, 2).flatten(2, 3)  # noqa: E731
    k, v = (_values(of(c[n]), of(c[n + "_scales"])) for n in ("k", "v"))  # [B, H, tokens, D]
    score = torch.matmul(st["q"].float().reshape(B, H, G, D) / math.sqrt(D), k.transpose(2, 3))
    at, n = torch.arange(k.shape[2], device=k.device), st["lengths"].long().unsqueeze(1)
    seen = at < n
    if case["window"]:
        seen = seen & (at >= n - case["window"])
    seen = seen[:, None, None]
    score = score.masked_fill(~seen, -math.inf)
    most = score.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(score - most)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.clamp_min(1e-30)
    out = out.reshape(B, H * G, D).to(st["q"].dtype)
    if not case["lse"]:
        return out
    return out, torch.where(total > 0, most + total.log(), -math.inf).reshape(B, H * G)


def _activated(p, act):
    if act == "gelu":
        return 0.5 * p * (1.0 + torch.erf(p * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * p * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (p + 0.044715 * p * p * p)))
    if act == "silu":
        return p * torch.sigmoid(p)
    if act == "relu":
        return torch.clamp_min(p, 0.0)
    if act == "swiglu":
        a = p[..., 0::2]
        return a * torch.sigmoid(a) * p[..., 1::2]
    return p


def _plain_linear(st):
    case = st["case"]
    p = torch.mm(st["x"].float(), _values(st["codes"], st["scales"]).T)
    if "bias" in st:
        p = p + st["bias"]
    p = _activated(p, case["act"])
    if "residual" in st:
        p = st["residual"].float() + st["gate"].repeat_interleave(case["M"] // BATCHES, 0) * p
    return p.to(_DTYPE[case["out"]])


def _row_bytes(case):
    """Of one token and head in one of a cache's two halves."""
    D, bits = case["D"], _BITS[case["form"]]
    return D * bits // 8 + (0 if bits == 16 else D // 32)


def work(case):
    size = lambda n: 2 if case[n] == BF16 else 4  # noqa: E731
    if case["op"] == "rope":
        T, n = case["T"], case["T"] * case["H"] * case["D"]
        return {"bytes": 2 * n * size("x") + T * len(_axes(case)) * (8 if case["pos"] == "int64" else 4), "flops": 3 * n}
    if case["op"] == "cache":
        T, R, H, D = case["B"] * case["T"], case["B"] * case["R"], case["H"], case["D"]
        return {"bytes": 2 * H * (T * (D * size("x") + _row_bytes(case)) + R * (_row_bytes(case) + 2 * D)) + 8 * (T + R),
                "flops": 2 * H * D * (4 * T + R)}
    if case["op"] == "attn":
        H, Hq, D = case["H"], case["H"] * case["G"], case["D"]
        seen = sum(min(n, case["window"] or n) for n in _lengths(case))
        return {"bytes": 2 * H * seen * _row_bytes(case) + 2 * case["B"] * Hq * D * size("q"), "flops": 4 * Hq * D * seen}
    M, K, N = case["M"], case["K"], case["N"]
    No = N // 2 if case["act"] == "swiglu" else N
    return {"bytes": N * K * 17 // 32 + M * K * size("x") + M * No * size("out") * (2 if case["residual"] else 1) + 4 * N * case["bias"]
            + (4 * BATCHES * N if case["residual"] else 0), "flops": 2 * M * N * K}


# ------------------------------------------------------------------ in 64 bits

def _exact_rope(case, seed):
    """Pairs as complex numbers; the gradient by autograd, from the forward formula alone."""
    st = _prepare_rope(case, seed)
    axes, x, pos = _axes(case), st["x"].double().contiguous(), st["positions"].double()
    n = sum(axes)
    freq = torch.cat([torch.exp(-math.log(case["theta"]) * 2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d) for d in axes])
    axis = torch.repeat_interleave(torch.arange(len(axes), device="cuda"), torch.tensor([d // 2 for d in axes], device="cuda"))
    unit = torch.polar(torch.ones_like(pos[:, axis]), pos[:, axis] * freq).unsqueeze(1)

    def turn(x):
        z = x[..., :n].unflatten(-1, (n // 2, 2) if case["pairing"] == "pairs" else (2, n // 2))
        z = torch.complex(*z.unbind(-1 if case["pairing"] == "pairs" else -2)) * unit
        return torch.cat([torch.stack([z.real, z.imag], -1 if case["pairing"] == "pairs" else -2).flatten(-2), x[..., n:]], -1)

    if not case["back"]:
        return turn(x)
    at = torch.zeros_like(x).requires_grad_()
    return torch.autograd.grad(turn(at), at, x)[0]


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _rounded64(x, form):
    """The nearest values that a cache holds for x [.., D]."""
    if form == "bf16":
        return x.to(torch.bfloat16).double()
    v = x.double().unflatten(-1, (-1, 32))
    top = v.abs().amax(-1, keepdim=True)
    unit = torch.exp2((torch.floor(torch.log2(top)) - (2 if form == "mxfp4" else 8)).clamp_min(-127.0))
    v = torch.where(top > 0, v / unit, torch.zeros_like(v))
    if form == "mxfp8":
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3.0)
        return (torch.clamp(torch.round(v / step) * step, -448.0, 448.0) * unit).flatten(-2)
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    m = v.abs().unsqueeze(-1)
    low = (grid <= m).sum(-1) - 1
    high = (low + 1).clamp_max(7)
    up, down = grid[high] - m.squeeze(-1), m.squeeze(-1) - grid[low]
    pick = torch.where((up < down) | ((up == down) & (low % 2 == 1)), high, low)
    return (torch.copysign(grid[pick], v) * unit).flatten(-2)


def _decoded64(codes, scales):
    if scales is None:
        return codes.double()
    if codes.shape[-1] == 32 * scales.shape[-1]:
        c = codes.long()
        e, m = c >> 3 & 15, (c & 7).double()
        mag = torch.where(e > 0, (1.0 + m / 8.0) * torch.pow(2.0, e.double() - 7.0), m * 2.0 ** -9)
        v = torch.where(c >= 128, -mag, mag)
    else:
        c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
        mag = torch.tensor(_E2M1, dtype=torch.float64, device=codes.device)[c & 7]
        v = torch.where(c >= 8, -mag, mag)
    return v * torch.pow(2.0, scales.double() - 127.0).repeat_interleave(32, -1)


def _exact_cache(case, seed):
    st = _prepare_cache(case, seed)
    page, out = case["page"], []
    for n in ("k", "v"):
        e, s = st["cache"][n], st["cache"][n + "_scales"]
        p, o = st["read"] // page, st["read"] % page
        got = _decoded64(e[p, :, o], None if s is None else s[p, :, o])
        where = {slot: i for i, slot in enumerate(st["slots"].tolist())}
        rows = [(i, where[slot]) for i, slot in enumerate(st["read"].tolist()) if slot in where]
        i, j = (torch.tensor(t, device="cuda") for t in zip(*rows))
        got[i] = _rounded64(st["new_" + n][j], case["form"])
        out.append(got)
    return tuple(out)


def _exact_attn(case, seed):
    """Sequence by sequence, over the tokens that count."""
    st = _prepare_attn(case, seed)
    H, G, D, c = case["H"], case["G"], case["D"], st["cache"]
    out = torch.zeros(case["B"], H * G, D, dtype=torch.float64, device="cuda")
    lse = torch.full((case["B"], H * G), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case)):
        at = torch.arange(max(0, n - case["window"]) if case["window"] else 0, n, device="cuda")
        if not len(at):
            continue
        p, o = st["table"][b].long()[at // case["page"]], at % case["page"]
        k, v = (_decoded64(c[m][p, :, o], None if c[m + "_scales"] is None else c[m + "_scales"][p, :, o]).transpose(0, 1) for m in ("k", "v"))
        score = st["q"][b].double().reshape(H, G, D) @ k.transpose(1, 2).contiguous() * D ** -0.5
        out[b] = (torch.softmax(score, -1) @ v.contiguous()).reshape(H * G, D)
        lse[b] = torch.logsumexp(score, -1).reshape(-1)
    return (out, lse) if case["lse"] else out


def _act64(p, act):
    if act == "gelu":
        return p * 0.5 * torch.special.erfc(-p / math.sqrt(2.0))
    if act == "gelu_tanh":
        z = math.sqrt(2.0 / math.pi) * (p + 0.044715 * p ** 3)
        return p / (1.0 + torch.exp(-2.0 * z))
    if act == "silu":
        return p / (1.0 + torch.exp(-p))
    if act == "relu":
        return torch.where(p > 0, p, torch.zeros_like(p))
    if act == "swiglu":
        a, b = p.unflatten(-1, (p.shape[-1] // 2, 2)).unbind(-1)
        return a * b / (1.0 + torch.exp(-a))
    return p


def _exact_linear(case, seed):
    st = _prepare_linear(case, seed)
    p = st["x"].double() @ _decoded64(st["codes"], st["scales"]).T
    if "bias" in st:
        p += st["bias"].double()
    p = _act64(p, case["act"])
    if "residual" in st:
        rows = torch.arange(case["M"], device="cuda") // (case["M"] // BATCHES)
        p = st["residual"].double() + st["gate"].double()[rows] * p
    return p


def exact(case, seed):
    return {"rope": _exact_rope, "cache": _exact_cache, "attn": _exact_attn, "linear": _exact_linear}[case["op"]](case, seed)
